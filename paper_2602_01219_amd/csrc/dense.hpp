// dense.hpp - building blocks of the dense attention kernels: row tiles staged
// in LDS, 32x32 MFMA products of a tile with operands held in registers, and the
// block order.
//
// A wave owns 32 columns (query rows in the forward and the query side of the
// backward, keys in its key side); lane l = 32 g + n belongs to column n. A tile
// holds 32 or 64 rows of D elements (keys and values, or queries and their
// gradients). Two products are formed with it:
//   rows:  C[i][n] = sum_d X[i][d] B[d][n]     (32 tile rows by 32 columns; B in registers)
//   cols:  A[d][n] += sum_i X[i][d] P[i][n]    (P as it left a `rows` product)
// A v_mfma_f32_32x32 accumulator holds C[8 (i / 4) + 4 g + i % 4][n], i = 0..15.
// As the B operand of the next product a lane needs rows of its own group g, and
// which rows a group takes is free as long as both operands agree: the
// accumulator's own rows serve, so P never moves between lanes.
// bf16: one v_mfma_f32_32x32x16_bf16 per 16-long reduction step. fp32: each operand
// as three bf16 numbers that add up to it exactly, and six of the nine products (see
// Split for the three left out). That takes 6 x 32 cycles of the matrix cores per 16-long step where the
// fp32 instruction takes 8 x 64, and splitting an operand on the way (44 VALU
// instructions per 8 elements and lane) runs beside it: 16 heads of 2048 tokens, d =
// 128, 310 -> 224 us forward and 1049 -> 800 backward, 154 TFLOP/s of fp32 products.
#pragma once
#include "cdna4.hpp"
#include "flash.hpp"

namespace mita {

typedef __attribute__((ext_vector_type(16))) float f32x16;

__device__ __forceinline__ f32x16 splat16(float x) {
  return f32x16{x, x, x, x, x, x, x, x, x, x, x, x, x, x, x, x};
}
// The tile row of accumulator element i for lane group g.
__device__ __forceinline__ int acc_row(int i, int g) { return 8 * (i >> 2) + 4 * g + (i & 3); }

template <typename T, int D> struct RowTile {
  static constexpr int RB = D * (int)sizeof(T);  // bytes per row
  static constexpr int CPR = RB / 16;            // 16-byte chunks per row
  static constexpr int RPI = 64 / CPR;           // rows one wave-wide copy fills
  static constexpr int NS = CPR / 2;             // pairs of chunks, one per lane group
  static constexpr int NB = D / 32;              // 32-wide blocks of d
  static constexpr int TR = sizeof(T) == 2 ? 64 : 32;  // rows per staged tile
  // Slot s of row r holds chunk s ^ swz(r). LDS serves 256 bytes per cycle: 16
  // lanes of the 16-byte reads (16 consecutive rows at one chunk), 32 lanes of
  // the transposing 8-byte reads (4 rows by 4 chunks), 64 lanes of fp32's 4-byte
  // reads (8 chunks of two rows 4 apart). With these each falls into 16
  // different 16-byte columns.
  __device__ __forceinline__ static int swz(int r) {
    if (sizeof(T) == 4) return ((r >> 2) & 1) << 3 | ((r >> 3) & 1) << 2 | (r & 3);
    if (CPR == 8) return ((r >> 1) & 1) << 2 | ((r >> 2) & 3);
    return (r & 3) << 2 | ((r >> 2) & 3);
  }
};

// LDS DMA of 16 (4) bytes per lane: lane l's go to LDS address at + 16 l (4 l). Written as
// instructions because around the builtin the compiler sets waits of its own before
// LDS reads that it cannot tell apart from the copy (for every copy in flight, where
// control flow meets): the caller waits with wait_copies or tile_barrier. base and
// at are the same for the whole wave, off the lane's bytes behind base.
__device__ __forceinline__ uint32_t lds_at(char *p) {  // address of the workgroup's LDS
  return __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(lds_void_t *)p);
}
__device__ __forceinline__ void copy16_unwaited(const char *base, uint32_t off, uint32_t at) {
  asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(off), "s"(base), "{m0}"(at) : "memory");
}

__device__ __forceinline__ void copy16_unwaited(const char *src, uint32_t at) {  // any 64-bit address per lane
  asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(src), "{m0}"(at) : "memory");
}
__device__ __forceinline__ void copy4_unwaited(const char *base, uint32_t off, uint32_t at) {
  asm volatile("s_nop 0\n\tglobal_load_lds_dword %0, %1" ::"v"(off), "s"(base), "{m0}"(at) : "memory");
}

// The copies this wave issued have landed, and those of every wave once all are
// here. (The barrier alone does not wait for them: a wave that reads none of the
// tile, or reads it behind the barrier, would pass with its own in flight.)
__device__ __forceinline__ void tile_barrier() {
  wait_loads();
  __syncthreads();
}

// All but this wave's last N copies have landed; all its LDS reads have returned.
template <int N> __device__ __forceinline__ void wait_copies() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt((N & 15) | (N >> 4) << 14 | 0x0f70);
  asm volatile("" ::: "memory");
}
__device__ __forceinline__ void wait_lds() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0xc07f);
  asm volatile("" ::: "memory");
}

// A tile's copy into LDS by DMA (global_load_lds_dwordx4), NW waves: lane l of
// copy `ins` fills slot l % CPR of row ins * RPI + l / CPR. swz is linear over the
// bits of the row, and a wave's copies j differ in bits of their own, so copy j's
// chunk is that of its first XOR swz(j RPI).
template <typename T, int D, int NW> struct TileCopy {
  using RT = RowTile<T, D>;
  static constexpr int PW = RT::TR / RT::RPI / NW;  // copies per wave
  static_assert(PW >= 1 && RT::TR % (RT::RPI * NW) == 0, "whole copies per wave");
  int w;           // the wave, as a scalar
  uint32_t row0;   // the lane's row of the wave's first copy
  uint32_t chunk0; // byte offset of its chunk in the row
  __device__ __forceinline__ void init() {
    w = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int lane = threadIdx.x & 63, r = w * PW * RT::RPI + lane / RT::CPR;
    row0 = (uint32_t)r;
    chunk0 = (uint32_t)(((lane % RT::CPR) ^ RT::swz(r)) << 4);
  }
  __device__ __forceinline__ void forget() {  // (see TileAddr)
    pin(row0);
    pin(chunk0);
  }
  __device__ __forceinline__ uint32_t row(int j) const { return row0 + j * RT::RPI; }
  __device__ __forceinline__ uint32_t chunk(int j) const { return chunk0 ^ (uint32_t)(RT::swz(j * RT::RPI) << 4); }
  // rows `first` .. of a matrix whose rows are `stride` bytes apart (off0 = row0
  // stride); of the tile's rows only the first nrows (>= 1) exist, the others
  // repeat the last of them
  __device__ __forceinline__ void issue(uint32_t tile, const char *base, int first, uint32_t stride, uint32_t off0,
                                        int nrows) const {
    const char *src = base + (int64_t)first * stride;
    if (nrows >= RT::TR) {
#pragma unroll
      for (int j = 0; j < PW; ++j)
        copy16_unwaited(src + (uint64_t)(j * RT::RPI) * stride, off0 + chunk(j), tile + (w * PW + j) * 1024);
    } else {
#pragma unroll
      for (int j = 0; j < PW; ++j)
        copy16_unwaited(src, min(row(j), (uint32_t)(nrows - 1)) * stride + chunk(j), tile + (w * PW + j) * 1024);
    }
  }
};

// The tiles of a workgroup in the order it takes them: position p < nfull is tile
// f0 + p, seen whole by every row; the others (which the window or an end cuts)
// follow, those in front of the full ones first.
struct TileOrder {
  int f0, nfull, h0, nhead, r0, total;
  // tiles [t0, t1), of which [fa, fb) are seen whole
  __device__ __forceinline__ TileOrder(int t0, int t1, int fa, int fb) {
    const int f1 = max(t0, min(fb, t1));
    f0 = min(max(fa, t0), f1);
    nfull = f1 - f0;
    h0 = t0;
    nhead = f0 - t0;
    r0 = f1;
    total = max(0, t1 - t0);
  }
  __device__ __forceinline__ int at(int p) const {
    const int m = p - nfull;
    return m < 0 ? f0 + p : m < nhead ? h0 + m : r0 + m - nhead;
  }
};

// Per-lane LDS addresses of the two products, fixed for every tile.
template <typename T, int D> struct TileAddr {
  using RT = RowTile<T, D>;
  uint32_t r0;  // `rows`: chunk g of row n; step s is r0 ^ (s << 5)
  uint32_t c0;  // `cols`: see col
  __device__ __forceinline__ void init() {
    const int lane = threadIdx.x & 63, n = lane & 31, g = lane >> 5;
    r0 = (uint32_t)(n * RT::RB + ((g ^ RT::swz(n)) << 4));
    if constexpr (sizeof(T) == 2) {
      // 16-lane groups read 4 x 16 blocks transposed (ds_read_b64_tr_b16: lane
      // 4 e + p addresses piece p of row e, lane i receives column i)
      const int e = (lane & 15) >> 2, p = lane & 3, half = (lane >> 4) & 1, r = 4 * g + e;
      c0 = (uint32_t)(r * RT::RB + (((2 * half + (p >> 1)) ^ RT::swz(r)) << 4) + ((p & 1) << 3));
    } else {
      // row 8 q + 4 g + r, element n of block db: c0 ^ (db << 7) ^ swizzle(q, r), + (8 q + r) rows
      c0 = (uint32_t)(4 * g * RT::RB + (((n >> 2) ^ (g << 3)) << 4) + ((n & 3) << 2));
    }
  }
  // bf16: rows 8 h + 4 g + e of 16, columns 32 db + 16 ((lane >> 4) & 1) + i
  __device__ __forceinline__ uint32_t col(int db, int h) const {
    return (c0 ^ (uint32_t)(((4 * db) ^ RT::swz(8 * h)) << 4)) + (uint32_t)(8 * h * RT::RB);
  }
  // Addresses that derive from these are formed again where they are used from
  // here on, instead of being kept in registers.
  __device__ __forceinline__ void forget() {
    pin(r0);
    pin(c0);
  }
};

__device__ __forceinline__ f32x16 mma32(const uint4 &a, const uint4 &b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0,
                                                 0);
}

// Eight fp32 values as bf16 numbers h + m + l = x. `cut`: h and m are the upper halves
// of x and of x - h, and l, what is left, has at most 8 bits; all have x's sign. `near`:
// h and m are x and x - h rounded to nearest (the largest fp32 numbers to the largest
// bf16 one), so that m and l have either sign; for operands that are split once.
// The products m l', l m' and l l' are left out. With one operand `near` (a column: rows
// times columns) they are at most 2^-22.4 of the product, of either sign and 0 on
// average. With both `cut` (the sums of rows weighted by P or dS, where splitting P
// `near` for every tile costs 1 to 4% of the call) they are at most 2^-21 and have the
// product's sign: such a product is low by 2^-24.7 of itself on average, 0.6 of half an
// fp32 step.
struct Split {
  uint4 h, m, l;
  __device__ __forceinline__ static uint4 upper(const uint32_t (&v)[8]) {
    return make_uint4(__builtin_amdgcn_perm(v[1], v[0], 0x07060302u), __builtin_amdgcn_perm(v[3], v[2], 0x07060302u),
                      __builtin_amdgcn_perm(v[5], v[4], 0x07060302u), __builtin_amdgcn_perm(v[7], v[6], 0x07060302u));
  }
  __device__ __forceinline__ void cut(const float (&x)[8]) {
    uint32_t u[3][8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      u[0][i] = __float_as_uint(x[i]);
      const float r = x[i] - __uint_as_float(u[0][i] & 0xffff0000u);
      u[1][i] = __float_as_uint(r);
      u[2][i] = __float_as_uint(r - __uint_as_float(u[1][i] & 0xffff0000u));
    }
    h = upper(u[0]);
    m = upper(u[1]);
    l = upper(u[2]);
  }
  __device__ __forceinline__ void near(const float (&x)[8]) {
    const float most = __uint_as_float(0x7f7f0000u);
    uint32_t a[4], b[4], c[8];
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
      a[i / 2] = pack_bf16x2(__builtin_amdgcn_fmed3f(x[i], -most, most), __builtin_amdgcn_fmed3f(x[i + 1], -most, most));
      const float r[2] = {x[i] - __uint_as_float(a[i / 2] << 16), x[i + 1] - __uint_as_float(a[i / 2] & 0xffff0000u)};
      b[i / 2] = pack_bf16x2(r[0], r[1]);
      c[i] = __float_as_uint(r[0] - __uint_as_float(b[i / 2] << 16));
      c[i + 1] = __float_as_uint(r[1] - __uint_as_float(b[i / 2] & 0xffff0000u));
    }
    h = make_uint4(a[0], a[1], a[2], a[3]);
    m = make_uint4(b[0], b[1], b[2], b[3]);
    l = upper(c);
  }
  __device__ __forceinline__ static void floats(float (&x)[8], const uint4 &a, const uint4 &b) {
    x[0] = __uint_as_float(a.x), x[1] = __uint_as_float(a.y), x[2] = __uint_as_float(a.z), x[3] = __uint_as_float(a.w);
    x[4] = __uint_as_float(b.x), x[5] = __uint_as_float(b.y), x[6] = __uint_as_float(b.z), x[7] = __uint_as_float(b.w);
  }
};
// The six products of the largest parts.
__device__ __forceinline__ f32x16 mma32(const Split &a, const Split &b, f32x16 c) {
  c = mma32(a.l, b.h, c);
  c = mma32(a.h, b.l, c);
  c = mma32(a.m, b.m, c);
  c = mma32(a.m, b.h, c);
  c = mma32(a.h, b.m, c);
  return mma32(a.h, b.h, c);
}

// A lane's column as B operand of `rows`, from its row in memory (zero without one):
// bf16 holds chunk 2 s + g for step s, fp32 chunks 4 t + g and 4 t + 2 + g for step t.
template <typename T, int D> struct Column;
template <int D> struct Column<bf16_t, D> {
  static constexpr int NS = RowTile<bf16_t, D>::NS;
  uint4 b[NS];
  __device__ __forceinline__ void load(const char *row, bool valid) {
    const int g = (threadIdx.x & 63) >> 5;
#pragma unroll
    for (int s = 0; s < NS; ++s)
      b[s] = valid ? *reinterpret_cast<const uint4 *>(row + 32 * s + 16 * g) : make_uint4(0, 0, 0, 0);
  }
};
template <int D> struct Column<float, D> {
  static constexpr int NS = RowTile<float, D>::NS / 2;
  Split b[NS];
  __device__ __forceinline__ void load(const char *row, bool valid) {
    const int g = (threadIdx.x & 63) >> 5;
    uint4 x[2 * NS];
#pragma unroll
    for (int s = 0; s < 2 * NS; ++s)
      x[s] = valid ? *reinterpret_cast<const uint4 *>(row + 32 * s + 16 * g) : make_uint4(0, 0, 0, 0);
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      float y[8];
      Split::floats(y, x[2 * s], x[2 * s + 1]);
      b[s].near(y);
    }
  }
};
// The scalar product of a column's rows x and y (0 without them), in both its lanes' parts.
template <typename T, int D> __device__ __forceinline__ float column_dot(const char *x, const char *y, bool valid) {
  const int g = (threadIdx.x & 63) >> 5;
  float d = 0.f;
  if (valid) {
#pragma unroll
    for (int s = 0; s < RowTile<T, D>::NS; ++s) {
      float u[16 / sizeof(T)], v[16 / sizeof(T)];
      unpack16(*reinterpret_cast<const uint4 *>(x + 32 * s + 16 * g), u, (const T *)nullptr);
      unpack16(*reinterpret_cast<const uint4 *>(y + 32 * s + 16 * g), v, (const T *)nullptr);
#pragma unroll
      for (int j = 0; j < 16 / (int)sizeof(T); ++j) d = __builtin_fmaf(u[j], v[j], d);
    }
  }
  return d;
}

// c + X B for the 32 tile rows from 32 kb on.
template <int D>
__device__ __forceinline__ f32x16 tile_rows(const char *tile, const TileAddr<bf16_t, D> &ad, int kb,
                                            const Column<bf16_t, D> &col, f32x16 c) {
  using RT = RowTile<bf16_t, D>;
#pragma unroll
  for (int s = 0; s < RT::NS; ++s)
    c = mma32(*reinterpret_cast<const uint4 *>(tile + (ad.r0 ^ (uint32_t)(s << 5)) + kb * 32 * RT::RB), col.b[s], c);
  return c;
}
template <int D>
__device__ __forceinline__ f32x16 tile_rows(const char *tile, const TileAddr<float, D> &ad, int kb,
                                            const Column<float, D> &col, f32x16 c) {
  using RT = RowTile<float, D>;
#pragma unroll
  for (int s = 0; s < RT::NS; s += 2) {
    float x[8];
    Split::floats(x, *reinterpret_cast<const uint4 *>(tile + (ad.r0 ^ (uint32_t)(s << 5)) + kb * 32 * RT::RB),
                  *reinterpret_cast<const uint4 *>(tile + (ad.r0 ^ (uint32_t)((s + 1) << 5)) + kb * 32 * RT::RB));
    Split a;
    a.cut(x);
    c = mma32(a, col.b[s / 2], c);
  }
  return c;
}

// P as the B operand, 16 rows each: bf16 rounds it (up to 2^-8 of each weight; errors of o
// against float64 go from 0.0017, the rounding of o itself, to 0.0021 - 0.0024, where
// two bf16 numbers per weight would cost half as many products again), fp32 splits it.
template <typename T> struct ColsOperand;
template <> struct ColsOperand<bf16_t> {
  uint4 b[2];
  __device__ __forceinline__ explicit ColsOperand(const f32x16 &p) {
#pragma unroll
    for (int s = 0; s < 2; ++s)
      b[s] = make_uint4(pack_bf16x2(p[8 * s], p[8 * s + 1]), pack_bf16x2(p[8 * s + 2], p[8 * s + 3]),
                        pack_bf16x2(p[8 * s + 4], p[8 * s + 5]), pack_bf16x2(p[8 * s + 6], p[8 * s + 7]));
  }
};
template <> struct ColsOperand<float> {
  Split b[2];
  __device__ __forceinline__ explicit ColsOperand(const f32x16 &p) {
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const float x[8] = {p[8 * s],     p[8 * s + 1], p[8 * s + 2], p[8 * s + 3],
                          p[8 * s + 4], p[8 * s + 5], p[8 * s + 6], p[8 * s + 7]};
      b[s].cut(x);
    }
  }
};

// acc[db] += X^T P for the 32 tile rows from 32 kb on.
template <int D>
__device__ __forceinline__ void tile_cols(f32x16 (&acc)[D / 32], const char *tile, const TileAddr<bf16_t, D> &ad, int kb,
                                          const ColsOperand<bf16_t> &P) {
  using RT = RowTile<bf16_t, D>;
#pragma unroll
  for (int s = 0; s < 2; ++s)
#pragma unroll
    for (int db = 0; db < RT::NB; ++db) {
      uint2 h[2];
#pragma unroll
      for (int i = 0; i < 2; ++i)
        h[i] = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                                             (lds_v4i16_t *)(tile + ad.col(db, i) + (32 * kb + 16 * s) * RT::RB)));
      acc[db] = mma32(make_uint4(h[0].x, h[0].y, h[1].x, h[1].y), P.b[s], acc[db]);
    }
}
template <int D>
__device__ __forceinline__ void tile_cols(f32x16 (&acc)[D / 32], const char *tile, const TileAddr<float, D> &ad, int kb,
                                          const ColsOperand<float> &P) {
  using RT = RowTile<float, D>;
#pragma unroll
  for (int s = 0; s < 2; ++s)
#pragma unroll
    for (int db = 0; db < RT::NB; ++db) {
      float x[8];  // rows acc_row(8 s + e, g), element n of block db
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int q = 2 * s + (e >> 2), r = e & 3;
        x[e] = *reinterpret_cast<const float *>(
            tile + (ad.c0 ^ (uint32_t)(((q & 1) << 2 | r) << 4) ^ (uint32_t)(db << 7)) + (32 * kb + 8 * q + r) * RT::RB);
      }
      Split a;
      a.cut(x);
      acc[db] = mma32(a, P.b[s], acc[db]);
    }
}

// The column's accumulators (d = 32 db + acc_row(i, g)) times `mul` to its row,
// 16 bytes per lane and store: bf16 lanes n and n + 32 exchange half of their
// 4-wide pieces, so each holds 8 consecutive elements.
template <int D>
__device__ __forceinline__ void store_column(float *row, const f32x16 (&acc)[D / 32], float mul, bool valid) {
  const int g = (threadIdx.x & 63) >> 5;
  if (!valid) return;
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int q = 0; q < 4; ++q)
      *reinterpret_cast<float4 *>(row + 32 * db + 8 * q + 4 * g) = make_float4(
          acc[db][4 * q] * mul, acc[db][4 * q + 1] * mul, acc[db][4 * q + 2] * mul, acc[db][4 * q + 3] * mul);
}
template <int D>
__device__ __forceinline__ void store_column(bf16_t *row, const f32x16 (&acc)[D / 32], float mul, bool valid) {
  const int g = (threadIdx.x & 63) >> 5;
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int q = 0; q < 4; q += 2) {
      uint32_t x[2], y[2];  // pieces q and q + 1
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        x[i] = pack_bf16x2(acc[db][4 * q + 2 * i] * mul, acc[db][4 * q + 2 * i + 1] * mul);
        y[i] = pack_bf16x2(acc[db][4 * q + 4 + 2 * i] * mul, acc[db][4 * q + 5 + 2 * i] * mul);
      }
      // first: piece q of the low half's lanes, q + 1 of the low half's in the
      // high lanes; second: the high half's
      const auto a = __builtin_amdgcn_permlane32_swap(x[0], y[0], false, false);
      const auto b = __builtin_amdgcn_permlane32_swap(x[1], y[1], false, false);
      if (valid) *reinterpret_cast<uint4 *>(row + 32 * db + 8 * (q + g)) = make_uint4(a[0], b[0], a[1], b[1]);
    }
}

// Sum (maximum) of x over the two lanes of a column.
__device__ __forceinline__ float column_sum(float x) {
  const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(a[0]) + __uint_as_float(a[1]);
}
__device__ __forceinline__ float column_max(float x) {
  const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
}

// ---------------------------------------------------------------------------
// Arguments and index arithmetic
// ---------------------------------------------------------------------------
struct DenseMat {
  const char *p;
  int64_t b, h;  // bytes between batch elements and heads
  uint32_t n;    // bytes between tokens
};
struct DenseArgs {
  DenseMat q, k, v, o, dO;        // o is written by the forward
  DenseMat dq, dk, dv;            // written
  const int32_t *q_len, *k_len;
  float *lse;                     // [B, H, N], written by the forward; may be NULL there
  float *part_o, *part_lse;       // the forward's splits
  float *row_lse, *row_D;         // the backward's rows (log2 units; see dense_backward.hip), padded to tiles
  float *part_q, *part_k, *part_v;
  int B, H, Hkv, G, N, Nk, R;
  int left, right;
  uint64_t magic;                 // 2^40 / G + 1
  float scale, sl2;               // sl2 = scale * log2(e)
  int tiles, splits;
  bool near;                      // a slice's rows of q and dO lie within 2^32 bytes
};

// r / G for r < 2^27, G <= 2^12: r * (2^40 / G + 1) errs by less than r / 2^40
// of a quotient step, below 1 / G
__device__ __forceinline__ int div_group(const DenseArgs &a, int r) {
  return (int)(((uint64_t)(uint32_t)r * a.magic) >> 40);
}

struct DenseSlice {
  int b, hk, qlen, klen, off;  // off: position of query 0
};
__device__ __forceinline__ DenseSlice dense_slice(const DenseArgs &a, int s) {
  DenseSlice x;
  x.b = s / a.Hkv;
  x.hk = s - x.b * a.Hkv;
  x.qlen = a.q_len ? min(max(a.q_len[x.b], 0), a.N) : a.N;
  x.klen = a.k_len ? min(max(a.k_len[x.b], 0), a.Nk) : a.Nk;
  x.off = x.klen - x.qlen;
  return x;
}
// Keys [lo, hi) that query `tok` sees (hi <= lo: none).
__device__ __forceinline__ int first_key(const DenseArgs &a, const DenseSlice &x, int tok) {
  return max(0, tok + x.off - a.left);
}
__device__ __forceinline__ int end_key(const DenseArgs &a, const DenseSlice &x, int tok) {
  return min(x.klen, tok + x.off + a.right + 1);
}

// Block id -> (slice, work item of the slice). Consecutive ids go to the eight
// XCDs in turn; a slice's items stay on one XCD, whose L2 then holds the rows
// they share, except for the last S % 8 slices, whose items go round all XCDs. The
// slices come to the XCDs in snake order, which evens out lengths that fall (or
// rise) over the batch.
__device__ __forceinline__ void dense_block(int id, int S, int items, int &slice, int &item, bool snake = true) {
  const int whole = S & ~7;
  if (id < whole * items) {
    const int j = id >> 3, round = j / items;
    slice = 8 * round + (snake && (round & 1) ? 7 - (id & 7) : id & 7);
    item = j - round * items;
  } else {
    const int j = id - whole * items, rest = S - whole;
    // items outermost: the heavy first items of every slice start first
    slice = whole + j % rest;
    item = j / rest;
  }
}

}  // namespace mita
