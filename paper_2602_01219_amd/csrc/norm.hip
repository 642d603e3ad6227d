// norm.hip - layer norm of rows and its gradients.
//
// Forward: y = (x - mean) rstd w + b. Backward, with h = (x - mean) rstd and
// g = dy w: dx = rstd (g - mean(g) - h mean(g h)), dw = sum dy h, db = sum dy.
// Both are bound by HBM: a row is read once into registers, its sums go across
// the lanes that share it (DPP within a wave), and it is written once (see norm_plan
// for the widest rows that fit; wider ones are read once per pass). The variance
// is summed about the mean from the registers (a one-pass sum of squares cancels
// where the mean is large). Loads and stores share one counter, so a loop that
// fetches the next row early waits for the stores of the last: rows come in waves
// that end instead (forward) or enough waves (backward). In the backward each lane
// keeps the sums of dw and db of its own columns over all rows its workgroup takes;
// one partial sum per workgroup goes to memory, and a second launch adds them in a
// fixed order. Measured: queries of 2 x 12 heads x 16384 tokens, d = 64, bf16, 19.9 us
// (104 MB: 5.3 TB/s; 26.0 as a persistent loop); backward of 32768 x 768 bf16
// 30 us and 4 for the sums (151 MB, 5 TB/s in the first; 37 as a loop that
// prefetched). Wide rows are further from it. 2048 rows forward: 8192 elements fp32 22
// us (22 at 6.2 TB/s) and bf16 15 (11), 16384 bf16 32 (22), 12288 fp32 in three passes 91 (32).
// Backward: 8192 bf16 38 (16), 16384 bf16 76 (32), 12288 fp32 138 (49): with 1024
// threads per row there are 128 registers for each, and the kernels that hold dw and db
// spill 23 (16-byte pieces of bf16) to 75 (two-element pieces) of them.
#include "cdna4.hpp"
#include "kernels.hpp"
#include "layer_check.hpp"

namespace mita {

namespace {

struct NormRows {
  int64_t s[3];  // distances in elements, in the order of the walk
  bool flat;     // rows of the walk are s[2] apart all over
};
struct NormArgs {
  const void *x, *dy, *w, *b;
  void *y, *dx, *dw, *db;
  const float *mean_in, *rstd_in;
  float *mean, *rstd, *part;
  // rows are walked in the order of x in memory, dimensions 0, 1, 2 from the
  // outside in; `stat` is the place of the row's statistics
  NormRows sx, sy, sdy, sdx, stat;
  int rows, n1, n2, C;
  uint32_t m1, m2;  // for quotients by n1 and n2
  int h1, h2;
  bool w16;  // weights in bf16
  float eps, invC;
};

// r / n for r < 2^31 with l = ceil(log2 n), m = 2^(31 + l) / n + 1 (floored, below
// 2^32 + 1 and so below 2^32 for n > 1), h = l - 1: r m exceeds 2^(31 + l) r / n by
// at most r < 2^31, less than a step of 1 / n. n = 1: h < 0.
__device__ __forceinline__ int quotient(int r, uint32_t m, int h) { return h < 0 ? r : (int)(__umulhi((uint32_t)r, m) >> h); }

__device__ __forceinline__ int64_t row_at(const NormArgs &a, const NormRows &s, int r) {
  if (s.flat) return (int64_t)r * s.s[2];
  const int t = quotient(r, a.m2, a.h2), i2 = r - t * a.n2, i0 = quotient(t, a.m1, a.h1), i1 = t - i0 * a.n1;
  return i0 * s.s[0] + i1 * s.s[1] + i2 * s.s[2];
}

// The pieces of a row that one thread holds: piece j is elements (j TPR + t) VE ..
template <typename T, int VE> struct Piece;
template <typename T> struct Piece<T, 16 / sizeof(T)> {
  uint4 v;
  __device__ __forceinline__ void load(const T *p) { v = *reinterpret_cast<const uint4 *>(p); }
  __device__ __forceinline__ void get(float *f) const { unpack16(v, f, (const T *)nullptr); }
};
template <> struct Piece<bf16_t, 2> {
  uint32_t v;
  __device__ __forceinline__ void load(const bf16_t *p) { v = *reinterpret_cast<const uint32_t *>(p); }
  __device__ __forceinline__ void get(float *f) const {
    f[0] = __uint_as_float(v << 16);
    f[1] = __uint_as_float(v & 0xffff0000u);
  }
};
template <> struct Piece<float, 2> {
  float2 v;
  __device__ __forceinline__ void load(const float *p) { v = *reinterpret_cast<const float2 *>(p); }
  __device__ __forceinline__ void get(float *f) const {
    f[0] = v.x;
    f[1] = v.y;
  }
};
template <typename T> struct Piece<T, 1> {
  T v;
  __device__ __forceinline__ void load(const T *p) { v = *p; }
  __device__ __forceinline__ void get(float *f) const { f[0] = to_f32(v); }
};
template <typename T, int VE> __device__ __forceinline__ void put(T *p, const float *f) {
  if constexpr (VE == 1) {
    *p = from_f32<T>(f[0]);
  } else if constexpr (VE == 2 && sizeof(T) == 4) {
    *reinterpret_cast<float2 *>(p) = make_float2(f[0], f[1]);
  } else if constexpr (VE == 2) {
    *reinterpret_cast<uint32_t *>(p) = pack_bf16x2(f[0], f[1]);
  } else if constexpr (sizeof(T) == 4) {
    *reinterpret_cast<float4 *>(p) = make_float4(f[0], f[1], f[2], f[3]);
  } else {
    *reinterpret_cast<uint4 *>(p) = make_uint4(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]),
                                               pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7]));
  }
}

template <typename T, int VE, int TPR, int P> struct RowRegs {
  Piece<T, VE> c[P];
  // pieces past the row repeat its last one (see `get`)
  __device__ __forceinline__ void load(const T *row, int C, int t) {
#pragma unroll
    for (int j = 0; j < P; ++j) c[j].load(row + min((j * TPR + t) * VE, C - VE));
  }
  // piece j in fp32, zero past the row
  __device__ __forceinline__ void get(float (&f)[VE], int j, int C, int t) const {
    c[j].get(f);
    const bool in = (j * TPR + t) * VE < C;
#pragma unroll
    for (int e = 0; e < VE; ++e) f[e] = in ? f[e] : 0.f;
  }
};

// The thread's weights (`missing` without any): column (j TPR + t) VE + e. Past the
// row they repeat its last columns.
template <int VE, int TPR, int P>
__device__ __forceinline__ void weights(float (&f)[P][VE], const void *w, bool w16, int C, int t, float missing) {
  if (!w) {
#pragma unroll
    for (int j = 0; j < P; ++j)
#pragma unroll
      for (int e = 0; e < VE; ++e) f[j][e] = missing;
  } else if (w16) {
    uint16_t u[P][VE];
#pragma unroll
    for (int j = 0; j < P; ++j)
#pragma unroll
      for (int e = 0; e < VE; ++e) u[j][e] = ((const uint16_t *)w)[min((j * TPR + t) * VE, C - VE) + e];
#pragma unroll
    for (int j = 0; j < P; ++j)
#pragma unroll
      for (int e = 0; e < VE; ++e) f[j][e] = bf16_to_f32(u[j][e]);
  } else {
#pragma unroll
    for (int j = 0; j < P; ++j)
#pragma unroll
      for (int e = 0; e < VE; ++e) f[j][e] = ((const float *)w)[min((j * TPR + t) * VE, C - VE) + e];
  }
}

// Sum over the lanes of a group of W (a power of two), the same in each: lanes are
// paired within quads, halves and rows of 16 by DPP, then across rows by swaps.
template <int W> __device__ __forceinline__ float group_sum(float x) {
  auto dpp = [](float v, auto ctrl) {
    return __uint_as_float(
        (uint32_t)__builtin_amdgcn_mov_dpp((int)__float_as_uint(v), decltype(ctrl)::value, 0xf, 0xf, true));
  };
  x += dpp(x, std::integral_constant<int, 0xb1>{});   // quad_perm 1 0 3 2
  x += dpp(x, std::integral_constant<int, 0x4e>{});   // quad_perm 2 3 0 1
  x += dpp(x, std::integral_constant<int, 0x141>{});  // row_half_mirror
  if constexpr (W >= 16) x += dpp(x, std::integral_constant<int, 0x140>{});  // row_mirror
  if constexpr (W >= 32) {
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  }
  if constexpr (W >= 64) {
    const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  }
  return x;
}

// Sums over the TPR threads of a row. Those of several waves go through `red`,
// whose halves consecutive calls use in turn.
template <int TPR, int THREADS, int K> struct RowSum {
  static constexpr int W = TPR > 64 ? TPR / 64 : 1, ROWS = THREADS / TPR;
  float (*red)[ROWS][W][K];  // [2]
  int turn = 0;
  __device__ __forceinline__ void operator()(float (&x)[K]) {
#pragma unroll
    for (int k = 0; k < K; ++k) x[k] = group_sum<(TPR < 64 ? TPR : 64)>(x[k]);
    if constexpr (W > 1) {
      const int sub = threadIdx.x / TPR, w = (threadIdx.x % TPR) >> 6;
      float(*r)[K] = red[turn][sub];
      turn ^= 1;
      if ((threadIdx.x & 63) == 0) {
#pragma unroll
        for (int k = 0; k < K; ++k) r[w][k] = x[k];
      }
      __syncthreads();
#pragma unroll
      for (int k = 0; k < K; ++k) {
        float y = r[0][k];
#pragma unroll
        for (int i = 1; i < W; ++i) y += r[i][k];
        x[k] = y;
      }
    }
  }
};

// U rows per thread group, all loaded before the first is reduced; a workgroup
// does not go on to others: nothing would wait for its stores, but the next loads
// would (loads and stores share one counter).
template <int TPR> constexpr int fwd_threads = TPR > NORM_FWD_THREADS ? TPR : NORM_FWD_THREADS;
// Workgroups along x: a dimension of a launch has less than 2^32 threads.
constexpr int NORM_GRID_X = 1 << 21;
inline dim3 norm_grid(int blocks) {
  return dim3((unsigned)std::min(blocks, NORM_GRID_X), (unsigned)((blocks + NORM_GRID_X - 1) / NORM_GRID_X));
}
template <int TPR> constexpr int bwd_threads = TPR > NORM_BWD_THREADS ? TPR : NORM_BWD_THREADS;
template <typename T, int VE, int TPR, int P, int U>
__global__ void __launch_bounds__(fwd_threads<TPR>) norm_fwd_kernel(NormArgs a) {
  using Sum = RowSum<TPR, fwd_threads<TPR>, 1>;
  constexpr int RPB = Sum::ROWS;
  __shared__ float red[2][Sum::ROWS][Sum::W][1];
  Sum row_sum{red};
  const int block = blockIdx.y * NORM_GRID_X + blockIdx.x;
  const int t = threadIdx.x % TPR, r0 = block * RPB * U + threadIdx.x / TPR;
  RowRegs<T, VE, TPR, P> x[U];
#pragma unroll
  for (int u = 0; u < U; ++u)
    x[u].load((const T *)a.x + row_at(a, a.sx, min(r0 + u * RPB, a.rows - 1)), a.C, t);
  float w[P][VE], b[P][VE];
  weights<VE, TPR, P>(w, a.w, a.w16, a.C, t, 1.f);
  weights<VE, TPR, P>(b, a.b, a.w16, a.C, t, 0.f);
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int r = r0 + u * RPB;
    float v[P][VE], sum[1] = {0.f};
#pragma unroll
    for (int j = 0; j < P; ++j) {
      x[u].get(v[j], j, a.C, t);
#pragma unroll
      for (int e = 0; e < VE; ++e) sum[0] += v[j][e];
    }
    row_sum(sum);
    const float mean = sum[0] * a.invC;
    float var[1] = {0.f};
#pragma unroll
    for (int j = 0; j < P; ++j) {
      const bool in = (j * TPR + t) * VE < a.C;
#pragma unroll
      for (int e = 0; e < VE; ++e) {
        v[j][e] = in ? v[j][e] - mean : 0.f;
        var[0] = __builtin_fmaf(v[j][e], v[j][e], var[0]);
      }
    }
    row_sum(var);
    const float rstd = 1.f / sqrtf(var[0] * a.invC + a.eps);
    if (r < a.rows) {
      T *y = (T *)a.y + row_at(a, a.sy, r);
#pragma unroll
      for (int j = 0; j < P; ++j) {
        const int i = (j * TPR + t) * VE;
        float o[VE];
#pragma unroll
        for (int e = 0; e < VE; ++e) o[e] = __builtin_fmaf(v[j][e] * rstd, w[j][e], b[j][e]);
        if (i < a.C) put<T, VE>(y + i, o);
      }
      if (t == 0 && (a.mean || a.rstd)) {
        const int64_t at = row_at(a, a.stat, r);
        if (a.mean) a.mean[at] = mean;
        if (a.rstd) a.rstd[at] = rstd;
      }
    }
  }
}

// WG: are dw and db wanted? A workgroup goes over rows gridDim.x * RPB apart and
// keeps its columns' sums.
template <typename T, int VE, int TPR, int P, bool WG>
__global__ void __launch_bounds__(bwd_threads<TPR>) norm_bwd_kernel(NormArgs a) {
  using Sum = RowSum<TPR, bwd_threads<TPR>, 2>;
  constexpr int RPB = Sum::ROWS;
  __shared__ float red[2][Sum::ROWS][Sum::W][2];
  __shared__ float sums[WG ? bwd_threads<TPR> * VE : 1];
  Sum row_sum{red};
  const int t = threadIdx.x % TPR, sub = threadIdx.x / TPR;
  float w[P][VE], dw[P][VE], db[P][VE];
  weights<VE, TPR, P>(w, a.w, a.w16, a.C, t, 1.f);
#pragma unroll
  for (int j = 0; j < P; ++j)
#pragma unroll
    for (int e = 0; e < VE; ++e) {
      dw[j][e] = 0.f;
      db[j][e] = 0.f;
    }
  // the loop is uniform over the workgroup: rows past the last weigh nothing
  for (int r0 = blockIdx.x * RPB; r0 < a.rows; r0 += gridDim.x * RPB) {
    const int r = r0 + sub, rc = min(r, a.rows - 1);
    RowRegs<T, VE, TPR, P> x, y;
    x.load((const T *)a.x + row_at(a, a.sx, rc), a.C, t);
    y.load((const T *)a.dy + row_at(a, a.sdy, rc), a.C, t);
    const int64_t at = row_at(a, a.stat, rc);
    const float mean = a.mean_in[at], rstd = a.rstd_in[at];
    // lanes past the last row hold its dy, or, with dx in dy's place, what its own
    // lanes have written there by now
    const bool on = r < a.rows;
    float sm[2] = {0.f, 0.f};
#pragma unroll
    for (int j = 0; j < P; ++j) {
      float xv[VE], yv[VE];
      x.c[j].get(xv);
      y.get(yv, j, a.C, t);
#pragma unroll
      for (int e = 0; e < VE; ++e) {
        const float h = (xv[e] - mean) * rstd, gw = yv[e] * w[j][e];
        // elements past the row have dy = 0
        sm[0] += gw;
        sm[1] = __builtin_fmaf(gw, h, sm[1]);
        if (WG) {
          dw[j][e] = on ? __builtin_fmaf(yv[e], h, dw[j][e]) : dw[j][e];
          db[j][e] = on ? db[j][e] + yv[e] : db[j][e];
        }
      }
    }
    if (!a.dx) continue;
    row_sum(sm);
    const float s1 = sm[0] * a.invC, s2 = sm[1] * a.invC;
    if (r < a.rows) {
      T *dx = (T *)a.dx + row_at(a, a.sdx, r);
#pragma unroll
      for (int j = 0; j < P; ++j) {
        const int i = (j * TPR + t) * VE;
        float xv[VE], yv[VE];
        x.c[j].get(xv);
        y.c[j].get(yv);
#pragma unroll
        for (int e = 0; e < VE; ++e) {
          const float h = (xv[e] - mean) * rstd;
          yv[e] = rstd * (__builtin_fmaf(yv[e], w[j][e], -s1) - h * s2);
        }
        if (i < a.C) put<T, VE>(dx + i, yv);
      }
    }
  }
  if constexpr (WG) {
    // the workgroup's sums, its rows' parts in a fixed order
    float *part = a.part + (int64_t)blockIdx.x * 2 * a.C;
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int j = 0; j < P; ++j) {
        __syncthreads();
#pragma unroll
        for (int e = 0; e < VE; ++e) sums[threadIdx.x * VE + e] = k ? db[j][e] : dw[j][e];
        __syncthreads();
        for (int c = threadIdx.x; c < TPR * VE; c += bwd_threads<TPR>) {
          const int i = j * TPR * VE + c;
          if (i < a.C) {
            float y = 0.f;
#pragma unroll 8
            for (int q = 0; q < RPB; ++q) y += sums[q * TPR * VE + c];
            part[k * a.C + i] = y;
          }
        }
      }
  }
}

// dw and db: the workgroups' partial sums, sixteen interleaved sequences per
// column added in a fixed order.
__global__ void __launch_bounds__(512) norm_sum_kernel(NormArgs a, int parts) {
  __shared__ float s[16][33];
  const int c = threadIdx.x & 31, q = threadIdx.x >> 5, i = blockIdx.x * 32 + c;
  float y = 0.f;
  if (i < 2 * a.C) {
#pragma unroll 16
    for (int p = q; p < parts; p += 16) y += a.part[(int64_t)p * 2 * a.C + i];
  }
  s[q][c] = y;
  __syncthreads();
  if (q != 0 || i >= 2 * a.C) return;
  y = 0.f;
#pragma unroll
  for (int k = 0; k < 16; ++k) y += s[k][c];
  void *out = i < a.C ? a.dw : a.db;
  const int at = i < a.C ? i : i - a.C;
  if (!out) return;
  if (a.w16)
    ((bf16_t *)out)[at] = from_f32<bf16_t>(y);
  else
    ((float *)out)[at] = y;
}

// Rows too wide for registers: a workgroup per row, which reads it once per pass.
__device__ __forceinline__ float block_sum(float x, float *red) {
  x = wave_sum(x);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = x;
  __syncthreads();
  float y = 0.f;
  for (int i = 0; i < (int)blockDim.x >> 6; ++i) y += red[i];
  return y;
}
__device__ __forceinline__ float weight_at(const void *w, bool w16, int i, float missing) {
  return !w ? missing : w16 ? to_f32(((const bf16_t *)w)[i]) : ((const float *)w)[i];
}
template <typename T> __global__ void __launch_bounds__(512) norm_fwd_wide_kernel(NormArgs a) {
  __shared__ float red[8];
  for (int r = blockIdx.x; r < a.rows; r += gridDim.x) {
    const T *x = (const T *)a.x + row_at(a, a.sx, r);
    T *y = (T *)a.y + row_at(a, a.sy, r);
    float s = 0.f;
    for (int i = threadIdx.x; i < a.C; i += blockDim.x) s += to_f32(x[i]);
    const float mean = block_sum(s, red) * a.invC;
    s = 0.f;
    for (int i = threadIdx.x; i < a.C; i += blockDim.x) {
      const float d = to_f32(x[i]) - mean;
      s += d * d;
    }
    const float rstd = 1.f / sqrtf(block_sum(s, red) * a.invC + a.eps);
    for (int i = threadIdx.x; i < a.C; i += blockDim.x)
      y[i] = from_f32<T>(__builtin_fmaf((to_f32(x[i]) - mean) * rstd, weight_at(a.w, a.w16, i, 1.f),
                                        weight_at(a.b, a.w16, i, 0.f)));
    if (threadIdx.x == 0) {
      const int64_t at = row_at(a, a.stat, r);
      if (a.mean) a.mean[at] = mean;
      if (a.rstd) a.rstd[at] = rstd;
    }
  }
}
template <typename T> __global__ void __launch_bounds__(512) norm_dx_wide_kernel(NormArgs a) {
  __shared__ float red[8];
  for (int r = blockIdx.x; r < a.rows; r += gridDim.x) {
    const T *x = (const T *)a.x + row_at(a, a.sx, r), *dy = (const T *)a.dy + row_at(a, a.sdy, r);
    T *dx = (T *)a.dx + row_at(a, a.sdx, r);
    const int64_t at = row_at(a, a.stat, r);
    const float mean = a.mean_in[at], rstd = a.rstd_in[at];
    float s1 = 0.f, s2 = 0.f;
    for (int i = threadIdx.x; i < a.C; i += blockDim.x) {
      const float gw = to_f32(dy[i]) * weight_at(a.w, a.w16, i, 1.f);
      s1 += gw;
      s2 = __builtin_fmaf(gw, (to_f32(x[i]) - mean) * rstd, s2);
    }
    s1 = block_sum(s1, red) * a.invC;
    s2 = block_sum(s2, red) * a.invC;
    for (int i = threadIdx.x; i < a.C; i += blockDim.x) {
      const float gw = to_f32(dy[i]) * weight_at(a.w, a.w16, i, 1.f);
      dx[i] = from_f32<T>(rstd * (gw - s1 - (to_f32(x[i]) - mean) * rstd * s2));
    }
  }
}
// Workgroup (i, p): columns 512 i .., every gridDim.y-th row from p on.
template <typename T> __global__ void __launch_bounds__(512) norm_dw_wide_kernel(NormArgs a) {
  const int i = blockIdx.x * 512 + threadIdx.x;
  if (i >= a.C) return;
  float dw = 0.f, db = 0.f;
#pragma unroll 4
  for (int r = blockIdx.y; r < a.rows; r += gridDim.y) {
    const int64_t at = row_at(a, a.stat, r);
    const float x = to_f32(((const T *)a.x)[row_at(a, a.sx, r) + i]);
    const float dy = to_f32(((const T *)a.dy)[row_at(a, a.sdy, r) + i]);
    dw = __builtin_fmaf(dy, (x - a.mean_in[at]) * a.rstd_in[at], dw);
    db += dy;
  }
  float *part = a.part + (int64_t)blockIdx.y * 2 * a.C;
  part[i] = dw;
  part[a.C + i] = db;
}

// The largest power of two up to 16 bytes, in elements, that divides the width and
// every row's place.
int row_align(const mita_norm_cfg_t &c, const Strided &s, const void *p, int align) {
  if (!p) return align;
  auto divides = [&](int64_t v) { return c.C % v == 0 && (uintptr_t)p % (v * elem_bytes(c)) == 0 &&
                                         (s.n[0] == 1 || s.s[0] % v == 0) && (s.n[1] == 1 || s.s[1] % v == 0) &&
                                         (s.n[2] == 1 || s.s[2] % v == 0); };
  while (align > 1 && !divides(align)) align /= 2;
  return align;
}

// The arguments of a call on `tensors` strided tensors, whose distances go to
// `to`; the statistics come last. The walk goes over the dimensions in the order of
// the first tensor's distances.
NormArgs norm_args(const mita_norm_cfg_t &c, const Strided *t, int tensors, NormRows NormArgs::*const *to) {
  NormArgs a{};
  const int64_t stat[3] = {(int64_t)c.n[1] * c.n[2], c.n[2], 1};
  int order[3] = {0, 1, 2};  // dimensions of one row outermost
  std::stable_sort(order, order + 3, [&](int x, int y) {
    if ((c.n[x] == 1) != (c.n[y] == 1)) return c.n[x] == 1;
    return c.n[x] > 1 && t[0].s[x] > t[0].s[y];
  });
  int64_t n[3];
  for (int k = 0; k < 3; ++k) n[k] = c.n[order[k]];
  for (int i = 0; i <= tensors; ++i) {
    NormRows &r = i < tensors ? a.*to[i] : a.stat;
    for (int k = 0; k < 3; ++k) r.s[k] = n[k] == 1 ? 0 : i < tensors ? t[i].s[order[k]] : stat[order[k]];
    r.flat = (n[1] == 1 || r.s[1] == n[2] * r.s[2]) && (n[0] == 1 || r.s[0] == n[1] * n[2] * r.s[2]);
  }
  auto magic = [](int64_t d, uint32_t &m, int &h) {
    int l = 0;
    while (((int64_t)1 << l) < d) ++l;
    h = l - 1;
    m = d == 1 ? 0u : (uint32_t)(((uint64_t)1 << (31 + l)) / (uint64_t)d + 1);
  };
  a.n1 = (int)n[1];
  a.n2 = (int)n[2];
  magic(n[1], a.m1, a.h1);
  magic(n[2], a.m2, a.h2);
  a.rows = (int)norm_rows(c);
  a.C = c.C;
  a.w16 = c.wdtype == MITA_BF16;
  a.eps = c.eps;
  a.invC = 1.f / (float)c.C;
  return a;
}

template <typename T, int VE, int TPR, int P> hipError_t fwd_p(const NormArgs &a, hipStream_t st) {
  // as many rows per thread as give four pieces, once that leaves eight workgroups per CU
  constexpr int N = fwd_threads<TPR>, RPB = N / TPR, U = P >= 4 ? 1 : P >= 2 ? 2 : 4;
  if (U > 1 && a.rows >= RPB * U * 8 * CUS)
    norm_fwd_kernel<T, VE, TPR, P, U><<<norm_grid((a.rows + RPB * U - 1) / (RPB * U)), N, 0, st>>>(a);
  else
    norm_fwd_kernel<T, VE, TPR, P, 1><<<norm_grid((a.rows + RPB - 1) / RPB), N, 0, st>>>(a);
  return launched("norm_fwd_kernel", st);
}
template <typename T, int VE, int TPR, int P> hipError_t bwd_p(const NormArgs &a, int blocks, hipStream_t st) {
  if (a.dw || a.db)
    norm_bwd_kernel<T, VE, TPR, P, true><<<dim3((unsigned)blocks), bwd_threads<TPR>, 0, st>>>(a);
  else
    norm_bwd_kernel<T, VE, TPR, P, false><<<dim3((unsigned)blocks), bwd_threads<TPR>, 0, st>>>(a);
  return launched("norm_bwd_kernel", st);
}

// f.run<VE, TPR, P>() for the plan's geometry
template <int VE, typename F> hipError_t with_plan_odd(const NormPlan &p, F &f) {
  if (p.tpr == 64) {
    if (p.p <= 4) return p.p == 2 ? f.template run<VE, 64, 2>() : f.template run<VE, 64, 4>();
    return p.p == 6 ? f.template run<VE, 64, 6>() : f.template run<VE, 64, 8>();
  }
  if (p.tpr == 256) return p.p == 4 ? f.template run<VE, 256, 4>() : f.template run<VE, 256, 8>();
  return f.template run<VE, 1024, 8>();
}
template <typename T, typename F> hipError_t with_plan(const NormPlan &p, F &&f) {
  constexpr int V = 16 / (int)sizeof(T);
  if (p.ve == V) {
    if (p.tpr == 8) return f.template run<V, 8, 1>();
    if (p.tpr == 16) return p.p == 1 ? f.template run<V, 16, 1>() : f.template run<V, 16, 3>();
    if (p.tpr == 32) return p.p == 1 ? f.template run<V, 32, 1>() : f.template run<V, 32, 3>();
    if (p.tpr == 64) {
      if (p.p == 1) return f.template run<V, 64, 1>();
      if (p.p == 2) return f.template run<V, 64, 2>();
      if (p.p == 3) return f.template run<V, 64, 3>();
      return f.template run<V, 64, 4>();
    }
    if (p.tpr == 256) return p.p == 2 ? f.template run<V, 256, 2>() : f.template run<V, 256, 4>();
    return f.template run<V, 1024, 2>();
  }
  return p.ve == 2 ? with_plan_odd<2>(p, f) : with_plan_odd<1>(p, f);
}
template <typename T> struct RunFwd {
  const NormArgs &a;
  hipStream_t st;
  template <int VE, int TPR, int P> hipError_t run() { return fwd_p<T, VE, TPR, P>(a, st); }
};
template <typename T> struct RunBwd {
  const NormArgs &a;
  int blocks;
  hipStream_t st;
  template <int VE, int TPR, int P> hipError_t run() { return bwd_p<T, VE, TPR, P>(a, blocks, st); }
};

template <typename T> hipError_t forward_t(const NormArgs &a, const NormPlan &p, hipStream_t st) {
  if (p.p) return with_plan<T>(p, RunFwd<T>{a, st});
  norm_fwd_wide_kernel<T><<<dim3((unsigned)std::min(a.rows, 4 * CUS)), 512, 0, st>>>(a);
  return launched("norm_fwd_wide_kernel", st);
}
template <typename T> hipError_t backward_t(const NormArgs &a, const NormPlan &p, int blocks, hipStream_t st) {
  const bool wg = a.dw || a.db;
  hipError_t e = hipSuccess;
  if (p.p) {
    e = with_plan<T>(p, RunBwd<T>{a, blocks, st});
    if (e != hipSuccess) return e;
  } else {
    if (wg) {  // before dx, which may take dy's place
      norm_dw_wide_kernel<T><<<dim3((unsigned)((a.C + 511) / 512), (unsigned)blocks), 512, 0, st>>>(a);
      e = launched("norm_dw_wide_kernel", st);
      if (e != hipSuccess) return e;
    }
    if (a.dx) {
      norm_dx_wide_kernel<T><<<dim3((unsigned)std::min(a.rows, 4 * CUS)), 512, 0, st>>>(a);
      e = launched("norm_dx_wide_kernel", st);
      if (e != hipSuccess) return e;
    }
  }
  if (!wg) return e;
  norm_sum_kernel<<<dim3((unsigned)((2 * a.C + 31) / 32)), 512, 0, st>>>(a, blocks);
  return launched("norm_sum_kernel", st);
}

}  // namespace

hipError_t launch_norm_forward(const mita_norm_cfg_t &c, const void *x, const void *w, const void *b, void *y,
                               float *mean, float *rstd, hipStream_t st) {
  const Strided t[2] = {strided_rows(c, c.x), strided_rows(c, c.y)};
  NormRows NormArgs::*const to[2] = {&NormArgs::sx, &NormArgs::sy};
  NormArgs a = norm_args(c, t, 2, to);
  a.x = x;
  a.w = w;
  a.b = b;
  a.y = y;
  a.mean = mean;
  a.rstd = rstd;
  const NormPlan p = norm_plan(c, row_align(c, t[1], y, row_align(c, t[0], x, 16 / (int)elem_bytes(c))));
  return c.dtype == MITA_F32 ? forward_t<float>(a, p, st) : forward_t<bf16_t>(a, p, st);
}

hipError_t launch_norm_backward(const mita_norm_cfg_t &c, const void *x, const void *w, const float *mean,
                                const float *rstd, const void *dy, void *dx, void *dw, void *db, void *ws,
                                hipStream_t st) {
  const Strided t[3] = {strided_rows(c, c.x), strided_rows(c, c.dy), strided_rows(c, c.dx)};
  NormRows NormArgs::*const to[3] = {&NormArgs::sx, &NormArgs::sdy, &NormArgs::sdx};
  NormArgs a = norm_args(c, t, 3, to);
  a.x = x;
  a.w = w;
  a.mean_in = mean;
  a.rstd_in = rstd;
  a.dy = dy;
  a.dx = dx;
  a.dw = dw;
  a.db = db;
  a.part = (float *)ws;
  const NormPlan p = norm_plan(c, row_align(c, t[2], dx, row_align(c, t[1], dy, row_align(c, t[0], x, 16 / (int)elem_bytes(c)))));
  const int blocks = norm_bwd_blocks(c, p);
  return c.dtype == MITA_F32 ? backward_t<float>(a, p, blocks, st) : backward_t<bf16_t>(a, p, blocks, st);
}

}  // namespace mita
