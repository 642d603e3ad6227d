// rows.hpp - rows of strided tensors held in the registers of the threads that
// share them: the walk over the rows, pieces of 16 bytes (or fewer where rows
// are not aligned so), sums over a row's threads. For the kernels of the norms.
#pragma once
#include <algorithm>

#include "cdna4.hpp"
#include "layer_check.hpp"

namespace mita {

struct RowPlaces {
  int64_t s[3];  // distances in elements, in the order of the walk
  bool flat;     // rows of the walk are s[2] apart all over
};

// Rows are walked in the order of the first tensor in memory, dimensions 0, 1, 2 from
// the outside in.
struct RowWalk {
  int rows, n1, n2, C;  // C: elements of a row
  uint32_t m1, m2;  // for quotients by n1 and n2
  int h1, h2;
};

// r / n for r < 2^31 with l = ceil(log2 n), m = 2^(31 + l) / n + 1 (floored, below
// 2^32 + 1 and so below 2^32 for n > 1), h = l - 1: r m exceeds 2^(31 + l) r / n by
// at most r < 2^31, less than a step of 1 / n. n = 1: h < 0.
__device__ __forceinline__ int quotient(int r, uint32_t m, int h) { return h < 0 ? r : (int)(__umulhi((uint32_t)r, m) >> h); }

__device__ __forceinline__ int64_t row_at(const RowWalk &a, const RowPlaces &s, int r) {
  if (s.flat) return (int64_t)r * s.s[2];
  const int t = quotient(r, a.m2, a.h2), i2 = r - t * a.n2, i0 = quotient(t, a.m1, a.h1), i1 = t - i0 * a.n1;
  return i0 * s.s[0] + i1 * s.s[1] + i2 * s.s[2];
}

// The pieces of a row that one thread holds: piece j is elements (j TPR + t) VE ..
template <typename T, int VE> struct Piece;
template <typename T> struct Piece<T, 16 / sizeof(T)> {
  uint4 v;
  __device__ __forceinline__ void load(const T *p) { v = *reinterpret_cast<const uint4 *>(p); }
  // of tensors that caches do not keep until they are read again
  __device__ __forceinline__ void load_once(const T *p) {
    typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
    v = __builtin_bit_cast(uint4, __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(p)));
  }
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
  template <bool ONCE = false> __device__ __forceinline__ void load(const T *row, int C, int t) {
#pragma unroll
    for (int j = 0; j < P; ++j) {
      const T *p = row + min((j * TPR + t) * VE, C - VE);
      if constexpr (ONCE)
        c[j].load_once(p);
      else
        c[j].load(p);
    }
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

// The largest of x over the lanes of a group of W, the same in each (NaN is passed over).
template <int W> __device__ __forceinline__ float group_max(float x) {
  auto dpp = [](float v, auto ctrl) {
    return __uint_as_float(
        (uint32_t)__builtin_amdgcn_mov_dpp((int)__float_as_uint(v), decltype(ctrl)::value, 0xf, 0xf, true));
  };
  x = fmaxf(x, dpp(x, std::integral_constant<int, 0xb1>{}));
  x = fmaxf(x, dpp(x, std::integral_constant<int, 0x4e>{}));
  x = fmaxf(x, dpp(x, std::integral_constant<int, 0x141>{}));
  if constexpr (W >= 16) x = fmaxf(x, dpp(x, std::integral_constant<int, 0x140>{}));
  if constexpr (W >= 32) {
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  }
  if constexpr (W >= 64) {
    const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
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
// Workgroups along x: a dimension of a launch has less than 2^32 threads.
constexpr int ROWS_GRID_X = 1 << 21;
inline dim3 rows_grid(int blocks) {
  return dim3((unsigned)std::min(blocks, ROWS_GRID_X), (unsigned)((blocks + ROWS_GRID_X - 1) / ROWS_GRID_X));
}
// The largest power of two up to 16 bytes, in elements, that divides the width and
// every row's place (elements of so many bytes; no tensor: as it was).
inline int row_align(const Strided &s, size_t bytes, const void *p, int align) {
  if (!p) return align;
  auto divides = [&](int64_t v) { return s.len % v == 0 && (uintptr_t)p % (v * bytes) == 0 &&
                                         (s.n[0] == 1 || s.s[0] % v == 0) && (s.n[1] == 1 || s.s[1] % v == 0) &&
                                         (s.n[2] == 1 || s.s[2] % v == 0); };
  while (align > 1 && !divides(align)) align /= 2;
  return align;
}

// The walk over the rows of t[0] and the places of every tensor's rows; those of the
// rows' statistics (contiguous) come last.
inline RowWalk row_walk(const Strided *t, int tensors, RowPlaces *places) {
  RowWalk a{};
  const int64_t(&c)[3] = t[0].n;
  const int64_t stat[3] = {c[1] * c[2], c[2], 1};
  int order[3] = {0, 1, 2};  // dimensions of one row outermost
  std::stable_sort(order, order + 3, [&](int x, int y) {
    if ((c[x] == 1) != (c[y] == 1)) return c[x] == 1;
    return c[x] > 1 && t[0].s[x] > t[0].s[y];
  });
  int64_t n[3];
  for (int k = 0; k < 3; ++k) n[k] = c[order[k]];
  for (int i = 0; i <= tensors; ++i) {
    RowPlaces &r = places[i];
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
  a.rows = (int)(c[0] * c[1] * c[2]);
  a.C = (int)t[0].len;
  return a;
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
}  // namespace mita
