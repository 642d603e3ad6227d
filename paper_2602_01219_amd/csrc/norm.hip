// norm.hip - layer norm of rows and its gradients.
//
// Forward: y = (x - mean) rstd w + b. Backward, with h = (x - mean) rstd and
// g = dy w: dx = rstd (g - mean(g) - h mean(g h)), dw = sum dy h, db = sum dy.
// Both are bound by HBM: a row is read once into registers, its sums go across
// the lanes that share it, and it is written once; the next row's loads are
// issued before the current row is reduced. The variance is summed about the
// mean from the registers (a one-pass sum of squares cancels where the mean is
// large). In the backward each lane keeps the sums of dw and db of its own
// columns over all rows its workgroup takes; one partial sum per workgroup goes
// to memory, and a second launch adds them in a fixed order.
#include "cdna4.hpp"
#include "kernels.hpp"
#include "layer_check.hpp"

namespace mita {

namespace {

struct NormRows {
  int64_t s[3];  // distances in elements
};
struct NormArgs {
  const void *x, *dy, *w, *b;
  void *y, *dx, *dw, *db;
  const float *mean_in, *rstd_in;
  float *mean, *rstd, *part;
  NormRows sx, sy, sdy, sdx;
  int rows, n1, n2, C;
  bool flat, w16;  // flat: rows are s[2] apart all over; w16: weights in bf16
  float eps, invC;
};

__device__ __forceinline__ int64_t row_at(const NormArgs &a, const NormRows &s, int r) {
  if (a.flat) return (int64_t)r * s.s[2];
  const int i2 = r % a.n2, t = r / a.n2, i1 = t % a.n1, i0 = t / a.n1;
  return i0 * s.s[0] + i1 * s.s[1] + i2 * s.s[2];
}

// The pieces of a row that one thread holds: piece j is elements (j TPR + t) VE ..
template <typename T, int VE> struct Piece;
template <typename T> struct Piece<T, 16 / sizeof(T)> {
  uint4 v;
  __device__ __forceinline__ void zero() { v = make_uint4(0, 0, 0, 0); }
  __device__ __forceinline__ void load(const T *p) { v = *reinterpret_cast<const uint4 *>(p); }
  __device__ __forceinline__ void get(float *f) const { unpack16(v, f, (const T *)nullptr); }
};
template <typename T> struct Piece<T, 1> {
  T v;
  __device__ __forceinline__ void zero() { v = from_f32<T>(0.f); }
  __device__ __forceinline__ void load(const T *p) { v = *p; }
  __device__ __forceinline__ void get(float *f) const { f[0] = to_f32(v); }
};
template <typename T, int VE> __device__ __forceinline__ void put(T *p, const float *f) {
  if constexpr (VE == 1) {
    *p = from_f32<T>(f[0]);
  } else if constexpr (sizeof(T) == 4) {
    *reinterpret_cast<float4 *>(p) = make_float4(f[0], f[1], f[2], f[3]);
  } else {
    *reinterpret_cast<uint4 *>(p) = make_uint4(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]),
                                               pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7]));
  }
}

template <typename T, int VE, int TPR, int P> struct RowRegs {
  Piece<T, VE> c[P];
  __device__ __forceinline__ void load(const void *base, int64_t at, int C, int t, bool ok) {
#pragma unroll
    for (int j = 0; j < P; ++j) {
      const int i = (j * TPR + t) * VE;
      if (ok && i < C)
        c[j].load((const T *)base + at + i);
      else
        c[j].zero();
    }
  }
};

// VE weights from column i on (`missing` where there are none).
template <int VE> __device__ __forceinline__ void weights(float *f, const void *w, bool w16, int i, int C, float missing) {
#pragma unroll
  for (int e = 0; e < VE; ++e) f[e] = missing;
  if (!w || i >= C) return;
#pragma unroll
  for (int e = 0; e < VE; ++e) f[e] = w16 ? to_f32(((const bf16_t *)w)[i + e]) : ((const float *)w)[i + e];
}

// Sum over the TPR threads of a row (the same in all of them). `red` is used in
// turn by consecutive calls of a workgroup that shares a row.
template <int TPR> __device__ __forceinline__ void row_sum2(float &x, float &y, float2 (*red)[4], int &turn) {
  constexpr int W = TPR < 64 ? TPR : 64;
#pragma unroll
  for (int o = W / 2; o > 0; o >>= 1) {
    x += __shfl_xor(x, o);
    y += __shfl_xor(y, o);
  }
  if constexpr (TPR > 64) {
    const int sub = (threadIdx.x / TPR), w = (threadIdx.x % TPR) >> 6;
    float2(*r)[4] = red + 4 * turn;
    turn ^= 1;
    if ((threadIdx.x & 63) == 0) r[sub][w] = make_float2(x, y);
    __syncthreads();
    const float2 p0 = r[sub][0], p1 = r[sub][1], p2 = r[sub][2], p3 = r[sub][3];
    x = (p0.x + p1.x) + (p2.x + p3.x);
    y = (p0.y + p1.y) + (p2.y + p3.y);
  }
}

template <typename T, int VE, int TPR, int P>
__global__ void __launch_bounds__(NORM_FWD_THREADS) norm_fwd_kernel(NormArgs a) {
  constexpr int RPB = NORM_FWD_THREADS / TPR;
  __shared__ float2 red[8][4];
  int turn = 0;
  const int t = threadIdx.x % TPR, sub = threadIdx.x / TPR;
  float w[P][VE], b[P][VE];
#pragma unroll
  for (int j = 0; j < P; ++j) {
    weights<VE>(w[j], a.w, a.w16, (j * TPR + t) * VE, a.C, 1.f);
    weights<VE>(b[j], a.b, a.w16, (j * TPR + t) * VE, a.C, 0.f);
  }
  RowRegs<T, VE, TPR, P> next;
  int r = blockIdx.x * RPB + sub;
  next.load(a.x, row_at(a, a.sx, min(r, a.rows - 1)), a.C, t, r < a.rows);
  // the loop is uniform over the workgroup: rows past the last are not written
  for (int r0 = blockIdx.x * RPB; r0 < a.rows; r0 += gridDim.x * RPB) {
    r = r0 + sub;
    const RowRegs<T, VE, TPR, P> cur = next;
    const int rn = r + gridDim.x * RPB;
    if (r0 + gridDim.x * RPB < a.rows) next.load(a.x, row_at(a, a.sx, min(rn, a.rows - 1)), a.C, t, rn < a.rows);
    float v[P][VE], sum = 0.f, none = 0.f;
#pragma unroll
    for (int j = 0; j < P; ++j) {
      cur.c[j].get(v[j]);
#pragma unroll
      for (int e = 0; e < VE; ++e) sum += v[j][e];
    }
    row_sum2<TPR>(sum, none, red, turn);
    const float mean = sum * a.invC;
    float var = 0.f;
    none = 0.f;
#pragma unroll
    for (int j = 0; j < P; ++j) {
      const bool in = (j * TPR + t) * VE < a.C;
#pragma unroll
      for (int e = 0; e < VE; ++e) {
        v[j][e] = in ? v[j][e] - mean : 0.f;
        var += v[j][e] * v[j][e];
      }
    }
    row_sum2<TPR>(var, none, red, turn);
    const float rstd = 1.f / sqrtf(var * a.invC + a.eps);
    if (r < a.rows) {
      const int64_t at = row_at(a, a.sy, r);
#pragma unroll
      for (int j = 0; j < P; ++j) {
        const int i = (j * TPR + t) * VE;
        float y[VE];
#pragma unroll
        for (int e = 0; e < VE; ++e) y[e] = __builtin_fmaf(v[j][e] * rstd, w[j][e], b[j][e]);
        if (i < a.C) put<T, VE>((T *)a.y + at + i, y);
      }
      if (t == 0) {
        if (a.mean) a.mean[r] = mean;
        if (a.rstd) a.rstd[r] = rstd;
      }
    }
  }
}

// WG: are dw and db wanted?
template <typename T, int VE, int TPR, int P, bool WG>
__global__ void __launch_bounds__(NORM_BWD_THREADS) norm_bwd_kernel(NormArgs a) {
  constexpr int RPB = NORM_BWD_THREADS / TPR;
  __shared__ float2 red[8][4];
  __shared__ float sums[WG ? NORM_BWD_THREADS * VE : 1];
  int turn = 0;
  const int t = threadIdx.x % TPR, sub = threadIdx.x / TPR;
  float w[P][VE], dw[P][VE], db[P][VE];
#pragma unroll
  for (int j = 0; j < P; ++j) {
    weights<VE>(w[j], a.w, a.w16, (j * TPR + t) * VE, a.C, 1.f);
#pragma unroll
    for (int e = 0; e < VE; ++e) {
      dw[j][e] = 0.f;
      db[j][e] = 0.f;
    }
  }
  RowRegs<T, VE, TPR, P> nx, ny;
  float nm, nr;
  auto fetch = [&](int r) {
    const int rc = min(r, a.rows - 1);
    nx.load(a.x, row_at(a, a.sx, rc), a.C, t, r < a.rows);
    ny.load(a.dy, row_at(a, a.sdy, rc), a.C, t, r < a.rows);
    nm = a.mean_in[rc];
    nr = a.rstd_in[rc];
  };
  fetch(blockIdx.x * RPB + sub);
  for (int r0 = blockIdx.x * RPB; r0 < a.rows; r0 += gridDim.x * RPB) {
    const int r = r0 + sub;
    const RowRegs<T, VE, TPR, P> cx = nx, cy = ny;
    const float mean = nm, rstd = nr;
    if (r0 + gridDim.x * RPB < a.rows) fetch(r + gridDim.x * RPB);
    float s1 = 0.f, s2 = 0.f;
#pragma unroll
    for (int j = 0; j < P; ++j) {
      float xv[VE], yv[VE];
      cx.c[j].get(xv);
      cy.c[j].get(yv);
#pragma unroll
      for (int e = 0; e < VE; ++e) {
        const float h = (xv[e] - mean) * rstd, gw = yv[e] * w[j][e];
        // elements past the row, and rows past the last, have dy = 0
        s1 += gw;
        s2 = __builtin_fmaf(gw, h, s2);
        if (WG) {
          dw[j][e] = __builtin_fmaf(yv[e], h, dw[j][e]);
          db[j][e] += yv[e];
        }
      }
    }
    if (!a.dx) continue;
    row_sum2<TPR>(s1, s2, red, turn);
    s1 *= a.invC;
    s2 *= a.invC;
    if (r < a.rows) {
      const int64_t at = row_at(a, a.sdx, r);
#pragma unroll
      for (int j = 0; j < P; ++j) {
        const int i = (j * TPR + t) * VE;
        float xv[VE], yv[VE];
        cx.c[j].get(xv);
        cy.c[j].get(yv);
#pragma unroll
        for (int e = 0; e < VE; ++e) {
          const float h = (xv[e] - mean) * rstd;
          yv[e] = rstd * (__builtin_fmaf(yv[e], w[j][e], -s1) - h * s2);
        }
        if (i < a.C) put<T, VE>((T *)a.dx + at + i, yv);
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
        for (int c = threadIdx.x; c < TPR * VE; c += NORM_BWD_THREADS) {
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

// dw and db: the workgroups' partial sums, eight interleaved sequences per column
// added in a fixed order.
__global__ void __launch_bounds__(256) norm_sum_kernel(NormArgs a, int parts) {
  __shared__ float s[8][33];
  const int c = threadIdx.x & 31, q = threadIdx.x >> 5, i = blockIdx.x * 32 + c;
  float y = 0.f;
  if (i < 2 * a.C) {
#pragma unroll 8
    for (int p = q; p < parts; p += 8) y += a.part[(int64_t)p * 2 * a.C + i];
  }
  s[q][c] = y;
  __syncthreads();
  if (q != 0 || i >= 2 * a.C) return;
  y = 0.f;
#pragma unroll
  for (int k = 0; k < 8; ++k) y += s[k][c];
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
      if (a.mean) a.mean[r] = mean;
      if (a.rstd) a.rstd[r] = rstd;
    }
  }
}
template <typename T> __global__ void __launch_bounds__(512) norm_dx_wide_kernel(NormArgs a) {
  __shared__ float red[8];
  for (int r = blockIdx.x; r < a.rows; r += gridDim.x) {
    const T *x = (const T *)a.x + row_at(a, a.sx, r), *dy = (const T *)a.dy + row_at(a, a.sdy, r);
    T *dx = (T *)a.dx + row_at(a, a.sdx, r);
    const float mean = a.mean_in[r], rstd = a.rstd_in[r];
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
    const float x = to_f32(((const T *)a.x)[row_at(a, a.sx, r) + i]);
    const float dy = to_f32(((const T *)a.dy)[row_at(a, a.sdy, r) + i]);
    dw = __builtin_fmaf(dy, (x - a.mean_in[r]) * a.rstd_in[r], dw);
    db += dy;
  }
  float *part = a.part + (int64_t)blockIdx.y * 2 * a.C;
  part[i] = dw;
  part[a.C + i] = db;
}

bool row_vectors(const mita_norm_cfg_t &c, const Strided &s, const void *p) {
  const int64_t ve = 16 / (int64_t)elem_bytes(c);
  if (!p) return true;
  if (c.C % ve != 0 || ((uintptr_t)p & 15)) return false;
  for (int i = 0; i < 3; ++i)
    if (s.n[i] > 1 && s.s[i] % ve != 0) return false;
  return true;
}
// rows one distance apart over all dimensions: the distance of row r is r * s[2]
bool flatten(const Strided &s, NormRows &out) {
  for (int i = 0; i < 3; ++i) out.s[i] = s.s[i];
  int64_t d = 0, inner = 1;  // distance of the innermost dimension of more than one row
  bool ok = true;
  for (int i = 2; i >= 0; --i) {
    if (s.n[i] == 1) continue;
    if (inner == 1)
      d = s.s[i];
    else if (s.s[i] != d * inner)
      ok = false;
    inner *= s.n[i];
  }
  if (ok) out.s[2] = d;
  return ok;
}

NormArgs norm_args(const mita_norm_cfg_t &c) {
  NormArgs a{};
  a.rows = (int)norm_rows(c);
  a.n1 = c.n[1];
  a.n2 = c.n[2];
  a.C = c.C;
  a.w16 = c.wdtype == MITA_BF16;
  a.eps = c.eps;
  a.invC = 1.f / (float)c.C;
  return a;
}

template <typename T, int VE, int TPR, int P> hipError_t fwd_p(const NormArgs &a, hipStream_t st) {
  constexpr int RPB = NORM_FWD_THREADS / TPR;
  const int blocks = std::min((a.rows + RPB - 1) / RPB, 8 * CUS);
  norm_fwd_kernel<T, VE, TPR, P><<<dim3((unsigned)blocks), NORM_FWD_THREADS, 0, st>>>(a);
  return launched("norm_fwd_kernel", st);
}
template <typename T, int VE, int TPR, int P> hipError_t bwd_p(const NormArgs &a, int blocks, hipStream_t st) {
  if (a.dw || a.db)
    norm_bwd_kernel<T, VE, TPR, P, true><<<dim3((unsigned)blocks), NORM_BWD_THREADS, 0, st>>>(a);
  else
    norm_bwd_kernel<T, VE, TPR, P, false><<<dim3((unsigned)blocks), NORM_BWD_THREADS, 0, st>>>(a);
  return launched("norm_bwd_kernel", st);
}

// f.run<VE, TPR, P>() for the plan's geometry
template <typename T, typename F> hipError_t with_plan(const NormPlan &p, F &&f) {
  constexpr int V = 16 / (int)sizeof(T);
  if (p.ve > 1) {
    if (p.tpr == 8) return f.template run<V, 8, 1>();
    if (p.tpr == 16) return f.template run<V, 16, 1>();
    if (p.tpr == 32) return f.template run<V, 32, 1>();
    if (p.tpr == 64) {
      if (p.p == 1) return f.template run<V, 64, 1>();
      if (p.p == 2) return f.template run<V, 64, 2>();
      return f.template run<V, 64, 4>();
    }
    if (p.p == 2) return f.template run<V, 256, 2>();
    if (p.p == 4) return f.template run<V, 256, 4>();
    return f.template run<V, 256, 8>();
  }
  if (p.tpr == 64) return p.p == 2 ? f.template run<1, 64, 2>() : f.template run<1, 64, 8>();
  return p.p == 4 ? f.template run<1, 256, 4>() : f.template run<1, 256, 16>();
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
  norm_sum_kernel<<<dim3((unsigned)((2 * a.C + 31) / 32)), 256, 0, st>>>(a, blocks);
  return launched("norm_sum_kernel", st);
}

}  // namespace

hipError_t launch_norm_forward(const mita_norm_cfg_t &c, const void *x, const void *w, const void *b, void *y,
                               float *mean, float *rstd, hipStream_t st) {
  NormArgs a = norm_args(c);
  const Strided sx = strided_rows(c, c.x), sy = strided_rows(c, c.y);
  const bool fx = flatten(sx, a.sx), fy = flatten(sy, a.sy);
  a.flat = fx && fy;
  if (!a.flat) {
    for (int i = 0; i < 3; ++i) {
      a.sx.s[i] = sx.s[i];
      a.sy.s[i] = sy.s[i];
    }
  }
  a.x = x;
  a.w = w;
  a.b = b;
  a.y = y;
  a.mean = mean;
  a.rstd = rstd;
  const NormPlan p = norm_plan(c, row_vectors(c, sx, x) && row_vectors(c, sy, y));
  return c.dtype == MITA_F32 ? forward_t<float>(a, p, st) : forward_t<bf16_t>(a, p, st);
}

hipError_t launch_norm_backward(const mita_norm_cfg_t &c, const void *x, const void *w, const float *mean,
                                const float *rstd, const void *dy, void *dx, void *dw, void *db, void *ws,
                                hipStream_t st) {
  NormArgs a = norm_args(c);
  const Strided sx = strided_rows(c, c.x), sdy = strided_rows(c, c.dy), sdx = strided_rows(c, c.dx);
  const bool fx = flatten(sx, a.sx), fy = flatten(sdy, a.sdy), fd = flatten(sdx, a.sdx);
  a.flat = fx && fy && fd;
  if (!a.flat) {
    for (int i = 0; i < 3; ++i) {
      a.sx.s[i] = sx.s[i];
      a.sdy.s[i] = sdy.s[i];
      a.sdx.s[i] = sdx.s[i];
    }
  }
  a.x = x;
  a.w = w;
  a.mean_in = mean;
  a.rstd_in = rstd;
  a.dy = dy;
  a.dx = dx;
  a.dw = dw;
  a.db = db;
  a.part = (float *)ws;
  const NormPlan p = norm_plan(c, row_vectors(c, sx, x) && row_vectors(c, sdy, dy) && row_vectors(c, sdx, dx));
  const int blocks = norm_bwd_blocks(c, p);
  return c.dtype == MITA_F32 ? backward_t<float>(a, p, blocks, st) : backward_t<bf16_t>(a, p, blocks, st);
}

}  // namespace mita
