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
#include "kernels.hpp"
#include "layer_check.hpp"
#include "rows.hpp"

namespace mita {

namespace {

struct NormTensors {
  const void *x, *dy, *w, *b;
  void *y, *dx, *dw, *db;
  const float *mean_in, *rstd_in;
  float *mean, *rstd, *part;
  RowPlaces sx, sy, sdy, sdx, stat;  // `stat`: of the row's statistics
};
// (the tensors first, and a row's width beside the number of rows, as in the RMS norm: with
// others between them the instructions read their arguments at other places, and the
// backward of 32768 rows of 768 takes 35.0 us instead of 34.4)
struct NormArgs : NormTensors, RowWalk {
  bool w16;  // weights in bf16
  float eps, invC;
};

// U rows per thread group, all loaded before the first is reduced; a workgroup
// does not go on to others: nothing would wait for its stores, but the next loads
// would (loads and stores share one counter).
template <int TPR> constexpr int fwd_threads = TPR > NORM_FWD_THREADS ? TPR : NORM_FWD_THREADS;
template <int TPR> constexpr int bwd_threads = TPR > NORM_BWD_THREADS ? TPR : NORM_BWD_THREADS;
template <typename T, int VE, int TPR, int P, int U>
__global__ void __launch_bounds__(fwd_threads<TPR>) norm_fwd_kernel(NormArgs a) {
  using Sum = RowSum<TPR, fwd_threads<TPR>, 1>;
  constexpr int RPB = Sum::ROWS;
  __shared__ float red[2][Sum::ROWS][Sum::W][1];
  Sum row_sum{red};
  const int block = blockIdx.y * ROWS_GRID_X + blockIdx.x;
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

// The arguments of a call on `tensors` strided tensors, whose places go to `to`.
NormArgs norm_args(const mita_norm_cfg_t &c, const Strided *t, int tensors, RowPlaces NormArgs::*const *to) {
  NormArgs a{};
  RowPlaces places[4];
  static_cast<RowWalk &>(a) = row_walk(t, tensors, places);
  for (int i = 0; i < tensors; ++i) a.*to[i] = places[i];
  a.stat = places[tensors];
  a.w16 = c.wdtype == MITA_BF16;
  a.eps = c.eps;
  a.invC = 1.f / (float)c.C;
  return a;
}

template <typename T, int VE, int TPR, int P> hipError_t fwd_p(const NormArgs &a, hipStream_t st) {
  // as many rows per thread as give four pieces, once that leaves eight workgroups per CU
  constexpr int N = fwd_threads<TPR>, RPB = N / TPR, U = P >= 4 ? 1 : P >= 2 ? 2 : 4;
  if (U > 1 && a.rows >= RPB * U * 8 * CUS)
    norm_fwd_kernel<T, VE, TPR, P, U><<<rows_grid((a.rows + RPB * U - 1) / (RPB * U)), N, 0, st>>>(a);
  else
    norm_fwd_kernel<T, VE, TPR, P, 1><<<rows_grid((a.rows + RPB - 1) / RPB), N, 0, st>>>(a);
  return launched("norm_fwd_kernel", st);
}
template <typename T, int VE, int TPR, int P> hipError_t bwd_p(const NormArgs &a, int blocks, hipStream_t st) {
  if (a.dw || a.db)
    norm_bwd_kernel<T, VE, TPR, P, true><<<dim3((unsigned)blocks), bwd_threads<TPR>, 0, st>>>(a);
  else
    norm_bwd_kernel<T, VE, TPR, P, false><<<dim3((unsigned)blocks), bwd_threads<TPR>, 0, st>>>(a);
  return launched("norm_bwd_kernel", st);
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
  RowPlaces NormArgs::*const to[2] = {&NormArgs::sx, &NormArgs::sy};
  NormArgs a = norm_args(c, t, 2, to);
  a.x = x;
  a.w = w;
  a.b = b;
  a.y = y;
  a.mean = mean;
  a.rstd = rstd;
  const size_t e = elem_bytes(c);
  const NormPlan p = norm_plan(c, row_align(t[1], e, y, row_align(t[0], e, x, 16 / (int)e)));
  return c.dtype == MITA_F32 ? forward_t<float>(a, p, st) : forward_t<bf16_t>(a, p, st);
}

hipError_t launch_norm_backward(const mita_norm_cfg_t &c, const void *x, const void *w, const float *mean,
                                const float *rstd, const void *dy, void *dx, void *dw, void *db, void *ws,
                                hipStream_t st) {
  const Strided t[3] = {strided_rows(c, c.x), strided_rows(c, c.dy), strided_rows(c, c.dx)};
  RowPlaces NormArgs::*const to[3] = {&NormArgs::sx, &NormArgs::sdy, &NormArgs::sdx};
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
  const size_t e = elem_bytes(c);
  const NormPlan p = norm_plan(c, row_align(t[2], e, dx, row_align(t[1], e, dy, row_align(t[0], e, x, 16 / (int)e))));
  const int blocks = norm_bwd_blocks(c, p);
  return c.dtype == MITA_F32 ? backward_t<float>(a, p, blocks, st) : backward_t<bf16_t>(a, p, blocks, st);
}

}  // namespace mita
