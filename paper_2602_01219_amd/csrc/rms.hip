// rms.hip - root-mean-square norm of rows with the residual's addition, also to 8
// bits with scales, and its gradients.
//
// Forward: h = x + res, y = h rstd w, rstd = 1 / sqrt(mean(h^2) + eps). Backward, with
// u = h rstd and g = dy w: dx = dh + rstd (g - u mean(g u)), dw = sum dy u. Both are bound
// by HBM: a row is read once into registers, its sum goes across the threads that
// share it, and it is written once (see row_plan for the widest rows that fit; wider
// ones are read once per pass). An 8-bit output's scales are maxima over the
// registers too: 128 columns are 16 neighbouring lanes' pieces in bf16.
#include "kernels.hpp"
#include "layer_check.hpp"
#include "rows.hpp"

namespace mita {

namespace {

struct RmsTensors {
  const void *x, *res, *w, *dy, *dh;
  void *h, *y, *dx, *dw;
  const float *rstd_in;
  float *rstd, *scales, *part;
  RowPlaces sx, sres, sh, sy, sdy, sdh, sdx, stat;  // `stat`: of the row's statistics
};
// (the tensors first: the walk first gives the same instructions, which read their arguments
// at other places, and for the backward of 32768 rows of 768 39.8 us instead of 39.5)
struct RmsArgs : RmsTensors, RowWalk {
  int q8;      // y: 0 in the rows' type, 1 in 8 bits with a scale per row, 2 per 128 columns
  int groups;  // scales per row
  bool w16;    // weights in bf16
  float eps, invC;
  // The forward adds squares of v unit, unit = 2^-k with 4^k >= C, and multiplies their sum
  // by over = 4^k / C, below 4: it stays finite wherever the mean of squares is. Powers of
  // two change no rounding, but for means below 2^-124, whose sum is denormal.
  float unit, over;
};

constexpr float E4M3_MAX = 448.f;
// The scale of a group whose largest value is `top`: not 0, and its reciprocal finite.
__device__ __forceinline__ float e4m3_scale(float top) { return fmaxf(top, 0x1p-117f) / E4M3_MAX; }
// y / scale as fp32 division rounds it, with one reciprocal for several values: a quotient q
// off by a step or two is brought to one of the two nearest by its residual, and from there
// to the nearest, as the residual then is exact (Markstein's theorem, 1990; the reciprocal
// has to be rounded correctly). All of it times the power of two that brings the scale to
// [1, 2), so that no residual that counts is lost below 2^-149. An infinite scale gives
// 0, and NaN for infinite y. 16384 rows of 4096 without a residual, bf16: 49 us with a
// division per value, 42.6 so, 41 with products with the reciprocal, which differ where y /
// scale is next to the middle of two codes. Pieces of one or two elements are divided.
struct Quotient {
  float unit, s, inv;
  __device__ __forceinline__ explicit Quotient(float scale) {
    const uint32_t e = __float_as_uint(scale) & 0x7f800000u;
    unit = __uint_as_float(0x7f000000u - min(e, 0x7e800000u));
    s = scale * unit;
    inv = 1.f / s;
    s = e == 0x7f800000u ? 0.f : s;
  }
  __device__ __forceinline__ float operator()(float y) const {
    y *= unit;
    float q = y * inv;
    q = __builtin_fmaf(-__builtin_fmaf(q, s, -y), inv, q);  // (so written, -0 stays -0)
    return __builtin_fmaf(-__builtin_fmaf(q, s, -y), inv, q);
  }
};
template <int VE> __device__ __forceinline__ void divide(float (&o)[VE], const float (&y)[VE], float scale) {
  if constexpr (VE > 2) {
    const Quotient quotient(scale);
#pragma unroll
    for (int e = 0; e < VE; ++e) o[e] = quotient(y[e]);
  } else {
#pragma unroll
    for (int e = 0; e < VE; ++e) o[e] = y[e] / scale;
  }
}
// VE codes of values that are at most 448 (but for the last rounding, which the
// conversion takes back).
template <int VE> __device__ __forceinline__ void put_e4m3(uint8_t *p, const float *f) {
  if constexpr (VE == 1) {
    *p = (uint8_t)__builtin_amdgcn_cvt_pk_fp8_f32(f[0], 0.f, 0, false);
  } else if constexpr (VE == 2) {
    *reinterpret_cast<uint16_t *>(p) = (uint16_t)__builtin_amdgcn_cvt_pk_fp8_f32(f[0], f[1], 0, false);
  } else {
    uint32_t v[VE / 4];
#pragma unroll
    for (int i = 0; i < VE / 4; ++i)
      v[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(
          f[4 * i + 2], f[4 * i + 3], __builtin_amdgcn_cvt_pk_fp8_f32(f[4 * i], f[4 * i + 1], 0, false), true);
    if constexpr (VE == 4)
      *reinterpret_cast<uint32_t *>(p) = v[0];
    else
      *reinterpret_cast<uint2 *>(p) = make_uint2(v[0], v[1]);
  }
}

// The largest |y| of each piece's group, in every thread that holds a part of it: one
// row (`row`), or 128 columns. A group is a part of one piece's lanes, several pieces,
// or (single elements over several waves) two waves' parts of a piece.
template <int VE, int TPR, int P, int THREADS> struct GroupTop {
  static constexpr int W = TPR > 64 ? TPR / 64 : 1, ROWS = THREADS / TPR;
  static constexpr int E = TPR * VE;                            // columns of a piece
  static constexpr int PG = E < RMS_GROUP ? RMS_GROUP / E : 1;  // pieces of a group
  static constexpr int L = RMS_GROUP / VE < TPR ? RMS_GROUP / VE : TPR;  // threads of a group
  float (*red)[W][P];  // [ROWS]
  __device__ __forceinline__ void operator()(float (&top)[P], bool row) {
    const int sub = threadIdx.x / TPR, w = (threadIdx.x % TPR) >> 6;
    if (row) {
      float m = top[0];
#pragma unroll
      for (int j = 1; j < P; ++j) m = fmaxf(m, top[j]);
      m = group_max<(TPR < 64 ? TPR : 64)>(m);
      if constexpr (W > 1) {
        if ((threadIdx.x & 63) == 0) red[sub][w][0] = m;
        __syncthreads();
        m = red[sub][0][0];
#pragma unroll
        for (int i = 1; i < W; ++i) m = fmaxf(m, red[sub][i][0]);
      }
#pragma unroll
      for (int j = 0; j < P; ++j) top[j] = m;
      return;
    }
#pragma unroll
    for (int j = 0; j < P; j += PG) {
      float m = top[j];
#pragma unroll
      for (int i = 1; i < PG; ++i)
        if (j + i < P) m = fmaxf(m, top[j + i]);
      m = group_max<(L < 64 ? L : 64)>(m);
#pragma unroll
      for (int i = 0; i < PG; ++i)
        if (j + i < P) top[j + i] = m;
    }
    if constexpr (L > 64) {
      if ((threadIdx.x & 63) == 0) {
#pragma unroll
        for (int j = 0; j < P; ++j) red[sub][w][j] = top[j];
      }
      __syncthreads();
#pragma unroll
      for (int j = 0; j < P; ++j) top[j] = fmaxf(top[j], red[sub][w ^ 1][j]);
    }
  }
};

template <int TPR> constexpr int fwd_threads = TPR > NORM_FWD_THREADS ? TPR : NORM_FWD_THREADS;
template <int TPR> constexpr int bwd_threads = TPR > NORM_BWD_THREADS ? TPR : NORM_BWD_THREADS;

// One row per thread group and workgroup: what is in flight comes from the other
// workgroups (two and four rows per group, all loaded first, with ordinary reads: 84 us
// and 87 against 84 for 16384 rows of 4096, 9.6 and 12.0 against 8.7 for 2000 of 2048, 27 and
// 27 against 26 for 300000 of 64).
template <typename T, int VE, int TPR, int P, bool ONCE>
__global__ void __launch_bounds__(fwd_threads<TPR>) rms_fwd_kernel(RmsArgs a) {
  using Sum = RowSum<TPR, fwd_threads<TPR>, 1>;
  using Top = GroupTop<VE, TPR, P, fwd_threads<TPR>>;
  __shared__ float red[2][Sum::ROWS][Sum::W][1];
  __shared__ float tops[Sum::ROWS][Top::W][P];
  Sum row_sum{red};
  const int block = blockIdx.y * ROWS_GRID_X + blockIdx.x;
  const int t = threadIdx.x % TPR, r = block * Sum::ROWS + threadIdx.x / TPR, rc = min(r, a.rows - 1);
  const bool on = r < a.rows;
  RowRegs<T, VE, TPR, P> x, res;
  x.template load<ONCE>((const T *)a.x + row_at(a, a.sx, rc), a.C, t);
  if (a.res) res.template load<ONCE>((const T *)a.res + row_at(a, a.sres, rc), a.C, t);
  float w[P][VE];
  weights<VE, TPR, P>(w, a.w, a.w16, a.C, t, 1.f);
  float v[P][VE], sum[1] = {0.f};
#pragma unroll
  for (int j = 0; j < P; ++j) {
    x.get(v[j], j, a.C, t);
    if (a.res) {
      float z[VE];
      res.get(z, j, a.C, t);
#pragma unroll
      for (int e = 0; e < VE; ++e) v[j][e] += z[e];
    }
#pragma unroll
    for (int e = 0; e < VE; ++e) {
      const float z = v[j][e] * a.unit;
      sum[0] = __builtin_fmaf(z, z, sum[0]);
    }
  }
  row_sum(sum);
  const float rstd = 1.f / sqrtf(sum[0] * a.over + a.eps);
  if (a.h && on) {
    T *h = (T *)a.h + row_at(a, a.sh, r);
#pragma unroll
    for (int j = 0; j < P; ++j) {
      const int i = (j * TPR + t) * VE;
      if (i < a.C) put<T, VE>(h + i, v[j]);
    }
  }
#pragma unroll
  for (int j = 0; j < P; ++j)
#pragma unroll
    for (int e = 0; e < VE; ++e) v[j][e] = v[j][e] * rstd * w[j][e];
  if (a.q8 == 0) {
    if (on) {
      T *y = (T *)a.y + row_at(a, a.sy, r);
#pragma unroll
      for (int j = 0; j < P; ++j) {
        const int i = (j * TPR + t) * VE;
        if (i < a.C) put<T, VE>(y + i, v[j]);
      }
    }
  } else {
    float top[P];
#pragma unroll
    for (int j = 0; j < P; ++j) {  // (pieces past the row hold 0)
      top[j] = 0.f;
#pragma unroll
      for (int e = 0; e < VE; ++e) top[j] = fmaxf(top[j], fabsf(v[j][e]));
    }
    Top{tops}(top, a.q8 == 1);
    if (on) {
      uint8_t *y = (uint8_t *)a.y + row_at(a, a.sy, r);
      float *scales = a.scales + row_at(a, a.stat, r) * a.groups;
#pragma unroll
      for (int j = 0; j < P; ++j) {
        const int i = (j * TPR + t) * VE;
        const float s = e4m3_scale(top[j]);
        float o[VE];
        divide(o, v[j], s);
        if (i < a.C) {
          put_e4m3<VE>(y + i, o);
          if (a.q8 == 2 ? i % RMS_GROUP == 0 : i == 0) scales[a.q8 == 2 ? i / RMS_GROUP : 0] = s;
        }
      }
    }
  }
  if (on && t == 0 && a.rstd) a.rstd[row_at(a, a.stat, r)] = rstd;
}

// WG: is dw wanted? A workgroup goes over rows gridDim.x * RPB apart and keeps its
// columns' sums.
template <typename T, int VE, int TPR, int P, bool WG, bool ONCE>
__global__ void __launch_bounds__(bwd_threads<TPR>) rms_bwd_kernel(RmsArgs a) {
  using Sum = RowSum<TPR, bwd_threads<TPR>, 1>;
  constexpr int RPB = Sum::ROWS;
  __shared__ float red[2][Sum::ROWS][Sum::W][1];
  __shared__ float sums[WG ? bwd_threads<TPR> * VE : 1];
  Sum row_sum{red};
  const int t = threadIdx.x % TPR, sub = threadIdx.x / TPR;
  float w[P][VE], dw[P][VE];
  weights<VE, TPR, P>(w, a.w, a.w16, a.C, t, 1.f);
#pragma unroll
  for (int j = 0; j < P; ++j)
#pragma unroll
    for (int e = 0; e < VE; ++e) dw[j][e] = 0.f;
  // the loop is uniform over the workgroup: rows past the last weigh nothing
  for (int r0 = blockIdx.x * RPB; r0 < a.rows; r0 += gridDim.x * RPB) {
    const int r = r0 + sub, rc = min(r, a.rows - 1);
    RowRegs<T, VE, TPR, P> h, y, z;
    h.template load<ONCE>((const T *)a.x + row_at(a, a.sx, rc), a.C, t);
    y.template load<ONCE>((const T *)a.dy + row_at(a, a.sdy, rc), a.C, t);
    if (a.dh) z.template load<ONCE>((const T *)a.dh + row_at(a, a.sdh, rc), a.C, t);
    const float rstd = a.rstd_in[row_at(a, a.stat, rc)];
    // lanes past the last row hold its dy, or, with dx in dy's place, what its own
    // lanes have written there by now
    const bool on = r < a.rows;
    float sm[1] = {0.f};
#pragma unroll
    for (int j = 0; j < P; ++j) {
      float hv[VE], yv[VE];
      h.c[j].get(hv);
      y.get(yv, j, a.C, t);
#pragma unroll
      for (int e = 0; e < VE; ++e) {
        const float p = yv[e] * (hv[e] * rstd);
        // elements past the row have dy = 0
        sm[0] = __builtin_fmaf(p, w[j][e], sm[0]);
        if (WG) dw[j][e] = on ? dw[j][e] + p : dw[j][e];
      }
    }
    if (!a.dx) continue;
    row_sum(sm);
    const float s = sm[0] * a.invC;
    if (on) {
      T *dx = (T *)a.dx + row_at(a, a.sdx, r);
#pragma unroll
      for (int j = 0; j < P; ++j) {
        const int i = (j * TPR + t) * VE;
        float hv[VE], yv[VE];
        h.c[j].get(hv);
        y.c[j].get(yv);
#pragma unroll
        for (int e = 0; e < VE; ++e) yv[e] = rstd * __builtin_fmaf(yv[e], w[j][e], -(hv[e] * rstd) * s);
        if (a.dh) {
          z.c[j].get(hv);
#pragma unroll
          for (int e = 0; e < VE; ++e) yv[e] += hv[e];
        }
        if (i < a.C) put<T, VE>(dx + i, yv);
      }
    }
  }
  if constexpr (WG) {
    // the workgroup's sums, its rows' parts in a fixed order
    float *part = a.part + (int64_t)blockIdx.x * a.C;
#pragma unroll
    for (int j = 0; j < P; ++j) {
      __syncthreads();
#pragma unroll
      for (int e = 0; e < VE; ++e) sums[threadIdx.x * VE + e] = dw[j][e];
      __syncthreads();
      for (int c = threadIdx.x; c < TPR * VE; c += bwd_threads<TPR>) {
        const int i = j * TPR * VE + c;
        if (i < a.C) {
          float y = 0.f;
#pragma unroll 8
          for (int q = 0; q < RPB; ++q) y += sums[q * TPR * VE + c];
          part[i] = y;
        }
      }
    }
  }
}

// dw: the workgroups' partial sums, sixteen interleaved sequences per column added
// in a fixed order.
__global__ void __launch_bounds__(512) rms_sum_kernel(RmsArgs a, int parts) {
  __shared__ float s[16][33];
  const int c = threadIdx.x & 31, q = threadIdx.x >> 5, i = blockIdx.x * 32 + c;
  float y = 0.f;
  if (i < a.C) {
#pragma unroll 16
    for (int p = q; p < parts; p += 16) y += a.part[(int64_t)p * a.C + i];
  }
  s[q][c] = y;
  __syncthreads();
  if (q != 0 || i >= a.C) return;
  y = 0.f;
#pragma unroll
  for (int k = 0; k < 16; ++k) y += s[k][c];
  if (a.w16)
    ((bf16_t *)a.dw)[i] = from_f32<bf16_t>(y);
  else
    ((float *)a.dw)[i] = y;
}

// Rows too wide for registers: a workgroup per row, which reads it once per pass, element by
// element: 2000 rows of 32768, bf16, 385 us to 8 bits with a scale per row (three passes; 32
// at 6.2 TB/s), 470 with a residual to bf16 (85), backward 490.
// Outputs in an input's place are written in the last one, each element by the thread
// that has just read it.
template <typename T> __global__ void __launch_bounds__(512) rms_fwd_wide_kernel(RmsArgs a) {
  __shared__ float red[8];
  for (int r = blockIdx.x; r < a.rows; r += gridDim.x) {
    const T *x = (const T *)a.x + row_at(a, a.sx, r);
    const T *res = a.res ? (const T *)a.res + row_at(a, a.sres, r) : nullptr;
    T *h = a.h ? (T *)a.h + row_at(a, a.sh, r) : nullptr;
    auto at = [&](int i) { return res ? to_f32(x[i]) + to_f32(res[i]) : to_f32(x[i]); };
    auto weight = [&](int i) { return weight_at(a.w, a.w16, i, 1.f); };
    float s = 0.f;
    for (int i = threadIdx.x; i < a.C; i += blockDim.x) {
      const float z = at(i) * a.unit;
      s = __builtin_fmaf(z, z, s);
    }
    const float rstd = 1.f / sqrtf(block_sum(s, red) * a.over + a.eps);
    const int64_t stat = row_at(a, a.stat, r);
    if (threadIdx.x == 0 && a.rstd) a.rstd[stat] = rstd;
    if (a.q8 == 0) {
      T *y = (T *)a.y + row_at(a, a.sy, r);
      for (int i = threadIdx.x; i < a.C; i += blockDim.x) {
        const float v = at(i);
        if (h) h[i] = from_f32<T>(v);
        y[i] = from_f32<T>(v * rstd * weight(i));
      }
      continue;
    }
    float scale = 0.f;
    if (a.q8 == 1) {
      float top = 0.f;
      for (int i = threadIdx.x; i < a.C; i += blockDim.x) top = fmaxf(top, fabsf(at(i) * rstd * weight(i)));
      top = wave_max(top);
      __syncthreads();
      if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = top;
      __syncthreads();
#pragma unroll
      for (int i = 0; i < 8; ++i) top = fmaxf(top, red[i]);
      scale = e4m3_scale(top);
      if (threadIdx.x == 0) a.scales[stat] = scale;
    }
    // a wave takes 128 columns at a time, two per lane
    uint8_t *y = (uint8_t *)a.y + row_at(a, a.sy, r);
    for (int c = (threadIdx.x >> 6) * RMS_GROUP; c < a.C; c += (blockDim.x >> 6) * RMS_GROUP) {
      float v[2];
      int i[2];
      bool in[2];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        i[e] = c + 64 * e + (threadIdx.x & 63);
        in[e] = i[e] < a.C;
        v[e] = in[e] ? at(i[e]) : 0.f;
        if (in[e] && h) h[i[e]] = from_f32<T>(v[e]);
        v[e] = in[e] ? v[e] * rstd * weight(i[e]) : 0.f;
      }
      if (a.q8 == 2) {
        scale = e4m3_scale(wave_max(fmaxf(fabsf(v[0]), fabsf(v[1]))));
        if ((threadIdx.x & 63) == 0) a.scales[stat * a.groups + c / RMS_GROUP] = scale;
      }
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const float o = v[e] / scale;
        if (in[e]) put_e4m3<1>(y + i[e], &o);
      }
    }
  }
}
template <typename T> __global__ void __launch_bounds__(512) rms_dx_wide_kernel(RmsArgs a) {
  __shared__ float red[8];
  for (int r = blockIdx.x; r < a.rows; r += gridDim.x) {
    const T *h = (const T *)a.x + row_at(a, a.sx, r), *dy = (const T *)a.dy + row_at(a, a.sdy, r);
    const T *dh = a.dh ? (const T *)a.dh + row_at(a, a.sdh, r) : nullptr;
    T *dx = (T *)a.dx + row_at(a, a.sdx, r);
    const float rstd = a.rstd_in[row_at(a, a.stat, r)];
    auto weight = [&](int i) { return weight_at(a.w, a.w16, i, 1.f); };
    float s = 0.f;
    for (int i = threadIdx.x; i < a.C; i += blockDim.x)
      s = __builtin_fmaf(to_f32(dy[i]) * weight(i), to_f32(h[i]) * rstd, s);
    s = block_sum(s, red) * a.invC;
    for (int i = threadIdx.x; i < a.C; i += blockDim.x) {
      float v = rstd * __builtin_fmaf(to_f32(dy[i]), weight(i), -(to_f32(h[i]) * rstd) * s);
      if (dh) v += to_f32(dh[i]);
      dx[i] = from_f32<T>(v);
    }
  }
}
// Workgroup (i, p): columns 512 i .., every gridDim.y-th row from p on.
template <typename T> __global__ void __launch_bounds__(512) rms_dw_wide_kernel(RmsArgs a) {
  const int i = blockIdx.x * 512 + threadIdx.x;
  if (i >= a.C) return;
  float dw = 0.f;
#pragma unroll 4
  for (int r = blockIdx.y; r < a.rows; r += gridDim.y) {
    const float h = to_f32(((const T *)a.x)[row_at(a, a.sx, r) + i]);
    const float dy = to_f32(((const T *)a.dy)[row_at(a, a.sdy, r) + i]);
    dw = __builtin_fmaf(dy, h * a.rstd_in[row_at(a, a.stat, r)], dw);
  }
  a.part[(int64_t)blockIdx.y * a.C + i] = dw;
}

// Inputs of 128 MB and more are read past the caches' order (the last-level one holds 256
// MB). With it and with ordinary reads, us, inputs and outputs of three calls in turn, and (in
// brackets) where the outputs take the place of the call's before, bf16: 16384 rows of 4096
// with a residual to 8 bits, 268 MB, 84 and 85 (75 and 85); 8192 rows, 134 MB, 43 and 45 (40 and
// 40), to bf16 48 and 48 (43 and 43), backward, 201 MB, 49 and 55 (49 and 50); backward of 65536
// rows of 768, 201 MB, 60 and 61 (54 and 56), of 32768 with dh, 151 MB, 39 and 44 (39 and 40);
// but 4096 rows of 4096, 67 MB, 24 and 26 (24 and 21). Pieces of 16 bytes only.
template <typename T, int VE> bool read_once(const RmsArgs &a, int tensors) {
  return VE * sizeof(T) == 16 && (int64_t)tensors * a.rows * a.C * (int64_t)sizeof(T) >= (int64_t)1 << 27;
}
template <typename T, int VE, int TPR, int P> hipError_t fwd_p(const RmsArgs &a, hipStream_t st) {
  constexpr int N = fwd_threads<TPR>, RPB = N / TPR;
  constexpr bool WHOLE = VE * sizeof(T) == 16;
  const dim3 grid = rows_grid((a.rows + RPB - 1) / RPB);
  if (read_once<T, VE>(a, a.res ? 2 : 1))
    rms_fwd_kernel<T, VE, TPR, P, WHOLE><<<grid, N, 0, st>>>(a);
  else
    rms_fwd_kernel<T, VE, TPR, P, false><<<grid, N, 0, st>>>(a);
  return launched("rms_fwd_kernel", st);
}
template <typename T, int VE, int TPR, int P> hipError_t bwd_p(const RmsArgs &a, int blocks, hipStream_t st) {
  constexpr bool WHOLE = VE * sizeof(T) == 16;
  const bool once = read_once<T, VE>(a, a.dh ? 3 : 2);
  if (a.dw && once)
    rms_bwd_kernel<T, VE, TPR, P, true, WHOLE><<<dim3((unsigned)blocks), bwd_threads<TPR>, 0, st>>>(a);
  else if (a.dw)
    rms_bwd_kernel<T, VE, TPR, P, true, false><<<dim3((unsigned)blocks), bwd_threads<TPR>, 0, st>>>(a);
  else if (once)
    rms_bwd_kernel<T, VE, TPR, P, false, WHOLE><<<dim3((unsigned)blocks), bwd_threads<TPR>, 0, st>>>(a);
  else
    rms_bwd_kernel<T, VE, TPR, P, false, false><<<dim3((unsigned)blocks), bwd_threads<TPR>, 0, st>>>(a);
  return launched("rms_bwd_kernel", st);
}
template <typename T> struct RunFwd {
  const RmsArgs &a;
  hipStream_t st;
  template <int VE, int TPR, int P> hipError_t run() { return fwd_p<T, VE, TPR, P>(a, st); }
};
template <typename T> struct RunBwd {
  const RmsArgs &a;
  int blocks;
  hipStream_t st;
  template <int VE, int TPR, int P> hipError_t run() { return bwd_p<T, VE, TPR, P>(a, blocks, st); }
};

template <typename T> hipError_t forward_t(const RmsArgs &a, const NormPlan &p, hipStream_t st) {
  if (p.p) return with_plan<T>(p, RunFwd<T>{a, st});
  rms_fwd_wide_kernel<T><<<dim3((unsigned)std::min(a.rows, 4 * CUS)), 512, 0, st>>>(a);
  return launched("rms_fwd_wide_kernel", st);
}
template <typename T> hipError_t backward_t(const RmsArgs &a, const NormPlan &p, int blocks, hipStream_t st) {
  hipError_t e = hipSuccess;
  if (p.p) {
    e = with_plan<T>(p, RunBwd<T>{a, blocks, st});
    if (e != hipSuccess) return e;
  } else {
    if (a.dw) {  // before dx, which may take dy's place
      rms_dw_wide_kernel<T><<<dim3((unsigned)((a.C + 511) / 512), (unsigned)blocks), 512, 0, st>>>(a);
      e = launched("rms_dw_wide_kernel", st);
      if (e != hipSuccess) return e;
    }
    if (a.dx) {
      rms_dx_wide_kernel<T><<<dim3((unsigned)std::min(a.rows, 4 * CUS)), 512, 0, st>>>(a);
      e = launched("rms_dx_wide_kernel", st);
      if (e != hipSuccess) return e;
    }
  }
  if (!a.dw) return e;
  rms_sum_kernel<<<dim3((unsigned)((a.C + 31) / 32)), 512, 0, st>>>(a, blocks);
  return launched("rms_sum_kernel", st);
}

RmsArgs rms_args(const mita_rms_cfg_t &c) {
  RmsArgs a{};
  a.q8 = c.ytype != MITA_E4M3 ? 0 : c.group ? 2 : 1;
  a.groups = rms_scales(c);
  a.w16 = c.wdtype == MITA_BF16;
  a.eps = c.eps;
  a.invC = 1.f / (float)c.C;
  int k = 0;
  while (((int64_t)1 << 2 * k) < c.C) ++k;
  a.unit = 1.f / (float)(1 << k);
  a.over = (float)((int64_t)1 << 2 * k) * a.invC;
  return a;
}

}  // namespace

hipError_t launch_rms_forward(const mita_rms_cfg_t &c, const void *x, const void *res, const void *w, void *h, void *y,
                              float *scales, float *rstd, hipStream_t st) {
  const Strided t[4] = {strided_rows(c, c.x), strided_rows(c, c.res), strided_rows(c, c.h), strided_rows(c, c.y)};
  RowPlaces places[5];
  RmsArgs a = rms_args(c);
  static_cast<RowWalk &>(a) = row_walk(t, 4, places);
  a.sx = places[0];
  a.sres = places[1];
  a.sh = places[2];
  a.sy = places[3];
  a.stat = places[4];
  a.x = x;
  a.res = res;
  a.w = w;
  a.h = h;
  a.y = y;
  a.scales = scales;
  a.rstd = rstd;
  const size_t e = elem_bytes(c);
  int align = row_align(t[0], e, x, 16 / (int)e);
  align = row_align(t[3], y_bytes(c), y, row_align(t[2], e, h, row_align(t[1], e, res, align)));
  const NormPlan p = row_plan(e, c.C, align);
  return c.dtype == MITA_F32 ? forward_t<float>(a, p, st) : forward_t<bf16_t>(a, p, st);
}

hipError_t launch_rms_backward(const mita_rms_cfg_t &c, const void *h, const void *w, const float *rstd, const void *dy,
                               const void *dh, void *dx, void *dw, void *ws, hipStream_t st) {
  const Strided t[4] = {strided_rows(c, c.h), strided_rows(c, c.dy), strided_rows(c, c.dh), strided_rows(c, c.dx)};
  RowPlaces places[5];
  RmsArgs a = rms_args(c);
  static_cast<RowWalk &>(a) = row_walk(t, 4, places);
  a.sx = places[0];
  a.sdy = places[1];
  a.sdh = places[2];
  a.sdx = places[3];
  a.stat = places[4];
  a.x = h;
  a.w = w;
  a.rstd_in = rstd;
  a.dy = dy;
  a.dh = dh;
  a.dx = dx;
  a.dw = dw;
  a.part = (float *)ws;
  const size_t e = elem_bytes(c);
  int align = row_align(t[0], e, h, 16 / (int)e);
  align = row_align(t[3], e, dx, row_align(t[2], e, dh, row_align(t[1], e, dy, align)));
  const NormPlan p = row_plan(e, c.C, align);
  const int blocks = row_bwd_blocks(norm_rows(c), p);
  return c.dtype == MITA_F32 ? backward_t<float>(a, p, blocks, st) : backward_t<bf16_t>(a, p, blocks, st);
}

}  // namespace mita
