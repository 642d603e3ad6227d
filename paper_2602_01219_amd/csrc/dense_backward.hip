// dense_backward.hip - gradients of dense attention from q, k, v, o, the rows'
// log-sum-exps and dO. With P = exp(scale Q K^T - lse), D = rowsum(dO o) and
// dS = P (dO V^T - D): dQ = scale dS K, dK = scale dS^T Q, dV = P^T dO.
//
// Two passes form P and dP each, so that every sum has one owner and no atomics:
// the query side (32 rows per wave, over the keys) sums dQ, the key side (32 keys
// per wave, over the rows of all query heads of the key head) sums dK and dV.
// That is 14 D flops per pair where 10 D would do with dQ added atomically. Both are
// bound by the MFMAs: 24 heads of 16384 tokens, d = 64, take 2.2 ms (query side)
// and 3.1 ms (key side), 1.1 PFLOP/s of the products formed; 16 heads of 8192, d =
// 128, 1.7 ms in all. Where registers are short (the key side at d = 128 holds 192
// of them in operands and sums) addresses are formed again: a spilled one's load waits
// for the tile copies in flight (1968 us before, 1707 after). What
// is left spilled: 12 registers of the key side in bf16 at d = 128, 21 in fp32 at d = 64
// and 19 at d = 128, 2 of the query side in fp32 at d = 64.
#include "dense.hpp"
#include "kernels.hpp"
#include "layer_check.hpp"

namespace mita {

DenseArgs dense_args(const mita_dense_cfg_t &c);

// exp(scale q.k - lse) of a raw dot and the row's log-sum-exp in log2 units.
__device__ __forceinline__ float prob(float s, float sl2, float l) {
  return __builtin_amdgcn_exp2f(__builtin_fmaf(s, sl2, -l));
}

// The query side: dQ, and for the key side the rows' log-sum-exps (log2 units;
// +infinity, weight 0, for rows that see nothing or do not exist) and D.
template <typename T, int D>
__global__ void __launch_bounds__(256, sizeof(T) * D == 128 ? 3 : sizeof(T) * D == 256 ? 2 : 1) dense_dq_kernel(DenseArgs a) {
  using RT = RowTile<T, D>;
  constexpr int TR = RT::TR, BYTES = TR * RT::RB;
  __shared__ __align__(16) char ldsK[2 * BYTES];
  __shared__ __align__(16) char ldsV[2 * BYTES];
  int s, item;
  dense_block(blockIdx.x, a.B * a.Hkv, a.tiles * a.splits, s, item);
  const int sp = item % a.splits;
  const int tile = a.tiles - 1 - item / a.splits;
  const DenseSlice x = dense_slice(a, s);
  const int lane = threadIdx.x & 63, n = lane & 31, g = lane >> 5;
  const int w = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);

  const int row = tile * DENSE_TQ + 32 * w + n;
  const int tok = div_group(a, row), head = x.hk * a.G + row - tok * a.G;
  const bool exists = row < a.R, valid = exists && tok < x.qlen;
  Column<T, D> q, dO;
  q.load(a.q.p + x.b * a.q.b + head * a.q.h + (int64_t)tok * a.q.n, valid);
  const char *const dOrow = a.dO.p + x.b * a.dO.b + head * a.dO.h + (int64_t)tok * a.dO.n;
  dO.load(dOrow, valid);
  const float Dr = column_sum(
      column_dot<T, D>(a.o.p + x.b * a.o.b + head * a.o.h + (int64_t)tok * a.o.n, dOrow, valid));
  float lse2 = INFINITY;
  if (valid) {
    const float l = a.lse[((int64_t)x.b * a.H + head) * a.N + tok];
    lse2 = l == -INFINITY ? INFINITY : l * LOG2E;
  }
  if (sp == 0 && lane < 32) {
    const int64_t at = ((int64_t)s * a.tiles + tile) * DENSE_TQ + 32 * w + n;
    a.row_lse[at] = lse2;
    a.row_D[at] = Dr;
  }
  const int lo = valid ? first_key(a, x, tok) : 0, hi = valid ? end_key(a, x, tok) : 0;

  const int b0 = div_group(a, tile * DENSE_TQ);
  const int b1 = min(div_group(a, min(tile * DENSE_TQ + DENSE_TQ, a.R) - 1), x.qlen - 1);
  const int kbeg = first_key(a, x, b0), kend = b0 <= b1 ? end_key(a, x, b1) : 0;
  const int nt = kend > kbeg ? (kend - kbeg + TR - 1) / TR : 0;
  const int per = (nt + a.splits - 1) / a.splits;
  const int t0 = sp * per, t1 = min(nt, t0 + per);
  const TileOrder order(t0, t1, (first_key(a, x, b1) - kbeg + TR - 1) / TR, max(0, end_key(a, x, b0) - kbeg) / TR);

  // keys that some row of the wave sees (none: the wave only copies)
  const int wr = tile * DENSE_TQ + 32 * w;
  const int w0 = wr < a.R ? div_group(a, wr) : x.qlen, w1 = min(div_group(a, min(wr + 32, a.R) - 1), x.qlen - 1);
  const int wlo = first_key(a, x, w0), whi = w0 <= w1 ? end_key(a, x, w1) : 0;

  TileAddr<T, D> ad;
  ad.init();
  TileCopy<T, D, 4> copy;
  copy.init();
  const uint32_t offK = copy.row0 * a.k.n, offV = copy.row0 * a.v.n;
  const char *kb = a.k.p + x.b * a.k.b + x.hk * a.k.h, *vb = a.v.p + x.b * a.v.b + x.hk * a.v.h;
  f32x16 dq[D / 32];
#pragma unroll
  for (int i = 0; i < D / 32; ++i) dq[i] = splat16(0.f);

  const uint32_t atK = lds_at(ldsK), atV = lds_at(ldsV);
  auto issue = [&](int p) {
    const int k0 = kbeg + order.at(p) * TR;
    copy.issue(atK + (p & 1) * BYTES, kb, k0, a.k.n, offK, x.klen - k0);
    copy.issue(atV + (p & 1) * BYTES, vb, k0, a.v.n, offV, x.klen - k0);
  };
  auto next = [&](int p) {
    tile_barrier();
    if (p + 1 < order.total) issue(p + 1);
  };
  auto tiles = [&](int p, int end, auto masked) {
    for (; p < end; ++p) {
      next(p);
      const int k0 = kbeg + order.at(p) * TR;
      const char *Kt = ldsK + (p & 1) * BYTES, *Vt = ldsV + (p & 1) * BYTES;
#pragma unroll (D == 64 ? 2 : 1)
      for (int h = 0; h < TR / 32; ++h) {
        if (decltype(masked)::value && (k0 + 32 * h >= whi || k0 + 32 * h + 32 <= wlo)) continue;
        f32x16 z = tile_rows<D>(Kt, ad, h, q, splat16(0.f));
        const f32x16 dp = tile_rows<D>(Vt, ad, h, dO, splat16(-Dr));
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int j = k0 + 32 * h + acc_row(i, g);
          const float y = prob(z[i], a.sl2, lse2) * dp[i];
          z[i] = !decltype(masked)::value || (j >= lo && j < hi) ? y : 0.f;
        }
        tile_cols<D>(dq, Kt, ad, h, ColsOperand<T>(z));
      }
    }
  };
  if (order.total > 0) issue(0);
  if (w0 <= w1) {
    tiles(0, order.nfull, std::false_type{});
    tiles(order.nfull, order.total, std::true_type{});
  } else {
    for (int p = 0; p < order.total; ++p) next(p);
  }
  if (a.splits == 1)
    store_column<D>((T *)(a.dq.p + x.b * a.dq.b + head * a.dq.h + (int64_t)tok * a.dq.n), dq, a.scale, exists);
  else
    store_column<D>(a.part_q + (((int64_t)s * a.R + row) * a.splits + sp) * D, dq, a.scale, exists);
}

// The key side: dK and dV of 32 keys per wave, over the rows that see them.
template <typename T, int D>
__global__ void __launch_bounds__(256, sizeof(T) * D <= 256 ? 2 : 1) dense_dkv_kernel(DenseArgs a, int ktiles, int ksplits) {
  using RT = RowTile<T, D>;
  constexpr int TR = RT::TR;
  constexpr int BYTES = TR * RT::RB;
  __shared__ __align__(16) char ldsQ[2 * BYTES];
  __shared__ __align__(16) char ldsG[2 * BYTES];  // the queries' gradients
  __shared__ __align__(16) char ldsL[2 * 512];    // their log-sum-exps (64) and D (64)
  int s, item;
  dense_block(blockIdx.x, a.B * a.Hkv, ktiles * ksplits, s, item);
  const int sp = item % ksplits, kt = item / ksplits;  // causal: the first keys are seen most
  const DenseSlice x = dense_slice(a, s);
  const int lane = threadIdx.x & 63, n = lane & 31, g = lane >> 5;
  const int w = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);

  const int key = kt * DENSE_KB + 32 * w + n;
  const bool exists = key < a.Nk, valid = key < x.klen;
  Column<T, D> kf, vf;
  kf.load(a.k.p + x.b * a.k.b + x.hk * a.k.h + (int64_t)key * a.k.n, valid);
  vf.load(a.v.p + x.b * a.v.b + x.hk * a.v.h + (int64_t)key * a.v.n, valid);

  // tokens [first, end) see key j; in rows, times G
  const int Rv = x.qlen * a.G;  // rows that exist
  auto first_row = [&](int j) { return min(max(0, j - x.off - a.right), x.qlen) * a.G; };
  auto end_row = [&](int j) { return max(0, min(x.qlen, j - x.off + a.left + 1)) * a.G; };
  const int lo = first_row(key), hi = end_row(key);
  const int k0 = kt * DENSE_KB, k1 = min(k0 + DENSE_KB, x.klen);
  // rows that see some key of the wave (none: the wave only copies)
  const int wk0 = k0 + 32 * w, wk1 = min(wk0 + 32, x.klen) - 1;
  const int wlo = first_row(wk0), whi = wk0 <= wk1 ? end_row(wk1) : 0;
  // whole tiles, counted from a multiple of TR
  const int rbeg = k0 < k1 ? first_row(k0) / TR * TR : 0, rend = k0 < k1 ? end_row(k1 - 1) : 0;
  const int nt = rend > rbeg ? (rend - rbeg + TR - 1) / TR : 0;
  const int per = (nt + ksplits - 1) / ksplits;
  const int t0 = sp * per, t1 = min(nt, t0 + per);
  // tiles whose rows all see the block's keys (rows past the last have no weight)
  const TileOrder order(t0, t1, (first_row(k1 - 1) - rbeg + TR - 1) / TR,
                        end_row(k0) >= Rv ? nt : max(0, end_row(k0) - rbeg) / TR);

  TileAddr<T, D> ad;
  ad.init();
  TileCopy<T, D, 4> copy;
  copy.init();
  const char *qb = a.q.p + x.b * a.q.b + (int64_t)x.hk * a.G * a.q.h;
  const char *db = a.dO.p + x.b * a.dO.b + (int64_t)x.hk * a.G * a.dO.h;
  const float *rl = a.row_lse + (int64_t)s * a.tiles * DENSE_TQ, *rd = a.row_D + (int64_t)s * a.tiles * DENSE_TQ;

  const uint32_t atQ = lds_at(ldsQ), atG = lds_at(ldsG), atL = lds_at(ldsL);
  auto issue = [&](int p) {
    if (sizeof(T) * D >= 256) copy.forget();
    const int r0 = rbeg + order.at(p) * TR;
    const uint32_t qt = atQ + (p & 1) * BYTES, gt = atG + (p & 1) * BYTES, lt = atL + (p & 1) * 512;
    if (a.G == 1) {
      copy.issue(qt, qb, r0, a.q.n, copy.row0 * a.q.n, Rv - r0);
      copy.issue(gt, db, r0, a.dO.n, copy.row0 * a.dO.n, Rv - r0);
    } else {
#pragma unroll
      for (int j = 0; j < copy.PW; ++j) {
        const int r = min(r0 + (int)copy.row(j), Rv - 1), tk = div_group(a, r), h = r - tk * a.G;
        const int at = (w * copy.PW + j) * 1024;
        if (a.near) {
          copy16_unwaited(qb, (uint32_t)h * (uint32_t)a.q.h + (uint32_t)tk * a.q.n + copy.chunk(j), qt + at);
          copy16_unwaited(db, (uint32_t)h * (uint32_t)a.dO.h + (uint32_t)tk * a.dO.n + copy.chunk(j), gt + at);
        } else {
          copy16_unwaited(qb + h * a.q.h + (int64_t)tk * a.q.n + copy.chunk(j), qt + at);
          copy16_unwaited(db + h * a.dO.h + (int64_t)tk * a.dO.n + copy.chunk(j), gt + at);
        }
      }
    }
    const uint32_t at4 = 4 * lanes_below(~(uint64_t)0);
    if (w == 0) copy4_unwaited((const char *)(rl + r0), at4, lt);
    if (w == 1) copy4_unwaited((const char *)(rd + r0), at4, lt + 256);
  };

  f32x16 dk[D / 32], dv[D / 32];
#pragma unroll
  for (int i = 0; i < D / 32; ++i) {
    dk[i] = splat16(0.f);
    dv[i] = splat16(0.f);
  }
  auto next = [&](int p) {
    tile_barrier();
    if (p + 1 < order.total) issue(p + 1);
  };
  auto tiles = [&](int p, int end, auto masked) {
    for (; p < end; ++p) {
      next(p);
      const int r0 = rbeg + order.at(p) * TR;
      const char *qt = ldsQ + (p & 1) * BYTES, *gt = ldsG + (p & 1) * BYTES;
#pragma unroll (D == 64 ? 2 : 1)
      for (int h = 0; h < TR / 32; ++h) {
        if (sizeof(T) * D >= 256) ad.forget();  // (registers are short)
        if (decltype(masked)::value && (r0 + 32 * h >= whi || r0 + 32 * h + 32 <= wlo)) continue;
        const float *ls = (const float *)(ldsL + (p & 1) * 512) + 32 * h + 4 * g, *ds = ls + 64;
        f32x16 z = tile_rows<D>(qt, ad, h, kf, splat16(0.f));
        f32x16 dp;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const float4 y = *reinterpret_cast<const float4 *>(ds + 8 * c);
          dp[4 * c] = -y.x;
          dp[4 * c + 1] = -y.y;
          dp[4 * c + 2] = -y.z;
          dp[4 * c + 3] = -y.w;
        }
        dp = tile_rows<D>(gt, ad, h, vf, dp);
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const float4 y = *reinterpret_cast<const float4 *>(ls + 8 * c);
          const float l[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int i = 4 * c + r, at = r0 + 32 * h + acc_row(i, g);
            const float e = prob(z[i], a.sl2, l[r]);
            z[i] = !decltype(masked)::value || (at >= lo && at < hi) ? e : 0.f;
            dp[i] *= z[i];
          }
        }
        tile_cols<D>(dv, gt, ad, h, ColsOperand<T>(z));
        tile_cols<D>(dk, qt, ad, h, ColsOperand<T>(dp));
      }
    }
  };
  if (order.total > 0) issue(0);
  if (wk0 <= wk1) {
    tiles(0, order.nfull, std::false_type{});
    tiles(order.nfull, order.total, std::true_type{});
  } else {
    for (int p = 0; p < order.total; ++p) next(p);
  }
  if (!valid) {
#pragma unroll
    for (int i = 0; i < D / 32; ++i) {
      dk[i] = splat16(0.f);
      dv[i] = splat16(0.f);
    }
  }
  if (ksplits == 1) {
    store_column<D>((T *)(a.dk.p + x.b * a.dk.b + x.hk * a.dk.h + (int64_t)key * a.dk.n), dk, a.scale, exists);
    store_column<D>((T *)(a.dv.p + x.b * a.dv.b + x.hk * a.dv.h + (int64_t)key * a.dv.n), dv, 1.f, exists);
  } else {
    const int64_t at = (((int64_t)s * a.Nk + key) * ksplits + sp) * D;
    store_column<D>(a.part_k + at, dk, a.scale, exists);
    store_column<D>(a.part_v + at, dv, 1.f, exists);
  }
}

// Adds the splits of each row in their order: blockIdx.y 0 .. 2 dQ, dK, dV (from `first` on).
template <typename T, int D> __global__ void __launch_bounds__(256) dense_add_kernel(DenseArgs a, int first, int ksplits) {
  constexpr int L = D / 4;
  const int which = first + blockIdx.y;
  const int rows = which == 0 ? a.R : a.Nk, splits = which == 0 ? a.splits : ksplits;
  const int64_t i = (int64_t)blockIdx.x * (256 / L) + threadIdx.x / L;
  const int c = threadIdx.x % L;
  if (i >= (int64_t)a.B * a.Hkv * rows) return;
  const int s = (int)(i / rows), r = (int)(i - (int64_t)s * rows), b = s / a.Hkv, hk = s - b * a.Hkv;
  const float *part = (which == 0 ? a.part_q : which == 1 ? a.part_k : a.part_v) + i * splits * D + 4 * c;
  float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int j = 0; j < splits; ++j) {
    const float4 z = *reinterpret_cast<const float4 *>(part + (int64_t)j * D);
    y.x += z.x;
    y.y += z.y;
    y.z += z.z;
    y.w += z.w;
  }
  const DenseMat &m = which == 0 ? a.dq : which == 1 ? a.dk : a.dv;
  const int tok = which == 0 ? div_group(a, r) : r, head = which == 0 ? hk * a.G + r - tok * a.G : hk;
  T *out = (T *)(m.p + b * m.b + head * m.h + (int64_t)tok * m.n) + 4 * c;
  out[0] = from_f32<T>(y.x);
  out[1] = from_f32<T>(y.y);
  out[2] = from_f32<T>(y.z);
  out[3] = from_f32<T>(y.w);
}

namespace {
template <typename T, int D> hipError_t backward_t(const DenseArgs &a, const DenseBwdPlan &p, hipStream_t st) {
  const unsigned S = (unsigned)(a.B * a.Hkv);
  dense_dq_kernel<T, D><<<dim3(S * p.qtiles * p.qsplits), 256, 0, st>>>(a);
  hipError_t e = launched("dense_dq_kernel", st);
  if (e != hipSuccess) return e;
  dense_dkv_kernel<T, D><<<dim3(S * p.ktiles * p.ksplits), 256, 0, st>>>(a, p.ktiles, p.ksplits);
  e = launched("dense_dkv_kernel", st);
  if (e != hipSuccess || (p.qsplits == 1 && p.ksplits == 1)) return e;
  const int first = p.qsplits > 1 ? 0 : 1, last = p.ksplits > 1 ? 2 : 0;
  const int64_t rows = (int64_t)S * (first == 0 && (last == 0 || a.R > a.Nk) ? a.R : a.Nk), per = 256 / (D / 4);
  dense_add_kernel<T, D><<<dim3((unsigned)((rows + per - 1) / per), last - first + 1), 256, 0, st>>>(a, first, p.ksplits);
  return launched("dense_add_kernel", st);
}
}  // namespace

hipError_t launch_dense_backward(const mita_dense_cfg_t &c, const void *q, const void *k, const void *v, const void *o,
                                 const float *lse, const void *dO, const int32_t *q_len, const int32_t *k_len, void *dq,
                                 void *dk, void *dv, void *ws, hipStream_t st) {
  DenseArgs a = dense_args(c);
  const DenseBwdPlan p = dense_bwd_plan(c);
  const DenseBwdLayout L = dense_backward_layout(c);
  a.q.p = (const char *)q;
  a.k.p = (const char *)k;
  a.v.p = (const char *)v;
  a.o.p = (const char *)o;
  a.dO.p = (const char *)dO;
  a.dq.p = (const char *)dq;
  a.dk.p = (const char *)dk;
  a.dv.p = (const char *)dv;
  a.q_len = q_len;
  a.k_len = k_len;
  a.lse = const_cast<float *>(lse);
  a.tiles = p.qtiles;
  a.splits = p.qsplits;
  char *w = (char *)ws;
  a.row_lse = (float *)(w + L.lse);
  a.row_D = (float *)(w + L.D);
  a.part_q = (float *)(w + L.part_q);
  a.part_k = (float *)(w + L.part_k);
  a.part_v = (float *)(w + L.part_v);
  if (c.dtype == MITA_F32) return c.d == 64 ? backward_t<float, 64>(a, p, st) : backward_t<float, 128>(a, p, st);
  return c.d == 64 ? backward_t<bf16_t, 64>(a, p, st) : backward_t<bf16_t, 128>(a, p, st);
}

}  // namespace mita
