// dense_forward.hip - dense attention: o = softmax(scale Q K^T) V over the keys
// each query sees, and the rows' log-sum-exps, with an online softmax.
//
// The query heads of one key head are rows of one matrix (row r: query r / G of
// head r % G), so grouped heads share the staged keys, and one token of many
// heads fills a tile.
#include "dense.hpp"
#include "kernels.hpp"
#include "layer_check.hpp"

namespace mita {

// A wave's 32 rows: o^T accumulators, the reference -m of the weights exp2(z - m)
// (log2 units), the raw dot above which the reference moves, and the lane's part
// of the weight sum.
template <int D> struct DenseState {
  f32x16 o[D / 32];
  float nm, thr, l;
  __device__ __forceinline__ void init() {
#pragma unroll
    for (int i = 0; i < D / 32; ++i) o[i] = splat16(0.f);
    nm = 0.f;
    thr = -INFINITY;
    l = 0.f;
  }
};

// Scores hidden from the column become -infinity: keys j of the 32 outside [lo, hi).
__device__ __forceinline__ void dense_mask(f32x16 &s, int lo, int hi) {
  const int g = (threadIdx.x & 63) >> 5;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int j = acc_row(i, g);
    s[i] = j >= lo && j < hi ? s[i] : -INFINITY;
  }
}

// The reference moves only where a score passes it by more than RESCALE_LOG2 (and
// at the column's first visible key): any reference gives the same softmax.
// Near DENSE_MAX_LOG2 = 2^27 fp32 numbers are 8 or 16 apart: z - m of the largest
// score is up to 4 off 0, and thr up to 24 + 4 off its place, so that weights reach
// 2^40 at most and their sums stay finite. A larger score makes its row NaN; scores
// below -2^27 weigh nothing, and a row with no others is 0 / 0.
constexpr float DENSE_MAX_LOG2 = 134217728.f;
template <int D> __device__ __forceinline__ void dense_reference(DenseState<D> &st, const f32x16 &s, float sl2) {
  float mx = s[0];
#pragma unroll
  for (int i = 1; i < 16; ++i) mx = fmaxf(mx, s[i]);
  if (__ballot(mx > st.thr)) {
    const float cm = column_max(mx);
    const bool up = cm > st.thr;
    const float top = cm * sl2;
    const float m = !up ? -st.nm : top > DENSE_MAX_LOG2 ? NAN : fmaxf(top, -DENSE_MAX_LOG2);
    const float alpha = st.thr == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(-st.nm - m);
    st.nm = -m;
    st.thr = up ? (m + RESCALE_LOG2) * __builtin_amdgcn_rcpf(sl2) : st.thr;
    st.l *= alpha;
#pragma unroll
    for (int i = 0; i < D / 32; ++i) st.o[i] *= alpha;
  }
}

// The weights exp2(s sl2 - m) as they multiply the values; their sum takes them
// before that rounding (the rounded ones would put the log-sum-exp off by about
// 2^-9 over the root of the number of keys).
template <typename T, int D>
__device__ __forceinline__ ColsOperand<T> dense_weights(DenseState<D> &st, f32x16 s, float sl2) {
  float l[2] = {st.l, 0.f};
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    s[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i], sl2, st.nm));
    l[i & 1] += s[i];
  }
  st.l = l[0] + l[1];
  return ColsOperand<T>(s);
}

// 1 / l of a row's weight sum l, and its log-sum-exp for the reference m (log2
// units). `none`: the row has no keys here, 0 and -infinity. A row that has keys but
// no weight, or weights that are NaN, is NaN.
__device__ __forceinline__ void dense_norm(bool none, float l, float m, float &inv, float &lse2) {
  inv = none ? 0.f : 1.f / l;
  lse2 = none ? -INFINITY : l == 0.f ? NAN : __builtin_amdgcn_logf(l) + m;
}

// The log-sum-exp of a split without weight whose row sees keys, here or elsewhere.
constexpr float DENSE_NO_WEIGHT = -3.4028235e38f;

// A column's result (weight sum l, reference m in log2 units) to o and lse, or to
// its split's place. `sees`: the row sees keys.
template <typename T, int D>
__device__ __forceinline__ void dense_write(const DenseArgs &a, const DenseSlice &x, int s, int sp, int row, int tok,
                                            int head, bool exists, bool sees, float l, float m, f32x16 (&o)[D / 32]) {
  const bool none = !sees || (a.splits > 1 && l == 0.f);
  if (none) {
#pragma unroll
    for (int i = 0; i < D / 32; ++i) o[i] = splat16(0.f);
  }
  float inv, lse2;
  dense_norm(none, l, m, inv, lse2);
  if (none && sees) lse2 = DENSE_NO_WEIGHT;
  const bool first = exists && (threadIdx.x & 63) < 32;
  if (a.splits == 1) {
    store_column<D>((T *)(a.o.p + x.b * a.o.b + head * a.o.h + (int64_t)tok * a.o.n), o, inv, exists);
    if (a.lse && first) a.lse[((int64_t)x.b * a.H + head) * a.N + tok] = lse2 * 0.69314718055994531f;
  } else {
    const int64_t at = ((int64_t)s * a.R + row) * a.splits + sp;
    store_column<D>(a.part_o + at * D, o, inv, exists);
    if (first) a.part_lse[at] = lse2;
  }
}

// Bound by the MFMA and VALU issue of long sequences (per score 4 D flops against
// one exp2, a quarter-rate instruction, and about three full-rate ones). A wave
// forms the scores of the next tile while it weighs the present one, so that its
// MFMAs have VALU work to run beside, and two waves share a SIMD (three in bf16 at
// d = 64).
// Tiles seen whole have a loop of their own: with masked and unmasked steps in one
// loop the accumulators were copied on every step. 16 heads of 16384 tokens, d = 128:
// 1.96 - 2.04 ms, 1.1 PFLOP/s (a large bf16 matrix product reaches 1.31); with one
// loop and the tile's own scores first 2.41 ms. 24 heads, d = 64: 1.84 ms, 0.9
// PFLOP/s: half the MFMA work for the same VALU work per score.
template <typename T, int D>
__global__ void __launch_bounds__(256, sizeof(T) * D <= 256 ? 2 : 1) dense_fwd_kernel(DenseArgs a) {
  using RT = RowTile<T, D>;
  constexpr int TR = RT::TR, HT = TR / 32, BYTES = TR * RT::RB;
  __shared__ __align__(16) char ldsK[2 * BYTES];
  __shared__ __align__(16) char ldsV[2 * BYTES];
  int s, item;
  dense_block(blockIdx.x, a.B * a.Hkv, a.tiles * a.splits, s, item);
  const int sp = item % a.splits;
  const int tile = a.tiles - 1 - item / a.splits;  // causal: the longest first
  const DenseSlice x = dense_slice(a, s);
  const int n = threadIdx.x & 31;
  const int w = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);

  // the keys of the block
  const int b0 = div_group(a, tile * DENSE_TQ);
  const int b1 = min(div_group(a, min(tile * DENSE_TQ + DENSE_TQ, a.R) - 1), x.qlen - 1);
  const int kbeg = first_key(a, x, b0), kend = b0 <= b1 ? end_key(a, x, b1) : 0;
  const int nt = kend > kbeg ? (kend - kbeg + TR - 1) / TR : 0;
  const int per = (nt + a.splits - 1) / a.splits;
  const int t0 = sp * per, t1 = min(nt, t0 + per);
  // of these, tiles that every row sees whole: keys [first_key(b1), end_key(b0))
  const TileOrder order(t0, t1, (first_key(a, x, b1) - kbeg + TR - 1) / TR, max(0, end_key(a, x, b0) - kbeg) / TR);

  TileAddr<T, D> ad;
  ad.init();
  TileCopy<T, D, 4> copy;
  copy.init();
  const uint32_t offK = copy.row0 * a.k.n, offV = copy.row0 * a.v.n;
  const char *kb = a.k.p + x.b * a.k.b + x.hk * a.k.h, *vb = a.v.p + x.b * a.v.b + x.hk * a.v.h;
  const uint32_t atK = lds_at(ldsK), atV = lds_at(ldsV);
  auto issue_k = [&](int p) {
    const int k0 = kbeg + order.at(p) * TR;
    copy.issue(atK + (p & 1) * BYTES, kb, k0, a.k.n, offK, x.klen - k0);
  };
  auto issue_v = [&](int p) {
    const int k0 = kbeg + order.at(p) * TR;
    copy.issue(atV + (p & 1) * BYTES, vb, k0, a.v.n, offV, x.klen - k0);
  };
  if (order.total > 0) issue_k(0);

  // the lane's row
  const int row = tile * DENSE_TQ + 32 * w + n;
  const int tok = div_group(a, row), head = x.hk * a.G + row - tok * a.G;
  const bool exists = row < a.R, valid = exists && tok < x.qlen;
  Column<T, D> q;
  q.load(a.q.p + x.b * a.q.b + head * a.q.h + (int64_t)tok * a.q.n, valid);
  const int lo = valid ? first_key(a, x, tok) : 0, hi = valid ? end_key(a, x, tok) : 0;
  const bool sees = lo < hi;
  // keys that some row of the wave sees (none: the wave only copies)
  const int wr = tile * DENSE_TQ + 32 * w;
  const int w0 = wr < a.R ? div_group(a, wr) : x.qlen, w1 = min(div_group(a, min(wr + 32, a.R) - 1), x.qlen - 1);
  const int wlo = first_key(a, x, w0), whi = w0 <= w1 ? end_key(a, x, w1) : 0;
  DenseState<D> st;
  st.init();

  f32x16 sc[HT];
  auto scores = [&](int p, int h) { return tile_rows<D>(ldsK + (p & 1) * BYTES, ad, h, q, splat16(0.f)); };
  auto next = [&](int p) {
    tile_barrier();
    if (p + 2 < order.total) issue_k(p + 2);
    if (p + 1 < order.total) issue_v(p + 1);
  };
  auto tiles = [&](int p, int end, auto masked) {
    for (; p < end; ++p) {
      next(p);
      const int k0 = kbeg + order.at(p) * TR;
#pragma unroll
      for (int h = 0; h < HT; ++h) {
        f32x16 now = sc[h];
        const int kh = k0 + 32 * h;
        if (decltype(masked)::value) {
          if (kh >= whi || kh + 32 <= wlo) {
            sc[h] = scores(p + 1, h);
            continue;
          }
          dense_mask(now, lo - kh, hi - kh);
        }
        dense_reference<D>(st, now, a.sl2);
        sc[h] = scores(p + 1, h);  // (past the last tile: unused)
        tile_cols<D>(st.o, ldsV + (p & 1) * BYTES, ad, h, dense_weights<T, D>(st, now, a.sl2));
      }
    }
  };
  if (order.total > 0) {
    tile_barrier();
    if (order.total > 1) issue_k(1);
    issue_v(0);
    if (w0 <= w1) {
#pragma unroll
      for (int h = 0; h < HT; ++h) sc[h] = scores(0, h);
      tiles(0, order.nfull, std::false_type{});
      tiles(order.nfull, order.total, std::true_type{});
    } else {
      for (int p = 0; p < order.total; ++p) next(p);
    }
  }
  dense_write<T, D>(a, x, s, sp, row, tok, head, exists, sees, column_sum(st.l), -st.nm, st.o);
}

// Few rows (single tokens, small problems): the four waves of a workgroup share 32
// rows and take the block's 32-key tiles in turn, each with tiles of its own in LDS
// and no barrier, so that every wave streams keys. Bound by the bytes of K and V,
// or in small problems by one wave's chain over its quarter of the keys: a wave
// refills its K tile while the values multiply and its V tile while the next scores
// form. The waves' results are joined at the end by their reference maxima. One
// token of 24 sequences of up to 16384 keys, 8 key heads, d = 128: 207 us with the
// join, 5.5 TB/s (plain reads reach 6.2); 8 causal heads of 1000 tokens over 2 key
// heads, d = 64: 10 us, 18.5 with the 128-row tiles of dense_fwd_kernel.
template <typename T, int D> struct FewTile {
  using RT = RowTile<T, D>;
  static constexpr int NW = 4, BYTES = 32 * RT::RB, NI = 32 / RT::RPI;  // copies per tile and wave
};

// The wave's next tile: rows past the last repeat it.
template <typename T, int D>
__device__ __forceinline__ void few_copy(uint32_t tile, const char *base, int first, uint32_t stride, int nrows) {
  using RT = RowTile<T, D>;
  const int lane = threadIdx.x & 63;
  const char *src = base + (int64_t)first * stride;
#pragma unroll
  for (int j = 0; j < FewTile<T, D>::NI; ++j) {
    const int r = j * RT::RPI + lane / RT::CPR;
    copy16_unwaited(src, (uint32_t)min(r, nrows - 1) * stride + (uint32_t)(((lane % RT::CPR) ^ RT::swz(r)) << 4),
                    tile + j * 1024);
  }
}

// (bf16 at d = 64: four workgroups fit a CU's LDS, and 128 registers suffice)
template <typename T, int D>
__global__ void __launch_bounds__(256, sizeof(T) * D == 128 ? 4 : sizeof(T) * D == 256 ? 2 : 1) dense_few_kernel(DenseArgs a) {
  using RT = RowTile<T, D>;
  using FT = FewTile<T, D>;
  __shared__ __align__(16) char ldsK[FT::NW * FT::BYTES];
  __shared__ __align__(16) char ldsV[FT::NW * FT::BYTES];
  __shared__ float join_m[FT::NW][32], join_l[FT::NW][32];
  int s, item;
  dense_block(blockIdx.x, a.B * a.Hkv, a.tiles * a.splits, s, item, false);
  const int sp = item % a.splits;
  const int tile = a.tiles - 1 - item / a.splits;  // causal: the longest first
  const DenseSlice x = dense_slice(a, s);
  const int lane = threadIdx.x & 63, n = lane & 31;
  const int w = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);

  const int row = 32 * tile + n;
  const int tok = div_group(a, row), head = x.hk * a.G + row - tok * a.G;
  const bool exists = row < a.R, valid = exists && tok < x.qlen;
  const int b0 = div_group(a, 32 * tile), b1 = min(div_group(a, min(32 * tile + 32, a.R) - 1), x.qlen - 1);
  const int kbeg = first_key(a, x, b0), kend = b0 <= b1 ? end_key(a, x, b1) : 0;
  const int nt = kend > kbeg ? (kend - kbeg + 31) / 32 : 0;
  const int per = (nt + a.splits - 1) / a.splits;
  const int t1 = min(nt, (sp + 1) * per);
  const char *kb = a.k.p + x.b * a.k.b + x.hk * a.k.h, *vb = a.v.p + x.b * a.v.b + x.hk * a.v.h;
  const char *Kt = ldsK + w * FT::BYTES, *Vt = ldsV + w * FT::BYTES;
  const uint32_t atK = lds_at(ldsK) + w * FT::BYTES, atV = lds_at(ldsV) + w * FT::BYTES;

  Column<T, D> q;
  q.load(a.q.p + x.b * a.q.b + head * a.q.h + (int64_t)tok * a.q.n, valid);
  const int lo = valid ? first_key(a, x, tok) : 0, hi = valid ? end_key(a, x, tok) : 0;
  const bool sees = lo < hi;
  // keys in [lo1, hi0) are seen by every query
  const int lo1 = first_key(a, x, b1), hi0 = end_key(a, x, b0);
  TileAddr<T, D> ad;
  ad.init();
  DenseState<D> st;
  st.init();
  int t = sp * per + w;
  if (t < t1) {
    const int k0 = kbeg + 32 * t;
    few_copy<T, D>(atK, kb, k0, a.k.n, x.klen - k0);
    few_copy<T, D>(atV, vb, k0, a.v.n, x.klen - k0);
  }
  wait_copies<0>();  // (the queries too: no wait for them inside the loop)
  for (; t < t1; t += FT::NW) {
    const int k0 = kbeg + 32 * t, k1 = k0 + 32 * FT::NW;
    const bool more = t + FT::NW < t1;
    wait_copies<FT::NI>();  // K is here, V may be in flight
    f32x16 sc = tile_rows<D>(Kt, ad, 0, q, splat16(0.f));
    wait_lds();  // and has been read
    if (more) few_copy<T, D>(atK, kb, k1, a.k.n, x.klen - k1);
    if (!(k0 >= lo1 && k0 + 32 <= hi0)) dense_mask(sc, lo - k0, hi - k0);
    dense_reference<D>(st, sc, a.sl2);
    const ColsOperand<T> P = dense_weights<T, D>(st, sc, a.sl2);
    if (more)
      wait_copies<FT::NI>();  // V is here, the next K may be in flight
    else
      wait_copies<0>();
    tile_cols<D>(st.o, Vt, ad, 0, P);
    wait_lds();
    if (more) few_copy<T, D>(atV, vb, k1, a.v.n, x.klen - k1);
  }

  // every wave's sums relative to the common maximum, added in pairs: waves 0 and
  // 2, 1 and 3, then both (element e of a lane's accumulators at 64 e + lane). A wave
  // without weights adds 0; one whose sum is NaN stays in the sum.
  const float l = column_sum(st.l);
  if (lane < 32) join_m[w][n] = l == 0.f ? -INFINITY : -st.nm;
  __syncthreads();  // (also: every wave is done with its tiles)
  float m = join_m[0][n];
#pragma unroll
  for (int i = 1; i < FT::NW; ++i) m = fmaxf(m, join_m[i][n]);
  const float f = l == 0.f ? 0.f : __builtin_amdgcn_exp2f(-st.nm - m);
  if (lane < 32) join_l[w][n] = l * f;
  float *const jk = (float *)ldsK + lane, *const jv = (float *)ldsV + lane;
  auto each = [&](auto &&op) {
#pragma unroll
    for (int i = 0; i < D / 32; ++i)
#pragma unroll
      for (int e = 0; e < 16; ++e) st.o[i][e] = op(st.o[i][e], 16 * i + e);
  };
  each([&](float o, int) { return f == 0.f ? 0.f : o * f; });
  if (w >= 2) each([&](float o, int e) { return jk[((w - 2) * (D / 2) + e) * 64] = o; });
  __syncthreads();
  if (w < 2) each([&](float o, int e) { return o + jk[(w * (D / 2) + e) * 64]; });
  if (w == 1) each([&](float o, int e) { return jv[e * 64] = o; });
  __syncthreads();
  if (w >= 1) return;
  each([&](float o, int e) { return o + jv[e * 64]; });
  dense_write<T, D>(a, x, s, sp, row, tok, head, exists, sees,
                    (join_l[0][n] + join_l[2][n]) + (join_l[1][n] + join_l[3][n]), m, st.o);
}

// Joins a row's splits by their log-sum-exps: D / 4 lanes per row.
template <typename T, int D> __global__ void __launch_bounds__(256) dense_join_kernel(DenseArgs a) {
  constexpr int L = D / 4;
  const int64_t i = (int64_t)blockIdx.x * (256 / L) + threadIdx.x / L;
  const int c = threadIdx.x % L;
  if (i >= (int64_t)a.B * a.Hkv * a.R) return;
  const int s = (int)(i / a.R), row = (int)(i - (int64_t)s * a.R);
  const int b = s / a.Hkv, tok = div_group(a, row), head = (s - b * a.Hkv) * a.G + row - tok * a.G;
  float m = -INFINITY, l = 0.f;
  bool sees = false;
  for (int j = 0; j < a.splits; ++j) {
    const float z = a.part_lse[i * a.splits + j];
    sees |= z != -INFINITY;
    m = fmaxf(m, z);
  }
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int j = 0; j < a.splits; ++j) {
    const float z = a.part_lse[i * a.splits + j];
    if (z <= DENSE_NO_WEIGHT) continue;
    const float f = __builtin_amdgcn_exp2f(z - m);
    const float4 y = *reinterpret_cast<const float4 *>(a.part_o + (i * a.splits + j) * D + 4 * c);
    l += f;
    o.x += f * y.x;
    o.y += f * y.y;
    o.z += f * y.z;
    o.w += f * y.w;
  }
  float inv, lse2;
  dense_norm(!sees, l, m, inv, lse2);
  T *out = (T *)(a.o.p + b * a.o.b + head * a.o.h + (int64_t)tok * a.o.n) + 4 * c;
  out[0] = from_f32<T>(o.x * inv);
  out[1] = from_f32<T>(o.y * inv);
  out[2] = from_f32<T>(o.z * inv);
  out[3] = from_f32<T>(o.w * inv);
  if (a.lse && c == 0) a.lse[((int64_t)b * a.H + head) * a.N + tok] = lse2 * 0.69314718055994531f;
}

DenseArgs dense_args(const mita_dense_cfg_t &c) {
  DenseArgs a{};
  const size_t e = elem_bytes(c);
  auto mat = [&](const mita_strides_t &s0, bool key) {
    const mita_strides_t s = key ? strides_or(s0, c.H_kv, c.N_k, c.d) : strides_or(s0, c.H, c.N, c.d);
    const int64_t n = key ? c.N_k : c.N;
    return DenseMat{nullptr, s.b * (int64_t)e, s.h * (int64_t)e, n > 1 ? (uint32_t)(s.n * e) : 0u};
  };
  a.q = mat(c.q, false);
  a.k = mat(c.k, true);
  a.v = mat(c.v, true);
  a.o = mat(c.o, false);
  a.dO = mat(c.dO, false);
  a.dq = mat(c.dq, false);
  a.dk = mat(c.dk, true);
  a.dv = mat(c.dv, true);
  a.B = c.B;
  a.H = c.H;
  a.Hkv = c.H_kv;
  a.G = group(c);
  a.N = c.N;
  a.Nk = c.N_k;
  a.R = (int)dense_rows(c);
  a.left = window(c.left);
  a.right = window(c.right);
  a.magic = ((uint64_t)1 << 40) / (uint64_t)a.G + 1;
  a.scale = eff_scale(c);
  a.sl2 = a.scale * LOG2E;
  a.near = true;
  for (const DenseMat *m : {&a.q, &a.dO})
    a.near = a.near && (a.G - 1) * m->h + (int64_t)a.N * m->n + 1024 < ((int64_t)1 << 32);
  return a;
}

namespace {
template <typename T, int D> hipError_t forward_t(const DenseArgs &a, bool few, hipStream_t st) {
  const dim3 grid((unsigned)(a.B * a.Hkv) * a.tiles * a.splits);
  if (few)
    dense_few_kernel<T, D><<<grid, 256, 0, st>>>(a);
  else
    dense_fwd_kernel<T, D><<<grid, 256, 0, st>>>(a);
  hipError_t e = launched(few ? "dense_few_kernel" : "dense_fwd_kernel", st);
  if (e != hipSuccess || a.splits == 1) return e;
  const int64_t rows = (int64_t)a.B * a.Hkv * a.R, per = 256 / (D / 4);
  dense_join_kernel<T, D><<<dim3((unsigned)((rows + per - 1) / per)), 256, 0, st>>>(a);
  return launched("dense_join_kernel", st);
}
}  // namespace

hipError_t launch_dense_forward(const mita_dense_cfg_t &c, const void *q, const void *k, const void *v,
                                const int32_t *q_len, const int32_t *k_len, void *o, float *lse, void *ws,
                                hipStream_t st) {
  DenseArgs a = dense_args(c);
  const DensePlan p = dense_plan(c);
  const DenseFwdLayout L = dense_forward_layout(c);
  a.q.p = (const char *)q;
  a.k.p = (const char *)k;
  a.v.p = (const char *)v;
  a.o.p = (const char *)o;
  a.q_len = q_len;
  a.k_len = k_len;
  a.lse = lse;
  a.tiles = p.tiles;
  a.splits = p.splits;
  if (p.splits > 1) {
    a.part_o = (float *)((char *)ws + L.part_o);
    a.part_lse = (float *)((char *)ws + L.part_lse);
  }
  if (c.dtype == MITA_F32) return c.d == 64 ? forward_t<float, 64>(a, p.few, st) : forward_t<float, 128>(a, p.few, st);
  return c.d == 64 ? forward_t<bf16_t, 64>(a, p.few, st) : forward_t<bf16_t, 128>(a, p.few, st);
}

}  // namespace mita
