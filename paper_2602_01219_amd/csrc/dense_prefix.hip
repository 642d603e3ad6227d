// dense_prefix.hip - dense attention of sequences that share prefixes: each query
// attends over its prefix's keys and its sequence's own, with an online softmax.
//
// Two ways. Where a sequence's rows fill tiles, a row tile goes through the prefix's
// keys and then its own: one softmax, no parts, and the sequences of a prefix find its
// keys in L2. Where they are few (single tokens) that would read the prefix once per
// sequence: there the rows of all sequences of a prefix are rows of one matrix that goes
// through its keys, split over the workgroups, others take each sequence's own keys in
// the same launch, and a second one joins a row's parts by their log-sum-exps.
//
// Prompts are bound by the MFMA and VALU issue, as dense_fwd_kernel: 32 sequences of 512
// tokens, 16 heads of 4 key heads, behind 8000 keys, d = 128: 1005 us, 1.10 PFLOP/s. Single
// tokens are bound by the bytes of the keys and by latencies: a token of 32 sequences, 32
// heads of 8 key heads, behind 32768 keys and up to 1024 of their own, d = 128: 46 us and
// 5 for the join (228 MB: 37 at 6.2 TB/s); of these 3 us pass before the first copy
// and 2.5 with the writing of the parts, 64 KB of each workgroup.
#include "dense.hpp"
#include "dense_softmax.hpp"
#include "kernels.hpp"
#include "layer_check.hpp"

namespace mita {

namespace {

struct PrefixArgs {
  DenseMat q, kp, vp, k, v, o;  // o is written
  const int32_t *q_len, *p_len, *k_len;
  float *lse;                // [B, H, N] or NULL
  float *part_o, *part_lse;  // [rows, slots (, D)], if slots > 1
  int B, Bp, S, H, Hkv, G, N, P, Nk;
  int rows;                  // N * G: of a sequence
  int left, right;
  uint64_t magic, magic_rows;  // 2^40 / G + 1, 2^40 / rows + 1
  float sl2;                 // scale * log2(e)
  int tiles, splits, otiles, osplits, slots;
  int blocks;                // of the prefixes' part
};

// r / n for r n < 2^40 and magic = 2^40 / n + 1, which errs by less than r / 2^40 of a
// quotient step, below 1 / n.
__device__ __forceinline__ int div_by(uint64_t magic, int r) { return (int)(((uint64_t)(uint32_t)r * magic) >> 40); }

// What a workgroup works on: rows of nb sequences from b0 on (of one prefix, of which
// row r is row r % rows of sequence b0 + r / rows), from row0 on, and the keys of their
// prefix, or their own, or both one after the other; of these the sp-th of `splits` parts.
struct PrefixItem {
  int bp, hk, b0, nb, row0;
  bool pre, own;
  int sp, splits, slot;
};

// A lane's row: its token, the keys it sees [lo, hi) with the own ones behind the
// prefix's, and those there are.
struct PrefixRow {
  int b, tok, head, in;  // in: row of its sequence
  int pl, kl, lo, hi;
  bool exists, valid;
};
__device__ __forceinline__ void sees_keys(const PrefixArgs &a, int p, int m, int &lo, int &hi) {
  lo = max(0, p - a.left);
  hi = min(m, p + a.right + 1);
}
__device__ __forceinline__ PrefixRow prefix_row(const PrefixArgs &a, const PrefixItem &it, int row) {
  PrefixRow x;
  x.exists = row < it.nb * a.rows;
  const int bs = it.nb > 1 ? min(div_by(a.magic_rows, row), it.nb - 1) : 0;
  x.b = it.b0 + bs;
  x.in = row - bs * a.rows;
  x.tok = div_by(a.magic, x.in);
  x.head = it.hk * a.G + x.in - x.tok * a.G;
  const int ql = a.q_len ? min(max(a.q_len[x.b], 0), a.N) : a.N;
  x.kl = a.k_len ? min(max(a.k_len[x.b], 0), a.Nk) : a.Nk;
  x.pl = a.p_len ? min(max(a.p_len[it.bp], 0), a.P) : a.P;
  x.valid = x.exists && x.tok < ql;
  sees_keys(a, x.pl + x.kl - ql + x.tok, x.pl + x.kl, x.lo, x.hi);
  if (!x.valid) x.lo = x.hi = 0;
  return x;
}

// Of the rows that there are: the first key that any sees, the first that all see, the
// end of those that all see and of those that any sees.
struct PrefixBounds {
  int lo0, lo1, hi0, hi1;
};
__device__ __forceinline__ int wave_min_i32(int x) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) x = min(x, __shfl_xor(x, o));
  return x;
}
__device__ __forceinline__ int wave_max_i32(int x) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) x = max(x, __shfl_xor(x, o));
  return x;
}
constexpr int PREFIX_FAR = 1 << 28;
__device__ __forceinline__ PrefixBounds wave_bounds(const PrefixRow &x) {
  PrefixBounds w;
  w.lo0 = __builtin_amdgcn_readfirstlane(wave_min_i32(x.valid ? x.lo : PREFIX_FAR));
  w.lo1 = __builtin_amdgcn_readfirstlane(wave_max_i32(x.valid ? x.lo : 0));
  w.hi0 = __builtin_amdgcn_readfirstlane(wave_min_i32(x.valid ? x.hi : PREFIX_FAR));
  w.hi1 = __builtin_amdgcn_readfirstlane(wave_max_i32(x.valid ? x.hi : 0));
  return w;
}

// The tiles of TR keys that a workgroup's rows see some of: np of the prefix from key
// pb on, then those of the sequence's own from ob on.
template <int TR> struct PrefixTiles {
  int pl, kl, pb, ob, np, total;
  __device__ __forceinline__ PrefixTiles(const PrefixItem &it, int pl_, int kl_, const PrefixBounds &w) {
    pl = __builtin_amdgcn_readfirstlane(pl_);
    kl = __builtin_amdgcn_readfirstlane(kl_);
    pb = min(w.lo0, pl);
    ob = min(max(w.lo0 - pl, 0), kl);
    const int pe = it.pre ? min(w.hi1, pl) : pb, oe = it.own ? min(w.hi1 - pl, kl) : ob;
    np = pe > pb ? (pe - pb + TR - 1) / TR : 0;
    total = np + (oe > ob ? (oe - ob + TR - 1) / TR : 0);
  }
  __device__ __forceinline__ bool own(int t) const { return t >= np; }
  __device__ __forceinline__ int key(int t) const { return t >= np ? ob + (t - np) * TR : pb + t * TR; }
};

// Tiles [t0, t1) in the order a workgroup takes them: those seen whole by every row
// first, of the prefix and then the own ones, then the others.
struct PrefixOrder {
  int s0, s1, s2, s3, s4, s5, e0, e1, e2, e3, e4;  // position p of segment i (up to ei) is tile si + p
  int nfull, total;
  template <int TR>
  __device__ __forceinline__ PrefixOrder(const PrefixTiles<TR> &x, int t0, int t1, const PrefixBounds &w) {
    // the prefix's whole tiles [a0, a1), the own ones [b0, b1), as tile numbers
    auto up = [](int y) { return y > 0 ? (y + TR - 1) / TR : 0; };
    auto down = [](int y) { return y > 0 ? y / TR : 0; };
    const int m = max(t0, min(x.np, t1));
    const int a1 = max(t0, min(down(min(w.hi0, x.pl) - x.pb), m));
    const int a0 = min(max(up(w.lo1 - x.pb), t0), a1);
    const int b1 = max(m, min(x.np + down(w.hi0 - x.pl - x.ob), t1));
    const int b0 = min(max(x.np + up(w.lo1 - x.pl - x.ob), m), b1);
    s0 = a0, e0 = a1 - a0;
    s1 = b0 - e0, e1 = e0 + b1 - b0;
    s2 = t0 - e1, e2 = e1 + a0 - t0;
    s3 = a1 - e2, e3 = e2 + m - a1;
    s4 = m - e3, e4 = e3 + b0 - m;
    s5 = b1 - e4;
    nfull = e1;
    total = max(0, t1 - t0);
  }
  __device__ __forceinline__ int at(int p) const {
    return p + (p < e0 ? s0 : p < e1 ? s1 : p < e2 ? s2 : p < e3 ? s3 : p < e4 ? s4 : s5);
  }
};

// A column's result (weight sum l, reference m in log2 units) to o and lse, or to
// its slot (dense_write of dense_forward.hip, with a row's parts in `slots` places).
template <typename T, int D>
__device__ __forceinline__ void prefix_write(const PrefixArgs &a, const PrefixItem &it, const PrefixRow &x, float l,
                                             float m, f32x16 (&o)[D / 32]) {
  const bool sees = x.lo < x.hi, none = !sees || (a.slots > 1 && l == 0.f);
  if (none) {
#pragma unroll
    for (int i = 0; i < D / 32; ++i) o[i] = splat16(0.f);
  }
  float inv, lse2;
  dense_norm(none, l, m, inv, lse2);
  if (none && sees) lse2 = DENSE_NO_WEIGHT;
  const bool first = x.exists && (threadIdx.x & 63) < 32;
  if (a.slots == 1) {
    store_column<D>((T *)(a.o.p + x.b * a.o.b + x.head * a.o.h + (int64_t)x.tok * a.o.n), o, inv, x.exists);
    if (a.lse && first) a.lse[((int64_t)x.b * a.H + x.head) * a.N + x.tok] = lse2 * 0.69314718055994531f;
  } else {
    const int64_t at = (((int64_t)x.b * a.Hkv + it.hk) * a.rows + x.in) * a.slots + it.slot;
    store_column<D>(a.part_o + at * D, o, inv, x.exists);
    if (first) a.part_lse[at] = lse2;
  }
}

// A value that is the same for the whole wave, as a scalar.
__device__ __forceinline__ const char *scalar(const char *p) {
  const uint64_t x = (uint64_t)(uintptr_t)p;
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)x), hi = __builtin_amdgcn_readfirstlane((uint32_t)(x >> 32));
  return (const char *)(uintptr_t)((uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ uint32_t scalar(uint32_t x) { return __builtin_amdgcn_readfirstlane(x); }
template <typename T, int D> __device__ __forceinline__ const char *key_base(const DenseMat &m, int b, int h) {
  return m.p + b * m.b + h * m.h;
}

// 128 rows, 32 per wave, which share tiles of 64 (fp32: 32) keys: a wave forms the scores
// of the next tile while it weighs the present one, as dense_fwd_kernel does.
template <typename T, int D, bool ONCE>
__device__ __forceinline__ void prefix_tile(const PrefixArgs &a, const PrefixItem &it, char *ldsK, char *ldsV,
                                            PrefixBounds *join) {
  using RT = RowTile<T, D>;
  constexpr int TR = RT::TR, HT = TR / 32, BYTES = TR * RT::RB;
  const int n = threadIdx.x & 31;
  const int w = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const PrefixRow x = prefix_row(a, it, it.row0 + 32 * w + n);
  Column<T, D> q;
  q.load(a.q.p + x.b * a.q.b + x.head * a.q.h + (int64_t)x.tok * a.q.n, x.valid);
  const PrefixBounds mine = wave_bounds(x);
  if ((threadIdx.x & 63) == 0) join[w] = mine;
  __syncthreads();
  PrefixBounds all = join[0];
#pragma unroll
  for (int i = 1; i < 4; ++i) {
    all.lo0 = min(all.lo0, join[i].lo0);
    all.lo1 = max(all.lo1, join[i].lo1);
    all.hi0 = min(all.hi0, join[i].hi0);
    all.hi1 = max(all.hi1, join[i].hi1);
  }
  all.lo0 = __builtin_amdgcn_readfirstlane(all.lo0);
  all.lo1 = __builtin_amdgcn_readfirstlane(all.lo1);
  all.hi0 = __builtin_amdgcn_readfirstlane(all.hi0);
  all.hi1 = __builtin_amdgcn_readfirstlane(all.hi1);
  const PrefixTiles<TR> tl(it, x.pl, x.kl, all);
  const int per = (tl.total + it.splits - 1) / it.splits;
  const PrefixOrder order(tl, min(it.sp * per, tl.total), min(tl.total, it.sp * per + per), all);

  TileAddr<T, D> ad;
  ad.init();
  TileCopy<T, D, 4, ONCE> copy;
  copy.init();
  const char *kpb = key_base<T, D>(a.kp, it.bp, it.hk), *vpb = key_base<T, D>(a.vp, it.bp, it.hk);
  const char *kb = key_base<T, D>(a.k, it.b0, it.hk), *vb = key_base<T, D>(a.v, it.b0, it.hk);
  const uint32_t atK = lds_at(ldsK), atV = lds_at(ldsV);
  auto issue = [&](uint32_t to, int p, const char *pre, uint32_t pre_n, const char *own, uint32_t own_n) {
    const int t = order.at(p), k0 = tl.key(t);
    const bool o = tl.own(t);
    const uint32_t stride = scalar(o ? own_n : pre_n);
    copy.issue(to + (p & 1) * BYTES, scalar((o ? own : pre) + (int64_t)k0 * stride), 0, stride, copy.row0 * stride,
               (o ? tl.kl : tl.pl) - k0);
  };
  auto issue_k = [&](int p) { issue(atK, p, kpb, a.kp.n, kb, a.k.n); };
  auto issue_v = [&](int p) { issue(atV, p, vpb, a.vp.n, vb, a.v.n); };
  if (order.total > 0) issue_k(0);

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
      const int t = order.at(p);
      const int k0 = tl.own(t) ? tl.pl + tl.key(t) : tl.key(t);  // the place of its first key
#pragma unroll
      for (int h = 0; h < HT; ++h) {
        f32x16 now = sc[h];
        if (decltype(masked)::value) {
          const int kh = k0 + 32 * h, last = tl.own(t) ? x.hi : min(x.hi, tl.pl);
          if (kh >= mine.hi1 || kh + 32 <= mine.lo0) {
            sc[h] = scores(p + 1, h);
            continue;
          }
          dense_mask(now, x.lo - kh, last - kh);
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
    if (mine.hi1 > 0) {
#pragma unroll
      for (int h = 0; h < HT; ++h) sc[h] = scores(0, h);
      tiles(0, order.nfull, std::false_type{});
      tiles(order.nfull, order.total, std::true_type{});
    } else {
      for (int p = 0; p < order.total; ++p) next(p);
    }
  }
  prefix_write<T, D>(a, it, x, column_sum(st.l), -st.nm, st.o);
}

// 32 rows whose keys four waves take in turn, 32 at a time, each with tiles of its own in
// LDS and no barrier, as dense_few_kernel does.
template <typename T, int D, bool ONCE>
__device__ __forceinline__ void prefix_few(const PrefixArgs &a, const PrefixItem &it, char *ldsK, char *ldsV,
                                           float (*join_m)[32], float (*join_l)[32]) {
  using FT = FewTile<T, D>;
  const int lane = threadIdx.x & 63, n = lane & 31;
  const int w = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const PrefixRow x = prefix_row(a, it, it.row0 + n);
  Column<T, D> q;
  q.load(a.q.p + x.b * a.q.b + x.head * a.q.h + (int64_t)x.tok * a.q.n, x.valid);
  const PrefixBounds all = wave_bounds(x);
  const PrefixTiles<32> tl(it, x.pl, x.kl, all);
  const int per = (tl.total + it.splits - 1) / it.splits;
  const int t1 = min(tl.total, it.sp * per + per);
  const char *kpb = key_base<T, D>(a.kp, it.bp, it.hk), *vpb = key_base<T, D>(a.vp, it.bp, it.hk);
  const char *kb = key_base<T, D>(a.k, it.b0, it.hk), *vb = key_base<T, D>(a.v, it.b0, it.hk);
  const char *Kt = ldsK + w * FT::BYTES, *Vt = ldsV + w * FT::BYTES;
  const uint32_t atK = lds_at(ldsK) + w * FT::BYTES, atV = lds_at(ldsV) + w * FT::BYTES;
  auto copy_k = [&](int t) {
    const bool o = tl.own(t);
    const int k0 = tl.key(t);
    const uint32_t stride = scalar(o ? a.k.n : a.kp.n);
    few_copy<T, D, ONCE>(atK, scalar((o ? kb : kpb) + (int64_t)k0 * stride), 0, stride, (o ? tl.kl : tl.pl) - k0);
  };
  auto copy_v = [&](int t) {
    const bool o = tl.own(t);
    const int k0 = tl.key(t);
    const uint32_t stride = scalar(o ? a.v.n : a.vp.n);
    few_copy<T, D, ONCE>(atV, scalar((o ? vb : vpb) + (int64_t)k0 * stride), 0, stride, (o ? tl.kl : tl.pl) - k0);
  };
  TileAddr<T, D> ad;
  ad.init();
  DenseState<D> st;
  st.init();
  int t = it.sp * per + w;
  if (t < t1) {
    copy_k(t);
    copy_v(t);
  }
  wait_copies<0>();  // (the queries too: no wait for them inside the loop)
  for (; t < t1; t += FT::NW) {
    const bool more = t + FT::NW < t1;
    wait_copies<FT::NI>();  // K is here, V may be in flight
    f32x16 sc = tile_rows<D>(Kt, ad, 0, q, splat16(0.f));
    wait_lds();  // and has been read
    if (more) copy_k(t + FT::NW);
    const int end = tl.own(t) ? tl.pl + tl.kl : tl.pl, k0 = tl.own(t) ? tl.pl + tl.key(t) : tl.key(t);
    if (!(k0 >= all.lo1 && k0 + 32 <= min(all.hi0, end))) dense_mask(sc, x.lo - k0, min(x.hi, end) - k0);
    dense_reference<D>(st, sc, a.sl2);
    const ColsOperand<T> P = dense_weights<T, D>(st, sc, a.sl2);
    if (more)
      wait_copies<FT::NI>();  // V is here, the next K may be in flight
    else
      wait_copies<0>();
    tile_cols<D>(st.o, Vt, ad, 0, P);
    wait_lds();
    if (more) copy_v(t + FT::NW);
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
  prefix_write<T, D>(a, it, x, (join_l[0][n] + join_l[2][n]) + (join_l[1][n] + join_l[3][n]), m, st.o);
}

// Ways of a launch: a sequence's rows by tiles of 128 or 32 over all their keys, or the
// prefixes' rows by tiles of 128 or 32 and each sequence's by 32.
enum { WAY_TILE, WAY_FEW, WAY_SHARED_TILE, WAY_SHARED_FEW };

template <typename T, int D, int WAY, bool ONCE>
__global__ void __launch_bounds__(256, WAY == WAY_FEW || WAY == WAY_SHARED_FEW ? (sizeof(T) * D == 128 ? 4 : sizeof(T) * D == 256 ? 2 : 1)
                                                                              : sizeof(T) * D <= 256 ? 2 : 1)
    prefix_kernel(PrefixArgs a) {
  using RT = RowTile<T, D>;
  constexpr bool tile = WAY == WAY_TILE || WAY == WAY_SHARED_TILE, shared = WAY == WAY_SHARED_TILE || WAY == WAY_SHARED_FEW;
  constexpr int TILE = 2 * RT::TR * RT::RB, FEW = FewTile<T, D>::NW * FewTile<T, D>::BYTES;
  constexpr int BYTES = WAY == WAY_TILE || TILE > FEW ? TILE : FEW;
  __shared__ __align__(16) char ldsK[BYTES];
  __shared__ __align__(16) char ldsV[BYTES];
  __shared__ union {
    PrefixBounds bounds[4];
    float of[2][FewTile<T, D>::NW][32];
  } join;
  PrefixItem it;
  int unit, part;
  if (!shared) {
    // the sequences of a prefix, and their tiles and splits, on one XCD
    dense_block(blockIdx.x, a.Bp * a.Hkv, a.S * a.tiles * a.splits, unit, part, false);
    it.bp = unit / a.Hkv;
    it.hk = unit - it.bp * a.Hkv;
    it.sp = part % a.splits;
    part /= a.splits;
    // causal: the longest first
    const int t = part / a.S;
    it.b0 = it.bp * a.S + part - t * a.S;
    it.nb = 1;
    it.row0 = (a.tiles - 1 - t) * (tile ? DENSE_TQ : DENSE_FEW);
    it.pre = it.own = true;
    it.splits = a.splits;
    it.slot = it.sp;
  } else if ((int)blockIdx.x < a.blocks) {
    // the row tiles that read the same keys follow one another on one XCD
    dense_block(blockIdx.x, a.Bp * a.Hkv * a.splits, a.tiles, unit, part, false);
    it.sp = unit % a.splits;
    unit /= a.splits;
    it.bp = unit / a.Hkv;
    it.hk = unit - it.bp * a.Hkv;
    it.b0 = it.bp * a.S;
    it.nb = a.S;
    it.row0 = part * (tile ? DENSE_TQ : DENSE_FEW);
    it.pre = true;
    it.own = false;
    it.splits = a.splits;
    it.slot = it.sp;
  } else {
    int id = blockIdx.x - a.blocks;
    it.sp = id % a.osplits;
    id /= a.osplits;
    it.row0 = id % a.otiles * DENSE_FEW;
    id /= a.otiles;
    it.b0 = id / a.Hkv;
    it.hk = id - it.b0 * a.Hkv;
    it.bp = it.b0 / a.S;
    it.nb = 1;
    it.pre = false;
    it.own = true;
    it.splits = a.osplits;
    it.slot = a.splits + it.sp;
  }
  if (tile && (!shared || (int)blockIdx.x < a.blocks))
    prefix_tile<T, D, ONCE>(a, it, ldsK, ldsV, join.bounds);
  else if (WAY != WAY_TILE)
    prefix_few<T, D, ONCE>(a, it, ldsK, ldsV, join.of[0], join.of[1]);
}

// Joins a row's parts by their log-sum-exps. ROWS = 1: a workgroup per row, whose groups
// of D / 4 lanes take the parts in turn and add theirs in a fixed order; else a group per
// row.
template <typename T, int D, int ROWS> __global__ void __launch_bounds__(256) prefix_join_kernel(PrefixArgs a) {
  constexpr int L = D / 4, GROUPS = 256 / L;
  static_assert(ROWS == 1 || ROWS == GROUPS, "a row per workgroup or per group");
  __shared__ float weight[ROWS == 1 ? 2 * PREFIX_MAX_SPLITS : 1];
  __shared__ float4 sums[ROWS == 1 ? GROUPS : 1][L];
  const int c = threadIdx.x % L, g = threadIdx.x / L;
  const int64_t block = (int64_t)blockIdx.y * gridDim.x + blockIdx.x, i = ROWS == 1 ? block : block * ROWS + g;
  if (i >= (int64_t)a.B * a.Hkv * a.rows) return;
  const float *lse = a.part_lse + i * a.slots;
  const float *part = a.part_o + i * a.slots * D + 4 * c;
  float m = -INFINITY, l = 0.f;
  bool sees;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  auto add = [&](float f, const float4 &y) {
    o.x = __builtin_fmaf(f, y.x, o.x);
    o.y = __builtin_fmaf(f, y.y, o.y);
    o.z = __builtin_fmaf(f, y.z, o.z);
    o.w = __builtin_fmaf(f, y.w, o.w);
  };
  if constexpr (ROWS == 1) {
    // every wave forms the weights of all parts, two per lane; parts that weigh nothing hold 0
    const int lane = threadIdx.x & 63;
    const float z0 = lane < a.slots ? lse[lane] : -INFINITY, z1 = lane + 64 < a.slots ? lse[lane + 64] : -INFINITY;
    sees = __ballot(z0 != -INFINITY || z1 != -INFINITY) != 0;
    m = wave_max(fmaxf(z0, z1));  // (passes over NaN, whose weight then is NaN)
    const float f0 = z0 <= DENSE_NO_WEIGHT ? 0.f : __builtin_amdgcn_exp2f(z0 - m);
    const float f1 = z1 <= DENSE_NO_WEIGHT ? 0.f : __builtin_amdgcn_exp2f(z1 - m);
    l = wave_sum(f0 + f1);
    if (threadIdx.x < 64) {
      weight[lane] = f0;
      weight[lane + 64] = f1;
    }
    __syncthreads();
#pragma unroll 4
    for (int j = g; j < a.slots; j += GROUPS) add(weight[j], *reinterpret_cast<const float4 *>(part + j * D));
    sums[g][c] = o;
    __syncthreads();
    if (g > 0) return;
#pragma unroll
    for (int k = 1; k < GROUPS; ++k) add(1.f, sums[k][c]);
  } else {
    sees = false;
    for (int j = 0; j < a.slots; ++j) {
      sees |= lse[j] != -INFINITY;
      m = fmaxf(m, lse[j]);
    }
#pragma unroll 4
    for (int j = 0; j < a.slots; ++j) {
      const float z = lse[j], f = z <= DENSE_NO_WEIGHT ? 0.f : __builtin_amdgcn_exp2f(z - m);
      l += f;
      add(f, *reinterpret_cast<const float4 *>(part + j * D));
    }
  }
  const int s = (int)(i / a.rows), row = (int)(i - (int64_t)s * a.rows);
  const int b = s / a.Hkv, tok = div_by(a.magic, row), head = (s - b * a.Hkv) * a.G + row - tok * a.G;
  float inv, lse2;
  dense_norm(!sees, l, m, inv, lse2);
  T *out = (T *)(a.o.p + b * a.o.b + head * a.o.h + (int64_t)tok * a.o.n) + 4 * c;
  out[0] = from_f32<T>(o.x * inv);
  out[1] = from_f32<T>(o.y * inv);
  out[2] = from_f32<T>(o.z * inv);
  out[3] = from_f32<T>(o.w * inv);
  if (a.lse && c == 0) a.lse[((int64_t)b * a.H + head) * a.N + tok] = lse2 * 0.69314718055994531f;
}

template <typename T, int D> hipError_t forward_t(const PrefixArgs &a, const PrefixPlan &p, hipStream_t st) {
  const dim3 grid((unsigned)(p.blocks + p.oblocks));
  if (p.shared && p.few && p.once)
    prefix_kernel<T, D, WAY_SHARED_FEW, true><<<grid, 256, 0, st>>>(a);
  else if (p.shared && p.few)
    prefix_kernel<T, D, WAY_SHARED_FEW, false><<<grid, 256, 0, st>>>(a);
  else if (p.shared && p.once)
    prefix_kernel<T, D, WAY_SHARED_TILE, true><<<grid, 256, 0, st>>>(a);
  else if (p.shared)
    prefix_kernel<T, D, WAY_SHARED_TILE, false><<<grid, 256, 0, st>>>(a);
  else if (p.few && p.once)
    prefix_kernel<T, D, WAY_FEW, true><<<grid, 256, 0, st>>>(a);
  else if (p.few)
    prefix_kernel<T, D, WAY_FEW, false><<<grid, 256, 0, st>>>(a);
  else
    prefix_kernel<T, D, WAY_TILE, false><<<grid, 256, 0, st>>>(a);
  const hipError_t e = launched("prefix_kernel", st);
  if (e != hipSuccess || p.slots == 1) return e;
  const int64_t rows = (int64_t)a.B * a.Hkv * a.rows;
  constexpr int PER = 256 / (D / 4);
  // (a dimension of a launch has less than 2^32 threads)
  auto grid2 = [](int64_t blocks) {
    constexpr int64_t X = 1 << 20;
    return dim3((unsigned)std::min(blocks, X), (unsigned)((blocks + X - 1) / X));
  };
  if (p.slots > 4)
    prefix_join_kernel<T, D, 1><<<grid2(rows), 256, 0, st>>>(a);
  else
    prefix_join_kernel<T, D, PER><<<grid2((rows + PER - 1) / PER), 256, 0, st>>>(a);
  return launched("prefix_join_kernel", st);
}

}  // namespace

hipError_t launch_prefix_forward(const mita_prefix_cfg_t &c, const void *q, const void *kp, const void *vp,
                                 const void *k, const void *v, const int32_t *q_len, const int32_t *p_len,
                                 const int32_t *k_len, void *o, float *lse, void *ws, hipStream_t st) {
  PrefixArgs a{};
  const size_t e = elem_bytes(c);
  auto mat = [&](const void *p, const Strided &s) {
    return DenseMat{(const char *)p, s.s[0] * (int64_t)e, s.s[1] * (int64_t)e, s.n[2] > 1 ? (uint32_t)(s.s[2] * e) : 0u};
  };
  a.q = mat(q, strided_q(c, c.q));
  a.kp = mat(kp, strided_p(c, c.kp));
  a.vp = mat(vp, strided_p(c, c.vp));
  a.k = mat(k, strided_k(c, c.k));
  a.v = mat(v, strided_k(c, c.v));
  a.o = mat(o, strided_q(c, c.o));
  a.q_len = q_len;
  a.p_len = p_len;
  a.k_len = k_len;
  a.lse = lse;
  a.B = c.B;
  a.Bp = c.Bp;
  a.S = c.B / c.Bp;
  a.H = c.H;
  a.Hkv = c.H_kv;
  a.G = group(c);
  a.N = c.N;
  a.P = c.P;
  a.Nk = c.N_k;
  a.rows = (int)dense_rows(c);
  a.left = window(c.left);
  a.right = window(c.right);
  a.magic = ((uint64_t)1 << 40) / (uint64_t)a.G + 1;
  a.magic_rows = ((uint64_t)1 << 40) / (uint64_t)a.rows + 1;
  a.sl2 = eff_scale(c) * LOG2E;
  const PrefixPlan p = prefix_plan(c);
  const PrefixLayout L = prefix_layout(c);
  a.tiles = p.tiles;
  a.splits = p.splits;
  a.otiles = p.otiles;
  a.osplits = p.osplits;
  a.slots = p.slots;
  a.blocks = (int)p.blocks;
  if (p.slots > 1) {
    a.part_o = (float *)((char *)ws + L.part_o);
    a.part_lse = (float *)((char *)ws + L.part_lse);
  }
  if (c.dtype == MITA_F32) return c.d == 64 ? forward_t<float, 64>(a, p, st) : forward_t<float, 128>(a, p, st);
  return c.d == 64 ? forward_t<bf16_t, 64>(a, p, st) : forward_t<bf16_t, 128>(a, p, st);
}

}  // namespace mita
