// layer_check.hpp - host-only validation, launch plans and workspace layouts of
// the dense attention, whole and over shared prefixes, of the layer norm and the RMS
// norm, and of the rotary positions, with their turns per position. Header-only, no HIP
// dependency: the host test builds it with g++.
#pragma once
#include <algorithm>
#include <cmath>
#include <cstdint>
#include <string>

#include "check.hpp"
#include "mita.h"

namespace mita {

constexpr int DENSE_TQ = 128;  // query rows of a dense attention workgroup (32 per wave)
constexpr int DENSE_FEW = 32;   // ... and of one whose waves share the rows
constexpr int DENSE_KB = 128;  // keys of a key-side backward workgroup
constexpr int CUS = 256;       // compute units of the MI355X
constexpr int DENSE_MAX_SPLITS = 64;

// ---------------------------------------------------------------------------
// Strided [n0, n1, n2, len] tensors.
// ---------------------------------------------------------------------------
struct Strided {
  int64_t n[3], s[3], len;  // outermost first; distances in elements
};

// Sort the dimensions by distance, largest first; dimensions of one entry go.
inline int sorted_dims(const Strided &t, int64_t (&n)[3], int64_t (&s)[3]) {
  int k = 0;
  for (int i = 0; i < 3; ++i)
    if (t.n[i] > 1) {
      n[k] = t.n[i];
      s[k++] = t.s[i];
    }
  for (int i = 1; i < k; ++i)
    for (int j = i; j > 0 && s[j] > s[j - 1]; --j) {
      std::swap(s[j], s[j - 1]);
      std::swap(n[j], n[j - 1]);
    }
  return k;
}

// Elements from the first to one past the last.
inline int64_t span_of(const Strided &t) {
  int64_t e = t.len;
  for (int i = 0; i < 3; ++i) e += (t.n[i] - 1) * t.s[i];
  return e;
}

// Does every index have an element of its own? (Sufficient: each distance is
// at least what the dimensions inside it span.)
inline bool nested(const Strided &t) {
  int64_t n[3], s[3], e = t.len;
  for (int k = sorted_dims(t, n, s) - 1; k >= 0; --k) {
    if (s[k] < e) return false;
    e += (n[k] - 1) * s[k];
  }
  return true;
}

// Do two nested tensors with the same distances, the second one's first element
// `delta` elements behind the first one's, share an element? Dimension i of
// distance s[i] shifts by t entries; only the two shifts that leave less than
// s[i] can matter, as the inner dimensions span no more.
inline bool shares(const int64_t (&s)[3], const int64_t (&na)[3], const int64_t (&nb)[3], int64_t len, int64_t delta,
                   int level) {
  if (level == 3) return delta > -len && delta < len;
  if (s[level] == 0) return shares(s, na, nb, len, delta, level + 1);
  int64_t t = delta / s[level];
  if (delta < 0 && t * s[level] != delta) --t;  // floor
  for (int i = 0; i < 2; ++i, ++t)
    if (t < na[level] && -t < nb[level] && shares(s, na, nb, len, delta - t * s[level], level + 1)) return true;
  return false;
}

// May an element of [a] and one of [b] (element size e) share memory? Tensors
// interleaved in one buffer (the slices of a fused projection's gradient) are
// told apart when they have the same distances, others by their spans.
inline bool may_overlap(const void *pa, const Strided &a, const void *pb, const Strided &b, size_t e) {
  if (!pa || !pb) return false;
  if (!overlaps(pa, (size_t)span_of(a) * e, pb, (size_t)span_of(b) * e)) return false;
  const int64_t bytes = (int64_t)((intptr_t)pb - (intptr_t)pa);
  bool same = a.len == b.len && bytes % (int64_t)e == 0 && nested(a) && nested(b);
  int order[3] = {0, 1, 2};
  int64_t s[3], na[3], nb[3];
  for (int i = 0; i < 3; ++i) {
    // a dimension of one entry takes the other tensor's distance
    const int64_t sa = a.n[i] > 1 ? a.s[i] : b.s[i], sb = b.n[i] > 1 ? b.s[i] : a.s[i];
    if (sa != sb) same = false;
    s[i] = a.n[i] > 1 || b.n[i] > 1 ? sa : 0;
  }
  if (!same) return true;
  std::sort(order, order + 3, [&](int x, int y) { return s[x] > s[y]; });
  int64_t so[3];
  for (int i = 0; i < 3; ++i) {
    so[i] = s[order[i]];
    na[i] = a.n[order[i]];
    nb[i] = b.n[order[i]];
  }
  // the distances must nest for both counts together
  int64_t ext = a.len;
  for (int i = 2; i >= 0; --i) {
    if (so[i] == 0) continue;
    if (so[i] < ext) return true;
    ext += (std::max(na[i], nb[i]) - 1) * so[i];
  }
  return shares(so, na, nb, a.len, bytes / (int64_t)e, 0);
}

// ---------------------------------------------------------------------------
// Dense attention
// ---------------------------------------------------------------------------
inline size_t elem_bytes(const mita_dense_cfg_t &c) { return c.dtype == MITA_F32 ? 4 : 2; }
inline float eff_scale(const mita_dense_cfg_t &c) { return c.scale != 0.f ? c.scale : 1.0f / std::sqrt((float)c.d); }
// Query heads of one key head. They read the same keys, so the kernels see
// them as rows of one matrix: row r of a (batch, key head) slice is query
// r / G of its head r % G, R = N * G rows in all.
inline int group(const mita_dense_cfg_t &c) { return c.H / c.H_kv; }
inline int64_t dense_rows(const mita_dense_cfg_t &c) { return (int64_t)c.N * group(c); }
inline int64_t slices(const mita_dense_cfg_t &c) { return (int64_t)c.B * c.H_kv; }

inline mita_strides_t strides_or(const mita_strides_t &s, int64_t h, int64_t n, int64_t d) {
  if (s.b == 0 && s.h == 0 && s.n == 0) return mita_strides_t{h * n * d, n * d, d};
  return s;
}
inline Strided strided_q(const mita_dense_cfg_t &c, const mita_strides_t &s0) {
  const mita_strides_t s = strides_or(s0, c.H, c.N, c.d);
  return Strided{{c.B, c.H, c.N}, {s.b, s.h, s.n}, c.d};
}
inline Strided strided_k(const mita_dense_cfg_t &c, const mita_strides_t &s0) {
  const mita_strides_t s = strides_or(s0, c.H_kv, c.N_k, c.d);
  return Strided{{c.B, c.H_kv, c.N_k}, {s.b, s.h, s.n}, c.d};
}

inline int check_dense(const mita_dense_cfg_t *c, std::string *err) {
  auto fail = [&](int st, const std::string &msg) {
    if (err) *err = msg;
    return st;
  };
  if (!c) return fail(MITA_ERR_INVALID_ARG, "cfg is NULL");
  if (c->B < 1 || c->H < 1 || c->H_kv < 1 || c->N < 1 || c->N_k < 1 || c->d < 1)
    return fail(MITA_ERR_INVALID_ARG, "B, H, H_kv, N, N_k, d must be >= 1");
  if (c->H % c->H_kv != 0) return fail(MITA_ERR_INVALID_ARG, "H_kv must divide H");
  if (c->dtype != MITA_F32 && c->dtype != MITA_BF16)
    return fail(MITA_ERR_UNSUPPORTED, "dtype must be MITA_F32 or MITA_BF16");
  if (c->d != 64 && c->d != 128) return fail(MITA_ERR_UNSUPPORTED, "d must be 64 or 128");
  if (c->N > MITA_DENSE_MAX_N || c->N_k > MITA_DENSE_MAX_N)
    return fail(MITA_ERR_UNSUPPORTED, "N and N_k must not exceed MITA_DENSE_MAX_N");
  if (c->left < -1 || c->right < -1) return fail(MITA_ERR_INVALID_ARG, "left and right must be >= -1");
  if (!(c->scale >= 0.f) || std::isinf(c->scale)) return fail(MITA_ERR_INVALID_ARG, "scale must be finite and >= 0");
  if (c->H > 4096) return fail(MITA_ERR_UNSUPPORTED, "H must not exceed 4096");
  // row numbers are 32-bit, and so are the grids
  if (dense_rows(*c) > (1 << 27)) return fail(MITA_ERR_UNSUPPORTED, "N * (H / H_kv) must not exceed 2^27");
  // (workgroups of 256 threads, of which a launch has less than 2^32)
  if (slices(*c) * ((dense_rows(*c) + 31) / 32) >= (1 << 24) || slices(*c) * ((c->N_k + 31) / 32) >= (1 << 24))
    return fail(MITA_ERR_UNSUPPORTED, "too many heads and tokens for one launch");
  const int64_t unit = 16 / (int64_t)elem_bytes(*c);
  const struct {
    const char *name;
    const mita_strides_t *s;
    bool key, out;
  } all[8] = {{"q", &c->q, false, false},  {"k", &c->k, true, false},   {"v", &c->v, true, false},
              {"o", &c->o, false, true},   {"dO", &c->dO, false, false}, {"dq", &c->dq, false, true},
              {"dk", &c->dk, true, true},  {"dv", &c->dv, true, true}};
  for (const auto &t : all) {
    const Strided x = t.key ? strided_k(*c, *t.s) : strided_q(*c, *t.s);
    for (int i = 0; i < 3; ++i) {
      if (x.s[i] < 0 || x.s[i] > (int64_t)1 << 40)
        return fail(MITA_ERR_INVALID_ARG, std::string("strides of ") + t.name + " must be in [0, 2^40]");
      if (x.n[i] > 1 && x.s[i] % unit != 0)
        return fail(MITA_ERR_INVALID_ARG, std::string("strides of ") + t.name + " must be multiples of 16 bytes");
    }
    if (x.n[2] > 1 && (x.s[2] < c->d || x.s[2] > MITA_DENSE_MAX_STRIDE))
      return fail(MITA_ERR_INVALID_ARG,
                  std::string("token stride of ") + t.name + " must be in [d, MITA_DENSE_MAX_STRIDE]");
    if (t.out && !nested(x))
      return fail(MITA_ERR_INVALID_ARG, std::string("strides of ") + t.name + " give elements the same address");
  }
  return MITA_OK;
}

// The window as the kernels use it: bounds past every key mean none.
inline int window(int w) {
  const int none = 4 * MITA_DENSE_MAX_N;
  return w < 0 || w > none ? none : w;
}

// Launch plan of the forward. A workgroup takes DENSE_TQ rows of a slice, or, where
// those leave CUs without work, DENSE_FEW rows whose keys its waves share. While
// workgroups are few (two fit a CU) the keys of each are split, at least 512 keys
// each; the splits' results are joined by their log-sum-exps.
// Below 256 tiles of DENSE_TQ rows, bf16, us by DENSE_FEW rows and by DENSE_TQ: d = 64,
// heads of 1000 tokens: 8 heads 11 and 19, 16 13 and 19, 30 (240 tiles) 19.2 and 20.3; two
// heads of 8192 59 and 63, of 16256 (254 tiles) 204 and 184. d = 128: 8 heads of 1000 15
// and 24, 16 20 and 25, 24 (192 tiles) 30 and 26; two heads of 8192 97 and 85, of 16256 366
// and 281: there, and for few long heads, DENSE_TQ wins from about 128 tiles on, which
// this rule does not use.
struct DensePlan {
  bool few;    // DENSE_FEW rows per workgroup
  int tiles;   // row tiles per slice
  int splits;  // key splits per row tile
};
inline int keys_seen(const mita_dense_cfg_t &c) {  // most keys one row tile reads
  const int64_t span = (DENSE_TQ + group(c) - 1) / group(c) + 1;
  int64_t m = c.N_k;
  if (c.left >= 0 && c.right >= 0) m = std::min<int64_t>(m, span + c.left + (int64_t)c.right);
  return (int)m;
}
// `uneven`: the window gives workgroups different lengths, which even out over two
// rounds of them (16 heads of 4 key heads, 8192 tokens, causal, d = 128, backward:
// 1718 us in one round, 1126 in two).
inline int splits_for(int64_t blocks, int64_t len, int64_t least, bool uneven) {
  // (rounded down: 960 workgroups of a causal forward, 5 sequences of 2039 tokens,
  // d = 128, take 62 us whole and 103 split in two, by the partial results)
  const int64_t want = (uneven ? 4 : 2) * CUS / blocks;
  return (int)std::max<int64_t>(1, std::min<int64_t>({want, len / least, (int64_t)DENSE_MAX_SPLITS}));
}
inline bool uneven(const mita_dense_cfg_t &c) { return (c.left >= 0) != (c.right >= 0); }
inline DensePlan dense_plan(const mita_dense_cfg_t &c) {
  DensePlan p;
  p.tiles = (int)((dense_rows(c) + DENSE_TQ - 1) / DENSE_TQ);
  p.few = dense_rows(c) <= DENSE_FEW || slices(c) * p.tiles < CUS;
  if (!p.few) {
    p.splits = splits_for(slices(c) * p.tiles, keys_seen(c), 512, uneven(c));
    return p;
  }
  p.tiles = (int)((dense_rows(c) + DENSE_FEW - 1) / DENSE_FEW);
  // just over two workgroups per CU (192 slices of up to 16384 keys, d = 128: 208 us;
  // one per CU 228, four 212, eight 218, as every workgroup starts with nothing in
  // flight), 256 keys each at least (1024 of more rows, whose join takes 4 us)
  const int64_t blocks = slices(c) * p.tiles, want = (2 * CUS) / blocks + (dense_rows(c) <= DENSE_FEW ? 1 : 0);
  const int64_t least = dense_rows(c) <= DENSE_FEW ? 256 : 1024;
  p.splits = (int)std::max<int64_t>(1, std::min<int64_t>({want, keys_seen(c) / least, (int64_t)DENSE_MAX_SPLITS}));
  return p;
}

// Launch plan of the backward: the query side as the forward (its splits' sums
// are added), the key side by DENSE_KB keys, its rows split the same way.
struct DenseBwdPlan {
  int qtiles, qsplits, ktiles, ksplits;
};
inline DenseBwdPlan dense_bwd_plan(const mita_dense_cfg_t &c) {
  DenseBwdPlan p;
  // the shortest piece (an fp32 step takes six times a bf16 one's MFMA time): 8
  // causal heads of 1000 bf16 tokens, d = 64, take 38 us at 256, 40 at 128, 48 at
  // 512; 8 heads of 500 fp32 tokens 50 us at 64, 60 at 128, 114 at 256, 58 at 32
  const int64_t least = c.dtype == MITA_F32 ? 64 : 256;
  p.qtiles = (int)((dense_rows(c) + DENSE_TQ - 1) / DENSE_TQ);
  p.qsplits = splits_for(slices(c) * p.qtiles, keys_seen(c), least, uneven(c));
  p.ktiles = (c.N_k + DENSE_KB - 1) / DENSE_KB;
  int64_t rows = dense_rows(c);
  if (c.left >= 0 && c.right >= 0)
    rows = std::min<int64_t>(rows, (DENSE_KB + (int64_t)c.left + c.right + 1) * group(c));
  p.ksplits = splits_for(slices(c) * p.ktiles, rows, least, uneven(c));
  return p;
}

// Workspace layouts (byte offsets).
struct DenseFwdLayout {
  size_t part_o, part_lse, total;  // per row and split: normalised output and log2-sum-exp
};
inline DenseFwdLayout dense_forward_layout(const mita_dense_cfg_t &c) {
  DenseFwdLayout L{};
  const DensePlan p = dense_plan(c);
  if (p.splits == 1) return L;
  const size_t rows = (size_t)slices(c) * dense_rows(c) * p.splits;
  L.part_o = 0;
  L.part_lse = align_up(rows * c.d * sizeof(float));
  L.total = L.part_lse + align_up(rows * sizeof(float));
  return L;
}
struct DenseBwdLayout {
  size_t lse, D, part_q, part_k, part_v, total;
};
inline DenseBwdLayout dense_backward_layout(const mita_dense_cfg_t &c) {
  DenseBwdLayout L{};
  const DenseBwdPlan p = dense_bwd_plan(c);
  const size_t rows = (size_t)slices(c) * dense_rows(c), keys = (size_t)slices(c) * c.N_k;
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t here = at;
    at += align_up(bytes);
    return here;
  };
  // the rows' log-sum-exps and D, whole row tiles per slice and one more piece,
  // as the key side copies 64 at a time
  const size_t padded = (size_t)slices(c) * p.qtiles * DENSE_TQ + 64;
  L.lse = take(padded * sizeof(float));
  L.D = take(padded * sizeof(float));
  L.part_q = take(p.qsplits > 1 ? rows * p.qsplits * c.d * sizeof(float) : 0);
  L.part_k = take(p.ksplits > 1 ? keys * p.ksplits * c.d * sizeof(float) : 0);
  L.part_v = take(p.ksplits > 1 ? keys * p.ksplits * c.d * sizeof(float) : 0);
  L.total = at;
  return L;
}
inline size_t dense_workspace_size(const mita_dense_cfg_t *c, int which) {
  if (check_dense(c, nullptr) != MITA_OK) return 0;
  if (which == MITA_WS_FORWARD) return dense_forward_layout(*c).total;
  if (which == MITA_WS_BACKWARD) return dense_backward_layout(*c).total;
  return 0;
}

// ---------------------------------------------------------------------------
// Layer norm
// ---------------------------------------------------------------------------
inline size_t elem_bytes(const mita_norm_cfg_t &c) { return c.dtype == MITA_F32 ? 4 : 2; }
inline int64_t norm_rows(const mita_norm_cfg_t &c) { return (int64_t)c.n[0] * c.n[1] * c.n[2]; }
template <typename Cfg> Strided strided_rows(const Cfg &c, const int64_t (&s)[3]) {  // (of the norms)
  if (s[0] == 0 && s[1] == 0 && s[2] == 0)
    return Strided{{c.n[0], c.n[1], c.n[2]}, {(int64_t)c.n[1] * c.n[2] * c.C, (int64_t)c.n[2] * c.C, c.C}, c.C};
  return Strided{{c.n[0], c.n[1], c.n[2]}, {s[0], s[1], s[2]}, c.C};
}

// The same rows in the same places (an output that may take its input's place)?
inline bool same_rows(const void *pa, const Strided &a, const void *pb, const Strided &b) {
  if (pa != pb || !nested(a)) return false;
  for (int i = 0; i < 3; ++i)
    if (a.n[i] > 1 && a.s[i] != b.s[i]) return false;
  return true;
}

inline int check_norm(const mita_norm_cfg_t *c, std::string *err) {
  auto fail = [&](int st, const std::string &msg) {
    if (err) *err = msg;
    return st;
  };
  if (!c) return fail(MITA_ERR_INVALID_ARG, "cfg is NULL");
  if (c->n[0] < 1 || c->n[1] < 1 || c->n[2] < 1 || c->C < 1) return fail(MITA_ERR_INVALID_ARG, "n and C must be >= 1");
  for (int t : {c->dtype, c->wdtype})
    if (t != MITA_F32 && t != MITA_BF16)
      return fail(MITA_ERR_UNSUPPORTED, "dtype and wdtype must be MITA_F32 or MITA_BF16");
  if (c->C > MITA_NORM_MAX_C) return fail(MITA_ERR_UNSUPPORTED, "C must not exceed MITA_NORM_MAX_C");
  if (!(c->eps > 0.f) || std::isinf(c->eps)) return fail(MITA_ERR_INVALID_ARG, "eps must be finite and > 0");
  // row numbers are 32-bit, with room for a workgroup past the last
  if ((int64_t)c->n[0] * c->n[1] > MITA_NORM_MAX_ROWS || norm_rows(*c) > MITA_NORM_MAX_ROWS)
    return fail(MITA_ERR_UNSUPPORTED, "more than MITA_NORM_MAX_ROWS rows");
  const struct {
    const char *name;
    const int64_t (&s)[3];
    bool out;
  } all[4] = {{"x", c->x, false}, {"y", c->y, true}, {"dy", c->dy, false}, {"dx", c->dx, true}};
  for (const auto &t : all) {
    const Strided x = strided_rows(*c, t.s);
    for (int i = 0; i < 3; ++i)
      if (x.s[i] < 0 || x.s[i] > (int64_t)1 << 40)
        return fail(MITA_ERR_INVALID_ARG, std::string("strides of ") + t.name + " must be in [0, 2^40]");
    if (t.out && !nested(x))
      return fail(MITA_ERR_INVALID_ARG, std::string("strides of ") + t.name + " give elements the same address");
  }
  return MITA_OK;
}

// Geometry of the norm kernels: `tpr` threads take a row, each `p` pieces of `ve`
// elements; p == 0: rows too wide for registers, read again in each pass. In
// registers: up to 16384 bf16 and 8192 fp32 elements in pieces of 16 bytes, 16384 in
// pieces of two elements, 8192 one by one.
constexpr int NORM_FWD_THREADS = 256, NORM_BWD_THREADS = 512;  // per workgroup, or tpr if that is more
struct NormPlan {
  int ve, tpr, p;
};
// `align`: every row of every tensor starts at, and C is, a multiple of so many
// elements, of `bytes` each.
inline NormPlan row_plan(size_t bytes, int C, int align) {
  const int full = 16 / (int)bytes;
  const int ve = align % full == 0 ? full : align % 2 == 0 ? 2 : 1;
  const int n = C / ve;  // pieces
  if (ve == full) {
    // within a wave: the fewest idle lanes (768 bf16 elements: 32 threads of three
    // pieces), then the fewest registers
    static const int g[12][2] = {{8, 1},  {16, 1}, {32, 1}, {16, 3},  {64, 1},  {32, 3},
                                 {64, 2}, {64, 3}, {64, 4}, {256, 2}, {256, 4}, {1024, 2}};
    for (const auto &x : g)
      if (n <= x[0] * x[1]) return {ve, x[0], x[1]};
  } else {
    static const int g[7][2] = {{64, 2}, {64, 4}, {64, 6}, {64, 8}, {256, 4}, {256, 8}, {1024, 8}};
    for (const auto &x : g)
      if (n <= x[0] * x[1]) return {ve, x[0], x[1]};
  }
  return {ve, 256, 0};
}
inline NormPlan norm_plan(const mita_norm_cfg_t &c, int align) { return row_plan(elem_bytes(c), c.C, align); }
// Workgroups of the backward, each with a partial sum of the weights' gradients: two
// per CU, or fewer where the rows do not fill them.
inline int row_bwd_blocks(int64_t rows, const NormPlan &p) {
  const int64_t per = p.p ? std::max(1, NORM_BWD_THREADS / p.tpr) : 64;
  return (int)std::min<int64_t>((rows + per - 1) / per, 2 * CUS);
}
inline int norm_bwd_blocks(const mita_norm_cfg_t &c, const NormPlan &p) { return row_bwd_blocks(norm_rows(c), p); }
inline size_t norm_workspace_size(const mita_norm_cfg_t *c) {
  if (check_norm(c, nullptr) != MITA_OK) return 0;
  // how rows are aligned is known only with the pointers
  int n = 0;
  for (int align = 1; align <= 8; align *= 2)
    if (c->C % align == 0) n = std::max(n, norm_bwd_blocks(*c, norm_plan(*c, align)));
  return align_up((size_t)n * 2 * c->C * sizeof(float));
}

// ---------------------------------------------------------------------------
// RMS norm with the residual's addition
// ---------------------------------------------------------------------------
constexpr int RMS_GROUP = 128;  // columns that share a scale of an 8-bit output
inline size_t elem_bytes(const mita_rms_cfg_t &c) { return c.dtype == MITA_F32 ? 4 : 2; }
inline size_t y_bytes(const mita_rms_cfg_t &c) { return c.ytype == MITA_E4M3 ? 1 : elem_bytes(c); }
inline int64_t norm_rows(const mita_rms_cfg_t &c) { return (int64_t)c.n[0] * c.n[1] * c.n[2]; }
inline int rms_scales(const mita_rms_cfg_t &c) {  // per row
  return c.ytype != MITA_E4M3 ? 0 : c.group ? (c.C + c.group - 1) / c.group : 1;
}

inline int check_rms(const mita_rms_cfg_t *c, std::string *err) {
  auto fail = [&](int st, const std::string &msg) {
    if (err) *err = msg;
    return st;
  };
  if (!c) return fail(MITA_ERR_INVALID_ARG, "cfg is NULL");
  if (c->n[0] < 1 || c->n[1] < 1 || c->n[2] < 1 || c->C < 1) return fail(MITA_ERR_INVALID_ARG, "n and C must be >= 1");
  for (int t : {c->dtype, c->wdtype})
    if (t != MITA_F32 && t != MITA_BF16)
      return fail(MITA_ERR_UNSUPPORTED, "dtype and wdtype must be MITA_F32 or MITA_BF16");
  if (c->ytype != c->dtype && c->ytype != MITA_E4M3)
    return fail(MITA_ERR_UNSUPPORTED, "ytype must be dtype or MITA_E4M3");
  if (c->group != 0 && (c->group != RMS_GROUP || c->ytype != MITA_E4M3))
    return fail(MITA_ERR_UNSUPPORTED, "group must be 0, or 128 with MITA_E4M3");
  if (c->C > MITA_NORM_MAX_C) return fail(MITA_ERR_UNSUPPORTED, "C must not exceed MITA_NORM_MAX_C");
  if (!(c->eps > 0.f) || std::isinf(c->eps)) return fail(MITA_ERR_INVALID_ARG, "eps must be finite and > 0");
  if ((int64_t)c->n[0] * c->n[1] > MITA_NORM_MAX_ROWS || norm_rows(*c) > MITA_NORM_MAX_ROWS)
    return fail(MITA_ERR_UNSUPPORTED, "more than MITA_NORM_MAX_ROWS rows");
  const struct {
    const char *name;
    const int64_t (&s)[3];
    bool out;
  } all[7] = {{"x", c->x, false},   {"res", c->res, false}, {"h", c->h, true},  {"y", c->y, true},
              {"dy", c->dy, false}, {"dh", c->dh, false},   {"dx", c->dx, true}};
  for (const auto &t : all) {
    const Strided x = strided_rows(*c, t.s);
    for (int i = 0; i < 3; ++i)
      if (x.s[i] < 0 || x.s[i] > (int64_t)1 << 40)
        return fail(MITA_ERR_INVALID_ARG, std::string("strides of ") + t.name + " must be in [0, 2^40]");
    if (t.out && !nested(x))
      return fail(MITA_ERR_INVALID_ARG, std::string("strides of ") + t.name + " give elements the same address");
  }
  return MITA_OK;
}
inline size_t rms_workspace_size(const mita_rms_cfg_t *c) {
  if (check_rms(c, nullptr) != MITA_OK) return 0;
  // how rows are aligned is known only with the pointers
  int n = 0;
  for (int align = 1; align <= 8; align *= 2)
    if (c->C % align == 0) n = std::max(n, row_bwd_blocks(norm_rows(*c), row_plan(elem_bytes(*c), c->C, align)));
  return align_up((size_t)n * c->C * sizeof(float));
}

// ---------------------------------------------------------------------------
// Rotary positions
// ---------------------------------------------------------------------------
inline size_t elem_bytes(const mita_rope_cfg_t &c) { return c.dtype == MITA_F32 ? 4 : 2; }
inline Strided strided_q(const mita_rope_cfg_t &c, const mita_strides_t &s0) {
  const mita_strides_t s = strides_or(s0, c.H, c.N, c.d);
  return Strided{{c.B, c.H, c.N}, {s.b, s.h, s.n}, c.d};
}
inline Strided strided_k(const mita_rope_cfg_t &c, const mita_strides_t &s0) {
  const mita_strides_t s = strides_or(s0, c.H_kv, c.N, c.d);
  return Strided{{c.B, c.H_kv, c.N}, {s.b, s.h, s.n}, c.d};
}
inline int check_rope(const mita_rope_cfg_t *c, std::string *err) {
  auto fail = [&](int st, const std::string &msg) {
    if (err) *err = msg;
    return st;
  };
  if (!c) return fail(MITA_ERR_INVALID_ARG, "cfg is NULL");
  if (c->B < 1 || c->H < 1 || c->H_kv < 1 || c->N < 1) return fail(MITA_ERR_INVALID_ARG, "B, H, H_kv, N must be >= 1");
  if (c->dtype != MITA_F32 && c->dtype != MITA_BF16)
    return fail(MITA_ERR_UNSUPPORTED, "dtype must be MITA_F32 or MITA_BF16");
  if (c->d < 2) return fail(MITA_ERR_INVALID_ARG, "d must be >= 2");
  if (c->d > MITA_ROPE_MAX_D) return fail(MITA_ERR_UNSUPPORTED, "d must not exceed MITA_ROPE_MAX_D");
  if (c->rot < 2 || c->rot > c->d || c->rot % 2 != 0) return fail(MITA_ERR_INVALID_ARG, "rot must be even and in [2, d]");
  if (c->H > 4096 || c->H_kv > 4096) return fail(MITA_ERR_UNSUPPORTED, "H and H_kv must not exceed 4096");
  // a thread for each piece of a token, of the queries and of the keys, of which a launch
  // has less than 2^32
  if ((int64_t)c->B * c->N > (1 << 30) || (int64_t)c->B * c->N * c->d > ((int64_t)1 << 31) - 512)
    return fail(MITA_ERR_UNSUPPORTED, "B * N * d must not exceed 2^31 - 512");
  if (c->scaling < MITA_ROPE_NONE || c->scaling > MITA_ROPE_PARTS)
    return fail(MITA_ERR_UNSUPPORTED, "scaling must be one of MITA_ROPE_*");
  if (!(c->base > 1.0) || std::isinf(c->base)) return fail(MITA_ERR_INVALID_ARG, "base must be finite and > 1");
  if (c->scaling != MITA_ROPE_NONE && (!(c->factor >= 1.0) || std::isinf(c->factor)))
    return fail(MITA_ERR_INVALID_ARG, "factor must be finite and >= 1");
  if (c->scaling == MITA_ROPE_PARTS) {
    if (c->trained < 1) return fail(MITA_ERR_INVALID_ARG, "trained must be >= 1");
    if (!(c->slow >= 0.0) || !(c->fast > c->slow) || std::isinf(c->fast))
      return fail(MITA_ERR_INVALID_ARG, "slow and fast must be finite with 0 <= slow < fast");
  }
  if (!(c->scale >= 0.f) || std::isinf(c->scale)) return fail(MITA_ERR_INVALID_ARG, "scale must be finite and >= 0");
  if (c->pos_b != 0 && c->pos_b != c->N) return fail(MITA_ERR_INVALID_ARG, "pos_b must be 0 or N");
  if (c->first < -((int64_t)1 << 31) || c->first > (int64_t)1 << 31)
    return fail(MITA_ERR_INVALID_ARG, "first must be in [-2^31, 2^31]");
  const struct {
    const char *name;
    const mita_strides_t *s;
    bool key, out;
  } all[4] = {{"q", &c->q, false, false}, {"k", &c->k, true, false}, {"qo", &c->qo, false, true}, {"ko", &c->ko, true, true}};
  for (const auto &t : all) {
    const Strided x = t.key ? strided_k(*c, *t.s) : strided_q(*c, *t.s);
    for (int i = 0; i < 3; ++i)
      if (x.s[i] < 0 || x.s[i] > (int64_t)1 << 40)
        return fail(MITA_ERR_INVALID_ARG, std::string("strides of ") + t.name + " must be in [0, 2^40]");
    if (t.out && !nested(x))
      return fail(MITA_ERR_INVALID_ARG, std::string("strides of ") + t.name + " give elements the same address");
  }
  return MITA_OK;
}
// Turns per position of each pair, rot / 2 of them: base^(-2 i / rot) as the product of
// two powers, of i's multiple of eight and of the rest (a call forms 16 powers for 64 pairs,
// not 64: 0.3 us of 9.4; two more roundings in 64 bits).
inline void rope_turns(const mita_rope_cfg_t &c, double *f) {
  const double two_pi = 6.283185307179586476925286766559;
  // (one pair alone has f = 1 for any base)
  const double base = c.scaling == MITA_ROPE_BASE && c.rot > 2 ? c.base * std::pow(c.factor, (double)c.rot / (c.rot - 2)) : c.base;
  const int n = c.rot / 2;
  double low[8], high[MITA_ROPE_MAX_D / 16 + 1];
  for (int i = 0; i < std::min(n, 8); ++i) low[i] = std::pow(base, -2.0 * i / c.rot) / two_pi;
  for (int i = 0; i < n; i += 8) high[i / 8] = std::pow(base, -2.0 * i / c.rot);
  for (int i = 0; i < n; ++i) {
    double t = high[i / 8] * low[i % 8];
    if (c.scaling == MITA_ROPE_LINEAR) t /= c.factor;
    if (c.scaling == MITA_ROPE_PARTS) {
      const double keep = std::min(1.0, std::max(0.0, (c.trained * t - c.slow) / (c.fast - c.slow)));
      t = keep * t + (1.0 - keep) * t / c.factor;
    }
    f[i] = t;
  }
}

// ---------------------------------------------------------------------------
// Dense attention over shared prefixes
// ---------------------------------------------------------------------------
inline size_t elem_bytes(const mita_prefix_cfg_t &c) { return c.dtype == MITA_F32 ? 4 : 2; }
inline float eff_scale(const mita_prefix_cfg_t &c) { return c.scale != 0.f ? c.scale : 1.0f / std::sqrt((float)c.d); }
inline int group(const mita_prefix_cfg_t &c) { return c.H / c.H_kv; }
// Rows that read the same keys: of a sequence (its own keys), and of the sequences
// that share a prefix.
inline int64_t dense_rows(const mita_prefix_cfg_t &c) { return (int64_t)c.N * group(c); }
inline int64_t shared_rows(const mita_prefix_cfg_t &c) { return dense_rows(c) * (c.B / c.Bp); }
inline int64_t slices(const mita_prefix_cfg_t &c) { return (int64_t)c.B * c.H_kv; }
inline Strided strided(int64_t b, int64_t h, int64_t n, int64_t d, const mita_strides_t &s0) {
  const mita_strides_t s = strides_or(s0, h, n, d);
  return Strided{{b, h, n}, {s.b, s.h, s.n}, d};
}
inline Strided strided_q(const mita_prefix_cfg_t &c, const mita_strides_t &s) { return strided(c.B, c.H, c.N, c.d, s); }
inline Strided strided_p(const mita_prefix_cfg_t &c, const mita_strides_t &s) { return strided(c.Bp, c.H_kv, c.P, c.d, s); }
inline Strided strided_k(const mita_prefix_cfg_t &c, const mita_strides_t &s) {
  return strided(c.B, c.H_kv, std::max(1, c.N_k), c.d, s);
}

inline int check_prefix(const mita_prefix_cfg_t *c, std::string *err) {
  auto fail = [&](int st, const std::string &msg) {
    if (err) *err = msg;
    return st;
  };
  if (!c) return fail(MITA_ERR_INVALID_ARG, "cfg is NULL");
  if (c->B < 1 || c->Bp < 1 || c->H < 1 || c->H_kv < 1 || c->N < 1 || c->P < 1 || c->N_k < 0 || c->d < 1)
    return fail(MITA_ERR_INVALID_ARG, "B, Bp, H, H_kv, N, P, d must be >= 1 and N_k >= 0");
  if (c->B % c->Bp != 0) return fail(MITA_ERR_INVALID_ARG, "Bp must divide B");
  if (c->H % c->H_kv != 0) return fail(MITA_ERR_INVALID_ARG, "H_kv must divide H");
  if (c->dtype != MITA_F32 && c->dtype != MITA_BF16)
    return fail(MITA_ERR_UNSUPPORTED, "dtype must be MITA_F32 or MITA_BF16");
  if (c->d != 64 && c->d != 128) return fail(MITA_ERR_UNSUPPORTED, "d must be 64 or 128");
  if (c->N > MITA_DENSE_MAX_N || c->P > MITA_DENSE_MAX_N || c->N_k > MITA_DENSE_MAX_N)
    return fail(MITA_ERR_UNSUPPORTED, "N, P and N_k must not exceed MITA_DENSE_MAX_N");
  if (c->left < -1 || c->right < -1) return fail(MITA_ERR_INVALID_ARG, "left and right must be >= -1");
  if (!(c->scale >= 0.f) || std::isinf(c->scale)) return fail(MITA_ERR_INVALID_ARG, "scale must be finite and >= 0");
  if (c->H > 4096) return fail(MITA_ERR_UNSUPPORTED, "H must not exceed 4096");
  // row numbers are 32-bit, and so are the grids (workgroups of 256 threads, of which a
  // launch has less than 2^32)
  if (shared_rows(*c) > (1 << 27)) return fail(MITA_ERR_UNSUPPORTED, "B / Bp * N * (H / H_kv) must not exceed 2^27");
  if (slices(*c) * ((dense_rows(*c) + 31) / 32) >= (1 << 23))
    return fail(MITA_ERR_UNSUPPORTED, "too many heads and tokens for one launch");
  const int64_t unit = 16 / (int64_t)elem_bytes(*c);
  const struct {
    const char *name;
    Strided x;
    bool out;
  } all[6] = {{"q", strided_q(*c, c->q), false}, {"kp", strided_p(*c, c->kp), false}, {"vp", strided_p(*c, c->vp), false},
              {"k", strided_k(*c, c->k), false}, {"v", strided_k(*c, c->v), false},   {"o", strided_q(*c, c->o), true}};
  for (const auto &t : all) {
    for (int i = 0; i < 3; ++i) {
      if (t.x.s[i] < 0 || t.x.s[i] > (int64_t)1 << 40)
        return fail(MITA_ERR_INVALID_ARG, std::string("strides of ") + t.name + " must be in [0, 2^40]");
      if (t.x.n[i] > 1 && t.x.s[i] % unit != 0)
        return fail(MITA_ERR_INVALID_ARG, std::string("strides of ") + t.name + " must be multiples of 16 bytes");
    }
    if (t.x.n[2] > 1 && (t.x.s[2] < c->d || t.x.s[2] > MITA_DENSE_MAX_STRIDE))
      return fail(MITA_ERR_INVALID_ARG,
                  std::string("token stride of ") + t.name + " must be in [d, MITA_DENSE_MAX_STRIDE]");
    if (t.out && !nested(t.x))
      return fail(MITA_ERR_INVALID_ARG, std::string("strides of ") + t.name + " give elements the same address");
  }
  return MITA_OK;
}

// Launch plan. `shared`: a prefix's keys are taken by the rows of all its sequences
// together, each sequence's own keys by its rows, and the parts are joined; else every
// row tile of a sequence goes through the prefix's keys and then its own.
constexpr int PREFIX_MAX_SPLITS = 64;
struct PrefixPlan {
  bool shared;
  bool few;           // DENSE_FEW rows per workgroup, else DENSE_TQ (shared: of the prefix's part; DENSE_FEW of the other)
  int tiles, splits;  // row tiles of a slice (shared: of a prefix's rows), key splits of each
  int otiles, osplits;  // shared: of a sequence's own part (0 without own keys)
  int64_t blocks, oblocks;  // workgroups
  int slots;          // parts of a row's result; 1: none is kept
  bool once;          // the keys are read once, or by a few row tiles at a time, and are more than caches keep
};
// Key splits of `tiles` row tiles of DENSE_TQ rows that go through `keys` keys each. A CU
// with n of their parts takes, per key, `alone` ns for one and `pair` for each of more,
// which share it two at a time (measured with 16000 keys: 256 tiles 281 us, 416 tiles 413
// in bf16, d = 128), a part about 150 keys more to begin and end, the join 10 TB/s and a
// launch. 416 tiles of 8518 keys: 214 us whole, 214, 192, 199 and 239 in two to five parts;
// 208 of 16000: 281, 227, 248, 241; 96 of 16000: 282, 152, 147, 124, and 126 in eight.
inline int prefix_splits(const mita_prefix_cfg_t &c, int64_t tiles, int64_t keys) {
  const bool f32 = c.dtype == MITA_F32, wide = c.d == 128;
  const double alone = f32 ? (wide ? 93 : 50) : wide ? 17.5 : 14.7, pair = f32 ? alone : wide ? 12.8 : 8.7;
  int best = 1;
  double least = 0;
  for (int s = 1; s <= 16 && (s == 1 || keys / s >= 256); ++s) {
    const int64_t n = (tiles * s + CUS - 1) / CUS;
    double t = (n == 1 ? alone : (double)n * pair) * ((double)keys / s + 150);
    if (s > 1) t += (double)slices(c) * dense_rows(c) * s * c.d * 8e-4 + 3000;
    if (s == 1 || t < least) best = s, least = t;
  }
  return best;
}
// Bytes of keys and values from which on caches are told to give them up first (the
// last-level one holds 256 MB). With it and without, us, inputs of three calls in turn: 32768
// prefix keys and 32 x 1024 own ones of 8 heads, d = 128 (268 MB) 57.9 and 65.1; four row
// tiles of 32768 keys (134 MB) 97.1 and 97.6; 4 x 5000 and 48 x 300 of 12 heads, d = 64 (106 MB)
// 26.0 and 27.0, and with lengths that leave 84 MB of them 22.8 and 22.7; 8000 and 16 x 256 of
// 8 heads, d = 128 (50 MB) 22.7 and 20.4.
constexpr int64_t PREFIX_ONCE = (int64_t)1 << 26;
inline PrefixPlan prefix_plan(const mita_prefix_cfg_t &c) {
  // (the window is not looked at: parts whose keys it hides find none, write zeros and are
  // joined. A token of 32 sequences, 32 heads of 8 key heads, behind 32768 keys, d = 128:
  // 55 us without one, 43 with left = 8192, 30 with 512)
  PrefixPlan p{};
  const int64_t rows = dense_rows(c), S = c.B / c.Bp, keys = (int64_t)c.P + c.N_k;
  const int64_t bytes = 2 * c.H_kv * ((int64_t)c.Bp * c.P + (int64_t)c.B * c.N_k) * c.d * (int64_t)elem_bytes(c);
  // Together and apart, us, bf16, d = 128, 8 key heads: 1 row of 64 sequences, 1000 prefix
  // keys 21 and 21, 4000 24 and 51; 4 rows of 16, 500 keys 12 and 13, 2000 15 and 18, 8000 19
  // and 35; 8 rows of 16, 1000 keys 16 and 15, 2000 17 and 18; 16 rows of 16, 2000 keys 20
  // and 19, 8000 28 and 35; 32 rows of 16, 8000 keys 39 and 37. Short prefixes have no
  // splits to join apart (250 keys, 4 rows of 4: 12 and 10). From 32 rows on the bound does not
  // look at how many sequences and keys there are: 40 rows of 16 and of 32 sequences, always
  // apart, 57 and 97 us behind 8000 keys, 242 and 450 behind 32768, 436 and 820 behind 60000.
  p.shared = S > 1 && rows < DENSE_FEW && c.P >= std::max<int64_t>(1024, 200 * rows);
  if (p.shared) {
    const int64_t prefixes = (int64_t)c.Bp * c.H_kv, all = shared_rows(c);
    p.few = all <= DENSE_FEW;
    p.tiles = (int)((all + (p.few ? DENSE_FEW : DENSE_TQ) - 1) / (p.few ? DENSE_FEW : DENSE_TQ));
    const int64_t blocks = prefixes * p.tiles;
    // one workgroup per CU, beside which others take the own keys (but for fp32 and d = 128,
    // where the LDS of either fills the CU, and they follow): a part of 128 rows is 64 KB to
    // write and read again (128 rows of 32768 keys and 8 key heads, each of 32 sequences up
    // to 1024 of its own, d = 128, ordinary reads: 61 us with 32 splits, 71 with 16, 72 with 64).
    // 32 rows, one, two and three workgroups per CU, us, 12 of the rows there: 12 heads behind 4
    // x 5000 and 300 keys, bf16, d = 64 22.9, 24.3 and 25.0, d = 128 39.3, 39.8 and 44.8, fp32
    // 42, 44 and 48; 16 rows, 8 heads, 32768 and 500 keys, d = 128 36.5, 38.5 and 38.2
    p.splits = (int)std::max<int64_t>(1, std::min<int64_t>({CUS / blocks, c.P / 128, PREFIX_MAX_SPLITS}));
    p.blocks = blocks * p.splits;
    if (c.N_k) {
      p.otiles = (int)((rows + DENSE_FEW - 1) / DENSE_FEW);
      const int64_t own = slices(c) * p.otiles;
      p.osplits = (int)std::max<int64_t>(1, std::min<int64_t>({2 * CUS / own, c.N_k / 512, PREFIX_MAX_SPLITS}));
      p.oblocks = own * p.osplits;
    }
    p.slots = p.splits + p.osplits;
    p.once = p.tiles <= 4 && bytes >= PREFIX_ONCE;
    return p;
  }
  // Rows by 32 and by 128, us, bf16, d = 128: 96 tiles of 128 rows and 1000 keys 17 and 25,
  // 4000 46 and 45, 16000 157 and 124; 208 tiles and 1000 keys 21 and 27, 4000 76 and 66; d =
  // 64: 96 tiles and 4000 keys 31 and 33, 16000 105 and 80; 208 tiles and 4000 43 and 45.
  p.tiles = (int)((rows + DENSE_TQ - 1) / DENSE_TQ);
  p.few = rows <= 64 || slices(c) * p.tiles * keys * (c.d / 64) < 1000000;
  if (p.few) {
    p.tiles = (int)((rows + DENSE_FEW - 1) / DENSE_FEW);
    const int64_t blocks = slices(c) * p.tiles, least = rows <= DENSE_FEW ? 256 : 1024;
    p.splits = (int)std::max<int64_t>(1, std::min<int64_t>({2 * CUS / blocks, keys / least, PREFIX_MAX_SPLITS}));
    p.once = S == 1 && p.tiles == 1 && bytes >= PREFIX_ONCE;
  } else {
    p.splits = prefix_splits(c, slices(c) * p.tiles, keys);
  }
  p.blocks = slices(c) * p.tiles * p.splits;
  p.slots = p.splits;
  return p;
}
struct PrefixLayout {
  size_t part_o, part_lse, total;  // per row and slot: normalised output and log2-sum-exp
};
inline PrefixLayout prefix_layout(const mita_prefix_cfg_t &c) {
  PrefixLayout L{};
  const PrefixPlan p = prefix_plan(c);
  if (p.slots == 1) return L;
  const size_t parts = (size_t)slices(c) * dense_rows(c) * p.slots;
  L.part_lse = align_up(parts * c.d * sizeof(float));
  L.total = L.part_lse + align_up(parts * sizeof(float));
  return L;
}
inline size_t prefix_workspace_size(const mita_prefix_cfg_t *c) {
  return check_prefix(c, nullptr) != MITA_OK ? 0 : prefix_layout(*c).total;
}

}  // namespace mita
