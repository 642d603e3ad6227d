// dense_softmax.hpp - the online softmax of a wave's 32 rows in the forward
// kernels of the dense attention: running reference, weights, normalisation, and
// the tiles of waves that take keys on their own.
#pragma once
#include "dense.hpp"

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

template <typename T, int D> struct FewTile {
  using RT = RowTile<T, D>;
  static constexpr int NW = 4, BYTES = 32 * RT::RB, NI = 32 / RT::RPI;  // copies per tile and wave
};

// The wave's next tile: rows past the last repeat it.
template <typename T, int D, bool ONCE = false>
__device__ __forceinline__ void few_copy(uint32_t tile, const char *base, int first, uint32_t stride, int nrows) {
  using RT = RowTile<T, D>;
  const int lane = threadIdx.x & 63;
  const char *src = base + (int64_t)first * stride;
#pragma unroll
  for (int j = 0; j < FewTile<T, D>::NI; ++j) {
    const int r = j * RT::RPI + lane / RT::CPR;
    copy16_unwaited<ONCE>(src, (uint32_t)min(r, nrows - 1) * stride + (uint32_t)(((lane % RT::CPR) ^ RT::swz(r)) << 4),
                          tile + j * 1024);
  }
}

}  // namespace mita
