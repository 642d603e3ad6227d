// rope.hip - rotary positions of queries and keys: (u, v) -> s (u cos a - v sin a,
// v cos a + u sin a) with a = pos f_i for each pair of a head's first elements, and its
// transpose for the gradients.
//
// Bound by HBM: every element is read and written once. A thread turns the same
// piece (of 16 bytes, or two of them where a head's halves form the pairs) of
// several heads of one token, so its angles' sines and cosines are formed once for
// all of them. 32768 tokens of 32 + 8 heads in token order, d = 128, bf16: 118 us, 5.7
// TB/s (a plain elementwise product reaches 6.2); 139 with the parts of a token's heads
// in distant workgroups, which touch the memory's pages in turn.
#include "cdna4.hpp"
#include "kernels.hpp"
#include "layer_check.hpp"

namespace mita {

namespace {

struct RopeMat {
  const char *in;
  char *out;
  int64_t ib, ih, in_n, ob, oh, on;  // bytes between batch elements, heads and tokens
  int heads;
  bool same;  // out is in: elements that do not turn stay where they are
};
struct RopeArgs {
  RopeMat m[2];  // queries, keys
  const int32_t *pos;
  int pos_b;
  int B, N, items;   // items: pieces of a token that a thread takes
  int turning;       // of these, the first so many turn
  int rot, per[2];      // heads of a thread
  int chunks, chunks_q; // parts of the heads, and those of the queries, which come first
  int64_t first;
  float scale;
  double f[MITA_ROPE_MAX_D / 2];  // turns per position
};

// Sine and cosine of `turns` whole turns: reduced to an eighth of a turn around a
// quarter in 64 bits (exactly, for turns below 2^53), then Taylor sums, whose next
// terms are below 2^-27 of the largest value.
__device__ __forceinline__ void sin_cos_turns(double turns, float &s, float &c) {
  const double r = turns - rint(turns), q = rint(4.0 * r);
  const float x = (float)(r - 0.25 * q) * 6.2831853071795865f, y = x * x;
  float sn = __builtin_fmaf(y, 2.7557319e-6f, -1.9841270e-4f);
  sn = __builtin_fmaf(y, sn, 8.3333333e-3f);
  sn = __builtin_fmaf(y, sn, -1.6666667e-1f);
  sn = __builtin_fmaf(x * y, sn, x);
  float cs = __builtin_fmaf(y, -2.7557319e-7f, 2.4801587e-5f);
  cs = __builtin_fmaf(y, cs, -1.3888889e-3f);
  cs = __builtin_fmaf(y, cs, 4.1666667e-2f);
  cs = __builtin_fmaf(y, cs, -0.5f);
  cs = __builtin_fmaf(y, cs, 1.f);
  const int k = (int)q;
  const float a = k & 1 ? cs : sn, b = k & 1 ? sn : cs;
  s = k & 2 ? -a : a;
  c = (k + 1) & 2 ? -b : b;
}

// V consecutive elements as they are in memory, and in fp32.
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
template <int BYTES> struct Bits;
template <> struct Bits<16> { using type = u32x4; };
template <> struct Bits<8> { using type = u32x2; };
template <> struct Bits<4> { using type = uint32_t; };
template <> struct Bits<2> { using type = uint16_t; };
template <typename T, int V> using BitsOf = typename Bits<V * (int)sizeof(T)>::type;

template <typename T, int V> __device__ __forceinline__ void unpack(const BitsOf<T, V> &x, float (&f)[V]) {
  if constexpr (V * sizeof(T) == 16) {
    unpack16(__builtin_bit_cast(uint4, x), f, (const T *)nullptr);
  } else if constexpr (V * sizeof(T) == 8) {
    f[0] = __uint_as_float(x.x);
    f[1] = __uint_as_float(x.y);
  } else if constexpr (sizeof(T) == 4) {
    f[0] = __uint_as_float(x);
  } else {
    f[0] = __uint_as_float((uint32_t)x << 16);
    if constexpr (V == 2) f[1] = __uint_as_float(x & 0xffff0000u);
  }
}
template <typename T, int V> __device__ __forceinline__ BitsOf<T, V> pack(const float (&f)[V]) {
  if constexpr (V * sizeof(T) == 16 && sizeof(T) == 4)
    return u32x4{__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])};
  else if constexpr (V * sizeof(T) == 16)
    return u32x4{pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7])};
  else if constexpr (V * sizeof(T) == 8)
    return u32x2{__float_as_uint(f[0]), __float_as_uint(f[1])};
  else if constexpr (sizeof(T) == 4)
    return __float_as_uint(f[0]);
  else if constexpr (V == 2)
    return pack_bf16x2(f[0], f[1]);
  else
    return f32_to_bf16(f[0]);
}

__device__ __forceinline__ void turn(float &u, float &v, float sn, float cs) {
  const float y = u, z = v;
  u = __builtin_fmaf(y, cs, -(z * sn));
  v = __builtin_fmaf(z, cs, y * sn);
}

// Thread x of its part of the heads takes piece x % items of token x / items; workgroups
// are the parts of the same tokens, then those of the next. Items below `turning` turn: V pairs of two pieces V long and
// rot / 2 apart, or (IL) the V / 2 pairs of one piece (V = 1: of two elements). The
// others are V elements that are copied.
template <typename T, int V, bool IL, bool ONCE> __global__ void __launch_bounds__(256) rope_kernel(RopeArgs a) {
  constexpr int NP = IL ? (V > 1 ? V / 2 : 1) : V;  // pairs of an item
  // neighbouring workgroups take the same tokens' heads, which a projection writes side by side
  const uint32_t block = blockIdx.x / (uint32_t)a.chunks;
  const int part = (int)(blockIdx.x - block * (uint32_t)a.chunks);
  const uint32_t x = block * 256 + threadIdx.x, t = x / (uint32_t)a.items;
  const int token = (int)t, item = (int)(x - t * (uint32_t)a.items);
  if (token >= a.B * a.N) return;
  const int b = token / a.N, n = token - b * a.N;
  const bool turns = item < a.turning;
  // the first element of the item, and where its pairs' other elements are
  const int e0 = turns ? (IL ? 2 * NP * item : V * item) : a.rot + V * (item - a.turning);
  using B = BitsOf<T, V>;
  constexpr bool second = !IL || V == 1;  // pairs of elements of two pieces
  const int apart = !turns ? 0 : IL ? (int)sizeof(T) : (a.rot / 2) * (int)sizeof(T);
  // a workgroup's heads are all queries' or all keys'
  const int key = part >= a.chunks_q;
  const RopeMat &m = a.m[key];
  int h = (part - key * a.chunks_q) * a.per[key];
  const int end = min(m.heads, h + a.per[key]);
  if (!turns && m.same) return;
  float sn[NP], cs[NP];
#pragma unroll
  for (int i = 0; i < NP; ++i) sn[i] = 0.f, cs[i] = 1.f;
  if (turns) {
    const double p = a.pos ? (double)a.pos[(int64_t)b * a.pos_b + n] : (double)(a.first + n);
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      sin_cos_turns(p * a.f[item * NP + i], sn[i], cs[i]);
      sn[i] *= a.scale;
      cs[i] *= fabsf(a.scale);
    }
  }
  const char *src = m.in + b * m.ib + n * m.in_n + e0 * (int)sizeof(T) + h * m.ih;
  char *dst = m.out + b * m.ob + n * m.on + e0 * (int)sizeof(T) + h * m.oh;
  const int64_t ih = m.ih, oh = m.oh;
  // U heads, all read before the first is written. Lanes whose elements do not turn do the
  // same with theirs, and write them as they were: with a branch of their own their loads
  // would wait for the others' (4 x 4096 tokens of 32 heads, 32 of 128 elements: 58 us).
  auto read = [](const char *p) {
    return ONCE ? __builtin_nontemporal_load(reinterpret_cast<const B *>(p)) : *reinterpret_cast<const B *>(p);
  };
  auto heads = [&](auto count) {
    constexpr int U = decltype(count)::value;
    B u[U], v[U];
#pragma unroll
    for (int i = 0; i < U; ++i) {
      u[i] = read(src + i * ih);
      if constexpr (second) v[i] = read(src + i * ih + apart);
    }
#pragma unroll
    for (int i = 0; i < U; ++i) {
      float x[V], y[V];
      unpack<T, V>(u[i], x);
      if constexpr (second) unpack<T, V>(v[i], y);
#pragma unroll
      for (int j = 0; j < NP; ++j) {
        if constexpr (second)
          turn(x[j], y[j], sn[j], cs[j]);
        else
          turn(x[2 * j], x[2 * j + 1], sn[j], cs[j]);
      }
      *reinterpret_cast<B *>(dst + i * oh) = turns ? pack<T, V>(x) : u[i];
      if constexpr (second) {
        if (turns) *reinterpret_cast<B *>(dst + i * oh + apart) = pack<T, V>(y);
      }
    }
  };
  for (; h + 4 <= end; h += 4, src += 4 * ih, dst += 4 * oh) heads(std::integral_constant<int, 4>{});
  for (; h + 2 <= end; h += 2, src += 2 * ih, dst += 2 * oh) heads(std::integral_constant<int, 2>{});
  if (h < end) heads(std::integral_constant<int, 1>{});
}

// The largest of 16 bytes, two elements and one that every piece of both tensors is
// aligned to, those that are copied as those that turn. 8192 tokens of 32 heads, bf16, us, and
// their bytes at 6.2 TB/s: d = 256, 16 bytes 51 (43), with 66 elements that turn, one by one,
// 92; d = 250, one by one 67 (42); d = 96 25.9 (16), with 24, by two elements, 27.6; d = 80
// 20.2 (13.5), with 20, by two, 22.2.
int rope_vector(const mita_rope_cfg_t &c, const Strided *t, const void *const *p) {
  const int e = (int)elem_bytes(c), full = 16 / e;
  auto fits = [&](int v) {
    if (c.d % v != 0 || c.rot % v != 0 || (!c.interleaved && (c.rot / 2) % v != 0)) return false;
    for (int i = 0; i < 4; ++i) {
      if (!p[i]) continue;
      if ((uintptr_t)p[i] % (v * e) != 0) return false;
      for (int k = 0; k < 3; ++k)
        if (t[i].n[k] > 1 && t[i].s[k] % v != 0) return false;
    }
    return true;
  };
  return fits(full) ? full : fits(2) ? 2 : 1;
}

// once: inputs of 128 MB and more are read past the caches' order, as in the RMS norm. With it
// and with ordinary reads, us, inputs and outputs of three calls in turn, and (in brackets) where
// the outputs take the place of the call's before: 4 x 8192 tokens of 32 heads, d = 128, 268
// MB, heads before tokens 98 and 102 (82 and 103), tokens before heads 93 to 96 and 95 (83 and
// 95); 4 x 4096, 134 MB, 54 and 56 (45 and 47), 51 and 51 (46 and 47); 32768 tokens of 32 + 8
// heads 118 and 117 (116 and 117); but 3277 tokens of 32 heads, 27 MB, 13 and 11.
template <typename T, int V> hipError_t rope_v(const RopeArgs &a, bool il, bool once, dim3 grid, hipStream_t st) {
  constexpr bool WHOLE = V * sizeof(T) == 16;
  if (il && once)
    rope_kernel<T, V, true, WHOLE><<<grid, 256, 0, st>>>(a);
  else if (il)
    rope_kernel<T, V, true, false><<<grid, 256, 0, st>>>(a);
  else if (once)
    rope_kernel<T, V, false, WHOLE><<<grid, 256, 0, st>>>(a);
  else
    rope_kernel<T, V, false, false><<<grid, 256, 0, st>>>(a);
  return launched("rope_kernel", st);
}

}  // namespace

hipError_t launch_rope(const mita_rope_cfg_t &c, const void *q, const void *k, const int32_t *pos, void *qo, void *ko,
                       bool back, hipStream_t st) {
  const Strided t[4] = {strided_q(c, c.q), strided_k(c, c.k), strided_q(c, c.qo), strided_k(c, c.ko)};
  const void *const p[4] = {q, k, qo, ko};
  const int e = (int)elem_bytes(c), v = rope_vector(c, t, p);
  RopeArgs a{};
  for (int i = 0; i < 2; ++i) {
    const Strided &x = t[i], &y = t[2 + i];
    a.m[i] = RopeMat{(const char *)p[i],
                     (char *)const_cast<void *>(p[2 + i]),
                     x.s[0] * e,
                     x.s[1] * e,
                     x.s[2] * e,
                     y.s[0] * e,
                     y.s[1] * e,
                     y.s[2] * e,
                     i == 0 ? c.H : k ? c.H_kv : 0,
                     p[i] == p[2 + i]};
  }
  a.pos = pos;
  a.pos_b = c.pos_b;
  a.B = c.B;
  a.N = c.N;
  a.rot = c.rot;
  const int pairs = c.interleaved ? std::max(1, v / 2) : v;
  a.turning = c.rot / 2 / pairs;
  a.items = a.turning + (a.m[0].same && (!k || a.m[1].same) ? 0 : (c.d - c.rot) / v);
  a.first = c.first;
  const float scale = c.scale != 0.f ? c.scale : 1.f;
  a.scale = back ? -scale : scale;
  const int heads = c.H + a.m[1].heads;
  rope_turns(c, a.f);
  const int64_t threads = (int64_t)c.B * c.N * a.items, blocks = (threads + 255) / 256;
  // Four heads per thread, whose loads are in flight together, or fewer where that leaves
  // less than two waves per SIMD; more only where a launch could not hold the threads. 32768
  // tokens of 40 heads, d = 128: 182 us with one head, 139 with two, 116 with four, 119
  // with eight; 64 x 196 tokens of 12 heads, d = 64: 11.0, 10.0, 10.0, 10.7; one token of
  // 24 sequences, 40 heads: 3.8, 4.1, 4.2, 5.2.
  int64_t per = std::max<int64_t>(1, std::min<int64_t>(4, threads * heads / (2 * 4 * 64 * CUS)));
  int chunks[2];
  for (;; per *= 2) {
    for (int i = 0; i < 2; ++i) {
      // (six heads, say, are one part and not two)
      const int all = a.m[i].heads, n = (int)std::max<int64_t>(1, (all + per / 4) / per);
      a.per[i] = std::max(1, (all + n - 1) / n);
      chunks[i] = (all + a.per[i] - 1) / a.per[i];
    }
    a.chunks_q = chunks[0];
    a.chunks = chunks[0] + chunks[1];
    if (256 * blocks * a.chunks <= ((int64_t)1 << 32) - 512) break;
    if (per > 8192) return hipErrorInvalidConfiguration;
  }
  const dim3 grid((unsigned)(blocks * a.chunks));
  const bool il = c.interleaved != 0, once = (int64_t)c.B * c.N * heads * c.d * e >= (int64_t)1 << 27;
  if (c.dtype == MITA_F32)
    return v == 4   ? rope_v<float, 4>(a, il, once, grid, st)
           : v == 2 ? rope_v<float, 2>(a, il, once, grid, st)
                    : rope_v<float, 1>(a, il, once, grid, st);
  return v == 8   ? rope_v<bf16_t, 8>(a, il, once, grid, st)
         : v == 2 ? rope_v<bf16_t, 2>(a, il, once, grid, st)
                  : rope_v<bf16_t, 1>(a, il, once, grid, st);
}

}  // namespace mita
