// Block attention over a cache held in 4 or 8 bits (kvq.h).
//
//   o_r = sum over the keys i that row r sees of softmax_i(scale q_r . k_i) v_i,    k_i, v_i = codes times 2^(e - 127) of their blocks, exactly.
//
// Row r of a kv head = (slot of the block) * group + query head.  A workgroup takes up to 16 RB of them and a range of keys, its four wavefronts a quarter of the range
// each, pages in pairs.  Codes become bf16 (fp32 models: fp32) in registers by the conversion instructions that take the block's scale, both exact (e2m1 and e4m3 numbers have
// 2 and 4 significant bits), but that 8-bit codes that stand for less than 2^-126 become 0 in bf16.  S^T = K Q^T leaves a lane four consecutive keys of a query column, which is how V^T P^T takes them.  Softmax in one pass,
// base 2, with a reference maximum that moves only when a score passes it by kSlack.  bf16 models: probabilities are hi + lo bf16 pairs, off by 2^-16 of themselves, as everywhere in them; by
// one number, off by 2^-8, the error against 64 bits was 0.0018 to 0.0020 of a row where the output's own rounding makes 0.0016.  All sums in fp32.
// Ranges of keys, each the mean of its values with its weights' sum and reference, are joined by kvq_merge_kernel in a fixed order: a call repeats itself bit for bit.
//
// Single tokens are bound by memory (32 of them behind 1k to 32k tokens, 32 heads over 8 of 128, 4 bits: 590 MB in 103 to 106 us, 5.6 TB/s; the copies by themselves 101); blocks of few pairs a
// wavefront by latency (16 x 16 rows behind up to 4k tokens: 34 us, and 6 for the merge); many rows by vector instructions, which share the issue with the MFMAs (pieces of 391 and 512 rows behind
// up to 6k tokens: 109 us with the merge, 500 TFLOP/s of the keys that the rows see).
#include <algorithm>
#include <type_traits>
#include <utility>

#include "kvq.h"
#include "plan.h"

namespace {

constexpr float kSlack = 8.f;   // probabilities up to 2^8 above the reference: nothing that fp32 sums or bf16 exponents notice
// Sums of finite values can pass fp32 where their weighted mean does not (a hundred keys of 2^122 and weight 1).  A wavefront whose sums are not finite takes its keys again with
// weights 2^-40 as large, which add up to less than 1 over any number of keys.  Not at once, so that values down to 2^-126 keep their bits where none is above 2^88.
constexpr float kLift = 40.f;
// A score times scale2 less a reference that was rounded after the same product is off by half a step of either: from scores of 2^31 on that is a power of 2^128 or of nothing.
// Such weights' sum is infinite, NaN or next to nothing where the reference's own is 1: those wavefronts, too, take their keys again, scores less the reference before the product.
constexpr float kLeast = 0x1p-20f;

__device__ __forceinline__ uint32_t pair_of(float a, float b) { return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2){a, b}, bf16x2)); }
__device__ __forceinline__ uint32_t finite_half(uint32_t x, uint32_t exponent) { return (x & exponent) == exponent ? 0u : x; }
__device__ __forceinline__ uint32_t finite_halves(uint32_t x) { return finite_half(x & 0xFFFFu, 0x7F80u) | finite_half(x & 0xFFFF0000u, 0x7F800000u); }
// the largest, NaN if one is (such a row is NaN whatever its reference): one instruction a pair of numbers, where fmaxf first quiets signalling NaNs
__device__ __forceinline__ float max3(float a, float b, float c) { return __builtin_elementwise_maximum(__builtin_elementwise_maximum(a, b), c); }
__device__ __forceinline__ bool odd_bits(float x) { return (__float_as_uint(x) & 0x7F800000u) == 0x7F800000u; }

// byte I of the scales of a lane's keys
template <int I, int N>
__device__ __forceinline__ float scale_at(const uint32_t (&w)[N]) { return kvq_scale<I % 4>(w[I / 4]); }

// A page as a lane has it: lane (g, key) of K, lane (g, n) of V.
template <int NB, int KB, int VB, bool F32>
struct Page {
  static constexpr int KW = NB * KB / 4, VW = NB * VB / 4, SROW = kvq_scale_row(NB);
  static constexpr bool OWN = !F32 && NB % 2 == 0;   // a lane's codes are of one block (one scale); else eight dims of every block
  uint32_t k[KW], v[VW], ks, vs[SROW];

  __device__ __forceinline__ void load_k(const unsigned char* unit, int lane) {
    const int g = lane >> 4, key = lane & 15;
    const unsigned char* p = unit;
    auto take = [&](int at, int words, const unsigned char* from) {
      if (words == 4) {
        const u32x4 w = *reinterpret_cast<const u32x4*>(from);
#pragma unroll
        for (int i = 0; i < 4; ++i) k[at + i] = w[i];
      } else if (words == 2) {
        const u32x2 w = *reinterpret_cast<const u32x2*>(from);
#pragma unroll
        for (int i = 0; i < 2; ++i) k[at + i] = w[i];
      } else {
        k[at] = *reinterpret_cast<const uint32_t*>(from);
      }
    };
    if constexpr (OWN && NB == 4) {
#pragma unroll
      for (int h = 0; h < KB / 4; ++h) take(4 * h, 4, p + ((h * 4 + g) * 16 + key) * 16);
    } else if constexpr (OWN) {
      if constexpr (KB == 4) take(0, 2, p + ((g >> 1) * 16 + key) * 16 + (g & 1) * 8);
      else take(0, 4, p + (((g & 1) * 2 + (g >> 1)) * 16 + key) * 16);
    } else {
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        if constexpr (KB == 4) take(b, 1, p + (b * 16 + key) * 16 + g * 4);
        else take(2 * b, 2, p + (((g >> 1) * NB + b) * 16 + key) * 16 + (g & 1) * 8);
      }
    }
    const unsigned char* s = unit + kvq_codes(NB, KB) + kvq_codes(NB, VB) + key * SROW;
    if constexpr (OWN) ks = s[NB == 4 ? g : g >> 1];
    else if constexpr (SROW == 4) ks = *reinterpret_cast<const uint32_t*>(s);
    else if constexpr (SROW == 2) ks = *reinterpret_cast<const uint16_t*>(s);
    else ks = s[0];
  }
  __device__ __forceinline__ void load_v(const unsigned char* unit, int lane) {
    const unsigned char* p = unit + kvq_codes(NB, KB);
    if constexpr (VB == 4 && NB == 3) {
#pragma unroll
      for (int b = 0; b < 3; ++b) v[b] = reinterpret_cast<const uint32_t*>(p)[lane * 3 + b];
    } else if constexpr (VB == 4) {
      typedef uint32_t words __attribute__((ext_vector_type(NB == 1 ? 2 : NB)));
      if constexpr (NB == 1) v[0] = reinterpret_cast<const uint32_t*>(p)[lane];
      else {
        const words w = reinterpret_cast<const words*>(p)[lane];
#pragma unroll
        for (int b = 0; b < NB; ++b) v[b] = w[b];
      }
    } else {
#pragma unroll
      for (int b = 0; b < NB; b += 2) {
        if (b + 1 < NB) {
          const u32x4 w = reinterpret_cast<const u32x4*>(p + (b / 2) * 1024)[lane];
#pragma unroll
          for (int i = 0; i < 4; ++i) v[2 * b + i] = w[i];
        } else {
          const u32x2 w = reinterpret_cast<const u32x2*>(p + (b / 2) * 1024)[lane];
          v[2 * b] = w[0];
          v[2 * b + 1] = w[1];
        }
      }
    }
    const uint32_t* s = reinterpret_cast<const uint32_t*>(p + kvq_codes(NB, VB) + DF_PAGE * SROW) + (lane >> 4) * SROW;
    if constexpr (SROW == 4) {
      const u32x4 w = *reinterpret_cast<const u32x4*>(s);
#pragma unroll
      for (int i = 0; i < 4; ++i) vs[i] = w[i];
    } else if constexpr (SROW == 2) {
      const u32x2 w = *reinterpret_cast<const u32x2*>(s);
      vs[0] = w[0];
      vs[1] = w[1];
    } else {
      vs[0] = s[0];
    }
  }
  // scale of chunk J of the lane's K codes
  template <int J>
  __device__ __forceinline__ float k_scale() const {
    if constexpr (OWN) return kvq_scale<0>(ks);
    else return kvq_scale<J>(ks);
  }
  template <int K, int B>
  __device__ __forceinline__ float v_scale() const { return scale_at<K * SROW + B>(vs); }
};

template <typename F, int... I>
__device__ __forceinline__ void each_of(F&& f, std::integer_sequence<int, I...>) { (f(std::integral_constant<int, I>()), ...); }
template <int N, typename F>
__device__ __forceinline__ void unrolled(F&& f) { each_of(f, std::make_integer_sequence<int, N>()); }

// ---- products ---------------------------------------------------------------------------------------------------------------------
template <typename T, int NB, int KB, int VB> struct Math;

template <int NB, int KB, int VB>
struct Math<bf16_t, NB, KB, VB> {
  using P = Page<NB, KB, VB, false>;
  struct Query { u32x4 q[NB]; };
  struct Sum { float l; };          // the lane's own keys
  struct Probs { u32x4 p, rest; };  // four keys of the first page, four of the second: hi + lo
  static __device__ __forceinline__ int dim(int g, int j) { return P::OWN ? 8 * (NB * g + j) : 8 * (4 * j + g); }
  static __device__ __forceinline__ void query(Query& f, const bf16_t* row, int hd, int lane) {
#pragma unroll
    for (int j = 0; j < NB; ++j) {
      const int d = dim(lane >> 4, j);
      f.q[j] = (u32x4){0u, 0u, 0u, 0u};
      if (row && d < hd) f.q[j] = *reinterpret_cast<const u32x4*>(row + d);
    }
  }
  struct Keys { u32x4 k[NB]; };
  static __device__ __forceinline__ void keys(Keys& f, const P& p) {
    unrolled<NB>([&](auto j_c) {
      constexpr int j = decltype(j_c)::value;
      const float s = p.template k_scale<j>();
      if constexpr (KB == 4)
        f.k[j] = (u32x4){kvq_bf16_of4<0>(p.k[j], s), kvq_bf16_of4<1>(p.k[j], s), kvq_bf16_of4<2>(p.k[j], s), kvq_bf16_of4<3>(p.k[j], s)};
      else
        f.k[j] = (u32x4){kvq_bf16_of8<0>(p.k[2 * j], s), kvq_bf16_of8<1>(p.k[2 * j], s), kvq_bf16_of8<0>(p.k[2 * j + 1], s), kvq_bf16_of8<1>(p.k[2 * j + 1], s)};
    });
  }
  static __device__ __forceinline__ f32x4 scores(const Keys& k, const Query& q) {
    f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < NB; ++j)
      s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, k.k[j]), __builtin_bit_cast(bf16x8, q.q[j]), s, 0, 0, 0);
    return s;
  }
  static __device__ __forceinline__ void probs(Probs& f, const float (&p)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f.p[i] = pair_of(p[2 * i], p[2 * i + 1]);
      f.rest[i] = pair_of(p[2 * i] - __uint_as_float(f.p[i] << 16), p[2 * i + 1] - __uint_as_float(f.p[i] & 0xFFFF0000u));
    }
  }
  static __device__ __forceinline__ void sum(Sum& l, const Probs&, const float (&p)[8]) {
    l.l += ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
  }
  static __device__ __forceinline__ void scale_sum(Sum& l, float f) { l.l *= f; }
  static __device__ __forceinline__ float total(const Sum& l) { return quarter_sum(l.l); }
  struct Values { u32x4 v[2]; };    // dims below 16 of a block, and those from 16 on
  template <int B>
  static __device__ __forceinline__ void values(Values& f, const P& a, const P& b) {
    uint32_t w[8];
    auto page = [&](int at, const P& p) {
      unrolled<4>([&](auto k_c) {
        constexpr int k = decltype(k_c)::value;
        const float s = p.template v_scale<k, B>();
        if constexpr (VB == 4) w[at + k] = kvq_bf16_of4<k>(p.v[B], s);
        else w[at + k] = kvq_bf16_of8<k & 1>(p.v[2 * B + k / 2], s);
      });
    };
    page(0, a);
    page(4, b);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f.v[0][i] = __builtin_amdgcn_perm(w[2 * i + 1], w[2 * i], 0x05040100u);
      f.v[1][i] = __builtin_amdgcn_perm(w[2 * i + 1], w[2 * i], 0x07060302u);
    }
  }
  // elements of keys that nobody sees (there: a bit a key) become 0; whether any that are left are not finite
  static __device__ __forceinline__ bool clear(Values& f, unsigned there) {
    uint32_t odd = 0;
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        f.v[h][i] &= (there >> (2 * i) & 1 ? 0x0000FFFFu : 0u) | (there >> (2 * i) & 2 ? 0xFFFF0000u : 0u);
        odd |= f.v[h][i] ^ finite_halves(f.v[h][i]);
      }
    return odd != 0;
  }
  // 1 for every element that is plus (minus) infinity or NaN
  static __device__ __forceinline__ void mark(Values& w, const Values& f, bool minus) {
    auto one = [&](uint32_t half) { return (half & 0x7F80u) == 0x7F80u && (half & 0x7Fu || (half >> 15 != 0) == minus) ? 0x3F80u : 0u; };
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int i = 0; i < 4; ++i) w.v[h][i] = one(f.v[h][i] & 0xFFFFu) | one(f.v[h][i] >> 16) << 16;
  }
  static __device__ __forceinline__ void drop(Values& f) {   // those become 0
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int i = 0; i < 4; ++i) f.v[h][i] = finite_halves(f.v[h][i]);
  }
  static __device__ __forceinline__ void add(f32x4& lo, f32x4& hi, const Values& v, const Probs& p) {
    lo = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, v.v[0]), __builtin_bit_cast(bf16x8, p.p), lo, 0, 0, 0);
    hi = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, v.v[1]), __builtin_bit_cast(bf16x8, p.p), hi, 0, 0, 0);
    lo = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, v.v[0]), __builtin_bit_cast(bf16x8, p.rest), lo, 0, 0, 0);
    hi = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, v.v[1]), __builtin_bit_cast(bf16x8, p.rest), hi, 0, 0, 0);
  }
};

template <int NB, int KB, int VB>
struct Math<float, NB, KB, VB> {
  using P = Page<NB, KB, VB, true>;
  struct Query { float q[NB * 8]; };   // dims 32 b + 8 g + i
  struct Sum { float l; };             // the lane's own keys
  struct Probs { float p[8]; };
  static __device__ __forceinline__ void query(Query& f, const float* row, int hd, int lane) {
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      const int d = 32 * b + 8 * (lane >> 4);
      f32x4 x = {0.f, 0.f, 0.f, 0.f}, y = x;
      if (row && d < hd) {
        x = reinterpret_cast<const f32x4*>(row + d)[0];
        y = reinterpret_cast<const f32x4*>(row + d)[1];
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        f.q[8 * b + i] = x[i];
        f.q[8 * b + 4 + i] = y[i];
      }
    }
  }
  struct Keys { float k[NB * 8]; };
  static __device__ __forceinline__ void keys(Keys& f, const P& p) {
    unrolled<NB>([&](auto b_c) {
      constexpr int b = decltype(b_c)::value;
      const float s = p.template k_scale<b>();
      auto two = [&](int i, f32x2 v) { f.k[8 * b + i] = v[0]; f.k[8 * b + i + 1] = v[1]; };
      if constexpr (KB == 4) {
        two(0, kvq_f32_of4<0>(p.k[b], s));
        two(2, kvq_f32_of4<1>(p.k[b], s));
        two(4, kvq_f32_of4<2>(p.k[b], s));
        two(6, kvq_f32_of4<3>(p.k[b], s));
      } else {
        two(0, kvq_f32_of8<0>(p.k[2 * b], s));
        two(2, kvq_f32_of8<1>(p.k[2 * b], s));
        two(4, kvq_f32_of8<0>(p.k[2 * b + 1], s));
        two(6, kvq_f32_of8<1>(p.k[2 * b + 1], s));
      }
    });
  }
  static __device__ __forceinline__ f32x4 scores(const Keys& k, const Query& q) {
    f32x4 s = {0.f, 0.f, 0.f, 0.f}, t = s;
#pragma unroll
    for (int i = 0; i < NB * 8; i += 2) {
      s = __builtin_amdgcn_mfma_f32_16x16x4f32(k.k[i], q.q[i], s, 0, 0, 0);
      t = __builtin_amdgcn_mfma_f32_16x16x4f32(k.k[i + 1], q.q[i + 1], t, 0, 0, 0);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) s[i] += t[i];
    return s;
  }
  static __device__ __forceinline__ void probs(Probs& f, const float (&p)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) f.p[i] = p[i];
  }
  static __device__ __forceinline__ void sum(Sum& l, const Probs&, const float (&p)[8]) {
    l.l += ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
  }
  static __device__ __forceinline__ void scale_sum(Sum& l, float f) { l.l *= f; }
  static __device__ __forceinline__ float total(const Sum& l) { return quarter_sum(l.l); }
  struct Values { float v[2][8]; };
  template <int B>
  static __device__ __forceinline__ void values(Values& f, const P& a, const P& b) {
    auto page = [&](int at, const P& p) {
      unrolled<4>([&](auto k_c) {
        constexpr int k = decltype(k_c)::value;
        const float s = p.template v_scale<k, B>();
        f32x2 x;
        if constexpr (VB == 4) x = kvq_f32_of4<k>(p.v[B], s);
        else x = kvq_f32_of8<k & 1>(p.v[2 * B + k / 2], s);
        f.v[0][at + k] = x[0];
        f.v[1][at + k] = x[1];
      });
    };
    page(0, a);
    page(4, b);
  }
  static __device__ __forceinline__ bool clear(Values& f, unsigned there) {
    bool odd = false;
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        f.v[h][i] = there >> i & 1 ? f.v[h][i] : 0.f;
        odd |= odd_bits(f.v[h][i]);
      }
    return odd;
  }
  static __device__ __forceinline__ void mark(Values& w, const Values& f, bool minus) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int i = 0; i < 8; ++i) w.v[h][i] = odd_bits(f.v[h][i]) && !(minus ? f.v[h][i] > 0.f : f.v[h][i] < 0.f) ? 1.f : 0.f;
  }
  static __device__ __forceinline__ void drop(Values& f) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int i = 0; i < 8; ++i) f.v[h][i] = odd_bits(f.v[h][i]) ? 0.f : f.v[h][i];
  }
  static __device__ __forceinline__ void add(f32x4& lo, f32x4& hi, const Values& v, const Probs& p) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      lo = __builtin_amdgcn_mfma_f32_16x16x4f32(v.v[0][i], p.p[i], lo, 0, 0, 0);
      hi = __builtin_amdgcn_mfma_f32_16x16x4f32(v.v[1][i], p.p[i], hi, 0, 0, 0);
    }
  }
};

template <typename T> __device__ __forceinline__ void store_row4(T* p, f32x4 v);
template <> __device__ __forceinline__ void store_row4<float>(float* p, f32x4 v) { *reinterpret_cast<f32x4*>(p) = v; }
template <> __device__ __forceinline__ void store_row4<bf16_t>(bf16_t* p, f32x4 v) { *reinterpret_cast<u32x2*>(p) = (u32x2){pair_of(v[0], v[1]), pair_of(v[2], v[3])}; }

// What a sequence's rows see: the same in the attention and the merge launch.
struct SeqRows {
  int len, count, n_tok;
  bool odd;   // a length or count that the call does not have
  __device__ __forceinline__ SeqRows(const KvqAttn& a, int s) {
    const int cap = a.mpps * DF_PAGE, c = a.counts ? a.counts[s] : a.rows, n = a.lens[s];
    len = min(max(n, 0), cap);
    count = min(max(c, 0), a.rows);
    n_tok = count > 0 ? min(len + count, cap) : 0;
    odd = c > a.rows || (count > 0 && (n < 0 || n > cap - count));
  }
  // keys in front of the first one that slot j does not see
  __device__ __forceinline__ int end(const KvqAttn& a, int j) const { return a.causal ? min(len + j + 1, n_tok) : n_tok; }
};

// slot and query head of a row; groups are powers of two as a rule, and a division costs 30 instructions
__device__ __forceinline__ void slot_of(int row, int group, int& slot, int& head) {
  if ((group & (group - 1)) == 0) {
    slot = row >> __builtin_ctz(group);
    head = row & (group - 1);
  } else {
    slot = row / group;
    head = row - slot * group;
  }
}

// Ranges.  The lengths are on the device, the host knows a bound: so the launch has a number of workgroups a head, and every one of them finds its share by itself.
// Ranges are as long for all sequences, so that about a.parts of them come out, and are counted through the sequences; workgroups behind the last one have nothing to do.
// (Cut by the longest sequence, 32 single tokens behind 1k to 32k tokens kept 72 % of the CUs busy.)
__device__ __forceinline__ int wave_scan(int x) {   // sum over the lanes up to this one
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);   // row_shr:1, 2, 4, 8
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);   // row_bcast:15, :31
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);
  return x;
}
struct Ranges {
  int chunk;   // keys, a multiple of 128
  int lane, own;   // page pairs of the sequence of this lane, of the first 64
  __device__ __forceinline__ static int pairs(const KvqAttn& a, int s) { return s < a.n_seqs ? (SeqRows(a, s).n_tok + 31) / 32 : 0; }
  __device__ __forceinline__ Ranges(const KvqAttn& a) : lane(threadIdx.x & 63), own(pairs(a, lane)) {
    float all = 0.f;   // in four pairs of pages
    for (int s0 = 0; s0 < a.n_seqs; s0 += 64) all += (float)__builtin_amdgcn_readlane(wave_scan(((s0 ? pairs(a, s0 + lane) : own) + 3) / 4), 63);
    chunk = kvq_chunk(all, a.parts);
  }
  __device__ __forceinline__ int count(int tokens) const { return (int)(((unsigned)tokens + (unsigned)chunk - 1) / (unsigned)chunk); }
  // the sequence that the f-th range belongs to, and the first of its ranges; false: there are not as many
  __device__ __forceinline__ bool find(const KvqAttn& a, int f, int& s, int& first) const {
    int before = 0;
    for (int s0 = 0; s0 < a.n_seqs; s0 += 64) {
      const int mine = ((s0 ? pairs(a, s0 + lane) : own) + chunk / 32 - 1) / (chunk / 32), upto = wave_scan(mine);
      const unsigned long long behind = __ballot(before + upto > f);
      if (behind) {
        const int at = __ffsll(behind) - 1;
        s = s0 + at;
        first = before + __builtin_amdgcn_readlane(upto - mine, at);
        return true;
      }
      before += __builtin_amdgcn_readlane(upto, 63);
    }
    return false;
  }
  __device__ __forceinline__ int first_of(const KvqAttn& a, int s) const {
    int before = 0;
    for (int s0 = 0; s0 < s; s0 += 64) {
      const int l = s0 + lane;
      before += __builtin_amdgcn_readlane(wave_scan(l < s ? ((s0 ? pairs(a, l) : own) + chunk / 32 - 1) / (chunk / 32) : 0), 63);
    }
    return before;
  }
};

// ---- a wavefront's rows: 16 RB of them, a column of 16 each ----------------------------------------------------------------------
// A pair of pages: where it begins, and whether its pages are there; a lane has keys 4g .. 4g + 3 of both.
struct Seen {
  int base, g;
  bool ok_a, ok_b;
  __device__ __forceinline__ unsigned before(int stop) const {   // those of the lane's eight keys in front of `stop` + 4 g, a bit each
    const int left = stop - base, a4 = ok_a ? min(max(left, 0), 4) : 0, b4 = ok_b ? min(max(left - DF_PAGE, 0), 4) : 0;
    return ((1u << a4) - 1) | ((1u << b4) - 1) << 4;
  }
};
template <typename M, int NB, int RB>
struct State {
  f32x4 acc[RB][2 * NB];
  typename M::Sum sum[RB];
  float m_run[RB];   // in units of the scores
  int row_end[RB];   // keys in front of the first one that the row does not see, less 4 g
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      m_run[rb] = -INFINITY;
      sum[rb] = {};
#pragma unroll
      for (int t = 0; t < 2 * NB; ++t) acc[rb][t] = (f32x4){0.f, 0.f, 0.f, 0.f};
    }
  }
  // sums that are infinite or NaN, or of weights that are next to nothing
  __device__ __forceinline__ bool unsound() const {
    float t = 0.f;
    bool odd = false;
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      const float l = M::total(sum[rb]);
      odd |= m_run[rb] != -INFINITY && !(l >= kLeast && l < INFINITY);
#pragma unroll
      for (int b = 0; b < 2 * NB; ++b)
#pragma unroll
        for (int i = 0; i < 4; ++i) t = __builtin_fmaf(acc[rb][b][i], 0.f, t);
    }
    return odd || t != 0.f;
  }
  // scores of both pages -> weights; masks where edge is set.  again: the second time
  __device__ __forceinline__ void weigh(typename M::Probs (&pr)[RB], const f32x4 (&sa)[RB], const f32x4 (&sb)[RB], const Seen& at, bool edge, float scale2, float slack, bool again) {
    float all[RB][8], ref[RB];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      float (&v)[8] = all[rb];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        v[k] = sa[rb][k];
        v[4 + k] = sb[rb][k];
      }
      if (edge) {
        asm volatile("");   // a branch, not selects in every turn
        const int left = row_end[rb] - at.base, left_a = at.ok_a ? left : 0, left_b = at.ok_b ? left - DF_PAGE : 0;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          v[k] = k < left_a ? v[k] : -INFINITY;
          v[4 + k] = k < left_b ? v[4 + k] : -INFINITY;
        }
      }
      float mx = max3(max3(v[0], v[1], v[2]), max3(v[3], v[4], v[5]), max3(v[5], v[6], v[7]));
      if (__ballot(mx > m_run[rb] + slack)) {   // (from minus infinity: the first keys)
        mx = fmaxf(quarter_max(mx), m_run[rb]);
        const float f = m_run[rb] == mx ? 1.f : __builtin_amdgcn_exp2f(scale2 * (m_run[rb] - mx));
        m_run[rb] = mx;
        M::scale_sum(sum[rb], f);
#pragma unroll
        for (int t = 0; t < 2 * NB; ++t) acc[rb][t] *= f;
      }
      ref[rb] = m_run[rb] == -INFINITY ? 0.f : scale2 * m_run[rb];
    }
    if (again) {
      asm volatile("");
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
#pragma unroll
        for (int k = 0; k < 8; ++k) all[rb][k] -= m_run[rb] == -INFINITY ? 0.f : m_run[rb];
        ref[rb] = kLift;
      }
    }
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      float p[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) p[k] = __builtin_amdgcn_exp2f(__builtin_fmaf(all[rb][k], scale2, -ref[rb]));
      M::probs(pr[rb], p);
      M::sum(sum[rb], pr[rb], p);
    }
  }
  // Values where some row does not see some key: those from `end` on are not there; those that are not finite, whose product with a weight of 0 would be NaN, are left out,
  // and whether there are any.
  __device__ __forceinline__ static bool finite_values(typename M::Values& v, const Seen& at, int end) {
    const bool odd = M::clear(v, at.before(end - 4 * at.g));
    if (__ballot(odd) == 0) return false;
    M::drop(v);
    return true;
  }
  // What was left out of a pair, behind the sweep (in it, sums that a rare branch changes would cost the registers a second time): how many such values a row sees, by sign,
  // are products too, and one is enough.
  template <typename P>
  __device__ __forceinline__ void add_left_out(const unsigned char* unit_a, const unsigned char* unit_b, const Seen& at, int end, int lane) {
    P pa, pb;
    pa.load_v(unit_a, lane);
    pb.load_v(unit_b, lane);
    unrolled<NB>([&](auto b_c) {
      constexpr int b = decltype(b_c)::value;
      typename M::Values v, w;
      M::template values<b>(v, pa, pb);
      M::clear(v, at.before(end - 4 * at.g));
#pragma unroll
      for (int sign = 0; sign < 2; ++sign) {
        M::mark(w, v, sign);
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
          const unsigned sees = at.before(row_end[rb]);
          float see[8];
#pragma unroll
          for (int k = 0; k < 8; ++k) see[k] = sees >> k & 1 ? 1.f : 0.f;
          typename M::Probs seen;
          M::probs(seen, see);
          f32x4 n[2] = {};
          M::add(n[0], n[1], w, seen);
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[rb][2 * b + h][i] += n[h][i] > 0.f ? (sign ? -INFINITY : INFINITY) : 0.f;
        }
      }
    });
  }
  template <int B>
  __device__ __forceinline__ void add(const typename M::Values& v, const typename M::Probs (&pr)[RB]) {
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) M::add(acc[rb][2 * B], acc[rb][2 * B + 1], v, pr[rb]);
  }
};

// A page of a head, UNIT contiguous bytes, from memory to LDS at byte `to`: 1 KB a copy (16 bytes a lane, offsets count on both sides), the last one by as many lanes as are left.
// One piece of assembly a page: whatever the compiler keeps in m0 is put back once, and the lanes are cut and restored without a branch.  All lanes have to be on.
template <int UNIT, bool NT>
__device__ __forceinline__ void copy_page(const unsigned char* from, unsigned to, unsigned voff) {
  constexpr int FULL = UNIT / 1024;
  constexpr unsigned long long REST = (1ull << (UNIT % 1024 / 16)) - 1;
  static_assert(FULL <= 4 && REST != 0, "offsets below 4096; scales are always left");
  to = __builtin_amdgcn_readfirstlane(to);
  unsigned keep_m0;
  unsigned long long keep_exec;
#define KVQ_BEGIN "s_mov_b32 %0, m0\n\ts_mov_b32 m0, %2\n\ts_mov_b64 %1, exec\n\ts_nop 0\n\t"
#define KVQ_COPY(off, nt) "global_load_lds_dwordx4 %3, %4 offset:" #off nt "\n\t"
#define KVQ_REST "s_mov_b64 exec, %5\n\ts_nop 0\n\t"
#define KVQ_END "s_mov_b64 exec, %1\n\ts_nop 0\n\ts_mov_b32 m0, %0"
#define KVQ_ASM(text) asm volatile(KVQ_BEGIN text KVQ_END : "=&s"(keep_m0), "=&s"(keep_exec) : "s"(to), "v"(voff), "s"(from), "s"(REST) : "memory")
#define KVQ_PAGE(nt)                                                                                                            \
  if constexpr (FULL == 0) KVQ_ASM(KVQ_REST KVQ_COPY(0, nt));                                                                   \
  else if constexpr (FULL == 1) KVQ_ASM(KVQ_COPY(0, nt) KVQ_REST KVQ_COPY(0x400, nt));                                          \
  else if constexpr (FULL == 2) KVQ_ASM(KVQ_COPY(0, nt) KVQ_COPY(0x400, nt) KVQ_REST KVQ_COPY(0x800, nt));                      \
  else if constexpr (FULL == 3) KVQ_ASM(KVQ_COPY(0, nt) KVQ_COPY(0x400, nt) KVQ_COPY(0x800, nt) KVQ_REST KVQ_COPY(0xc00, nt));  \
  else KVQ_ASM(KVQ_COPY(0, nt) KVQ_COPY(0x400, nt) KVQ_COPY(0x800, nt) KVQ_COPY(0xc00, nt))
  if constexpr (NT) { KVQ_PAGE(" nt"); }
  else { KVQ_PAGE(""); }
  if constexpr (FULL == 4) {   // the rest lies behind the largest offset
    from += 4096;
    to += 4096;
    if constexpr (NT) KVQ_ASM(KVQ_REST KVQ_COPY(0, " nt"));
    else KVQ_ASM(KVQ_REST KVQ_COPY(0, ""));
  }
#undef KVQ_PAGE
#undef KVQ_ASM
#undef KVQ_END
#undef KVQ_REST
#undef KVQ_COPY
#undef KVQ_BEGIN
}

// grid: kv heads (fastest) x row tiles x ranges, or sequences where each is one range (a.parts = 0)
template <typename T, int NB, int KB, int VB, int RB>
struct Launch {
  static constexpr int UNIT = kvq_unit(NB, KB, VB), LD = NB * 32 + 4, WAVES = 4;
  static constexpr bool F32 = std::is_same<T, float>::value, Q_LDS = RB == 4;   // the queries beside 64 rows' sums are too many for the registers
  // A wavefront's ring of page pairs as they lie in memory, filled by direct-to-LDS copies: what is on its way costs no registers.  Two pairs: three or four leave room for
  // fewer workgroups and gain nothing (an earlier form of the loop, single tokens 133, 133, 144 us; blocks of 16 rows 42, 42, 65).
  static constexpr int PAIR = 2 * UNIT, NI = 2 * ((UNIT + 1023) / 1024);   // bytes, copies a pair
  static constexpr int RING = WAVES * PAIR * 2, MERGE = WAVES * 16 * LD * 4, RAW = RING > MERGE ? RING : MERGE;
  // Where a sequence's rows are one tile nobody else reads these bytes, and they need no place in L2 (single tokens 125 -> 119 us).
  static constexpr bool ONCE = !F32 && (RB == 1 || (RB == 2 && kvq_tiles_of_64(NB, KB, VB)));
  static constexpr int ON_SIMD = RB == 1 && KB + VB < 16 ? 3 : 2;   // wavefronts
};
template <typename T, int NB, int KB, int VB, int RB>
__global__ __launch_bounds__((64 * Launch<T, NB, KB, VB, RB>::WAVES), (Launch<T, NB, KB, VB, RB>::ON_SIMD)) void kvq_attn_kernel(KvqAttn a) {
  using L = Launch<T, NB, KB, VB, RB>;
  using M = Math<T, NB, KB, VB>;
  using P = typename M::P;
  constexpr int UNIT = L::UNIT, LD = L::LD, PAIR = L::PAIR, NI = L::NI, WAVES = L::WAVES;
  constexpr bool Q_LDS = L::Q_LDS;
  constexpr int QP = sizeof(typename M::Query) / 16;   // 16-byte pieces of a lane's queries, a lane's neighbour's beside each (a lane's behind each other: four lanes a bank)
  __shared__ u32x4 s_q[Q_LDS ? RB : 1][QP][Q_LDS ? 64 : 1];
  __shared__ float s_m[WAVES][RB * 16], s_l[WAVES][RB * 16], s_lift[WAVES];
  __shared__ __attribute__((aligned(1024))) unsigned char s_raw[L::RAW];   // the ring, then the wavefronts' outputs
  float (*s_o)[16][LD] = reinterpret_cast<float (*)[16][LD]>(s_raw);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, g = lane >> 4, col = lane & 15;
  const int H = a.c.n_kv_heads, hd = a.c.hd, group = a.n_q_heads / H;
  const int kvh = blockIdx.x % H, tile = blockIdx.x / H % a.tiles, part = blockIdx.x / H / a.tiles;
  int s = part, first = part, chunk = 0x7FFFFF80;
  if (a.parts) {
    const Ranges ranges(a);
    chunk = ranges.chunk;
    if (!ranges.find(a, part, s, first)) return;
  }
  const int split = part - first;
  const SeqRows rows(a, s);
  const int row0 = tile * 16 * RB, n_rows = min(rows.count * group - row0, 16 * RB);
  if (rows.odd && split + kvh + tile == 0 && threadIdx.x == 0) atomicOr(a.status, DF_STATUS_CAPACITY);
  if (n_rows <= 0) return;
  const int end = rows.end(a, (row0 + n_rows - 1) / group);      // keys that some row of the tile sees
  const int all_see = rows.end(a, row0 / group);                 // ... that all rows see
  if (end <= split * (long long)chunk) return;
  const int c0 = split * chunk, c1 = min(end - c0, chunk) + c0;

  typename M::Query q[Q_LDS ? 1 : RB];
  State<M, NB, RB> st;
  st.clear();
  const T* q_base = static_cast<const T*>(a.q);
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    const int r = rb * 16 + col;
    int j, h;
    slot_of(row0 + min(r, n_rows - 1), group, j, h);
    const T* p = q_base + ((size_t)(s * (size_t)a.rows + j) * a.n_q_heads + kvh * group + h) * hd;
    st.row_end[rb] = rows.end(a, j) - 4 * g;
    if constexpr (Q_LDS) {
      if (wave == rb) {
        typename M::Query f;
        M::query(f, r < n_rows ? p : nullptr, hd, lane);
#pragma unroll
        for (int i = 0; i < QP; ++i) {
          u32x4 x;
          __builtin_memcpy(&x, reinterpret_cast<const char*>(&f) + 16 * i, 16);
          s_q[rb][i][lane] = x;
        }
      }
    } else {
      M::query(q[rb], r < n_rows ? p : nullptr, hd, lane);
    }
  }
  if constexpr (Q_LDS) __syncthreads();
  auto query = [&](int rb) {
    if constexpr (Q_LDS) {
      typename M::Query f;
#pragma unroll
      for (int i = 0; i < QP; ++i) {
        const u32x4 x = s_q[rb][i][lane];
        __builtin_memcpy(reinterpret_cast<char*>(&f) + 16 * i, &x, 16);
      }
      return f;
    } else {
      return q[rb];
    }
  };
  // this wavefront's pairs of pages
  const int pairs = (c1 - c0 + 31) / 32, per = (pairs + WAVES - 1) / WAVES;
  const int p0 = wave * per, p1 = min(p0 + per, pairs);
  const int32_t* table = a.table + (size_t)s * a.mpps + c0 / DF_PAGE;
  const int last_page = (c1 - c0 + DF_PAGE - 1) / DF_PAGE - 1;    // of the range
  const unsigned char* layer = a.c.data + (size_t)a.layer * a.c.n_pages * H * UNIT + (size_t)kvh * UNIT;
  const size_t page_bytes = (size_t)H * UNIT;
  const float scale2 = a.scale * 1.44269504088896340736f, slack = kSlack / scale2;

  // ids of 32 pairs at a time, lane l has page l of them (-1: not there); the next ones are asked for when a set has been used up, and waited for in a branch of their own: where
  // every turn used a register that a load may still be on its way to, the compiler would have every turn wait for all copies
  auto load_ids = [&](int p) { return table[min(2 * p + lane, last_page)]; };
  auto there_or_not = [&](int id) { return id >= 0 && id < a.c.n_pages ? id : -1; };
  int ids = load_ids(p0), ids_next = load_ids(p0 + 32), fresh = 0;
  const unsigned ring = (unsigned)(size_t)&s_raw[0] + (unsigned)wave * (PAIR * 2);
  const unsigned char* my_ring = s_raw + wave * (PAIR * 2);
  const unsigned voff = lane * 16;
  auto unit_of = [&](int id) { return layer + (uint64_t)(unsigned)max(id, 0) * (unsigned)page_bytes; };   // pages that are not there alias a readable one and weigh nothing
  struct Ids { int a, b; };
  auto fetch = [&](int k, int slot) {
    const int from = k & 32 ? ids_next : ids;
    const Ids id = {__builtin_amdgcn_readlane(from, (k & 31) * 2), __builtin_amdgcn_readlane(from, (k & 31) * 2 + 1)};
    copy_page<UNIT, L::ONCE>(unit_of(id.a), ring + slot * PAIR, voff);
    copy_page<UNIT, L::ONCE>(unit_of(id.b), ring + slot * PAIR + UNIT, voff);
    return id;
  };
  bool left_out = false;
  int again = 0;   // the second time
  auto work = [&](const unsigned char* pair, const Seen& at, bool edge) {   // edge: some row does not see some key
    typename M::Probs pr[RB];
    f32x4 sa[RB], sb[RB];
    {
      P page;
      typename M::Keys ka, kb;
      page.load_k(pair, lane);
      M::keys(ka, page);
      page.load_k(pair + UNIT, lane);
      M::keys(kb, page);
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        if constexpr (Q_LDS) asm volatile("" ::: "memory");   // one row block's queries at a time
        const typename M::Query f = query(rb);
        sa[rb] = M::scores(ka, f);
        sb[rb] = M::scores(kb, f);
      }
    }
    P pa, pb;
    pa.load_v(pair, lane);
    pb.load_v(pair + UNIT, lane);
    st.weigh(pr, sa, sb, at, edge, scale2, slack, again != 0);
    typename M::Values v[L::F32 ? 1 : NB];   // bf16: all blocks, and one branch for the edge; fp32: block by block
    auto block = [&](auto b_c) -> typename M::Values& { return v[L::F32 ? 0 : decltype(b_c)::value]; };
    unrolled<NB>([&](auto b_c) {
      constexpr int b = decltype(b_c)::value;
      M::template values<b>(block(b_c), pa, pb);
      if constexpr (L::F32) {
        if (edge) {
          asm volatile("");
          left_out |= st.finite_values(block(b_c), at, end);
        }
        st.template add<b>(block(b_c), pr);
      }
    });
    if constexpr (!L::F32) {
      if (edge) {
        asm volatile("");
#pragma unroll
        for (int b = 0; b < NB; ++b) left_out |= st.finite_values(v[b], at, end);
      }
      unrolled<NB>([&](auto b_c) { st.template add<decltype(b_c)::value>(block(b_c), pr); });
    }
  };
  if (p0 < p1) {
    const int n = p1 - p0;
    ids = there_or_not(ids);
    ids_next = there_or_not(ids_next);
    asm volatile("" : "+v"(ids), "+v"(ids_next));
#pragma unroll 1
    for (;;) {
      int slot = 0;   // of the ring, of the pair at hand
      Ids next = fetch(0, 0);
#pragma unroll 1
      for (int k = 0; k < n; ++k) {
        if ((k & 31) == 0 && k) fresh = load_ids(p0 + k + 32);
        if ((k & 31) == 16 && k > 16) {
          fresh = there_or_not(fresh);
          asm volatile("" : "+v"(fresh));
          if (k & 32) ids = fresh;
          else ids_next = fresh;
        }
        const Ids at = next;
        if (k + 1 < n) {   // into the slot that the pair before this one has left
          next = fetch(k + 1, slot ^ 1);
          __builtin_amdgcn_s_waitcnt(0x0F70 | NI);   // vmcnt: this pair's copies have landed
        } else {
          __builtin_amdgcn_s_waitcnt(0x0F70);
        }
        asm volatile("" ::: "memory");
        const int base = c0 + (p0 + k) * 32;
        const bool ok_a = at.a >= 0, ok_b = at.b >= 0;
        const unsigned char* pair = my_ring + slot * PAIR;
        work(pair, Seen{base, g, ok_a, ok_b}, base + 32 > all_see || !ok_a || !ok_b || again);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // the pair has been read before its slot is filled again
        slot ^= 1;
      }
      if (again || __ballot(st.unsound()) == 0) break;
      // again: smaller weights, and whatever value is not finite itself is left out of the products
      again = 1;
      left_out = false;
      st.clear();
      int p = p0;
      asm volatile("" : "+s"(p));   // (their places, worked out here)
      ids = there_or_not(load_ids(p));
      ids_next = there_or_not(load_ids(p + 32));
      asm volatile("" : "+v"(ids), "+v"(ids_next));
    }
    if (left_out)
#pragma unroll 1
      for (int k = 0; k < n; ++k) {
        const int base = c0 + (p0 + k) * 32, ia = there_or_not(table[min(2 * (p0 + k), last_page)]), ib = there_or_not(table[min(2 * (p0 + k) + 1, last_page)]);
        if (base + 32 > all_see || ia < 0 || ib < 0 || again) st.template add_left_out<P>(unit_of(ia), unit_of(ib), Seen{base, g, ia >= 0, ib >= 0}, end, lane);
      }
  }
  __syncthreads();   // the wavefronts' outputs overlay the ring

  // ---- the wavefronts' results become one ----
  unsigned thread = threadIdx.x;
  asm("" : "+v"(thread));   // places are worked out again: kept over the sweep they cost 64 rows' tiles registers that they do not have
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    const float l = M::total(st.sum[rb]);
    if ((thread & 48) == 0) {
      s_m[wave][rb * 16 + (thread & 15)] = st.m_run[rb];
      s_l[wave][rb * 16 + (thread & 15)] = again ? l * 0x1p40f : l;
    }
  }
  if ((thread & 63) == 0) s_lift[wave] = again ? 0x1p40f : 1.f;
  const bool whole = end <= chunk;   // the only range: nothing to merge
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    if (rb * 16 >= n_rows) break;
    if (rb) __syncthreads();
#pragma unroll
    for (int t = 0; t < 2 * NB; ++t) *reinterpret_cast<f32x4*>(&s_o[wave][thread & 15][t * 16 + (thread >> 4 & 3) * 4]) = st.acc[rb][t];
    __syncthreads();
    constexpr int LANES = WAVES * 4;   // of a row
    const int r = thread / LANES;
    if (rb * 16 + r < n_rows) {
      float m_all = -INFINITY, l = 0.f, f[WAVES];
#pragma unroll
      for (int w = 0; w < WAVES; ++w) m_all = fmaxf(m_all, s_m[w][rb * 16 + r]);
#pragma unroll
      for (int w = 0; w < WAVES; ++w) {
        const float m = s_m[w][rb * 16 + r];
        f[w] = m == m_all ? 1.f : __builtin_amdgcn_exp2f(scale2 * (m - m_all));   // (no key in any: all are minus infinity and all sums 0)
        l += f[w] * s_l[w][rb * 16 + r];
      }
      int j, h;
      slot_of(row0 + rb * 16 + r, group, j, h);
      h += kvh * group;
      const size_t at = (s * (size_t)a.rows + j) * a.n_q_heads + h, in_part = (part * (size_t)a.rows + j) * a.n_q_heads;
      const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
      for (int w = 0; w < WAVES; ++w) f[w] *= inv * s_lift[w];   // the sums' shares, before they are added: a mean is finite where a sum need not be
      for (int d = 4 * (thread % LANES); d < hd; d += 4 * LANES) {
        f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < WAVES; ++w) o += *reinterpret_cast<const f32x4*>(&s_o[w][r][d]) * f[w];
        if (whole) store_row4(static_cast<T*>(a.out) + at * hd + d, o);
        else *reinterpret_cast<f32x4*>(a.part_o + (in_part + h) * hd + d) = o;
      }
      if (!whole && thread % LANES == 0) a.part_ml[in_part + h] = make_float2(m_all, l);
    }
  }
}

// A row's ranges: 32 lanes (four dims a lane) a row, or eight times 32, which take every eighth range and are joined in their order (few rows of many ranges: 1024 rows of
// up to 12, 7.0 -> 4.2 us; 8192 rows of up to 5 are better off with 32 lanes, 11.9 -> 5.7 us; the host knows the rows, not the ranges that each has, and goes by the rows).  grid: rows of a sequence and heads / (8 / GROUPS), sequences.
template <typename T, int ROWS, int GROUPS>
__global__ __launch_bounds__(256) void kvq_merge_kernel(KvqAttn a) {
  __shared__ float s_m[8], s_l[8];
  __shared__ __attribute__((aligned(16))) float s_o[GROUPS][132];
  const int s = blockIdx.y, of = threadIdx.x >> 5, at = GROUPS == 8 ? blockIdx.x : blockIdx.x * 8 + of;
  const int group = a.n_q_heads / a.c.n_kv_heads;
  int j, h, kvh, in_group, last_slot, rest;
  slot_of(at, a.n_q_heads, j, h);
  slot_of(h, group, kvh, in_group);
  const SeqRows rows(a, s);
  const Ranges ranges(a);
  const int first = ranges.first_of(a, s);
  if (j >= rows.count) return;
  slot_of(min(((j * group + in_group) / ROWS + 1) * ROWS, rows.count * group) - 1, group, last_slot, rest);
  const int parts = ranges.count(rows.end(a, last_slot));   // of the row's tile
  if (parts <= 1) return;
  const int d = 4 * (threadIdx.x & 31), hd = a.c.hd;
  const size_t step = (size_t)a.rows * a.n_q_heads, from = (first * (size_t)a.rows + j) * a.n_q_heads + h;
  const float scale2 = a.scale * 1.44269504088896340736f;
  float m = -INFINITY, l = 0.f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  constexpr int AHEAD = 4;
  for (int p0 = GROUPS == 8 ? of : 0; p0 < parts; p0 += GROUPS * AHEAD) {
    float2 x[AHEAD];
    f32x4 y[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      const int p = min(p0 + i * GROUPS, parts - 1);
      x[i] = a.part_ml[from + p * step];
      y[i] = *reinterpret_cast<const f32x4*>(a.part_o + (from + p * step) * hd + min(d, hd - 4));
    }
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      if (p0 + i * GROUPS >= parts) break;
      const float top = fmaxf(m, x[i].x), f = m == top ? 1.f : __builtin_amdgcn_exp2f(scale2 * (m - top));
      const float fx = x[i].x == top ? 1.f : __builtin_amdgcn_exp2f(scale2 * (x[i].x - top));
      const float all = f * l + fx * x[i].y, inv = all == 0.f ? 0.f : __builtin_amdgcn_rcpf(all);
      o = o * (f * l * inv) + y[i] * (fx * x[i].y * inv);
      m = top;
      l = all;
    }
  }
  if constexpr (GROUPS == 8) {
    *reinterpret_cast<f32x4*>(&s_o[of][d]) = o;
    if (d == 0) {
      s_m[of] = m;
      s_l[of] = l;
    }
    __syncthreads();
    if (of) return;
    float m_all = -INFINITY, f[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) m_all = fmaxf(m_all, s_m[i]);
    l = 0.f;
    o = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      f[i] = s_l[i] * (s_m[i] == m_all ? 1.f : __builtin_amdgcn_exp2f(scale2 * (s_m[i] - m_all)));
      l += f[i];
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
    for (int i = 0; i < 8; ++i) o += *reinterpret_cast<const f32x4*>(&s_o[i][d]) * (f[i] * inv);
  }
  if (d < hd) store_row4(static_cast<T*>(a.out) + ((s * (size_t)a.rows + j) * a.n_q_heads + h) * hd + d, o);
}

template <typename T, int NB, int KB, int VB>
void launch(const KvqAttn& a, int tile, hipStream_t st) {
  const dim3 grid((unsigned)((long long)(a.n_seqs + a.parts) * a.tiles * a.c.n_kv_heads));
  auto go = [&](auto rb_c) {
    constexpr int RB = decltype(rb_c)::value;
    hipLaunchKernelGGL((kvq_attn_kernel<T, NB, KB, VB, RB>), grid, dim3(64 * Launch<T, NB, KB, VB, RB>::WAVES), 0, st, a);
  };
  if (tile == 16) go(std::integral_constant<int, 1>());
  else if constexpr (std::is_same<T, bf16_t>::value) {
    if (tile == 32) go(std::integral_constant<int, 2>());
    else if constexpr (kvq_tiles_of_64(NB, KB, VB)) go(std::integral_constant<int, 4>());
  }
}
template <typename T>
void launch_merge(const KvqAttn& a, int tile, hipStream_t st) {
  auto go = [&](auto rows_c) {
    constexpr int ROWS = decltype(rows_c)::value;
    const int rows = a.rows * a.n_q_heads;
    if ((long long)rows * a.n_seqs < 4096) hipLaunchKernelGGL((kvq_merge_kernel<T, ROWS, 8>), dim3(rows, a.n_seqs), dim3(256), 0, st, a);
    else hipLaunchKernelGGL((kvq_merge_kernel<T, ROWS, 1>), dim3((rows + 7) / 8, a.n_seqs), dim3(256), 0, st, a);
  };
  if (tile == 16) go(std::integral_constant<int, 16>());
  else if constexpr (std::is_same<T, bf16_t>::value) {
    if (tile == 32) go(std::integral_constant<int, 32>());
    else go(std::integral_constant<int, 64>());
  }
}
int tile_rows(const KvqAttn& a, bool bf16) {
  return kvq_tile_rows(bf16, a.rows * (a.n_q_heads / a.c.n_kv_heads), kvq_tiles_of_64(kvq_blocks(a.c.hd), a.c.k_bits, a.c.v_bits));
}
template <typename T, int NB>
void launch_bits(const KvqAttn& a, int rb, hipStream_t st) {
  if (a.c.k_bits == 4) a.c.v_bits == 4 ? launch<T, NB, 4, 4>(a, rb, st) : launch<T, NB, 4, 8>(a, rb, st);
  else a.c.v_bits == 4 ? launch<T, NB, 8, 4>(a, rb, st) : launch<T, NB, 8, 8>(a, rb, st);
}
template <typename T>
void launch_type(const KvqAttn& a, int rb, hipStream_t st) {
  switch (kvq_blocks(a.c.hd)) {
    case 1: launch_bits<T, 1>(a, rb, st); break;
    case 2: launch_bits<T, 2>(a, rb, st); break;
    case 3: launch_bits<T, 3>(a, rb, st); break;
    default: launch_bits<T, 4>(a, rb, st);
  }
}

}  // namespace

bool kvq_attn_plan(KvqAttn& a, bool bf16, int max_tokens, size_t part_rows) {
  const KvqPlan p = kvq_plan(a.n_seqs, a.rows, a.n_q_heads, a.c.n_kv_heads, bf16, kvq_tiles_of_64(kvq_blocks(a.c.hd), a.c.k_bits, a.c.v_bits), max_tokens, part_rows);
  a.tiles = p.tiles;
  a.parts = p.parts;
  return (a.n_seqs + (long long)a.parts) * a.c.n_kv_heads * a.tiles <= 0x7FFFFFFFll;
}

void kvq_attn_launch(const KvqAttn& a, bool bf16, hipStream_t st) {
  if (bf16) launch_type<bf16_t>(a, tile_rows(a, true), st);
  else launch_type<float>(a, tile_rows(a, false), st);
}
void kvq_merge_launch(const KvqAttn& a, bool bf16, hipStream_t st) {
  if (bf16) launch_merge<bf16_t>(a, tile_rows(a, true), st);
  else launch_merge<float>(a, tile_rows(a, false), st);
}
