// Block attention over a cache held in 4 or 8 bits (kvq.h).
//
//   o_r = sum over the keys i that row r sees of softmax_i(scale q_r . k_i) v_i,    k_i, v_i = codes times 2^(e - 127) of their blocks, exactly.
//
// Row r of a kv head = (slot of the block) * group + query head.  A workgroup takes up to 16 RB of them and a range of keys, its four wavefronts a quarter of the range
// each, pages in pairs.  Codes become bf16 (fp32 models: fp32) in registers by the conversion instructions that take the block's scale, both exact: e2m1 and e4m3 numbers have
// 2 and 4 significant bits.  S^T = K Q^T leaves a lane four consecutive keys of a query column, which is how V^T P^T takes them.  Softmax in one pass,
// base 2, with a reference maximum that moves only when a score passes it by kSlack.  bf16 models: probabilities are rounded to bf16, by 2^-9 of themselves each, where
// V itself is held to 2^-2 or 2^-4 of its block; their sum is taken over the rounded ones, so the weights still add up to one.  All sums in fp32.
// Ranges of keys are joined by kvq_merge_kernel in a fixed order: a call repeats itself bit for bit.
#include <algorithm>
#include <type_traits>
#include <utility>

#include "kvq.h"

namespace {

constexpr int kWaves = 4;
constexpr float kSlack = 8.f;   // probabilities up to 2^8 above the reference: nothing that fp32 sums or bf16 exponents notice

__device__ __forceinline__ uint32_t pair_of(float a, float b) { return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2){a, b}, bf16x2)); }
__device__ __forceinline__ uint32_t finite_half(uint32_t x, uint32_t exponent) { return (x & exponent) == exponent ? 0u : x; }
__device__ __forceinline__ uint32_t finite_halves(uint32_t x) { return finite_half(x & 0xFFFFu, 0x7F80u) | finite_half(x & 0xFFFF0000u, 0x7F800000u); }
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
  struct Sum { f32x4 l; };          // all four and all four lanes of a column the same
  struct Probs { u32x4 p; };        // four keys of the first page, four of the second
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
    for (int i = 0; i < 4; ++i) f.p[i] = pair_of(p[2 * i], p[2 * i + 1]);
  }
  static __device__ __forceinline__ void sum(Sum& l, const Probs& p, const float (&)[8]) {
    const u32x4 ones = {0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u};
    l.l = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, ones), __builtin_bit_cast(bf16x8, p.p), l.l, 0, 0, 0);
  }
  static __device__ __forceinline__ void scale_sum(Sum& l, float f) { l.l *= f; }
  static __device__ __forceinline__ float total(const Sum& l) { return l.l[0]; }
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
  // elements of keys that nobody sees (there: a bit a key) become 0, and so do those that are not finite; whether there were any of these
  static __device__ __forceinline__ bool clear(Values& f, unsigned there) {
    uint32_t odd = 0;
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t x = f.v[h][i] & ((there >> (2 * i) & 1 ? 0x0000FFFFu : 0u) | (there >> (2 * i) & 2 ? 0xFFFF0000u : 0u)), y = finite_halves(x);
        odd |= x ^ y;
        f.v[h][i] = y;
      }
    return odd != 0;
  }
  static __device__ __forceinline__ void add(f32x4& lo, f32x4& hi, const Values& v, const Probs& p) {
    lo = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, v.v[0]), __builtin_bit_cast(bf16x8, p.p), lo, 0, 0, 0);
    hi = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, v.v[1]), __builtin_bit_cast(bf16x8, p.p), hi, 0, 0, 0);
  }
  // one element as the products take it
  static __device__ __forceinline__ float element(uint32_t code, float scale, bool up) {
    const uint32_t w = VB == 4 ? kvq_bf16_of4<0>(code, scale) : kvq_bf16_of8<0>(code, scale);
    return __uint_as_float(up ? w & 0xFFFF0000u : w << 16);
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
        const float x = there >> i & 1 ? f.v[h][i] : 0.f;
        odd |= odd_bits(x);
        f.v[h][i] = odd_bits(x) ? 0.f : x;
      }
    return odd;
  }
  static __device__ __forceinline__ void add(f32x4& lo, f32x4& hi, const Values& v, const Probs& p) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      lo = __builtin_amdgcn_mfma_f32_16x16x4f32(v.v[0][i], p.p[i], lo, 0, 0, 0);
      hi = __builtin_amdgcn_mfma_f32_16x16x4f32(v.v[1][i], p.p[i], hi, 0, 0, 0);
    }
  }
  static __device__ __forceinline__ float element(uint32_t code, float scale, bool up) {
    const f32x2 v = VB == 4 ? kvq_f32_of4<0>(code, scale) : kvq_f32_of8<0>(code, scale);
    return up ? v[1] : v[0];
  }
};

// V elements that are not finite, of keys that some rows of a tile see and others do not (the block itself, under the causal mask): taken out of the products, where
// a weight of 0 would make them NaN, and added here to the rows that see them, whose sums become what they are.
template <typename M, int NB, int KB, int VB>
__device__ __forceinline__ void add_not_finite(f32x4 (&acc)[2 * NB], const unsigned char* unit, int n_keys, int lane) {
  constexpr int SROW = kvq_scale_row(NB);
  const unsigned char* codes = unit + kvq_codes(NB, KB);
  const unsigned char* scales = codes + kvq_codes(NB, VB) + DF_PAGE * SROW;
#pragma unroll 1
  for (int key = 0; key < n_keys; ++key)
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      const float s = kvq_scale_clean(scales[key * SROW + b]);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int n = 4 * (lane >> 4) + i, wide = NB - (b & ~1) < 2 ? 1 : 2;
        const uint32_t code = VB == 4 ? codes[(((key >> 2) * 16 + n) * NB + b) * 4 + (key & 3)]
                                      : *reinterpret_cast<const uint16_t*>(codes + (b >> 1) * 1024 + (((key >> 2) * 16 + n) * wide + (b & 1)) * 8 + (key & 3) * 2);
        const float lo = M::element(code, s, false), hi = M::element(code, s, true);
        acc[2 * b][i] += odd_bits(lo) ? lo : 0.f;
        acc[2 * b + 1][i] += odd_bits(hi) ? hi : 0.f;
      }
    }
}

template <typename T> __device__ __forceinline__ void store_row4(T* p, f32x4 v);
template <> __device__ __forceinline__ void store_row4<float>(float* p, f32x4 v) { *reinterpret_cast<f32x4*>(p) = v; }
template <> __device__ __forceinline__ void store_row4<bf16_t>(bf16_t* p, f32x4 v) { *reinterpret_cast<u32x2*>(p) = (u32x2){pair_of(v[0], v[1]), pair_of(v[2], v[3])}; }

// What a sequence's rows see: the same in the attention and the merge launch.
struct SeqRows {
  int len, count, n_tok;
  bool outgrown;
  __device__ __forceinline__ SeqRows(const KvqAttn& a, int s) {
    const int cap = a.mpps * DF_PAGE, c = a.counts ? a.counts[s] : a.rows, n = a.lens[s];
    len = min(max(n, 0), cap);
    count = min(max(c, 0), a.rows);
    n_tok = min(min(len + count, cap), a.limit);
    outgrown = c > a.rows || (count > 0 && (n > cap - count || n > a.limit - count));
  }
  // keys in front of the first one that slot j does not see
  __device__ __forceinline__ int end(const KvqAttn& a, int j) const { return a.causal ? min(len + j + 1, n_tok) : n_tok; }
};

// grid: kv heads (fastest) x ranges x row tiles x sequences
template <typename T, int NB, int KB, int VB, int RB>
__global__ __launch_bounds__(64 * kWaves, 2) void kvq_attn_kernel(KvqAttn a) {
  using M = Math<T, NB, KB, VB>;
  using P = typename M::P;
  constexpr int UNIT = kvq_unit(NB, KB, VB), LD = NB * 32 + 4;
  __shared__ float s_m[kWaves][RB * 16], s_l[kWaves][RB * 16];
  __shared__ __attribute__((aligned(16))) float s_o[kWaves][16][LD];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, g = lane >> 4, col = lane & 15;
  const int H = a.c.n_kv_heads, hd = a.c.hd, group = a.n_q_heads / H;
  int i = blockIdx.x;
  const int kvh = i % H;
  i /= H;
  const int split = i % a.splits;
  i /= a.splits;
  const int tile = i % a.tiles, s = i / a.tiles;
  const SeqRows rows(a, s);
  const int row0 = tile * 16 * RB, n_rows = min(rows.count * group - row0, 16 * RB);
  if (n_rows <= 0) {
    if (rows.outgrown && tile == 0 && split == 0 && kvh == 0 && threadIdx.x == 0) atomicOr(a.status, DF_STATUS_CAPACITY);
    return;
  }
  const int end = rows.end(a, (row0 + n_rows - 1) / group);      // keys that some row of the tile sees
  const int all_see = rows.end(a, row0 / group);                 // ... that all rows see
  const int c0 = split * a.chunk, c1 = min(c0 + a.chunk, end);
  if (c0 >= end && split > 0) return;
  if (rows.outgrown && split == 0 && kvh == 0 && tile == 0 && threadIdx.x == 0) atomicOr(a.status, DF_STATUS_CAPACITY);

  typename M::Query q[RB];
  int row_end[RB];
  const T* q_base = static_cast<const T*>(a.q);
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    const int r = rb * 16 + col, row = row0 + min(r, n_rows - 1), j = row / group, h = row % group;
    const T* p = q_base + ((size_t)(s * (size_t)a.rows + j) * a.n_q_heads + kvh * group + h) * hd;
    M::query(q[rb], r < n_rows ? p : nullptr, hd, lane);
    row_end[rb] = rows.end(a, j);
  }
  f32x4 acc[RB][2 * NB];
  typename M::Sum sum[RB];
  float m_run[RB];
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    m_run[rb] = -INFINITY;
    sum[rb] = {};
#pragma unroll
    for (int t = 0; t < 2 * NB; ++t) acc[rb][t] = (f32x4){0.f, 0.f, 0.f, 0.f};
  }

  // this wavefront's pairs of pages
  const int pairs = (c1 - c0 + 31) / 32, per = (pairs + kWaves - 1) / kWaves;
  const int p0 = wave * per, p1 = min(p0 + per, pairs);
  const int32_t* table = a.table + (size_t)s * a.mpps + c0 / DF_PAGE;
  const int last_page = (c1 - c0 + DF_PAGE - 1) / DF_PAGE - 1;    // of the range
  const unsigned char* layer = a.c.data + (size_t)a.layer * a.c.n_pages * H * UNIT + (size_t)kvh * UNIT;
  const size_t page_bytes = (size_t)H * UNIT;
  const float scale2 = a.scale * 1.44269504088896340736f;

  auto id_of = [&](int page) { return table[min(page, last_page)]; };
  auto valid = [&](int id) { return id >= 0 && id < a.c.n_pages; };
  auto unit_of = [&](int id) { return layer + (size_t)(valid(id) ? id : 0) * page_bytes; };
  struct Pair { P a, b; };
  auto load = [&](Pair& x, int ia, int ib) {
    const unsigned char *ua = unit_of(ia), *ub = unit_of(ib);
    x.a.load_k(ua, lane);
    x.b.load_k(ub, lane);
    x.a.load_v(ua, lane);
    x.b.load_v(ub, lane);
  };
  auto work = [&](const Pair& x, int base, int ia, int ib, auto edge_c) {
    constexpr bool EDGE = decltype(edge_c)::value;
    const bool ok_a = !EDGE || valid(ia), ok_b = !EDGE || valid(ib);
    typename M::Probs pr[RB];
    {
      typename M::Keys ka, kb;
      M::keys(ka, x.a);
      M::keys(kb, x.b);
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        const f32x4 sa = M::scores(ka, q[rb]), sb = M::scores(kb, q[rb]);
        float v[8], p[8];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          v[k] = sa[k];
          v[4 + k] = sb[k];
          if (EDGE) {
            if (!ok_a || base + 4 * g + k >= row_end[rb]) v[k] = -INFINITY;
            if (!ok_b || base + 16 + 4 * g + k >= row_end[rb]) v[4 + k] = -INFINITY;
          }
        }
        float mx = fmaxf(fmaxf(fmaxf(v[0], v[1]), fmaxf(v[2], v[3])), fmaxf(fmaxf(v[4], v[5]), fmaxf(v[6], v[7]))) * scale2;
        if (__ballot(mx > m_run[rb] + kSlack)) {   // (from minus infinity: the first keys)
          mx = fmaxf(quarter_max(mx), m_run[rb]);
          const float f = m_run[rb] == mx ? 1.f : __builtin_amdgcn_exp2f(m_run[rb] - mx);
          m_run[rb] = mx;
          M::scale_sum(sum[rb], f);
#pragma unroll
          for (int t = 0; t < 2 * NB; ++t) acc[rb][t] *= f;
        }
        const float mb = m_run[rb] == -INFINITY ? 0.f : m_run[rb];
#pragma unroll
        for (int k = 0; k < 8; ++k) p[k] = __builtin_amdgcn_exp2f(__builtin_fmaf(v[k], scale2, -mb));
        M::probs(pr[rb], p);
        M::sum(sum[rb], pr[rb], p);
      }
    }
    unsigned there = 0;
    if (EDGE) {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if (ok_a && base + 4 * g + k < end) there |= 1u << k;
        if (ok_b && base + 16 + 4 * g + k < end) there |= 16u << k;
      }
    }
    bool odd = false;
    unrolled<NB>([&](auto b_c) {
      constexpr int b = decltype(b_c)::value;
      typename M::Values v;
      M::template values<b>(v, x.a, x.b);
      if (EDGE) odd |= M::clear(v, there);
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) M::add(acc[rb][2 * b], acc[rb][2 * b + 1], v, pr[rb]);
    });
    if (EDGE && __ballot(odd)) {
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        if (ok_a) add_not_finite<M, NB, KB, VB>(acc[rb], unit_of(ia), min(max(row_end[rb] - base, 0), DF_PAGE), lane);
        if (ok_b) add_not_finite<M, NB, KB, VB>(acc[rb], unit_of(ib), min(max(row_end[rb] - base - DF_PAGE, 0), DF_PAGE), lane);
      }
    }
  };
  if (p0 < p1) {
    Pair cur, next;
    int ia = id_of(2 * p0), ib = id_of(2 * p0 + 1), na = id_of(2 * p0 + 2), nb = id_of(2 * p0 + 3);
    load(cur, ia, ib);
    for (int p = p0; p < p1; ++p) {
      const int base = c0 + p * 32;
      const int fa = id_of(2 * p + 4), fb = id_of(2 * p + 5);
      load(next, na, nb);
      if (base + 32 > all_see || base + 32 > c1 || !valid(ia) || !valid(ib)) work(cur, base, ia, ib, std::true_type());
      else work(cur, base, ia, ib, std::false_type());
      cur = next;
      ia = na;
      ib = nb;
      na = fa;
      nb = fb;
    }
  }

  // ---- the wavefronts' results become one ----
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    const float l = M::total(sum[rb]);
    if (g == 0) {
      s_m[wave][rb * 16 + col] = m_run[rb];
      s_l[wave][rb * 16 + col] = l;
    }
  }
  const int parts = (end + a.chunk - 1) / a.chunk;
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    if (rb * 16 >= n_rows) break;
    if (rb) __syncthreads();
#pragma unroll
    for (int t = 0; t < 2 * NB; ++t) *reinterpret_cast<f32x4*>(&s_o[wave][col][t * 16 + 4 * g]) = acc[rb][t];
    __syncthreads();
    const int r = threadIdx.x >> 4, row = row0 + rb * 16 + r;
    if (rb * 16 + r < n_rows) {
      float m_all = -INFINITY, l = 0.f, f[kWaves];
#pragma unroll
      for (int w = 0; w < kWaves; ++w) m_all = fmaxf(m_all, s_m[w][rb * 16 + r]);
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        const float m = s_m[w][rb * 16 + r];
        f[w] = m == m_all ? 1.f : __builtin_amdgcn_exp2f(m - m_all);   // (no key in any: all are minus infinity and all sums 0)
        l += f[w] * s_l[w][rb * 16 + r];
      }
      const int j = row / group, h = kvh * group + row % group;
      const size_t at = (s * (size_t)a.rows + j) * a.n_q_heads + h;
      const bool whole = parts <= 1;
      const float inv = whole ? (l == 0.f ? 0.f : 1.f / l) : 1.f;
      for (int d = 4 * (threadIdx.x & 15); d < hd; d += 64) {
        f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < kWaves; ++w) o += *reinterpret_cast<const f32x4*>(&s_o[w][r][d]) * f[w];
        o *= inv;
        if (whole) store_row4(static_cast<T*>(a.out) + at * hd + d, o);
        else *reinterpret_cast<f32x4*>(a.part_o + (at * a.splits + split) * hd + d) = o;
      }
      if (!whole && (threadIdx.x & 15) == 0) a.part_ml[at * a.splits + split] = make_float2(m_all, l);
    }
  }
}

// A row's ranges in their order: 32 lanes a row, four dims each.
template <typename T, int RB16>
__global__ __launch_bounds__(256) void kvq_merge_kernel(KvqAttn a, long long n_rows) {
  const long long at = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
  if (at >= n_rows) return;
  const int hq = (int)(at % a.n_q_heads), group = a.n_q_heads / a.c.n_kv_heads;
  const int j = (int)(at / a.n_q_heads % a.rows), s = (int)(at / a.n_q_heads / a.rows);
  const SeqRows rows(a, s);
  if (j >= rows.count) return;
  const int row = j * group + hq % group, tile = row / (16 * RB16);
  const int last = min((tile + 1) * 16 * RB16, rows.count * group) - 1;
  const int parts = (rows.end(a, last / group) + a.chunk - 1) / a.chunk;
  if (parts <= 1) return;
  const int d = 4 * (threadIdx.x & 31), hd = a.c.hd;
  const float2* ml = a.part_ml + at * a.splits;
  float m_all = -INFINITY;
  for (int p = 0; p < parts; ++p) m_all = fmaxf(m_all, ml[p].x);
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  float l = 0.f;
  for (int p = 0; p < parts; ++p) {
    const float2 x = ml[p];
    const float f = x.x == m_all ? 1.f : __builtin_amdgcn_exp2f(x.x - m_all);
    l += f * x.y;
    if (d < hd) o += *reinterpret_cast<const f32x4*>(a.part_o + (at * a.splits + p) * hd + d) * f;
  }
  if (d < hd) store_row4(static_cast<T*>(a.out) + at * hd + d, o * (l == 0.f ? 0.f : 1.f / l));
}

int row_blocks(bool bf16, int rows) { return rows <= 16 ? 1 : rows <= 32 || !bf16 ? 2 : 4; }

template <typename T, int NB, int KB, int VB>
void launch(const KvqAttn& a, int rb, hipStream_t st) {
  const dim3 grid((unsigned)((long long)a.n_seqs * a.tiles * a.splits * a.c.n_kv_heads)), block(64 * kWaves);
  const long long rows = (long long)a.n_seqs * a.rows * a.n_q_heads;
  const dim3 merge((unsigned)((rows + 7) / 8));
  auto go = [&](auto rb_c) {
    constexpr int RB = decltype(rb_c)::value;
    hipLaunchKernelGGL((kvq_attn_kernel<T, NB, KB, VB, RB>), grid, block, 0, st, a);
    if (a.splits > 1) hipLaunchKernelGGL((kvq_merge_kernel<T, RB>), merge, dim3(256), 0, st, a, rows);
  };
  if (rb == 1) go(std::integral_constant<int, 1>());
  else if (rb == 2) go(std::integral_constant<int, 2>());
  else if constexpr (std::is_same<T, bf16_t>::value) go(std::integral_constant<int, 4>());
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
  const int rows = a.rows * (a.n_q_heads / a.c.n_kv_heads), rb = row_blocks(bf16, rows);
  a.tiles = (rows + 16 * rb - 1) / (16 * rb);
  const long long wgs = (long long)a.n_seqs * a.c.n_kv_heads * a.tiles;
  const long long room = std::max<long long>(1, (long long)(part_rows / ((size_t)a.n_seqs * a.rows * a.n_q_heads)));
  const long long want = std::max<long long>(1, (2048 + wgs - 1) / wgs), most = std::max(1, max_tokens / 256);
  const int splits = (int)std::min(std::min(want, most), room);
  a.chunk = std::max(128, (int)(((long long)max_tokens + splits - 1) / splits + 127) / 128 * 128);
  a.splits = std::max(1, (max_tokens + a.chunk - 1) / a.chunk);
  a.limit = (int)std::min<long long>((long long)a.splits * a.chunk, 0x7FFFFFFF);
  return wgs * a.splits <= 0x7FFFFFFFll && ((long long)a.n_seqs * a.rows * a.n_q_heads + 7) / 8 <= 0x7FFFFFFFll;
}

void kvq_attn_launch(const KvqAttn& a, bool bf16, hipStream_t st) {
  const int rb = row_blocks(bf16, a.rows * (a.n_q_heads / a.c.n_kv_heads));
  if (bf16) launch_type<bf16_t>(a, rb, st);
  else launch_type<float>(a, rb, st);
}
