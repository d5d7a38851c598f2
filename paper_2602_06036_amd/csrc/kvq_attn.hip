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
  // elements that are not finite become 0 in f, and 1 in `up` (plus infinity and NaN) and `down` (minus infinity and NaN)
  static __device__ __forceinline__ void part(Values& f, Values& up, Values& down) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t x = f.v[h][i];
        auto mark = [&](uint32_t half, bool minus) { return (half & 0x7F80u) == 0x7F80u && (half & 0x7Fu || (half >> 15 != 0) == minus) ? 0x3F80u : 0u; };
        up.v[h][i] = mark(x & 0xFFFFu, false) | mark(x >> 16, false) << 16;
        down.v[h][i] = mark(x & 0xFFFFu, true) | mark(x >> 16, true) << 16;
        f.v[h][i] = finite_halves(x);
      }
  }
  static __device__ __forceinline__ void add(f32x4& lo, f32x4& hi, const Values& v, const Probs& p) {
    lo = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, v.v[0]), __builtin_bit_cast(bf16x8, p.p), lo, 0, 0, 0);
    hi = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, v.v[1]), __builtin_bit_cast(bf16x8, p.p), hi, 0, 0, 0);
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
  static __device__ __forceinline__ void part(Values& f, Values& up, Values& down) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float x = f.v[h][i];
        up.v[h][i] = odd_bits(x) && !(x < 0.f) ? 1.f : 0.f;
        down.v[h][i] = odd_bits(x) && !(x > 0.f) ? 1.f : 0.f;
        f.v[h][i] = odd_bits(x) ? 0.f : x;
      }
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
  constexpr bool Q_LDS = RB == 4 || (std::is_same<T, float>::value && RB == 2);   // the queries beside 64 rows' sums are too many for the registers
  // A wavefront's ring of page pairs as they lie in memory, filled by direct-to-LDS copies: what is on its way costs no registers.
  constexpr int PAIR = 2 * UNIT, D = kWaves * PAIR * 3 <= 53248 ? 3 : 2, NI = 2 * ((UNIT + 1023) / 1024);   // depth, copies a pair
  constexpr int RING = kWaves * PAIR * D, MERGE = kWaves * 16 * LD * 4;
  __shared__ typename M::Query s_q[Q_LDS ? RB : 1][64];
  __shared__ float s_m[kWaves][RB * 16], s_l[kWaves][RB * 16];
  __shared__ __attribute__((aligned(1024))) unsigned char s_raw[RING > MERGE ? RING : MERGE];   // the ring, then the wavefronts' outputs
  float (*s_o)[16][LD] = reinterpret_cast<float (*)[16][LD]>(s_raw);
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

  typename M::Query q[Q_LDS ? 1 : RB];
  int row_end[RB];
  const T* q_base = static_cast<const T*>(a.q);
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    const int r = rb * 16 + col, row = row0 + min(r, n_rows - 1), j = row / group, h = row % group;
    const T* p = q_base + ((size_t)(s * (size_t)a.rows + j) * a.n_q_heads + kvh * group + h) * hd;
    row_end[rb] = rows.end(a, j);
    if constexpr (Q_LDS) {
      if (wave == rb % kWaves) {
        typename M::Query f;
        M::query(f, r < n_rows ? p : nullptr, hd, lane);
        s_q[rb][lane] = f;
      }
    } else {
      M::query(q[rb], r < n_rows ? p : nullptr, hd, lane);
    }
  }
  if constexpr (Q_LDS) __syncthreads();
  auto query = [&](int rb) -> const typename M::Query& {
    if constexpr (Q_LDS) return s_q[rb][lane];
    else return q[rb];
  };
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

  auto valid = [&](int id) { return id >= 0 && id < a.c.n_pages; };
  // ids of 32 pairs at a time, lane l has page l of them; the next ones are asked for when a set has been used up, and waited for in a branch of their own: where every turn
  // used a register that a load may still be on its way to, the compiler would have every turn wait for all copies
  auto load_ids = [&](int p) { return table[min(2 * p + lane, last_page)]; };
  int ids = load_ids(p0), ids_next = load_ids(p0 + 32), fresh = 0;
  auto id_of = [&](int p, int i) { return __builtin_amdgcn_readlane((p - p0) & 32 ? ids_next : ids, ((p - p0) & 31) * 2 + i); };
  const unsigned ring = (unsigned)(size_t)&s_raw[0] + (unsigned)wave * (PAIR * D);
  const unsigned char* my_ring = s_raw + wave * (PAIR * D);
  const unsigned voff = lane * 16;
  auto copy = [&](const unsigned char* from, unsigned at) {   // 1 KB, or as far as the page goes
    const unsigned dst = __builtin_amdgcn_readfirstlane(ring + at);
    unsigned keep_m0;   // whatever the compiler keeps in m0 is put back
    asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, %3\n\ts_nop 0\n\ts_mov_b32 m0, %0"
                 : "=&s"(keep_m0) : "s"(dst), "v"(voff), "s"(from) : "memory");
  };
  auto fetch = [&](int p, int slot) {   // pages that are not there alias a readable one and weigh nothing
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int id = id_of(p, i);
      const unsigned char* unit = layer + (size_t)(valid(id) ? id : 0) * page_bytes;
#pragma unroll
      for (int c = 0; c < UNIT; c += 1024) {
        if (UNIT - c >= 1024) copy(unit + c, slot * PAIR + i * UNIT + c);
        else if (lane < (UNIT - c) / 16) copy(unit + c, slot * PAIR + i * UNIT + c);
      }
    }
  };
  // a lane's eight keys of a pair in front of `stop`, a bit each
  auto there = [&](bool ok_a, bool ok_b, int base, int stop) {
    const int left = stop - base - 4 * g, a4 = ok_a ? min(max(left, 0), 4) : 0, b4 = ok_b ? min(max(left - DF_PAGE, 0), 4) : 0;
    return ((1u << a4) - 1) | ((1u << b4) - 1) << 4;
  };
  auto work = [&](const unsigned char* pair, int base, bool ok_a, bool ok_b, bool edge) {   // edge: some row does not see some key
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
        const typename M::Query& f = query(rb);
        sa[rb] = M::scores(ka, f);
        sb[rb] = M::scores(kb, f);
      }
    }
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      float v[8], p[8];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        v[k] = sa[rb][k];
        v[4 + k] = sb[rb][k];
      }
      if (edge) {
        const int left = row_end[rb] - base - 4 * g, left_a = ok_a ? left : 0, left_b = ok_b ? left - DF_PAGE : 0;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          v[k] = k < left_a ? v[k] : -INFINITY;
          v[4 + k] = k < left_b ? v[4 + k] : -INFINITY;
        }
      }
      float mx = scale2 * max3(max3(v[0], v[1], v[2]), max3(v[3], v[4], v[5]), max3(v[5], v[6], v[7]));
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
    P pa, pb;
    pa.load_v(pair, lane);
    pb.load_v(pair + UNIT, lane);
    unrolled<NB>([&](auto b_c) {
      constexpr int b = decltype(b_c)::value;
      typename M::Values v;
      M::template values<b>(v, pa, pb);
      if (edge && __ballot(M::clear(v, there(ok_a, ok_b, base, end)))) {
        // V elements that are not finite, of keys that some rows see and others do not: a weight of 0 would make them NaN.  They leave the products, and how
        // many of them a row sees, by sign, are products too: one is enough.
        typename M::Values up, down;
        M::part(v, up, down);
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
          const unsigned sees = there(ok_a, ok_b, base, row_end[rb]);
          float see[8];
#pragma unroll
          for (int k = 0; k < 8; ++k) see[k] = sees >> k & 1 ? 1.f : 0.f;
          typename M::Probs seen;
          M::probs(seen, see);
          f32x4 n[4] = {};
          M::add(n[0], n[1], up, seen);
          M::add(n[2], n[3], down, seen);
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              acc[rb][2 * b + h][i] += n[h][i] > 0.f ? INFINITY : 0.f;
              acc[rb][2 * b + h][i] += n[2 + h][i] > 0.f ? -INFINITY : 0.f;
            }
        }
      }
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) M::add(acc[rb][2 * b], acc[rb][2 * b + 1], v, pr[rb]);
    });
  };
  if (p0 < p1) {
    const int n = p1 - p0;
    int asked = 0, slot = 0;   // pairs asked for, the ring's slot of the pair at hand
    for (; asked < D - 1 && asked < n; ++asked) fetch(p0 + asked, asked);
    asm volatile("" : "+v"(ids), "+v"(ids_next));
#pragma unroll 1
    for (int k = 0; k < n; ++k) {
      if ((k & 31) == 0 && k) fresh = load_ids(p0 + k + 32);
      if ((k & 31) == 16 && k > 16) {
        asm volatile("" : "+v"(fresh));
        if (k & 32) ids = fresh;
        else ids_next = fresh;
      }
      if (asked < n) {   // the slot that the pair before this one has left
        fetch(p0 + asked, slot == 0 ? D - 1 : slot - 1);
        ++asked;
        __builtin_amdgcn_s_waitcnt(0x0F70 | ((D - 1) * NI & 15) | ((D - 1) * NI >> 4 << 14));   // vmcnt: this pair's copies have landed
      } else if (D > 2 && k + 1 < n) {
        __builtin_amdgcn_s_waitcnt(0x0F70 | (NI & 15) | (NI >> 4 << 14));
      } else {
        __builtin_amdgcn_s_waitcnt(0x0F70);
      }
      asm volatile("" ::: "memory");
      const int base = c0 + (p0 + k) * 32;
      const bool ok_a = valid(id_of(p0 + k, 0)), ok_b = valid(id_of(p0 + k, 1));
      const unsigned char* pair = my_ring + slot * PAIR;
      work(pair, base, ok_a, ok_b, base + 32 > all_see || base + 32 > c1 || !ok_a || !ok_b);
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // the pair has been read before its slot is filled again
      slot = slot + 1 == D ? 0 : slot + 1;
    }
  }
  __syncthreads();   // the wavefronts' outputs overlay the ring

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
