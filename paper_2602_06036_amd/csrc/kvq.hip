// Rows and pages of caches held in 4 or 8 bits (kvq.h): quantised as they are written, read back, packed from a context's pool and unpacked into it.
// One wavefront takes one page of one kv head.  All of it is bound by memory; a block's 32 elements are in one lane (rows) or in the 16 lanes of a row of lanes (V of a pool's
// page), so a block's maximum costs no trip through LDS.
#include <algorithm>
#include <type_traits>

#include "kvq.h"

namespace {

template <typename T> struct Raw;   // elements as they lie in memory, 32 bytes' worth of them at a time
template <> struct Raw<bf16_t> {
  // 8 elements at p
  static __device__ __forceinline__ void load8(float (&x)[8], const bf16_t* p) {
    const u32x4 w = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
  }
  static __device__ __forceinline__ uint32_t two(float a, float b) {   // values of at most four significant bits: bf16 holds all but the smallest as they are
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2){a, b}, bf16x2));
  }
  static __device__ __forceinline__ void store8(bf16_t* p, const float (&x)[8]) {
    u32x4 w;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = two(x[2 * i], x[2 * i + 1]);
    *reinterpret_cast<u32x4*>(p) = w;
  }
  static __device__ __forceinline__ void load4(float (&x)[4], const bf16_t* p) {
    const u32x2 w = *reinterpret_cast<const u32x2*>(p);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
  }
  static __device__ __forceinline__ void store4(bf16_t* p, const float (&x)[4]) { *reinterpret_cast<u32x2*>(p) = (u32x2){two(x[0], x[1]), two(x[2], x[3])}; }
  static __device__ __forceinline__ void store1(bf16_t* p, float x) { *p = (bf16_t)two(x, x); }
};
template <> struct Raw<float> {
  static __device__ __forceinline__ void load8(float (&x)[8], const float* p) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const f32x4 w = reinterpret_cast<const f32x4*>(p)[h];
#pragma unroll
      for (int i = 0; i < 4; ++i) x[4 * h + i] = w[i];
    }
  }
  static __device__ __forceinline__ void store8(float* p, const float (&x)[8]) {
#pragma unroll
    for (int h = 0; h < 2; ++h) reinterpret_cast<f32x4*>(p)[h] = (f32x4){x[4 * h], x[4 * h + 1], x[4 * h + 2], x[4 * h + 3]};
  }
  static __device__ __forceinline__ void load4(float (&x)[4], const float* p) {
    const f32x4 w = *reinterpret_cast<const f32x4*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = w[i];
  }
  static __device__ __forceinline__ void store4(float* p, const float (&x)[4]) { *reinterpret_cast<f32x4*>(p) = (f32x4){x[0], x[1], x[2], x[3]}; }
  static __device__ __forceinline__ void store1(float* p, float x) { *p = x; }
};

__device__ __forceinline__ uint32_t magnitude(float x) { return __float_as_uint(x) & 0x7FFFFFFFu; }

// codes of two elements into byte (16-bit half) I of a word
template <int I>
__device__ __forceinline__ void put4(uint32_t& w, float a, float b, float scale) { w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, a, b, scale, I); }
template <int I>
__device__ __forceinline__ void put8(uint32_t& w, float a, float b, float scale) {
  w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(__builtin_bit_cast(i16x2, w), a, b, scale, I != 0));
}
// a block in one lane: e, and its elements without those of a block that is NaN
template <int BITS>
__device__ __forceinline__ int block_scale(float (&x)[32], float& scale) {
  uint32_t most = 0;
#pragma unroll
  for (int i = 0; i < 32; ++i) most = max(most, magnitude(x[i]));
  const int e = kvq_exponent<BITS>(most);
  if (e == 255)
#pragma unroll
    for (int i = 0; i < 32; ++i) x[i] = 0.f;
  scale = __uint_as_float(e == 255 ? 127u << 23 : (uint32_t)e << 23);
  return e;
}

// ---- K of one key and block <-> 32 values ------------------------------------------------------------------------------------
template <int BITS>
__device__ __forceinline__ int k_encode(float (&x)[32], unsigned char* codes, int nb, int key, int b) {
  float scale;
  const int e = block_scale<BITS>(x, scale);
  uint32_t w[BITS];
#pragma unroll
  for (int i = 0; i < BITS; ++i) {
    w[i] = 0;
    if constexpr (BITS == 4) {
      put4<0>(w[i], x[8 * i], x[8 * i + 1], scale);
      put4<1>(w[i], x[8 * i + 2], x[8 * i + 3], scale);
      put4<2>(w[i], x[8 * i + 4], x[8 * i + 5], scale);
      put4<3>(w[i], x[8 * i + 6], x[8 * i + 7], scale);
    } else {
      put8<0>(w[i], x[4 * i], x[4 * i + 1], scale);
      put8<1>(w[i], x[4 * i + 2], x[4 * i + 3], scale);
    }
  }
#pragma unroll
  for (int h = 0; h < BITS / 4; ++h)
    *reinterpret_cast<u32x4*>(codes + ((h * nb + b) * 16 + key) * 16) = (u32x4){w[4 * h], w[4 * h + 1], w[4 * h + 2], w[4 * h + 3]};
  return e;
}
// (codes are asked for and decoded apart: a call's bits are known at run time, and K's, V's and the scales are one trip to memory only if none is waited for in between)
template <int BITS>
__device__ __forceinline__ void k_load(uint32_t (&w)[8], const unsigned char* codes, int nb, int key, int b) {
#pragma unroll
  for (int h = 0; h < BITS / 4; ++h) {
    const u32x4 x = *reinterpret_cast<const u32x4*>(codes + ((h * nb + b) * 16 + key) * 16);
#pragma unroll
    for (int i = 0; i < 4; ++i) w[4 * h + i] = x[i];
  }
}
template <int BITS>
__device__ __forceinline__ void k_decode(float (&x)[32], const uint32_t (&w)[8], float scale) {
#pragma unroll
  for (int i = 0; i < BITS; ++i) {
    auto two = [&](int at, f32x2 v) { x[at] = v[0]; x[at + 1] = v[1]; };
    if constexpr (BITS == 4) {
      two(8 * i, kvq_f32_of4<0>(w[i], scale));
      two(8 * i + 2, kvq_f32_of4<1>(w[i], scale));
      two(8 * i + 4, kvq_f32_of4<2>(w[i], scale));
      two(8 * i + 6, kvq_f32_of4<3>(w[i], scale));
    } else {
      two(4 * i, kvq_f32_of8<0>(w[i], scale));
      two(4 * i + 2, kvq_f32_of8<1>(w[i], scale));
    }
  }
}

// ---- V of one key and block <-> 32 values; the four lanes of a quad have four keys that lie together -------------------------------
// where the four keys q of dim n (and n + 16) of block b lie
template <int BITS>
__device__ __forceinline__ int v_place(int nb, int q, int n, int b) {
  if (BITS == 4) return ((q * 16 + n) * nb + b) * 4;
  const int wide = min(2, nb - (b & ~1));
  return (b >> 1) * 1024 + ((q * 16 + n) * wide + (b & 1)) * 8;
}
template <int BITS>
__device__ __forceinline__ int v_encode(float (&x)[32], unsigned char* codes, int nb, int key, int b, bool there, bool quad) {
  float scale;
  const int e = block_scale<BITS>(x, scale), q = key >> 2, k = key & 3;
  uint32_t w[BITS];
#pragma unroll
  for (int i = 0; i < BITS; ++i) {
    w[i] = 0;
    if constexpr (BITS == 4) {
      put4<0>(w[i], x[4 * i], x[4 * i + 16], scale);
      put4<1>(w[i], x[4 * i + 1], x[4 * i + 17], scale);
      put4<2>(w[i], x[4 * i + 2], x[4 * i + 18], scale);
      put4<3>(w[i], x[4 * i + 3], x[4 * i + 19], scale);
    } else {
      put8<0>(w[i], x[2 * i], x[2 * i + 16], scale);
      put8<1>(w[i], x[2 * i + 1], x[2 * i + 17], scale);
    }
  }
  if (there && !quad) {   // a key whose neighbours are not the call's: by itself
#pragma unroll
    for (int n = 0; n < 16; ++n) {
      unsigned char* at = codes + v_place<BITS>(nb, q, n, b);
      if constexpr (BITS == 4) at[k] = (unsigned char)(w[n / 4] >> (n % 4 * 8));
      else *reinterpret_cast<uint16_t*>(at + 2 * k) = (uint16_t)(w[n / 2] >> (n % 2 * 16));
    }
  }
#pragma unroll
  for (int m = 0; m < 4; ++m) {
    unsigned char* at = codes + v_place<BITS>(nb, q, 4 * m + k, b);
    if constexpr (BITS == 4) {
      const uint32_t x4 = quad_bytes(w[m], k);
      if (quad) *reinterpret_cast<uint32_t*>(at) = x4;
    } else {
      uint32_t lo = w[2 * m], hi = w[2 * m + 1];
      quad_halves_in(lo, hi, k);
      quad_halves_swap(lo, hi, k);
      if (quad) *reinterpret_cast<u32x2*>(at) = (u32x2){lo, hi};
    }
  }
  return e;
}
template <int BITS>
__device__ __forceinline__ void v_load(uint32_t (&w)[8], const unsigned char* codes, int nb, int key, int b) {
#pragma unroll
  for (int m = 0; m < 4; ++m) {
    const unsigned char* at = codes + v_place<BITS>(nb, key >> 2, 4 * m + (key & 3), b);
    if constexpr (BITS == 4) {
      w[m] = *reinterpret_cast<const uint32_t*>(at);
    } else {
      const u32x2 x = *reinterpret_cast<const u32x2*>(at);
      w[2 * m] = x[0];
      w[2 * m + 1] = x[1];
    }
  }
}
template <int BITS>
__device__ __forceinline__ void v_decode(float (&x)[32], const uint32_t (&w)[8], int k, float scale) {   // k: the lane's place among the four of a quad
#pragma unroll
  for (int m = 0; m < 4; ++m) {
    auto two = [&](int n, f32x2 v) { x[n] = v[0]; x[n + 16] = v[1]; };
    if constexpr (BITS == 4) {
      const uint32_t y = quad_bytes(w[m], k);
      two(4 * m, kvq_f32_of4<0>(y, scale));
      two(4 * m + 1, kvq_f32_of4<1>(y, scale));
      two(4 * m + 2, kvq_f32_of4<2>(y, scale));
      two(4 * m + 3, kvq_f32_of4<3>(y, scale));
    } else {
      uint32_t lo = w[2 * m], hi = w[2 * m + 1];
      quad_halves_swap(lo, hi, k);
      quad_halves_in(lo, hi, k);
      two(4 * m, kvq_f32_of8<0>(lo, scale));
      two(4 * m + 1, kvq_f32_of8<1>(lo, scale));
      two(4 * m + 2, kvq_f32_of8<0>(hi, scale));
      two(4 * m + 3, kvq_f32_of8<1>(hi, scale));
    }
  }
}

// ---- rows [S, rows, Hkv, hd] <-> cache ----------------------------------------------------------------------------------------
// Codes: lane = (block b, key).  Rows: a wavefront moves them 16 bytes a lane, a row's pieces in neighbouring lanes, and they change places in LDS: a lane by itself would touch a
// quarter of 64 lines with every load or store (one layer of eight caches read back, 402 MB: 145 us, now 80; four prompts written and read, 207 MB: 66, now 48).
// grid: (pages that a sequence's rows may touch x kv heads / 4 wavefronts, 1, S), kv heads fastest.
constexpr int kRowWaves = 4;

template <typename T, int HD, bool WRITE>
__global__ __launch_bounds__(64 * kRowWaves) void kvq_rows_kernel(KvqRows a, int slots) {
  constexpr int NB = kvq_blocks(HD), SROW = kvq_scale_row(NB), E = 16 / sizeof(T);   // elements of 16 bytes
  constexpr int ROW = HD / E, PIECES = DF_PAGE * ROW, LD = ROW + 1;                   // 16-byte pieces; LD: rows 16 bytes further in LDS, so that a column lies in all banks
  __shared__ u32x4 s_rows[kRowWaves][DF_PAGE * LD];   // K, then V in its place, which leaves room for six wavefronts a SIMD instead of four
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int i = blockIdx.x * kRowWaves + wave, H = a.c.n_kv_heads;
  if (i >= slots * H) return;
  const int s = blockIdx.z, head = i % H, slot = i / H;
  const int first = a.first[s];
  int count = a.counts ? a.counts[s] : a.rows;
  if (count <= 0) return;
  bool odd = count > a.rows || first < 0;   // a range that the call does not have
  count = min(count, a.rows);
  const long long lo = first, hi = lo + count;
  const long long index = (lo < 0 ? 0 : lo >> 4) + slot;   // page of the sequence
  if (index * DF_PAGE >= hi) {
    if (odd && slot == 0 && head == 0 && lane == 0) atomicOr(a.status, DF_STATUS_CAPACITY);
    return;
  }
  const int page = index < a.mpps ? a.table[(size_t)s * a.mpps + index] : -1;
  // keys of the page that are the call's
  const int key0 = (int)max(lo - index * DF_PAGE, 0ll), key1 = (int)min(hi - index * DF_PAGE, (long long)DF_PAGE);
  const long long j0 = index * DF_PAGE - lo;   // row of key 0
  auto piece = [&](int p, int& key, int& c) {
    key = p / ROW;
    c = p % ROW;
    return p < PIECES && key >= key0 && key < key1;
  };
  auto place = [&](T* rows, int key, int c) { return reinterpret_cast<u32x4*>(rows + (((size_t)s * a.rows + (size_t)(j0 + key)) * H + head) * HD) + c; };
  u32x4* rows = s_rows[wave];
  const int key = lane & 15, b = lane >> 4, bc = min(b, NB - 1);
  const bool there = key >= key0 && key < key1 && b < NB;
  constexpr int N = (PIECES + 63) / 64;
  auto sync = [] {   // of one wavefront: its LDS accesses are done in order
    asm volatile("" ::: "memory");
    __builtin_amdgcn_wave_barrier();
  };
  auto block_at = [&](int e) { return rows + key * LD + (bc * 32 + e) / E; };
  if (page < 0 || page >= a.c.n_pages) odd = true;
  if (odd && head == 0 && lane == 0) atomicOr(a.status, DF_STATUS_CAPACITY);
  if (page < 0 || page >= a.c.n_pages) return;
  const int kb = a.c.k_bits, vb = a.c.v_bits;
  unsigned char* unit = a.c.data + (((size_t)a.layer * a.c.n_pages + page) * H + head) * kvq_unit(NB, kb, vb);
  unsigned char *kc = unit, *vc = kc + kvq_codes(NB, kb), *ks = vc + kvq_codes(NB, vb), *vs = ks + DF_PAGE * SROW;
  if constexpr (WRITE) {
    // all rows at once, behind the page's id: in front of it the rows of short batches are even and those of four prompts 49.0 us instead of 47.6
    u32x4 in[2][N];
#pragma unroll
    for (int kv = 0; kv < 2; ++kv)
#pragma unroll
      for (int n = 0; n < N; ++n) {
        int key2, c;
        in[kv][n] = (u32x4){0u, 0u, 0u, 0u};
        if (piece(lane + 64 * n, key2, c)) in[kv][n] = *place(static_cast<T*>(kv ? a.v : a.k), key2, c);
      }
    float x[32];
    auto take = [&](const u32x4 (&from)[N]) {
      sync();
#pragma unroll
      for (int n = 0; n < N; ++n)
        if (lane + 64 * n < PIECES) rows[(lane + 64 * n) / ROW * LD + (lane + 64 * n) % ROW] = from[n];
      sync();
#pragma unroll
      for (int e = 0; e < 32; e += 8) {
        float y[8];
#pragma unroll
        for (int i2 = 0; i2 < 8; ++i2) y[i2] = 0.f;
        if (HD % 32 == 0 || bc * 32 + e < HD) Raw<T>::load8(y, reinterpret_cast<const T*>(block_at(e)));
#pragma unroll
        for (int i2 = 0; i2 < 8; ++i2) x[e + i2] = y[i2];
      }
    };
    take(in[0]);
    if (there) {
      const int e = kb == 4 ? k_encode<4>(x, kc, NB, key, bc) : k_encode<8>(x, kc, NB, key, bc);
      ks[key * SROW + b] = (unsigned char)e;
    }
    take(in[1]);
    const bool quad = ((unsigned)(__ballot(there) >> (lane & ~3)) & 15u) == 15u;
    const int e = vb == 4 ? v_encode<4>(x, vc, NB, key, bc, there, quad) : v_encode<8>(x, vc, NB, key, bc, there, quad);
    if (there) vs[key * SROW + b] = (unsigned char)e;
  } else {
    float k[32], v[32];
    const unsigned ke = ks[key * SROW + bc], ve = vs[key * SROW + bc];
    uint32_t kw[8], vw[8];
    if (kb == 4) k_load<4>(kw, kc, NB, key, bc);
    else k_load<8>(kw, kc, NB, key, bc);
    if (vb == 4) v_load<4>(vw, vc, NB, key, bc);
    else v_load<8>(vw, vc, NB, key, bc);
    if (kb == 4) k_decode<4>(k, kw, kvq_scale_clean(ke));
    else k_decode<8>(k, kw, kvq_scale_clean(ke));
    if (vb == 4) v_decode<4>(v, vw, key & 3, kvq_scale_clean(ve));
    else v_decode<8>(v, vw, key & 3, kvq_scale_clean(ve));
    auto give = [&](const float (&x)[32], T* to) {
      sync();
#pragma unroll
      for (int e = 0; e < 32; e += 8) {
        float y[8];
#pragma unroll
        for (int i2 = 0; i2 < 8; ++i2) y[i2] = x[e + i2];
        if (b < NB && (HD % 32 == 0 || bc * 32 + e < HD)) Raw<T>::store8(reinterpret_cast<T*>(block_at(e)), y);
      }
      sync();
#pragma unroll
      for (int n = 0; n < N; ++n) {
        int key2, c;
        if (piece(lane + 64 * n, key2, c)) *place(to, key2, c) = rows[key2 * LD + c];
      }
    };
    give(k, static_cast<T*>(a.k));
    give(v, static_cast<T*>(a.v));
  }
}

// ---- pages of a pool <-> cache --------------------------------------------------------------------------------------------------
// K: lane = (block, key), 8 dims a load.  V: lane = (q, dim % 16) has four keys of a dim, as both layouts do; a block's maximum is that of two registers over the
// sixteen lanes of a row.  Bound by memory: four requests of 700 to 2050 tokens, 36 layers, taken up again 226 us (5.0 TB/s, the rate of a large copy); two put aside
// 147 us (3.8: V's maxima and two conversions an element take half of the issue).  grid: (pages x kv heads / 4 wavefronts, layers, S).
__device__ __forceinline__ uint32_t row_max(uint32_t x) {   // over 16 lanes
  auto step = [&](uint32_t y) { x = max(x, y); };
  step((uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0xB1, 0xf, 0xf, true));
  step((uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x4E, 0xf, 0xf, true));
  step((uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x141, 0xf, 0xf, true));
  step((uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x128, 0xf, 0xf, true));
  return x;
}
// the four keys' elements (dims n and n + 16) of a block -> codes
template <int BITS>
__device__ __forceinline__ void v_pack(float (&lo)[4], float (&hi)[4], uint32_t (&w)[BITS / 4], int (&e)[4]) {
#pragma unroll
  for (int i = 0; i < BITS / 4; ++i) w[i] = 0;
  float scale[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    e[k] = kvq_exponent<BITS>(row_max(max(magnitude(lo[k]), magnitude(hi[k]))));
    if (e[k] == 255) lo[k] = hi[k] = 0.f;
    scale[k] = __uint_as_float(e[k] == 255 ? 127u << 23 : (uint32_t)e[k] << 23);
  }
  if constexpr (BITS == 4) {
    put4<0>(w[0], lo[0], hi[0], scale[0]);
    put4<1>(w[0], lo[1], hi[1], scale[1]);
    put4<2>(w[0], lo[2], hi[2], scale[2]);
    put4<3>(w[0], lo[3], hi[3], scale[3]);
  } else {
    put8<0>(w[0], lo[0], hi[0], scale[0]);
    put8<1>(w[0], lo[1], hi[1], scale[1]);
    put8<0>(w[1], lo[2], hi[2], scale[2]);
    put8<1>(w[1], lo[3], hi[3], scale[3]);
  }
}
template <int BITS>
__device__ __forceinline__ void v_unpack(float (&lo)[4], float (&hi)[4], const uint32_t (&w)[BITS / 4], const float (&scale)[4]) {
  f32x2 v[4];
  if constexpr (BITS == 4) {
    v[0] = kvq_f32_of4<0>(w[0], scale[0]);
    v[1] = kvq_f32_of4<1>(w[0], scale[1]);
    v[2] = kvq_f32_of4<2>(w[0], scale[2]);
    v[3] = kvq_f32_of4<3>(w[0], scale[3]);
  } else {
    v[0] = kvq_f32_of8<0>(w[0], scale[0]);
    v[1] = kvq_f32_of8<1>(w[0], scale[1]);
    v[2] = kvq_f32_of8<0>(w[1], scale[2]);
    v[3] = kvq_f32_of8<1>(w[1], scale[3]);
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    lo[k] = v[k][0];
    hi[k] = v[k][1];
  }
}

template <typename T, int NB, bool PACK>
__global__ __launch_bounds__(64 * kRowWaves) void kvq_pages_kernel(KvqPages a) {
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int i = blockIdx.x * kRowWaves + wave, H = a.c.n_kv_heads;
  const int s = blockIdx.z, layer = blockIdx.y, head = i % H, index = i / H;
  const int len = min(max(a.lens[s], 0), a.mpps * DF_PAGE);
  if (i == 0 && layer == 0 && lane == 0 && (a.lens[s] < 0 || a.lens[s] > a.max_pages * DF_PAGE || a.lens[s] > a.mpps * DF_PAGE)) atomicOr(a.status, DF_STATUS_CAPACITY);
  if (index >= a.max_pages || index * DF_PAGE >= len) return;
  const int from = a.pool_table[(size_t)s * a.mpps + index], to = a.table[(size_t)s * a.mpps + index];
  if (from < 0 || from >= a.pool_pages || to < 0 || to >= a.c.n_pages) {
    if (head == 0 && layer == 0 && lane == 0) atomicOr(a.status, DF_STATUS_CAPACITY);
    return;
  }
  const int hd = a.c.hd, kb = a.c.k_bits, vb = a.c.v_bits;
  constexpr int SROW = kvq_scale_row(NB);
  unsigned char* unit = a.c.data + (((size_t)layer * a.c.n_pages + to) * H + head) * kvq_unit(NB, kb, vb);
  unsigned char *kc = unit, *vc = kc + kvq_codes(NB, kb), *ks = vc + kvq_codes(NB, vb), *vs = ks + DF_PAGE * SROW;
  T* pk = static_cast<T*>(a.pool) + kv_head_base(layer, a.pool_pages, from, H, head, hd);
  T* pv = pk + DF_PAGE * hd;
  const int n_rows = min(DF_PAGE, len - index * DF_PAGE);   // rows of the page that there are
  {
    const int key = lane & 15, b = lane >> 4;
    if (b < NB) {
      const int n8 = min(4, (hd - 32 * b) / 8);
      float x[32];
      if constexpr (PACK) {
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          float y[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) y[j] = 0.f;
          if (key < n_rows && c < n8) Raw<T>::load8(y, pk + (4 * b + c) * 128 + key * 8);
#pragma unroll
          for (int j = 0; j < 8; ++j) x[8 * c + j] = y[j];
        }
        ks[key * SROW + b] = (unsigned char)(kb == 4 ? k_encode<4>(x, kc, NB, key, b) : k_encode<8>(x, kc, NB, key, b));
      } else {
        const float scale = kvq_scale_clean(ks[key * SROW + b]);
        uint32_t w[8];
        if (kb == 4) k_load<4>(w, kc, NB, key, b);
        else k_load<8>(w, kc, NB, key, b);
        if (kb == 4) k_decode<4>(x, w, scale);
        else k_decode<8>(x, w, scale);
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          float y[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) y[j] = x[8 * c + j];
          if (key < n_rows && c < n8) Raw<T>::store8(pk + (4 * b + c) * 128 + key * 8, y);
        }
      }
    }
  }
  // V: all blocks' codes of a lane go to and fro together, 16 bytes of them where there are four blocks (block by block a store wrote 4 bytes in 16)
  auto v_part = [&](auto bits_c) {
    constexpr int BITS = decltype(bits_c)::value, W = BITS / 4;
    const int q = lane >> 4, n = lane & 15;
    const int there = min(max(n_rows - 4 * q, 0), 4);   // of the lane's four keys
    uint32_t sc[SROW], w[NB][W];                         // scales of its four keys, as they lie
    auto codes = [&](auto copy) {                        // (place, first block, blocks that lie together)
      if constexpr (BITS == 4) copy(vc + (q * 16 + n) * NB * 4, 0, std::integral_constant<int, NB>());
      else {
        if constexpr (NB >= 2) copy(vc + (q * 16 + n) * 16, 0, std::integral_constant<int, 2>());
        if constexpr (NB == 4) copy(vc + 1024 + (q * 16 + n) * 16, 2, std::integral_constant<int, 2>());
        if constexpr (NB & 1) copy(vc + (NB / 2) * 1024 + (q * 16 + n) * 8, NB - 1, std::integral_constant<int, 1>());
      }
    };
#pragma unroll
    for (int i2 = 0; i2 < SROW; ++i2) sc[i2] = PACK ? 0u : reinterpret_cast<const uint32_t*>(vs + 4 * q * SROW)[i2];
    if constexpr (!PACK)
      codes([&](const unsigned char* at, int b, auto n_c) {
        constexpr int N = decltype(n_c)::value * W;
        uint32_t x[N];
        __builtin_memcpy(x, __builtin_assume_aligned(at, N == 4 ? 16 : N == 2 ? 8 : 4), 4 * N);
#pragma unroll
        for (int i2 = 0; i2 < N; ++i2) w[b + i2 / W][i2 % W] = x[i2];
      });
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      const bool two = 32 * b + 16 < hd;
      float lo[4], hi[4];
      T* at = pv + (2 * b) * 256 + lane * 4;
      if constexpr (PACK) {
#pragma unroll
        for (int k = 0; k < 4; ++k) lo[k] = hi[k] = 0.f;
        if (there) {
          Raw<T>::load4(lo, at);
          if (two) Raw<T>::load4(hi, at + 256);
        }
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (k >= there) lo[k] = hi[k] = 0.f;
        int e[4];
        v_pack<BITS>(lo, hi, w[b], e);
#pragma unroll
        for (int k = 0; k < 4; ++k) sc[(k * SROW + b) / 4] |= (uint32_t)e[k] << ((k * SROW + b) % 4 * 8);
      } else {
        float scale[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) scale[k] = kvq_scale_clean(sc[(k * SROW + b) / 4] >> ((k * SROW + b) % 4 * 8));
        v_unpack<BITS>(lo, hi, w[b], scale);
        if (there == 4) {
          Raw<T>::store4(at, lo);
          if (two) Raw<T>::store4(at + 256, hi);
        } else {
#pragma unroll
          for (int k = 0; k < 4; ++k)
            if (k < there) {
              Raw<T>::store1(at + k, lo[k]);
              if (two) Raw<T>::store1(at + 256 + k, hi[k]);
            }
        }
      }
    }
    if constexpr (PACK) {
      codes([&](unsigned char* at, int b, auto n_c) {
        constexpr int N = decltype(n_c)::value * W;
        uint32_t x[N];
#pragma unroll
        for (int i2 = 0; i2 < N; ++i2) x[i2] = w[b + i2 / W][i2 % W];
        __builtin_memcpy(__builtin_assume_aligned(at, N == 4 ? 16 : N == 2 ? 8 : 4), x, 4 * N);
      });
      if (n == 0)
#pragma unroll
        for (int i2 = 0; i2 < SROW; ++i2) reinterpret_cast<uint32_t*>(vs + 4 * q * SROW)[i2] = sc[i2];
    }
  };
  if (vb == 4) v_part(std::integral_constant<int, 4>());
  else v_part(std::integral_constant<int, 8>());
}

template <bool WRITE>
void rows_launch(const KvqRows& a, bool bf16, hipStream_t st) {
  const int slots = (a.rows + 30) / 16;   // pages that a sequence's rows touch at most
  const dim3 grid((unsigned)(((long long)slots * a.c.n_kv_heads + kRowWaves - 1) / kRowWaves), 1, a.n_seqs), block(64 * kRowWaves);
  auto go = [&](auto hd) {
    constexpr int HD = decltype(hd)::value;
    if (bf16) hipLaunchKernelGGL((kvq_rows_kernel<bf16_t, HD, WRITE>), grid, block, 0, st, a, slots);
    else hipLaunchKernelGGL((kvq_rows_kernel<float, HD, WRITE>), grid, block, 0, st, a, slots);
  };
  switch (a.c.hd / 16) {
    case 1: go(std::integral_constant<int, 16>()); break;
    case 2: go(std::integral_constant<int, 32>()); break;
    case 3: go(std::integral_constant<int, 48>()); break;
    case 4: go(std::integral_constant<int, 64>()); break;
    case 5: go(std::integral_constant<int, 80>()); break;
    case 6: go(std::integral_constant<int, 96>()); break;
    case 7: go(std::integral_constant<int, 112>()); break;
    default: go(std::integral_constant<int, 128>());
  }
}
template <bool PACK>
void pages_launch(const KvqPages& a, bool bf16, hipStream_t st) {
  const dim3 grid((unsigned)(((long long)std::max(a.max_pages, 1) * a.c.n_kv_heads + kRowWaves - 1) / kRowWaves), a.n_layers, a.n_seqs), block(64 * kRowWaves);
  auto go = [&](auto nb) {
    constexpr int NB = decltype(nb)::value;
    if (bf16) hipLaunchKernelGGL((kvq_pages_kernel<bf16_t, NB, PACK>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((kvq_pages_kernel<float, NB, PACK>), grid, block, 0, st, a);
  };
  switch (kvq_blocks(a.c.hd)) {
    case 1: go(std::integral_constant<int, 1>()); break;
    case 2: go(std::integral_constant<int, 2>()); break;
    case 3: go(std::integral_constant<int, 3>()); break;
    default: go(std::integral_constant<int, 4>());
  }
}

}  // namespace

void kvq_write_launch(const KvqRows& a, bool bf16, hipStream_t st) { rows_launch<true>(a, bf16, st); }
void kvq_read_launch(const KvqRows& a, bool bf16, hipStream_t st) { rows_launch<false>(a, bf16, st); }
void kvq_pack_launch(const KvqPages& a, bool bf16, hipStream_t st) { pages_launch<true>(a, bf16, st); }
void kvq_unpack_launch(const KvqPages& a, bool bf16, hipStream_t st) { pages_launch<false>(a, bf16, st); }
