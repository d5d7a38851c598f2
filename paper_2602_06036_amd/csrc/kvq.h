// K/V caches held in 4 or 8 bits: what the host side hands to the kernels of kvq.hip and kvq_attn.hip, and the format itself.
//
// A row of K or V is cut into blocks of 32 dims; a block has a scale 2^(e - 127) (one byte e) and 32 codes: 4 bits (sign, 2 bits of exponent, 1 of mantissa: up to
// 6) or 8 bits (sign, 4, 3: up to 448).  e is the least at which the largest magnitude over the scale is at most 7 (464), half a step above the largest code:
// every element, the largest too, is off by half a step at most.  Codes round to nearest even.  e = 255: the block is NaN.
//
// cache[layer][page][kv head][K codes | V codes | K scales | V scales], NB blocks a row (the last one padded with zeros), key = 4 q + k of 16, dim d of block b:
//   K, 4 bits: [b][key][d / 2], even dim low                 K, 8 bits: [d / 16][b][key][d % 16]
//   V, 4 bits: [q][d % 16][b][k], dim below 16 low           V, 8 bits, per pair of blocks: [q][d % 16][b % 2][k][d / 16]
//   scales: [key][NB, of three 4]
// K: what lane (b, key) of a 16-key MFMA operand takes is contiguous, 16 bytes a load, and so is what a row's writer has.  V: lane (q, d % 16) takes four keys of two dims
// a block; the two halves of a byte (a 16-bit pair) are of one key, so they share a scale, and no two keys share a byte: single rows are written without a read.
#pragma once
#include "common.h"

__host__ __device__ __forceinline__ constexpr int kvq_blocks(int hd) { return (hd + 31) / 32; }
__host__ __device__ __forceinline__ constexpr int kvq_scale_row(int nb) { return nb == 3 ? 4 : nb; }   // bytes of a key's scales
__host__ __device__ __forceinline__ constexpr int kvq_codes(int nb, int bits) { return 64 * nb * bits; }   // bytes of the K or V codes of a page of a head
__host__ __device__ __forceinline__ constexpr int kvq_unit(int nb, int k_bits, int v_bits) {             // bytes of a page of a head
  return kvq_codes(nb, k_bits) + kvq_codes(nb, v_bits) + 2 * DF_PAGE * kvq_scale_row(nb);
}

// A cache as the kernels see it.
struct KvqCache {
  unsigned char* data;
  int32_t n_pages, n_kv_heads, hd, k_bits, v_bits;
};

// kvq_write / kvq_read: rows [S, rows, Hkv, hd] <-> positions first[s] .. of a layer
struct KvqRows {
  KvqCache c;
  int32_t layer, n_seqs, rows, mpps;
  const int32_t *first, *counts, *table;   // first position of a sequence's rows; counts null: all rows
  void *k, *v;                             // (only read where the cache is written)
  int32_t* status;
};
// kvq_pack / kvq_unpack: pages of a context's pool <-> pages of the cache, all layers
struct KvqPages {
  KvqCache c;
  int32_t n_layers, n_seqs, max_pages, mpps, pool_pages;
  const int32_t *lens, *pool_table, *table;
  void* pool;
  int32_t* status;
};
struct KvqAttn {
  KvqCache c;
  int32_t layer, n_seqs, rows, causal, n_q_heads, mpps;
  const int32_t *lens, *counts, *table;
  const void* q;
  void* out;
  float scale;
  int32_t parts, tiles;           // about how many ranges the keys of all sequences are cut into (0: a sequence is one), row tiles of a sequence
  float* part_o;                  // [range][row of a sequence][query head][hd] and without hd
  float2* part_ml;
  int32_t* status;
};

void kvq_write_launch(const KvqRows& a, bool bf16, hipStream_t st);
void kvq_read_launch(const KvqRows& a, bool bf16, hipStream_t st);
void kvq_pack_launch(const KvqPages& a, bool bf16, hipStream_t st);
void kvq_unpack_launch(const KvqPages& a, bool bf16, hipStream_t st);
// fills in parts and tiles: part_rows partial rows fit part_o and part_ml; max_tokens: the longest sequence with its rows.  False: no launch is that large
bool kvq_attn_plan(KvqAttn& a, bool bf16, int max_tokens, size_t part_rows);
void kvq_attn_launch(const KvqAttn& a, bool bf16, hipStream_t st);
void kvq_merge_launch(const KvqAttn& a, bool bf16, hipStream_t st);   // where a.parts is not 0

#ifdef __HIPCC__
// ---- device side ----------------------------------------------------------------------------------------------------------
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef short i16x2 __attribute__((ext_vector_type(2)));

// A scale as the conversion instructions take it: a float of whom they look at the exponent alone (checked for every code and scale against the format), so that
// one shift takes byte I out of four, whatever its neighbours leave in the sign and the mantissa.
template <int I>
__device__ __forceinline__ float kvq_scale(uint32_t four) {
  return __uint_as_float(I == 0 ? four << 23 : I == 1 ? four << 15 : I == 2 ? four << 7 : four >> 1);
}
__device__ __forceinline__ float kvq_scale_clean(uint32_t e) { return __uint_as_float((e & 255u) << 23); }

// codes -> two bf16 numbers (exact; e4m3 values below bf16's normal numbers become 0): byte I, or 16-bit half I, of a word
template <int I>
__device__ __forceinline__ uint32_t kvq_bf16_of4(uint32_t w, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, I));
}
template <int I>
__device__ __forceinline__ uint32_t kvq_bf16_of8(uint32_t w, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, I != 0));
}
template <int I>
__device__ __forceinline__ f32x2 kvq_f32_of4(uint32_t w, float scale) {
  return __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, I);
}
template <int I>
__device__ __forceinline__ f32x2 kvq_f32_of8(uint32_t w, float scale) {
  return __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, scale, I != 0);
}

// e of a block whose largest magnitude has these bits (an infinity or NaN: 255)
template <int BITS>
__device__ __forceinline__ int kvq_exponent(uint32_t most) {
  constexpr int top = BITS == 4 ? 2 : 8;
  constexpr uint32_t above = BITS == 4 ? 0x600000u : 0x680000u;   // 1.75 and 1.8125, mantissas of 7 and 464
  const int x = (int)(most >> 23);
  return x == 255 ? 255 : max(x - top + ((most & 0x7FFFFFu) > above ? 1 : 0), 0);
}

// four bytes of four neighbouring lanes: lane k gets byte k of each (its own inverse)
__device__ __forceinline__ uint32_t quad_dpp1(uint32_t x) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0xB1, 0xf, 0xf, true); }
__device__ __forceinline__ uint32_t quad_dpp2(uint32_t x) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x4E, 0xf, 0xf, true); }
__device__ __forceinline__ uint32_t quad_bytes(uint32_t w, int lane) {
  uint32_t o = quad_dpp1(w);
  w = __builtin_amdgcn_perm(o, w, lane & 1 ? 0x03070105u : 0x06020400u);
  o = quad_dpp2(w);
  return __builtin_amdgcn_perm(o, w, lane & 2 ? 0x03020706u : 0x05040100u);
}
// four 16-bit numbers (two words) of four neighbouring lanes, likewise
__device__ __forceinline__ void quad_halves_in(uint32_t& a, uint32_t& b, int lane) {
  const uint32_t sel = lane & 1 ? 0x03020706u : 0x05040100u;
  a = __builtin_amdgcn_perm(quad_dpp1(a), a, sel);
  b = __builtin_amdgcn_perm(quad_dpp1(b), b, sel);
}
__device__ __forceinline__ void quad_halves_swap(uint32_t& a, uint32_t& b, int lane) {
  const bool up = lane & 2;
  const uint32_t x = quad_dpp2(up ? a : b);
  if (up) a = x;
  else b = x;
}
#endif
