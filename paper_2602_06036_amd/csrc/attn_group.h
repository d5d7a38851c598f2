// Block attention for sequences that share pages.
//
// The batch is cut into groups of consecutive sequences.  The leading pages that the block-table rows of a group have in common are attended
// to once for all rows of the group (the prefix part), what lies behind them by each sequence for itself (its own part):
//     row r:  o = softmax(q K^T * scale) V over both parts = (sum of parts of 2^(m_i - m) o_i) / (sum of 2^(m_i - m) l_i),
// m_i, l_i, o_i a part's reference maximum, sum of exponentials (base 2, scores times log2 e) and unnormalised output, m the largest of the maxima.  Both
// parts are split along their keys into ranges of equal length, ranges in a fixed order in the sum, so a call repeats itself bit for bit.  A row that sees
// no key is zeros; a NaN among its scores makes it NaN; an infinity or NaN in a V row reaches the rows that see the key, and only them.
//
// What sequences share is found on the device, so a wrong grouping costs time and nothing else.
//
// Rows of a kv head, in the order of the batch: row = (sequence * block + slot) * group + query head of the kv head.
#pragma once
#include "attn_mfma.h"

typedef float f32x16 __attribute__((ext_vector_type(16)));

struct GroupArgs {
  int n_q_heads, n_kv_heads, layer, causal;
  int n_seqs, rows;         // query rows of a sequence and kv head = block size * (n_q_heads / n_kv_heads)
  int tile;                 // rows of a tile of the prefix part: 64 or 128
  int max_tiles;            // tiles of the prefix part, at most
  int own_tiles;            // tiles (of 64 rows) of a sequence's own part
  int prefix_splits, own_splits;   // prefix_splits 0: every sequence by itself from its first key, without a plan
  float scale;
  void* out;                // one range in all: the finished rows go here and no merge follows
  int operand;              // ... as GEMM operand (Act<T>), else plain rows of the model's type
};

constexpr int kOwnTile = 64;   // query rows of a workgroup of an own part

// Written by group_plan_kernel, read by the launches behind it.
struct GroupTables {
  int4* tiles;       // first row, rows (0: no tile), first sequence of the group, first one behind it
  int2* group;       // [n_seqs] first sequence of the sequence's group, first one behind it
  int32_t* common;   // [n_seqs] tokens that the sequence has in common with the first one of its group: whole pages, committed in both
};
// Tiles of the prefix part: a group that starts at sequence a and is the g-th has those from a * rows / tile + g on (rounded down: whatever the groups in
// front of it need lies below), so no group has to wait for another's count.
__host__ __device__ __forceinline__ int group_tile_slots(int n_seqs, int rows, int tile, int n_groups) { return (int)((long long)n_seqs * rows / tile) + n_groups; }

// Groups -> tiles, a workgroup a sequence: which group it belongs to (the caller's starts as their running maximum, inside the batch; the first is 0), what it has in
// common with the group's first sequence, and, of that one, the group's tiles.  n_groups = 1 needs no starts.  A chain of
// loads: the sequence's own entries are asked for while the starts are on their way (the launch in front of 32 x 1 rows behind 8192 tokens 4.1 -> 3.4 us).
__global__ __launch_bounds__(256) void group_plan_kernel(SeqGeom geo, const int32_t* __restrict__ starts, int n_groups, int n_seqs, int rows, int tile, int expected,
                                                      GroupTables gt) {
  constexpr int AHEAD = 4;   // entries of the sequence's row that a thread asks for before it knows the group
  __shared__ int s_next, s_start, s_end, s_after, s_pages;
  const int t = threadIdx.x, s = blockIdx.x, mpps = geo.max_pages_per_seq;
  const int32_t* row = geo.block_table + (size_t)s * mpps;
  const int len = geo.seq_lens[s];
  int ids[AHEAD];
#pragma unroll
  for (int k = 0; k < AHEAD; ++k) ids[k] = row[min(t + 256 * k, mpps - 1)];
  if (t == 0) {
    s_next = s_after = n_groups;   // the first groups whose starts lie behind this sequence and behind the group's end
    s_start = 0;
    s_end = n_seqs;
    s_pages = mpps;
  }
  auto first_behind = [&](int at, int* to) {   // of the groups whose starts lie behind `at`; a wavefront's lanes ask with one atomic
    for (int i0 = 0; i0 < n_groups; i0 += 256) {
      const int i = i0 + t;
      const unsigned long long behind = __ballot(i > 0 && i < n_groups && starts[min(i, n_groups - 1)] > at);
      if (behind && (t & 63) == 0) atomicMin(to, i + __ffsll(behind) - 1);
      if (behind) break;
    }
  };
  __syncthreads();
  if (n_groups > 1) {
    first_behind(s, &s_next);
    __syncthreads();
    const int next = s_next;
    for (int i = t; i < n_groups; i += 256) {
      const int at = starts[i];
      if (i > 0 && i < next) atomicMax(&s_start, min(max(at, 0), n_seqs));
      if (i == next) s_end = min(at, n_seqs);
      if (s == 0 && (i == 0 ? at != 0 : at < starts[i - 1] || at > n_seqs)) atomicOr(geo.status, DF_STATUS_CAPACITY);
    }
    __syncthreads();
    first_behind(s_end, &s_after);
  }
  const int g = s_next - 1, start = s_start, end = s_end;
  const int32_t* lead = geo.block_table + (size_t)start * mpps;
  int most = min(mpps, min(max(len, 0), max(geo.seq_lens[start], 0)) / DF_PAGE);
  if (end - start == 1) most = min(most, expected / DF_PAGE);   // a sequence by itself is cut where its launch's ranges expect it
  int theirs[AHEAD];
#pragma unroll
  for (int k = 0; k < AHEAD; ++k) theirs[k] = lead[min(t + 256 * k, mpps - 1)];
  int pages = most;
  auto look = [&](int p, int id, int mine) {
    if (p < pages && (id < 0 || id >= geo.n_pages || mine != id)) pages = p;
  };
#pragma unroll
  for (int k = 0; k < AHEAD; ++k) look(t + 256 * k, theirs[k], ids[k]);
  for (int p = t + 256 * AHEAD; p < pages; p += 256) look(p, lead[p], row[p]);
  if (pages < most) atomicMin(&s_pages, pages);
  __syncthreads();
  if (t == 0) {
    gt.group[s] = make_int2(start, end);
    gt.common[s] = min(most, s_pages) * DF_PAGE;
  }
  if (s != start) return;
  // this group's tiles, then empty ones up to those of the group that sequence `end` belongs to (groups without sequences lie between)
  const int row0 = start * rows, row1 = end * rows, slot0 = row0 / tile + g;
  const int slot1 = end < n_seqs ? row1 / tile + s_after - 1 : group_tile_slots(n_seqs, rows, tile, n_groups);
  for (int i = (s == 0 ? 0 : slot0) + t; i < slot1; i += 256) {
    const int r = row0 + (i - slot0) * tile;
    gt.tiles[i] = make_int4(r, i < slot0 ? 0 : max(0, min(tile, row1 - r)), start, end);
  }
}

// What a workgroup does: query rows, their keys' pages, and where the partial results go.
struct GroupWork {
  int row0, n_rows;         // rows of the kv head
  const int32_t* table;     // block-table row
  int c0, c1;               // keys from c0 to below c1
  int own_len;              // causal mask of a sequence's own part: tokens in front of its block; < 0: every row sees every key
  int part;                 // index of the partial result
  bool outgrown;            // the block-table row does not cover all rows of the sequence, and this is the workgroup that says so
};
// ... once its sweep is on its way: in front of it a branch would part the chain of loads that the sweep begins with (attend_token_f32 7.97 -> 8.14 us)
__device__ __forceinline__ void say_outgrown(const SeqGeom& geo, const GroupWork& w) {
  if (w.outgrown && threadIdx.x == 0) atomicOr(geo.status, DF_STATUS_CAPACITY);
}

// tokens that a group has in common (the same in all lanes)
__device__ __forceinline__ int group_prefix(const GroupTables& gt, int start, int end) {
  int c = 0x7FFFFFFF;
  for (int s = start + (threadIdx.x & 63); s < end; s += 64) c = min(c, gt.common[s]);
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) c = min(c, __shfl_xor(c, d, 64));
  return __builtin_amdgcn_readfirstlane(c);
}

// grid: (tiles of the prefix part x its key ranges, then tiles of the own parts x theirs) x kv heads, kv heads fastest: workgroups that read the same keys lie a
// multiple of 8 apart where heads x ranges divide by 8, so on one XCD.  False: there is nothing to do (a tile without rows), or a prefix range has no keys, which
// this writes down.
template <int THREADS>
__device__ __forceinline__ bool group_work(GroupWork& w, int& kvh, const SeqGeom& geo, const GroupArgs& ga, const GroupTables& gt, float2* part_ml) {
  int i = blockIdx.x / ga.n_kv_heads;
  kvh = blockIdx.x % ga.n_kv_heads;
  const int n_prefix = ga.max_tiles * ga.prefix_splits;
  if (i < n_prefix) {
    const int4 t = gt.tiles[i / ga.prefix_splits];
    if (t.y == 0) return false;
    const int split = i % ga.prefix_splits, prefix = group_prefix(gt, t.z, t.w);
    const int chunk = ((prefix + 31) / 32 + ga.prefix_splits - 1) / ga.prefix_splits * 32;
    w = {t.x, t.y, geo.block_table + (size_t)t.z * geo.max_pages_per_seq, min(split * chunk, prefix), min((split + 1) * chunk, prefix), -1, split, false};
    if (w.c0 < w.c1) return true;
    const int parts = ga.prefix_splits + ga.own_splits, group = ga.n_q_heads / ga.n_kv_heads;
    for (int r = threadIdx.x; r < t.y; r += THREADS) {
      const int row = t.x + r, s = row / ga.rows, at = row % ga.rows;
      part_ml[((size_t)(s * geo.block_size + at / group) * ga.n_q_heads + kvh * group + at % group) * parts + split] = make_float2(-INFINITY, 0.f);
    }
    return false;
  }
  i -= n_prefix;
  const int split = i % ga.own_splits, tile = i / ga.own_splits % ga.own_tiles, s = i / (ga.own_splits * ga.own_tiles);
  const int cap = geo.max_pages_per_seq * DF_PAGE;   // a length beyond the block-table row counts as that (whatever it is, its sum with the block stays a number of tokens)
  const int len = min(max(geo.seq_lens[s], 0), cap), n_tok = min(len + geo.block_size, cap);
  int first = 0;
  if (ga.prefix_splits) {
    const int2 g = gt.group[s];
    first = group_prefix(gt, g.x, g.y);
  }
  const int chunk = ((n_tok - first + 31) / 32 + ga.own_splits - 1) / ga.own_splits * 32;
  w = {s * ga.rows + tile * kOwnTile, min(kOwnTile, ga.rows - tile * kOwnTile), geo.block_table + (size_t)s * geo.max_pages_per_seq,
       min(first + split * chunk, n_tok), min(first + (split + 1) * chunk, n_tok), ga.causal && geo.block_size > 1 ? len : -1, ga.prefix_splits + split,
       len > cap - geo.block_size && split + tile + kvh == 0};   // (a single row sees every key)
  return true;
}

// ---- V rows of keys that some rows see and others do not (the block itself, under the causal mask) -------------------------------
// A row's weight of a key that it does not see is 0, and its product with an infinity or a NaN would be NaN.  In the pairs that reach into the block such elements are
// taken out of the products, and given to the rows that see them here: whatever the weight, it is above 0 and the sum becomes what they are.
__device__ __forceinline__ bool not_finite(float x) { return (__float_as_uint(x) & 0x7F800000u) == 0x7F800000u; }
__device__ __forceinline__ float widen(float x) { return x; }
__device__ __forceinline__ float widen(bf16_t x) { return __uint_as_float((uint32_t)x << 16); }
template <typename T, int DT>
__device__ __forceinline__ void add_not_finite(f32x4 (&acc)[DT], const T* v, int n_keys, int pos, int last, int lane) {   // of a page's first keys, from position pos
  n_keys = min(n_keys, last - pos + 1);
  const T* at = v + (lane >> 4) * 16;
#pragma unroll 1
  for (int k = 0; k < n_keys; ++k, at += k & 3 ? 1 : 61)
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float x = widen(at[dt * 256 + i * 4]);
        acc[dt][i] += not_finite(x) ? x : 0.f;
      }
}
// a pair of bf16 numbers without those that are not finite
__device__ __forceinline__ uint32_t finite_pair(uint32_t x) {
  return ((x & 0x7F80u) == 0x7F80u ? 0u : x & 0xFFFFu) | ((x & 0x7F800000u) == 0x7F800000u ? 0u : x & 0xFFFF0000u);
}

// ---- storage types: fragments of a page pair and their products ------------------------------------------------------------
// A pair of pages is 32 keys.  S^T = K . Q^T leaves a lane 4 consecutive keys (4g .. 4g+3, g = lane / 16) of query column lane % 16 of each page, and
// O^T += V^T . P^T takes them as they are.  bf16: 16x16x32 MFMAs, probabilities as a hi + lo pair (~16 bits, as everywhere in the bf16 model).  fp32: 16x16x4
// MFMAs, every product and sum in fp32.
template <typename T, int HD> struct PairFrags;

template <int HD>
struct PairFrags<bf16_t, HD> {
  static constexpr int KT = (HD + 31) / 32, DT = HD / 16;
  struct Query { u32x4 q[KT]; };
  struct Keys { u32x4 a[KT], b[KT]; };
  struct Values { uint2 a[DT], b[DT]; };
  static __device__ __forceinline__ u32x4 chunk(const bf16_t* p, int kt, int lane) {   // 16 rows x 32 dims; dims behind HD are zeros
    const int g = lane >> 4;
    if (HD % 32 && kt * 4 + g >= HD / 8) return (u32x4){0u, 0u, 0u, 0u};
    return reinterpret_cast<const u32x4*>(p)[kt * 64 + lane];
  }
  static __device__ __forceinline__ void query(Query& f, const bf16_t* row, int lane) {   // the row of lane % 16
    const int g = lane >> 4;
#pragma unroll
    for (int kt = 0; kt < KT; ++kt) {
      f.q[kt] = (u32x4){0u, 0u, 0u, 0u};
      if (row && (HD % 32 == 0 || kt * 4 + g < HD / 8)) f.q[kt] = reinterpret_cast<const u32x4*>(row)[kt * 4 + g];
    }
  }
  static __device__ __forceinline__ void keys(Keys& f, const bf16_t* a, const bf16_t* b, int lane) {
#pragma unroll
    for (int kt = 0; kt < KT; ++kt) {
      f.a[kt] = chunk(a, kt, lane);
      f.b[kt] = chunk(b, kt, lane);
    }
  }
  static __device__ __forceinline__ void values(Values& f, const bf16_t* a, const bf16_t* b, int lane) {
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {
      f.a[dt] = reinterpret_cast<const uint2*>(a + DF_PAGE * HD)[dt * 64 + lane];
      f.b[dt] = reinterpret_cast<const uint2*>(b + DF_PAGE * HD)[dt * 64 + lane];
    }
  }
  static __device__ __forceinline__ void scores(f32x4& sa, f32x4& sb, const Keys& k, const Query& q) {
    sa = sb = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int kt = 0; kt < KT; ++kt) {
      sa = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, k.a[kt]), __builtin_bit_cast(bf16x8, q.q[kt]), sa, 0, 0, 0);
      sb = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, k.b[kt]), __builtin_bit_cast(bf16x8, q.q[kt]), sb, 0, 0, 0);
    }
  }
  // V elements of keys that are not there (never written, another sequence's; there: a bit a key): 0 * whatever they hold must stay 0
  static __device__ __forceinline__ void clear(Values& f, unsigned there) {
    auto half = [&](int i) { return (there >> i & 1 ? 0x0000FFFFu : 0u) | (there >> i & 2 ? 0xFFFF0000u : 0u); };
    const unsigned m0 = half(0), m1 = half(2), m2 = half(4), m3 = half(6);
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {
      f.a[dt].x &= m0; f.a[dt].y &= m1;
      f.b[dt].x &= m2; f.b[dt].y &= m3;
    }
  }
  static __device__ __forceinline__ bool not_all_finite(const Values& f) {
    uint32_t odd = 0;
    auto look = [&](uint32_t x) { odd |= finite_pair(x) ^ x; };
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {
      look(f.a[dt].x); look(f.a[dt].y);
      look(f.b[dt].x); look(f.b[dt].y);
    }
    return odd != 0;
  }
  static __device__ __forceinline__ void drop_not_finite(Values& f) {
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {
      f.a[dt] = make_uint2(finite_pair(f.a[dt].x), finite_pair(f.a[dt].y));
      f.b[dt] = make_uint2(finite_pair(f.b[dt].x), finite_pair(f.b[dt].y));
    }
  }
  static __device__ __forceinline__ void add(f32x4 (&acc)[DT], const Values& v, const float (&p)[8]) {
    u32x4 hi, lo;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t h = pack_bf16_pair(p[2 * i], p[2 * i + 1]);
      hi[i] = h;
      lo[i] = pack_bf16_pair(p[2 * i] - __uint_as_float(h << 16), p[2 * i + 1] - __uint_as_float(h & 0xFFFF0000u));
    }
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {
      const u32x4 vf = {v.a[dt].x, v.a[dt].y, v.b[dt].x, v.b[dt].y};
      acc[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, vf), __builtin_bit_cast(bf16x8, hi), acc[dt], 0, 0, 0);
      acc[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, vf), __builtin_bit_cast(bf16x8, lo), acc[dt], 0, 0, 0);
    }
  }
};

template <int HD>
struct PairFrags<float, HD> {
  static constexpr int KT = HD / 8, DT = HD / 16;
  struct Query { float2 q[KT]; };          // dims 8 kt + 2g, + 1
  struct Keys { float2 a[KT], b[KT]; };
  struct Values { float4 a[DT], b[DT]; };
  static __device__ __forceinline__ void query(Query& f, const float* row, int lane) {
#pragma unroll
    for (int kt = 0; kt < KT; ++kt) {
      f.q[kt] = make_float2(0.f, 0.f);
      if (row) f.q[kt] = reinterpret_cast<const float2*>(row)[kt * 4 + (lane >> 4)];
    }
  }
  static __device__ __forceinline__ void keys(Keys& f, const float* a, const float* b, int lane) {
    const int at = (lane & 15) * 4 + (lane >> 4);
#pragma unroll
    for (int kt = 0; kt < KT; ++kt) {
      f.a[kt] = reinterpret_cast<const float2*>(a)[kt * 64 + at];
      f.b[kt] = reinterpret_cast<const float2*>(b)[kt * 64 + at];
    }
  }
  static __device__ __forceinline__ void values(Values& f, const float* a, const float* b, int lane) {
    const int at = (lane >> 4) * 16 + (lane & 15);
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {
      f.a[dt] = reinterpret_cast<const float4*>(a + DF_PAGE * HD)[dt * 64 + at];
      f.b[dt] = reinterpret_cast<const float4*>(b + DF_PAGE * HD)[dt * 64 + at];
    }
  }
  static __device__ __forceinline__ void scores(f32x4& sa, f32x4& sb, const Keys& k, const Query& q) {
    sa = sb = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int kt = 0; kt < KT; ++kt) {
      sa = __builtin_amdgcn_mfma_f32_16x16x4f32(k.a[kt].x, q.q[kt].x, sa, 0, 0, 0);
      sb = __builtin_amdgcn_mfma_f32_16x16x4f32(k.b[kt].x, q.q[kt].x, sb, 0, 0, 0);
      sa = __builtin_amdgcn_mfma_f32_16x16x4f32(k.a[kt].y, q.q[kt].y, sa, 0, 0, 0);
      sb = __builtin_amdgcn_mfma_f32_16x16x4f32(k.b[kt].y, q.q[kt].y, sb, 0, 0, 0);
    }
  }
  static __device__ __forceinline__ void clear(Values& f, unsigned there) {
    auto keep = [&](int i, float v) { return there >> i & 1 ? v : 0.f; };
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {
      f.a[dt] = make_float4(keep(0, f.a[dt].x), keep(1, f.a[dt].y), keep(2, f.a[dt].z), keep(3, f.a[dt].w));
      f.b[dt] = make_float4(keep(4, f.b[dt].x), keep(5, f.b[dt].y), keep(6, f.b[dt].z), keep(7, f.b[dt].w));
    }
  }
  static __device__ __forceinline__ bool not_all_finite(const Values& f) {
    uint32_t most = 0;
    auto look = [&](float x) { most = max(most, __float_as_uint(x) & 0x7FFFFFFFu); };
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {
      look(f.a[dt].x); look(f.a[dt].y); look(f.a[dt].z); look(f.a[dt].w);
      look(f.b[dt].x); look(f.b[dt].y); look(f.b[dt].z); look(f.b[dt].w);
    }
    return most >= 0x7F800000u;
  }
  static __device__ __forceinline__ void drop_not_finite(Values& f) {
    auto drop = [&](float& x) { x = not_finite(x) ? 0.f : x; };
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {
      drop(f.a[dt].x); drop(f.a[dt].y); drop(f.a[dt].z); drop(f.a[dt].w);
      drop(f.b[dt].x); drop(f.b[dt].y); drop(f.b[dt].z); drop(f.b[dt].w);
    }
  }
  static __device__ __forceinline__ void add(f32x4 (&acc)[DT], const Values& v, const float (&p)[8]) {
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {   // the product of lanes' i-th keys: keys i, 4 + i, 8 + i, 12 + i of a page
      acc[dt] = __builtin_amdgcn_mfma_f32_16x16x4f32(v.a[dt].x, p[0], acc[dt], 0, 0, 0);
      acc[dt] = __builtin_amdgcn_mfma_f32_16x16x4f32(v.a[dt].y, p[1], acc[dt], 0, 0, 0);
      acc[dt] = __builtin_amdgcn_mfma_f32_16x16x4f32(v.a[dt].z, p[2], acc[dt], 0, 0, 0);
      acc[dt] = __builtin_amdgcn_mfma_f32_16x16x4f32(v.a[dt].w, p[3], acc[dt], 0, 0, 0);
      acc[dt] = __builtin_amdgcn_mfma_f32_16x16x4f32(v.b[dt].x, p[4], acc[dt], 0, 0, 0);
      acc[dt] = __builtin_amdgcn_mfma_f32_16x16x4f32(v.b[dt].y, p[5], acc[dt], 0, 0, 0);
      acc[dt] = __builtin_amdgcn_mfma_f32_16x16x4f32(v.b[dt].z, p[6], acc[dt], 0, 0, 0);
      acc[dt] = __builtin_amdgcn_mfma_f32_16x16x4f32(v.b[dt].w, p[7], acc[dt], 0, 0, 0);
    }
  }
};

// four dims of a finished row (m_hq: its place among the query rows of all heads).  True: one of them is not finite, see below
template <typename T>
__device__ __forceinline__ bool group_store(const GroupArgs& ga, size_t m_hq, int hd, int d, float4 o, float l) {
  const float by = l != 0.f ? l : INFINITY;   // no visible key: zeros
  o = make_float4(o.x / by, o.y / by, o.z / by, o.w / by);
  T* out = static_cast<T*>(ga.out);
  if (ga.operand) Act<T>::store4(out, (int)(m_hq / ga.n_q_heads), (int)(m_hq % ga.n_q_heads) * hd + d, ga.n_q_heads * hd, o);
  else if constexpr (sizeof(T) == 2) *reinterpret_cast<uint2*>(out + m_hq * hd + d) = make_uint2(pack_bf16_pair(o.x, o.y), pack_bf16_pair(o.z, o.w));
  else *reinterpret_cast<float4*>(out + m_hq * hd + d) = o;
  return l > 0.f && (not_finite(o.x) || not_finite(o.y) || not_finite(o.z) || not_finite(o.w));   // (a NaN among the scores: the row is NaN)
}
// Four dims of a finished row, some of them not finite: those whose V is not finite in a key that the row sees are what such elements add up to.  The products need not have made
// that of them (a weight that is 0 in fp32; hi * inf + lo * inf with a lo of 0 or below it), and in which products they stand depends on how the keys are cut, which the row must not.
template <typename T>
__device__ __forceinline__ void group_store_not_finite(const SeqGeom& geo, const GroupArgs& ga, const T* pool, int m_hq, int hd, int d) {
  const int m = m_hq / ga.n_q_heads, hq = m_hq % ga.n_q_heads, s = m / geo.block_size, cap = geo.max_pages_per_seq * DF_PAGE;
  const int n_see = min(min(max(geo.seq_lens[s], 0), cap) + (ga.causal ? m % geo.block_size + 1 : geo.block_size), cap);
  float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
  for (int p = 0; p * DF_PAGE < n_see; ++p) {
    const int id = geo.block_table[(size_t)s * geo.max_pages_per_seq + p];
    if (id < 0 || id >= geo.n_pages) continue;
    const T* v = pool + kv_head_base(ga.layer, geo.n_pages, id, ga.n_kv_heads, hq / (ga.n_q_heads / ga.n_kv_heads), hd) + DF_PAGE * hd + v_in_page(0, d);
#pragma unroll
    for (int k = 0; k < DF_PAGE; ++k)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float x = widen(v[k / 4 * 64 + i * 4 + k % 4]);
        sum[i] += p * DF_PAGE + k < n_see && not_finite(x) ? x : 0.f;
      }
  }
  T* out = static_cast<T*>(ga.out);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (!not_finite(sum[i])) continue;
    if (ga.operand) Act<T>::store(out, m, hq * hd + d + i, ga.n_q_heads * hd, sum[i]);
    else out[(size_t)m_hq * hd + d + i] = Store<T>::from(sum[i]);
  }
}

// fp32, and bf16 with other head dims.  A wavefront sweeps 16 rows, pairs of pages straight from memory; the workgroup's four share its rows (up to 64) or, where there
// are fewer, the keys too, and add their parts in LDS.
template <typename T, int HD>
__global__ __launch_bounds__(256, 2) void group_attn_kernel(const T* __restrict__ q, const T* __restrict__ pool, SeqGeom geo, GroupArgs ga, GroupTables gt,
                                                            float* __restrict__ part_o, float2* __restrict__ part_ml) {
  typedef PairFrags<T, HD> F;
  constexpr int DT = HD / 16, LD = HD + 4;
  __shared__ float s_o[3][16][LD];
  __shared__ float2 s_ml[3][16];
  GroupWork w;
  int kvh;
  if (!group_work<256>(w, kvh, geo, ga, gt, part_ml)) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 15, g = lane >> 4;
  const int blocks = w.n_rows > 32 ? 4 : w.n_rows > 16 ? 2 : 1, shares = 4 / blocks;   // wavefronts that share rows, and that share keys
  const int block = wave % blocks, share = wave / blocks;
  const int group = ga.n_q_heads / ga.n_kv_heads;
  const bool valid = block * 16 + n < w.n_rows;
  const int row = w.row0 + (valid ? block * 16 + n : 0);
  const int s = row / ga.rows, slot = row % ga.rows / group, hq = kvh * group + row % group;   // rows is a multiple of the group
  const size_t m_hq = (size_t)(s * geo.block_size + slot) * ga.n_q_heads + hq;
  typename F::Query qf;
  F::query(qf, valid ? q + m_hq * HD : nullptr, lane);
  const int last = !valid ? -1 : (w.own_len >= 0 ? w.own_len + slot : 0x7FFFFFFF);

  float m_run = -INFINITY, l_run = 0.f;
  f32x4 acc[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) acc[dt] = (f32x4){0.f, 0.f, 0.f, 0.f};
  const float scale2 = ga.scale * 1.44269504088896341f;   // base-2 exponents

  struct Ids { int a, b; };
  auto ids_of = [&](int base) {   // foreign and missing pages as -1
    const int at = base / DF_PAGE;
    Ids p{-1, -1};
    if (base < w.c1) p.a = w.table[at];
    if (base + DF_PAGE < w.c1) p.b = w.table[at + 1];
    if (p.a < 0 || p.a >= geo.n_pages) p.a = -1;
    if (p.b < 0 || p.b >= geo.n_pages) p.b = -1;
    return p;
  };
  auto page = [&](int id) { return pool + kv_head_base(ga.layer, geo.n_pages, id, ga.n_kv_heads, kvh, HD); };
  const int step = 32 * shares;
  int base = w.c0 + 32 * share;
  Ids id = ids_of(base);
  typename F::Keys kf;
  typename F::Values vf;
  if (base < w.c1) F::keys(kf, page(max(id.a, 0)), page(id.b >= 0 ? id.b : max(id.a, 0)), lane);   // a page that may be read; its keys weigh nothing
  for (; base < w.c1; base += step) {
    const bool ok_a = id.a >= 0, ok_b = id.b >= 0;
    const T *page_a = page(max(id.a, 0)), *page_b = page(ok_b ? id.b : max(id.a, 0));
    F::values(vf, page_a, page_b, lane);
    id = ids_of(base + step);
    f32x4 sa, sb;
    F::scores(sa, sb, kf, qf);
    if (base + step < w.c1) F::keys(kf, page(max(id.a, 0)), page(id.b >= 0 ? id.b : max(id.a, 0)), lane);   // the next pair's, behind the softmax and the products
    float v[8], p[8];
    unsigned there = 0u;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int pos = base + (i >> 2) * DF_PAGE + 4 * g + (i & 3);
      const bool in = (i < 4 ? ok_a : ok_b) && pos < w.c1;
      there |= in ? 1u << i : 0u;
      v[i] = in && pos <= last ? (i < 4 ? sa[i & 3] : sb[i & 3]) * scale2 : -INFINITY;
    }
    float mx = fmaxf(fmaxf(fmaxf(v[0], v[1]), fmaxf(v[2], v[3])), fmaxf(fmaxf(v[4], v[5]), fmaxf(v[6], v[7])));
    mx = quarter_max(mx);
    const float m_new = fmaxf(m_run, mx), mb = m_new == -INFINITY ? 0.f : m_new;   // nothing visible yet: exp2(-inf - 0) = 0
    const float corr = m_run == -INFINITY ? (m_new == -INFINITY ? 1.f : 0.f) : exp2f(m_run - m_new);
#pragma unroll
    for (int i = 0; i < 8; ++i) p[i] = __builtin_amdgcn_exp2f(v[i] - mb);
    l_run = l_run * corr + (((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7])));
    m_run = m_new;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {
      acc[dt][0] *= corr; acc[dt][1] *= corr; acc[dt][2] *= corr; acc[dt][3] *= corr;
    }
    if (there != 0xFFu) F::clear(vf, there);
    if (w.own_len >= 0 && base + 32 > w.own_len && __builtin_amdgcn_ballot_w64(F::not_all_finite(vf)) != 0ull) {
      F::drop_not_finite(vf);
      add_not_finite(acc, page_a + DF_PAGE * HD, ok_a ? min(DF_PAGE, w.c1 - base) : 0, base, last, lane);
      add_not_finite(acc, page_b + DF_PAGE * HD, ok_b ? min(DF_PAGE, w.c1 - base - DF_PAGE) : 0, base + DF_PAGE, last, lane);
    }
    F::add(acc, vf, p);
  }
  say_outgrown(geo, w);
  float l = quarter_sum(l_run);
  if (shares > 1) {   // uniform over the workgroup
    if (share > 0) {
      const int to = (share - 1) * blocks + block;
      if (g == 0) s_ml[to][n] = make_float2(m_run, l);
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) *reinterpret_cast<float4*>(&s_o[to][n][dt * 16 + 4 * g]) = make_float4(acc[dt][0], acc[dt][1], acc[dt][2], acc[dt][3]);
    }
    __syncthreads();
    if (share > 0) return;
    for (int i = 1; i < shares; ++i) {
      const int from = (i - 1) * blocks + block;
      const float2 ml = s_ml[from][n];
      if (ml.y == 0.f) continue;   // no visible key
      const float m_new = fmaxf(m_run, ml.x);
      const float f0 = m_run == m_new ? 1.f : exp2f(m_run - m_new), f1 = ml.x == m_new ? 1.f : exp2f(ml.x - m_new);
      l = l * f0 + ml.y * f1;
      m_run = m_new;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        const float4 o = *reinterpret_cast<const float4*>(&s_o[from][n][dt * 16 + 4 * g]);
        acc[dt] = (f32x4){acc[dt][0] * f0 + o.x * f1, acc[dt][1] * f0 + o.y * f1, acc[dt][2] * f0 + o.z * f1, acc[dt][3] * f0 + o.w * f1};
      }
    }
  }
  if (!valid) return;
  if (ga.out) {
    bool again = false;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) again |= group_store<T>(ga, m_hq, HD, dt * 16 + 4 * g, make_float4(acc[dt][0], acc[dt][1], acc[dt][2], acc[dt][3]), l);
    if (again)
#pragma unroll 1
      for (int dt = 0; dt < DT; ++dt) group_store_not_finite(geo, ga, pool, (int)m_hq, HD, dt * 16 + 4 * g);
    return;
  }
  const size_t pr = m_hq * (ga.prefix_splits + ga.own_splits) + w.part;
  if (g == 0) part_ml[pr] = make_float2(m_run, l);
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
    *reinterpret_cast<float4*>(part_o + pr * HD + dt * 16 + 4 * g) = make_float4(acc[dt][0], acc[dt][1], acc[dt][2], acc[dt][3]);
}

// ---- bf16, head dims 32, 64, 96 and 128: wavefronts split the keys ------------------------------------------------------------------
// Four wavefronts take every fourth pair of pages each for all RB blocks of 16 query rows, from a ring of their own in LDS: the pages go there
// directly (global_load_lds), K refilled as soon as a pair's scores are done and V as soon as its products are, so nothing in flight costs a
// register and no wavefront waits for another before the end, where their partial results are added in LDS.  The loads are counted by hand (NI per half page,
// in order): the compiler would wait for all of them ahead of every LDS read.  Two workgroups a CU.
template <int HD>
struct KeySplit {
  static constexpr int KT = HD / 32, DT = HD / 16, NW = 4, LD = HD + 4;
  static constexpr int PART = DF_PAGE * HD * 2, NI = PART / 1024;   // bytes of the K or V part of a page, load instructions for it
  static constexpr int RING = NW * 4 * PART;                        // per wavefront: K of page A, of page B, V of page A, of page B
  // ring and queries; in the end two wavefronts' rows from the start and all wavefronts' maxima and sums behind them, then the rows' places
  static constexpr int OUT(int rb) { return 2 * rb * 16 * LD * 4; }
  static constexpr int ROWS_AT(int rb) { return OUT(rb) + NW * rb * 16 * 8; }
  static constexpr int bytes(int rb) { return RING + rb * KT * 1024 > ROWS_AT(rb) + rb * 16 * 4 ? RING + rb * KT * 1024 : ROWS_AT(rb) + rb * 16 * 4; }
};

// DIRECT: the launch may be one whose rows are finished here (ga.out)
template <int HD, int RB, bool DIRECT>
__device__ __forceinline__ void group_sweep_keys(char* s_raw, const GroupWork& w, int kvh, const bf16_t* __restrict__ q,
                                                 const bf16_t* __restrict__ pool, const SeqGeom& geo, const GroupArgs& ga, float* __restrict__ part_o,
                                                 float2* __restrict__ part_ml) {
  typedef KeySplit<HD> C;
  constexpr int KT = C::KT, DT = C::DT, NW = C::NW, LD = C::LD, PART = C::PART, NI = C::NI;
  float (*s_o)[RB * 16][LD] = reinterpret_cast<float (*)[RB * 16][LD]>(s_raw);
  float2 (*s_ml)[RB * 16] = reinterpret_cast<float2 (*)[RB * 16]>(s_raw + C::OUT(RB));
  u32x4* q_lds = reinterpret_cast<u32x4*>(s_raw + C::RING);                      // [rb][kt][lane]
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 15, g = lane >> 4;
  const int group = ga.n_q_heads / ga.n_kv_heads, page0 = w.c0 / DF_PAGE;
  // page ids of this wavefront's pairs, 32 pairs at a time: lane l holds page l % 2 of its pair k0 + l / 2; the next set is requested as a set comes into use
  auto load_ids = [&](int k0) { return w.table[min(page0 + 2 * (wave + NW * (k0 + (lane >> 1))) + (lane & 1), geo.max_pages_per_seq - 1)]; };
  int ids = load_ids(0);
  const int n_pairs = w.c1 > w.c0 ? (w.c1 - w.c0 + 31) >> 5 : 0, my_pairs = n_pairs > wave ? (n_pairs - wave + NW - 1) / NW : 0;
  int ids_next = my_pairs > 32 ? load_ids(32) : 0;
  u32x4 qr[KT];
  {
    const int r = (wave < RB ? wave : 0) * 16 + n, row = w.row0 + min(r, w.n_rows - 1);
    const int s = row / ga.rows, slot = row % ga.rows / group;
    const u32x4* qp = reinterpret_cast<const u32x4*>(q + ((size_t)(s * geo.block_size + slot) * ga.n_q_heads + kvh * group + row % group) * HD);
#pragma unroll
    for (int kt = 0; kt < KT; ++kt) qr[kt] = qp[kt * 4 + g];   // a row that is not there reads along and is not stored
  }
  int last[RB];   // last key that a lane's row sees (of a sequence's own part under the causal mask)
#pragma unroll
  for (int rb = 0; rb < RB; ++rb)
    last[rb] = w.own_len >= 0 ? w.own_len + (w.row0 + min(rb * 16 + n, w.n_rows - 1)) % ga.rows / group : 0x7FFFFFFF;
  const int n_all = w.own_len >= 0 ? min(w.c1, w.own_len) : w.c1;   // keys below this are visible to every row

  const unsigned ring = (unsigned)(size_t)s_raw + (unsigned)wave * (4 * PART), voff = lane * 16;
  auto fetch = [&](const bf16_t* src, unsigned at) {   // one part of a page into the ring at byte `at`
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const unsigned dst = __builtin_amdgcn_readfirstlane(ring + at + i * 1024);
      const bf16_t* from = src + i * 512;
      unsigned keep_m0;   // whatever the compiler keeps in m0 is put back
      asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, %3\n\ts_nop 0\n\ts_mov_b32 m0, %0"
                   : "=&s"(keep_m0) : "s"(dst), "v"(voff), "s"(from) : "memory");
    }
  };
  struct Pair {
    const bf16_t *a, *b;   // the pages' K parts (V follows)
    bool ok_a, ok_b;
  };
  auto pair_of = [&](int k) {   // this wavefront's k-th pair; foreign or missing pages alias a readable one and weigh nothing
    Pair p;
    const int pa = __builtin_amdgcn_readlane(ids, (k & 31) * 2), pb = __builtin_amdgcn_readlane(ids, (k & 31) * 2 + 1);
    p.ok_a = pa >= 0 && pa < geo.n_pages;
    p.ok_b = w.c0 + (wave + NW * k) * 32 + 16 < w.c1 && pb >= 0 && pb < geo.n_pages;
    const int a = p.ok_a ? pa : 0, b = p.ok_b ? pb : a;
    p.a = pool + kv_head_base(ga.layer, geo.n_pages, a, ga.n_kv_heads, kvh, HD);
    p.b = pool + kv_head_base(ga.layer, geo.n_pages, b, ga.n_kv_heads, kvh, HD);
    return p;
  };
  Pair cur{pool, pool, false, false};
  if (my_pairs > 0) {
    cur = pair_of(0);
    fetch(cur.a, 0);
    fetch(cur.b, PART);
    fetch(cur.a + DF_PAGE * HD, 2 * PART);
    fetch(cur.b + DF_PAGE * HD, 3 * PART);
  }
  if (wave < RB) {
#pragma unroll
    for (int kt = 0; kt < KT; ++kt) q_lds[(wave * KT + kt) * 64 + lane] = qr[kt];
  }
  __syncthreads();

  float m_run[RB], l_run[RB];
  f32x4 acc[RB][DT];
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    m_run[rb] = -INFINITY;
    l_run[rb] = 0.f;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) acc[rb][dt] = (f32x4){0.f, 0.f, 0.f, 0.f};
  }
  const float scale2 = ga.scale * 1.44269504088896341f;
  const char* my_ring = s_raw + wave * (4 * PART);

  f32x4 sc[RB][2];
  u32x4 ph[RB], pl[RB];   // probabilities as hi + lo pairs
  auto scores = [&](int k) {
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * NI) : "memory");   // this pair's K is there (its V still on the way)
    const u32x4* kp = reinterpret_cast<const u32x4*>(my_ring) + lane;
    u32x4 ka[KT], kb[KT];
#pragma unroll
    for (int kt = 0; kt < KT; ++kt) {
      ka[kt] = kp[kt * 64];
      kb[kt] = kp[PART / 16 + kt * 64];
    }
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      asm volatile("" ::: "memory");   // the query fragments of one row block at a time: together they would cost 64 registers
      sc[rb][0] = sc[rb][1] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int kt = 0; kt < KT; ++kt) {
        const u32x4 qf = q_lds[(rb * KT + kt) * 64 + lane];
        sc[rb][0] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, ka[kt]), __builtin_bit_cast(bf16x8, qf), sc[rb][0], 0, 0, 0);
        sc[rb][1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kb[kt]), __builtin_bit_cast(bf16x8, qf), sc[rb][1], 0, 0, 0);
      }
    }
    __builtin_amdgcn_s_waitcnt(0xC07F);   // lgkmcnt(0): the K half has been read
  };
  auto softmax = [&](const Pair& pr, int base) {
    if (!pr.ok_a || !pr.ok_b || base + 32 > n_all) {   // (n_all <= c1: keys behind the range as well)
      const int p0 = base + 4 * g;
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        const int upto = min(w.c1 - 1, last[rb]);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (!(pr.ok_a && p0 + i <= upto)) sc[rb][0][i] = -INFINITY;
          if (!(pr.ok_b && p0 + 16 + i <= upto)) sc[rb][1][i] = -INFINITY;
        }
      }
    }
    // Lazy reference maximum: it moves only when a row's has grown by more than 8 (in powers of two), decided from each lane's own scores, so the
    // accumulators are rescaled once or twice a sweep; until then the exponentials stay below 256.
    float lmx[RB];
    bool grew = false;
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      const f32x4 x = sc[rb][0], y = sc[rb][1];
      lmx[rb] = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(y[0], y[1]), fmaxf(y[2], y[3]))) * scale2;
      grew = grew || lmx[rb] > m_run[rb] + 8.f;
    }
    if (__builtin_amdgcn_ballot_w64(grew) != 0ull) {
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        const float mx = quarter_max(lmx[rb]);
        const bool grow = mx > m_run[rb] + 8.f;
        const float corr = grow ? (m_run[rb] == -INFINITY ? 0.f : exp2f(m_run[rb] - mx)) : 1.f;
        l_run[rb] *= corr;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) {
          acc[rb][dt][0] *= corr; acc[rb][dt][1] *= corr; acc[rb][dt][2] *= corr; acc[rb][dt][3] *= corr;
        }
        if (grow) m_run[rb] = mx;
      }
    }
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      const float mb = (m_run[rb] == -INFINITY) ? 0.f : m_run[rb];
      float pe[8];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        pe[i] = __builtin_amdgcn_exp2f(fmaf(sc[rb][0][i], scale2, -mb));
        pe[4 + i] = __builtin_amdgcn_exp2f(fmaf(sc[rb][1][i], scale2, -mb));
      }
      l_run[rb] += ((pe[0] + pe[1]) + (pe[2] + pe[3])) + ((pe[4] + pe[5]) + (pe[6] + pe[7]));
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t h = pack_bf16_pair(pe[2 * i], pe[2 * i + 1]);
        ph[rb][i] = h;
        pl[rb][i] = pack_bf16_pair(pe[2 * i] - __uint_as_float(h << 16), pe[2 * i + 1] - __uint_as_float(h & 0xFFFF0000u));
      }
    }
  };
  auto products = [&](const Pair& pr, int base) {
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * NI) : "memory");   // V is there (the next pair's K may still be on its way)
    uint2* va = reinterpret_cast<uint2*>(s_raw + wave * (4 * PART) + 2 * PART) + lane;
    if (base + 32 > n_all || !pr.ok_a || !pr.ok_b) {   // V of rows that were never written and of foreign pages: 0 * whatever is there must stay 0
      const int pos_a = base + 4 * g, pos_b = base + 16 + 4 * g;
      auto half = [&](bool ok, int p0) { return (ok && p0 < w.c1 ? 0x0000FFFFu : 0u) | (ok && p0 + 1 < w.c1 ? 0xFFFF0000u : 0u); };
      const unsigned a0 = half(pr.ok_a, pos_a), a1 = half(pr.ok_a, pos_a + 2), b0 = half(pr.ok_b, pos_b), b1 = half(pr.ok_b, pos_b + 2);
      uint32_t odd = 0;
#pragma unroll 1
      for (int dt = 0; dt < DT; ++dt) {
        uint2 a = va[dt * 64], b = va[PART / 8 + dt * 64];
        a = make_uint2(a.x & a0, a.y & a1);
        b = make_uint2(b.x & b0, b.y & b1);
        va[dt * 64] = a;
        va[PART / 8 + dt * 64] = b;
        odd |= (finite_pair(a.x) ^ a.x) | (finite_pair(a.y) ^ a.y) | (finite_pair(b.x) ^ b.x) | (finite_pair(b.y) ^ b.y);
      }
      asm volatile("" ::: "memory");
      if (w.own_len >= 0 && __builtin_amdgcn_ballot_w64(odd != 0) != 0ull) {
        const bf16_t* v = reinterpret_cast<const bf16_t*>(s_raw + wave * (4 * PART) + 2 * PART);
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
          add_not_finite(acc[rb], v, DF_PAGE, base, last[rb], lane);
          add_not_finite(acc[rb], v + PART / 2, DF_PAGE, base + DF_PAGE, last[rb], lane);
        }
        asm volatile("" ::: "memory");
#pragma unroll 1
        for (int dt = 0; dt < DT; ++dt) {
          const uint2 a = va[dt * 64], b = va[PART / 8 + dt * 64];
          va[dt * 64] = make_uint2(finite_pair(a.x), finite_pair(a.y));
          va[PART / 8 + dt * 64] = make_uint2(finite_pair(b.x), finite_pair(b.y));
        }
        asm volatile("" ::: "memory");
      }
    }
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {
      const uint2 a = va[dt * 64], b = va[PART / 8 + dt * 64];
      const u32x4 vf = {a.x, a.y, b.x, b.y};
#pragma unroll
      for (int rb = 0; rb < RB; ++rb)   // all hi products, then all lo products: two MFMAs on one accumulator are never back to back
        acc[rb][dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, vf), __builtin_bit_cast(bf16x8, ph[rb]), acc[rb][dt], 0, 0, 0);
#pragma unroll
      for (int rb = 0; rb < RB; ++rb)
        acc[rb][dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, vf), __builtin_bit_cast(bf16x8, pl[rb]), acc[rb][dt], 0, 0, 0);
    }
    __builtin_amdgcn_s_waitcnt(0xC07F);   // lgkmcnt(0): the V half has been read
  };
  if (my_pairs > 0) {
    Pair prev = cur;
    auto next = [&](int k) {   // the K of pair k on its way, after the last pair that one's again: the number of loads in flight stays the same
      if (k < my_pairs) {
        if ((k & 31) == 0) {
          ids = ids_next;
          if (k + 32 < my_pairs) ids_next = load_ids(k + 32);
          asm volatile("" : "+v"(ids_next));   // waited for here: left to the compiler it would be a wait for every copy at the end of every pair
        }
        cur = pair_of(k);
      }
      fetch(cur.a, 0);
      fetch(cur.b, PART);
    };
    scores(0);
    next(1);
    softmax(prev, w.c0 + wave * 32);
    for (int k = 1; k < my_pairs; ++k) {
      const int base = w.c0 + (wave + NW * k) * 32;
      products(prev, base - NW * 32);
      prev = cur;
      fetch(cur.a + DF_PAGE * HD, 2 * PART);
      fetch(cur.b + DF_PAGE * HD, 3 * PART);
      scores(k);
      next(k + 1);
      softmax(prev, base);
    }
    products(prev, w.c0 + (wave + NW * (my_pairs - 1)) * 32);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // nothing may still be on its way into the ring when it is overlaid
  }

  // ---- the wavefronts' parts together: the upper two hand theirs to the lower two, then all rows leave
  __syncthreads();   // every wavefront is done with the ring and the queries
  int* s_row = reinterpret_cast<int*>(s_raw + C::ROWS_AT(RB));   // the rows' places among the query rows of all heads: divisions once a row
  if ((int)threadIdx.x < w.n_rows) {
    const int row = w.row0 + threadIdx.x, at = row % ga.rows;
    s_row[threadIdx.x] = (row / ga.rows * geo.block_size + at / group) * ga.n_q_heads + kvh * group + at % group;
  }
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    const float l = quarter_sum(l_run[rb]);
    if (g == 0) s_ml[wave][rb * 16 + n] = make_float2(m_run[rb], l);
  }
  __syncthreads();
  float mine[RB];
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    float m_all = -INFINITY;
#pragma unroll
    for (int v = 0; v < NW; ++v) m_all = fmaxf(m_all, s_ml[v][rb * 16 + n].x);
    mine[rb] = m_run[rb] == m_all ? 1.f : __builtin_amdgcn_exp2f(m_run[rb] - m_all);   // (no key: both are -inf)
  }
  auto slot = [&](int v, int rb, int dt) { return reinterpret_cast<float4*>(&s_o[v][rb * 16 + n][dt * 16 + 4 * g]); };
  if (wave >= 2) {
#pragma unroll
    for (int rb = 0; rb < RB; ++rb)
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
        *slot(wave - 2, rb, dt) = make_float4(acc[rb][dt][0] * mine[rb], acc[rb][dt][1] * mine[rb], acc[rb][dt][2] * mine[rb], acc[rb][dt][3] * mine[rb]);
  }
  __syncthreads();
  if (wave < 2) {
#pragma unroll
    for (int rb = 0; rb < RB; ++rb)
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        float4* p = slot(wave, rb, dt);
        const float4 u = *p;
        *p = make_float4(acc[rb][dt][0] * mine[rb] + u.x, acc[rb][dt][1] * mine[rb] + u.y, acc[rb][dt][2] * mine[rb] + u.z, acc[rb][dt][3] * mine[rb] + u.w);
      }
  }
  __syncthreads();
  const int parts = ga.prefix_splits + ga.own_splits;
  bool again = false;
  for (int i = threadIdx.x; i < w.n_rows * (HD / 4); i += 64 * NW) {
    const int r = i / (HD / 4), d4 = i % (HD / 4);
    const size_t pr = (size_t)s_row[r] * parts + w.part;
    auto sum = [&]() {   // (maximum, sum) of the row
      float m_all = -INFINITY, l = 0.f;
#pragma unroll
      for (int v = 0; v < NW; ++v) m_all = fmaxf(m_all, s_ml[v][r].x);
#pragma unroll
      for (int v = 0; v < NW; ++v) {
        const float2 ml = s_ml[v][r];
        l += ml.y == 0.f ? 0.f : ml.y * (ml.x == m_all ? 1.f : __builtin_amdgcn_exp2f(ml.x - m_all));
      }
      return make_float2(m_all, l);
    };
    const float4 o = *reinterpret_cast<const float4*>(&s_o[0][r][d4 * 4]), o1 = *reinterpret_cast<const float4*>(&s_o[1][r][d4 * 4]);
    const float4 x = make_float4(o.x + o1.x, o.y + o1.y, o.z + o1.z, o.w + o1.w);
    if constexpr (DIRECT)
      if (ga.out) {
        again |= group_store<bf16_t>(ga, s_row[r], HD, d4 * 4, x, sum().y);
        continue;
      }
    *reinterpret_cast<float4*>(part_o + pr * HD + d4 * 4) = x;
    if (d4 == 0) part_ml[pr] = sum();
  }
  if (again)
#pragma unroll 1
    for (int i = threadIdx.x; i < w.n_rows * (HD / 4); i += 64 * NW) group_store_not_finite(geo, ga, pool, s_row[i / (HD / 4)], HD, i % (HD / 4) * 4);
}

// ---- bf16, head dims 32, 64, 96 and 128: tiles of 128 query rows of the prefix part -----------------------------------------------------
// Four wavefronts of 32 rows, the pages staged in an LDS ring that all four read (a stage is a pair of pages: K of page A, of page B, V of A, of B; every
// wavefront copies a quarter), one barrier a stage, two workgroups a CU.  32x32x16 MFMAs: S^T = K . Q^T leaves a lane 16 of the pair's keys (quartets h and h + 2
// of either page, h = lane / 32) of query column lane % 32, and O^T += V^T . P^T takes them as they are.
// Three stages of the sweep are in work at once, independent of each other: scores of pair i + 2, softmax of pair i + 1, products of pair i.  Matrix and vector
// instructions of one wavefront then run side by side, and the other workgroup's fill what is left.  Probabilities are a hi + lo bf16 pair, ~16 bits, as everywhere in the
// bf16 model.  (Rounded to bf16 once, for rows that leave in bf16 themselves, 32 x 16 rows behind 16384 tokens take 196 us instead of 233, nine smaller calls as long as
// with the pair, and the rows' error against 64 bits is 0.0023 instead of the 0.0017 of their own rounding.)
template <int HD>
struct TileSweep {
  static constexpr int KT = HD / 16, MT = HD / 32, NS = 5;
  static constexpr int PART = DF_PAGE * HD * 2, NI = PART / 1024, STAGE = 4 * PART, BYTES = NS * STAGE;   // PART: K or V of a page, NI copies of 1 KB
};

template <int HD>
__device__ __forceinline__ void group_sweep_tile(char* s_raw, const GroupWork& w, int kvh, const bf16_t* __restrict__ q, const bf16_t* __restrict__ pool,
                                                 const SeqGeom& geo, const GroupArgs& ga, float* __restrict__ part_o, float2* __restrict__ part_ml) {
  typedef TileSweep<HD> C;
  constexpr int KT = C::KT, MT = C::MT, NS = C::NS, PART = C::PART, NI = C::NI, STAGE = C::STAGE;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 31, h = lane >> 5;
  const int group = ga.n_q_heads / ga.n_kv_heads, n_pairs = (w.c1 - w.c0 + 31) >> 5, page0 = w.c0 / DF_PAGE;
  const int row = w.row0 + min(wave * 32 + n, w.n_rows - 1), rs = row / ga.rows, rat = row % ga.rows;   // a row that is not there reads along and is not stored
  const size_t out_row = (size_t)(rs * geo.block_size + rat / group) * ga.n_q_heads + kvh * group + rat % group;
  auto load_ids = [&](int p0) { return w.table[min(page0 + 2 * p0 + lane, geo.max_pages_per_seq - 1)]; };   // 32 pairs' page ids
  int ids = load_ids(0), ids_next = n_pairs > 32 ? load_ids(32) : 0;
  u32x4 qf[KT];   // dims 16 kt + 8 h .. + 7 of the lane's row
  {
    const u32x4* qp = reinterpret_cast<const u32x4*>(q + out_row * HD);
#pragma unroll
    for (int kt = 0; kt < KT; ++kt) qf[kt] = qp[kt * 2 + h];
  }
  const bool live = wave * 32 < w.n_rows;   // a wavefront without rows copies its quarters
  const bool half_pair = (w.c1 - w.c0) & DF_PAGE;   // the last pair has no page B: page A in its place, and its keys weigh nothing
  const unsigned lds = (unsigned)(size_t)s_raw + (unsigned)((wave & 1) * 2 + (wave >> 1)) * PART, voff = lane * 16;
  const size_t page_elems = (size_t)ga.n_kv_heads * 2 * DF_PAGE * HD;
  const bf16_t* mine = pool + kv_head_base(ga.layer, geo.n_pages, 0, ga.n_kv_heads, kvh, HD) + (size_t)(wave & 1) * DF_PAGE * HD;
  int fetch_slot = 0;
  // this wavefront's quarter of a stage: the K or V half (wave & 1) of page A or B (wave >> 1); past the end the last stage again, into a slot that nobody reads.
  // The pages of a prefix are all there (group_plan_kernel)
  auto fetch = [&](int st) {
    const int real = min(st, n_pairs - 1), at = (real & 31) * 2 + (half_pair && real == n_pairs - 1 ? 0 : wave >> 1);
    const bf16_t* src = mine + (size_t)__builtin_amdgcn_readlane(ids, at) * page_elems;
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const unsigned dst = __builtin_amdgcn_readfirstlane(lds + (unsigned)(fetch_slot * STAGE + i * 1024));
      const bf16_t* from = src + i * 512;
      unsigned keep_m0;   // whatever the compiler keeps in m0 is put back
      asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, %3\n\ts_nop 0\n\ts_mov_b32 m0, %0"
                   : "=&s"(keep_m0) : "s"(dst), "v"(voff), "s"(from) : "memory");
    }
    fetch_slot = fetch_slot + 1 == NS ? 0 : fetch_slot + 1;
  };
#pragma unroll
  for (int kt = 0; kt < KT; ++kt) asm volatile("" : "+v"(qf[kt]));   // waited for here: inside the loop that would be a wait for every copy
  asm volatile("" : "+v"(ids_next));
  for (int st = 0; st < NS - 1; ++st) fetch(st);

  float m_run = -INFINITY, neg_m = INFINITY, l_run = 0.f;   // no maximum yet: the first pair's sums are infinite
  f32x16 acc[MT];
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) acc[mt] = (f32x16){};
  const float scale2 = ga.scale * 1.44269504088896341f;   // base-2 exponents
  struct P { u32x4 v[2][2]; };   // hi and lo of page A's and page B's keys
  P p0, p1;
  f32x16 s0, s1;

  auto ready = [&]() {   // all stages but the youngest have landed, and everybody is done with the oldest
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(NI) : "memory");
    __builtin_amdgcn_s_waitcnt(0xC07F);   // lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };
  auto read_k = [&](u32x4 (&kf)[KT], int slot) {
    const u32x4* kp = reinterpret_cast<const u32x4*>(s_raw + slot * STAGE + (n >> 4) * PART) + h * 16 + (n & 15);
#pragma unroll
    for (int kt = 0; kt < KT; ++kt) kf[kt] = kp[kt * 32];
  };
  auto read_v = [&](u32x4 (&vf)[2][MT], int slot) {
    const uint2* vp = reinterpret_cast<const uint2*>(s_raw + slot * STAGE + 2 * PART) + (n >> 4) * 64 + h * 16 + (n & 15);
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const uint2 x = vp[mt * 128 + b * (PART / 8)], y = vp[mt * 128 + b * (PART / 8) + 32];   // quartets h and h + 2
        vf[b][mt] = (u32x4){x.x, x.y, y.x, y.y};
      }
  };
  auto qk = [&](f32x16& s, const u32x4& k, int kt) {
    s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, k), __builtin_bit_cast(bf16x8, qf[kt]), s, 0, 0, 0);
  };
  auto pv = [&](const u32x4& v, const u32x4& p, int mt) {
    acc[mt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, v), __builtin_bit_cast(bf16x8, p), acc[mt], 0, 0, 0);
  };
  // Probabilities of a pair.  The reference maximum is that of the sweep's first pair and stays while a lane's sum of exponentials, over all its keys so far, is at most
  // 2^20: the relative precision does not depend on it, and a row's weights are then at most 2^21 in all, which leaves room for values of 2^100.  So a pair costs no maximum,
  // only a look at the sum.
  auto soft = [&](const f32x16& s, P& p) {
    float e[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) e[i] = __builtin_amdgcn_exp2f(fmaf(s[i], scale2, neg_m));
    const float sum = (((e[0] + e[1]) + (e[2] + e[3])) + ((e[4] + e[5]) + (e[6] + e[7]))) + (((e[8] + e[9]) + (e[10] + e[11])) + ((e[12] + e[13]) + (e[14] + e[15])));
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float x = e[8 * b + 2 * i], y = e[8 * b + 2 * i + 1];
        const uint32_t v = pack_bf16_pair(x, y);
        p.v[0][b][i] = v;
        p.v[1][b][i] = pack_bf16_pair(x - __uint_as_float(v << 16), y - __uint_as_float(v & 0xFFFF0000u));
      }
    return sum;
  };
  // ... and the rest of it, when the products before it are in the accumulators: a row whose sum has grown too large (or that has no maximum yet) gets another
  // reference, by which everything there is is rescaled: this pair's maximum, or, where that is not far above the old one and many keys have made the sum, one 2^16 above it
  auto settle = [&](const f32x16& s, P& p, float sum) {
    constexpr float most = 0x1p20f;
    if (__builtin_amdgcn_ballot_w64(l_run + sum > most || sum != sum) != 0ull) {   // (nothing above -inf yet: the sum is infinite or a NaN)
      float mx = s[0];
#pragma unroll
      for (int i = 1; i < 16; ++i) mx = fmaxf(mx, s[i]);
      const LanePair x = lane_swap32(mx, mx), all = lane_swap32(l_run + sum, l_run + sum);
      mx = fmaxf(x.lo, x.hi) * scale2;
      if (m_run == -INFINITY ? mx > m_run : all.lo > most || all.hi > most) {
        const float ref = mx > m_run + 8.f ? mx : m_run + 16.f;
        const float corr = m_run == -INFINITY ? 0.f : exp2f(m_run - ref);
        l_run *= corr;
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) acc[mt] *= corr;
        m_run = ref;
        neg_m = -ref;
      }
      const float again = neg_m;
      if (m_run == -INFINITY) neg_m = 0.f;   // nothing above -inf yet: exp2(-inf - 0) = 0
      sum = soft(s, p);
      neg_m = again;
    }
    l_run += sum;
  };
  auto scores = [&](f32x16& s, int slot) {
    u32x4 kf[KT];
    read_k(kf, slot);
    s = (f32x16){};
#pragma unroll
    for (int kt = 0; kt < KT; ++kt) qk(s, kf[kt], kt);
  };
  auto without_b = [&](f32x16& s) {
#pragma unroll
    for (int i = 8; i < 16; ++i) s[i] = -INFINITY;
  };

  ready();   // stages 0, 1 and 2
  if (live) {
    scores(s0, 0);
    if (half_pair && n_pairs == 1) without_b(s0);
    settle(s0, p0, soft(s0, p0));
    if (n_pairs > 1) scores(s1, 1);
  }
  int slot = 0;   // of stage i
  auto step = [&](P& p, const f32x16& s, P& pn, f32x16& sn) {   // products with p, softmax of s into pn, scores into sn
    if (live) {
      u32x4 kf[KT], vf[2][MT];
      __builtin_amdgcn_sched_barrier(0);
      read_v(vf, slot);
      read_k(kf, slot + 2 >= NS ? slot + 2 - NS : slot + 2);
      sn = (f32x16){};
#pragma unroll
      for (int kt = 0; kt < KT; ++kt) {   // KT = 2 MT: the chain of the scores between products that do not wait for each other
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const int at = kt * 2 + j;
          pv(vf[at / MT % 2][at % MT], p.v[at / (2 * MT)][at / MT % 2], at % MT);
        }
        qk(sn, kf[kt], kt);
      }
      const float sum = soft(s, pn);
      __builtin_amdgcn_sched_barrier(0);
      settle(s, pn, sum);
    }
    slot = slot + 1 == NS ? 0 : slot + 1;
  };
  auto turn = [&](int i) {   // stage i + 2 is there; stage i + 4 goes where stage i - 1 was
    ready();
    const int ahead = i + NS - 1;
    if ((ahead & 31) == 0 && ahead < n_pairs) {   // uniform: the next set of page ids comes into use
      ids = ids_next;
      if (ahead + 32 < n_pairs) ids_next = load_ids(ahead + 32);
      asm volatile("" : "+v"(ids_next));
    }
    fetch(ahead);
  };
  int i = 0;
  for (; i + 3 < n_pairs; i += 2) {
    turn(i);
    step(p0, s1, p1, s0);
    turn(i + 1);
    step(p1, s0, p0, s1);
  }
  if (i + 2 < n_pairs) {
    turn(i);
    step(p0, s1, p1, s0);
    ++i;
    p0 = p1;
    s1 = s0;
  }
  ready();
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // nothing may still be on its way into LDS when the workgroup ends
  if (!live) return;
  auto last = [&](const P& p, bool cut) {
    u32x4 vf[2][MT];
    read_v(vf, slot);
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      if (cut) vf[1][mt] = (u32x4){0u, 0u, 0u, 0u};
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int pl = 0; pl < 2; ++pl) pv(vf[b][mt], p.v[pl][b], mt);
    }
    slot = slot + 1 == NS ? 0 : slot + 1;
  };
  if (i + 1 < n_pairs) {
    if (half_pair) without_b(s1);
    const float sum = soft(s1, p1);
    last(p0, false);
    settle(s1, p1, sum);
    p0 = p1;
  }
  last(p0, half_pair);
  const LanePair l = lane_swap32(l_run, l_run);
  if (wave * 32 + n >= w.n_rows) return;
  const size_t pr = out_row * (ga.prefix_splits + ga.own_splits) + w.part;
  if (h == 0) part_ml[pr] = make_float2(m_run, l.lo + l.hi);
#pragma unroll
  for (int mt = 0; mt < MT; ++mt)
#pragma unroll
    for (int j = 0; j < 4; ++j)
      *reinterpret_cast<float4*>(part_o + pr * HD + mt * 32 + 8 * j + 4 * h) = make_float4(acc[mt][4 * j], acc[mt][4 * j + 1], acc[mt][4 * j + 2], acc[mt][4 * j + 3]);
}

// RBP: row blocks (of 16) of the prefix part's key-split workgroups, 0: tiles of 128 rows.  RBO: row blocks of an own part's workgroup.
template <int HD, int RBP, int RBO>
__global__ __launch_bounds__(256, 2) void group_attn_mfma_kernel(const bf16_t* __restrict__ q, const bf16_t* __restrict__ pool, SeqGeom geo, GroupArgs ga,
                                                                 GroupTables gt, float* __restrict__ part_o, float2* __restrict__ part_ml) {
  constexpr int P_BYTES = RBP ? KeySplit<HD>::bytes(RBP) : TileSweep<HD>::BYTES, O_BYTES = KeySplit<HD>::bytes(RBO);
  __shared__ __attribute__((aligned(1024))) char s_raw[P_BYTES > O_BYTES ? P_BYTES : O_BYTES];
  static_assert(sizeof(s_raw) <= 80 * 1024, "two workgroups a CU");
  GroupWork w;
  int kvh;
  if (!group_work<256>(w, kvh, geo, ga, gt, part_ml)) return;
  constexpr bool DIRECT = RBP == RBO;   // (every sequence by itself: group_attn_launch)
  if (w.part >= ga.prefix_splits) {
    group_sweep_keys<HD, RBO, DIRECT>(s_raw, w, kvh, q, pool, geo, ga, part_o, part_ml);
    return say_outgrown(geo, w);
  }
  if constexpr (RBP == 0) group_sweep_tile<HD>(s_raw, w, kvh, q, pool, geo, ga, part_o, part_ml);
  else group_sweep_keys<HD, RBP, DIRECT>(s_raw, w, kvh, q, pool, geo, ga, part_o, part_ml);
}

// Parts -> rows, a wavefront a row, four dims a lane, as many parts side by side as that leaves room for (two of 128 dims) and four times that on their way.  A part
// without keys (its sum is exactly 0) is left out.
template <typename T>
__global__ __launch_bounds__(256) void group_merge_kernel(const float* __restrict__ part_o, const float2* __restrict__ part_ml, const T* __restrict__ pool, SeqGeom geo, GroupArgs ga,
                                                          int hd, int n_rows) {
  const int lane = threadIdx.x & 63, row = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);   // m * n_q_heads + hq
  if (row >= n_rows) return;
  const int parts = ga.prefix_splits + ga.own_splits;
  const int width = hd > 64 ? 32 : hd > 32 ? 16 : 8, beside = 64 / width, sub = lane / width, d = lane % width * 4;   // lanes of a part, parts side by side
  const float2 ml = lane < parts ? part_ml[(size_t)row * parts + lane] : make_float2(-INFINITY, 0.f);
  const bool some = ml.y != 0.f, mine = d < hd;
  const float mx = wave_reduce_max(some ? ml.x : -INFINITY);
  const float wgt = some ? __builtin_amdgcn_exp2f(ml.x - (mx == -INFINITY ? 0.f : mx)) : 0.f;
  const float L = wave_reduce_sum(some ? wgt * ml.y : 0.f);
  const unsigned long long live = __ballot(some);
  const float* po = part_o + (size_t)row * parts * hd + d;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int p0 = 0; p0 < parts; p0 += 4 * beside) {
    float4 x[4];
    bool on[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int p = p0 + u * beside + sub;
      on[u] = mine && p < parts && (live >> p & 1);
      x[u] = on[u] ? *reinterpret_cast<const float4*>(po + (size_t)p * hd) : make_float4(0.f, 0.f, 0.f, 0.f);
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const float w = __shfl(wgt, min(p0 + u * beside + sub, 63), 64);
      if (on[u]) {
        o.x += w * x[u].x; o.y += w * x[u].y; o.z += w * x[u].z; o.w += w * x[u].w;
      }
    }
  }
  for (int k = width; k < 64; k <<= 1) {
    o.x += __shfl_xor(o.x, k, 64); o.y += __shfl_xor(o.y, k, 64); o.z += __shfl_xor(o.z, k, 64); o.w += __shfl_xor(o.w, k, 64);
  }
  if (!mine || sub > 0) return;
  if (group_store<T>(ga, row, hd, d, o, L)) group_store_not_finite(geo, ga, pool, row, hd, d);
}

// whether the prefix part goes by tiles of 128 rows: the groups have more rows, on average, than a key-split workgroup
inline bool group_by_tiles(bool bf16, int hd, int n_seqs, int rows, int n_groups) {
  return bf16 && hd % 32 == 0 && (long long)n_seqs * rows > (long long)n_groups * kOwnTile;
}

template <typename T>
inline void group_attn_launch(hipStream_t st, const T* q, const T* pool, const SeqGeom& geo, const GroupArgs& ga, int hd, const GroupTables& gt, float* part_o,
                              float2* part_ml) {
  const dim3 grid((ga.max_tiles * ga.prefix_splits + ga.n_seqs * ga.own_tiles * ga.own_splits) * ga.n_kv_heads), block(256);
  if constexpr (sizeof(T) == 2) {
    const bool few = ga.rows <= 16, few_all = (long long)ga.n_seqs * ga.rows <= 16;
    auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, st, q, pool, geo, ga, gt, part_o, part_ml); };
    auto mfma = [&](auto c) {
      constexpr int HD = decltype(c)::value;
      if (!ga.prefix_splits || few_all) few ? launch(group_attn_mfma_kernel<HD, 1, 1>) : launch(group_attn_mfma_kernel<HD, 4, 4>);
      else if (ga.tile > kOwnTile) few ? launch(group_attn_mfma_kernel<HD, 0, 1>) : launch(group_attn_mfma_kernel<HD, 0, 4>);
      else few ? launch(group_attn_mfma_kernel<HD, 4, 1>) : launch(group_attn_mfma_kernel<HD, 4, 4>);
    };
    if (hd == 128) return mfma(std::integral_constant<int, 128>{});
    if (hd == 96) return mfma(std::integral_constant<int, 96>{});
    if (hd == 64) return mfma(std::integral_constant<int, 64>{});
    if (hd == 32) return mfma(std::integral_constant<int, 32>{});
  }
  auto go = [&](auto c) { hipLaunchKernelGGL((group_attn_kernel<T, decltype(c)::value>), grid, block, 0, st, q, pool, geo, ga, gt, part_o, part_ml); };
  switch (hd) {
    case 16: return go(std::integral_constant<int, 16>{});
    case 48: return go(std::integral_constant<int, 48>{});
    case 80: return go(std::integral_constant<int, 80>{});
    case 112: return go(std::integral_constant<int, 112>{});
    default: break;
  }
  if constexpr (sizeof(T) == 4) {
    if (hd == 32) return go(std::integral_constant<int, 32>{});
    if (hd == 64) return go(std::integral_constant<int, 64>{});
    if (hd == 96) return go(std::integral_constant<int, 96>{});
    go(std::integral_constant<int, 128>{});
  }
}
