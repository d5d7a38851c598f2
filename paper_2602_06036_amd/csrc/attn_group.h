// Block attention for sequences that share pages.
//
// The batch is cut into groups of consecutive sequences.  The leading pages that the block-table rows of a group have in common are attended
// to once for all rows of the group (the prefix part), what lies behind them by each sequence for itself (its own part):
//     row r:  o = softmax(q K^T * scale) V over both parts = (sum of parts of e^(m_i - m) o_i) / (sum of e^(m_i - m) l_i),
// m_i, l_i, o_i a part's running maximum, sum of exponentials and unnormalised output, m the largest of the maxima.  Both parts are split along their
// keys into ranges of equal length, ranges in a fixed order in the sum, so a call repeats itself bit for bit.  A row that sees no key is zeros; a NaN among
// its scores makes it NaN.
//
// What sequences share is found on the device, so a wrong grouping costs time and nothing else.
//
// Rows of a kv head, in the order of the batch: row = (sequence * block + slot) * group + query head of the kv head.
#pragma once
#include "attn_mfma.h"

constexpr int kGroupTile = 64;   // query rows of a workgroup

struct GroupArgs {
  int n_q_heads, n_kv_heads, layer, causal;
  int n_seqs, rows;         // query rows of a sequence and kv head = block size * (n_q_heads / n_kv_heads)
  int max_tiles;            // tiles of the prefix part, at most
  int own_tiles;            // tiles of a sequence's own part
  int prefix_splits, own_splits;
  float scale;
};

// Written by group_plan_kernel, read by the launches behind it.
struct GroupTables {
  int4* tiles;      // first row, rows (0: no tile), block-table row to read, tokens of the prefix
  int32_t* first;   // [n_seqs] tokens in front of a sequence's own part
};
// Tiles of the prefix part: group g, which starts at sequence a, has those from a * rows / kGroupTile + g on (rounded down: whatever the groups in
// front of it need lies below), so no group has to wait for another's count.
__host__ __device__ __forceinline__ int group_tile_slots(int n_seqs, int rows, int n_groups) { return (int)((long long)n_seqs * rows / kGroupTile) + n_groups; }

// Groups -> tiles, a workgroup each: where the group starts and ends (the caller's starts as their running maximum, inside the batch, the first 0 and the
// last end n_seqs), and how many leading pages its rows have in common and committed.  n_groups = 1 needs no starts.
__global__ __launch_bounds__(1024) void group_plan_kernel(SeqGeom geo, const int32_t* __restrict__ starts, int n_groups, int n_seqs, int rows, GroupTables gt) {
  __shared__ int s_start, s_end, s_pages;
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6, g = blockIdx.x;
  if (t == 0) {
    s_start = 0;
    s_end = g + 1 < n_groups ? 0 : n_seqs;
    s_pages = geo.max_pages_per_seq;
  }
  __syncthreads();
  if (n_groups > 1) {
    for (int i = t; i <= g + 1 && i < n_groups; i += 1024) {
      const int given = starts[i], at = i == 0 ? 0 : min(max(given, 0), n_seqs);
      if (given != at || (i + 1 < n_groups && starts[i + 1] < given)) atomicOr(geo.status, DF_STATUS_CAPACITY);
      if (i <= g) atomicMax(&s_start, at);
      atomicMax(&s_end, at);
    }
    __syncthreads();
  }
  const int start = s_start, end = s_end, size = end - start, mpps = geo.max_pages_per_seq;
  if (size > 0) {
    for (int s = start + t; s < end; s += 1024) atomicMin(&s_pages, size > 1 ? max(geo.seq_lens[s], 0) / DF_PAGE : 0);
    __syncthreads();
    const int32_t* lead = geo.block_table + (size_t)start * mpps;
    int most = s_pages;
    __syncthreads();
    for (int k = wave; k < size; k += 16) {   // the first one against the range of page ids, the others against it
      const int32_t* row = lead + (size_t)k * mpps;
      for (int p = lane; p < most; p += 64) {
        const int id = lead[p];
        if (k ? row[p] != id : (id < 0 || id >= geo.n_pages)) most = p;
      }
    }
    atomicMin(&s_pages, most);
    __syncthreads();
    for (int s = start + t; s < end; s += 1024) gt.first[s] = s_pages * DF_PAGE;
  }
  // this group's tiles, and the slots behind them up to the next group's
  const int row0 = start * rows, row1 = end * rows, slot0 = row0 / kGroupTile + g, slot1 = row1 / kGroupTile + g + 1;
  for (int i = slot0 + t; i < slot1; i += 1024) {
    const int r = row0 + (i - slot0) * kGroupTile;
    gt.tiles[i] = make_int4(r, size > 0 ? max(0, min(kGroupTile, row1 - r)) : 0, start, s_pages * DF_PAGE);
  }
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
  // V elements of keys that are not there (never written, another sequence's): 0 * whatever they hold must stay 0
  static __device__ __forceinline__ void clear(Values& f, const bool (&there)[8]) {
    auto half = [&](int i) { return (there[i] ? 0x0000FFFFu : 0u) | (there[i + 1] ? 0xFFFF0000u : 0u); };
    const unsigned m[4] = {half(0), half(2), half(4), half(6)};
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {
      f.a[dt].x &= m[0]; f.a[dt].y &= m[1];
      f.b[dt].x &= m[2]; f.b[dt].y &= m[3];
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
  static __device__ __forceinline__ void clear(Values& f, const bool (&there)[8]) {
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {
      f.a[dt] = make_float4(there[0] ? f.a[dt].x : 0.f, there[1] ? f.a[dt].y : 0.f, there[2] ? f.a[dt].z : 0.f, there[3] ? f.a[dt].w : 0.f);
      f.b[dt] = make_float4(there[4] ? f.b[dt].x : 0.f, there[5] ? f.b[dt].y : 0.f, there[6] ? f.b[dt].z : 0.f, there[7] ? f.b[dt].w : 0.f);
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

// What a workgroup does: query rows, their keys' pages, and where the partial results go.
struct GroupWork {
  int row0, n_rows;         // rows of the kv head
  const int32_t* table;     // block-table row
  int c0, c1, n_tok;        // keys from c0 to below c1; keys from n_tok on were never written
  int own_len;              // causal mask of a sequence's own part: tokens in front of its block; < 0: every row sees every key
  int part;                 // index of the partial result
};

// grid: (tiles of the prefix part x its key ranges, then tiles of the own parts x theirs) x kv heads, kv heads fastest: the tiles that share keys lie
// max_tiles apart in steps of a multiple of the heads and ranges
__device__ __forceinline__ bool group_work(GroupWork& w, int& kvh, const SeqGeom& geo, const GroupArgs& ga, const GroupTables& gt) {
  int i = blockIdx.x / ga.n_kv_heads;
  kvh = blockIdx.x % ga.n_kv_heads;
  const int n_prefix = ga.max_tiles * ga.prefix_splits;
  if (i < n_prefix) {
    const int4 t = gt.tiles[i / ga.prefix_splits];
    const int split = i % ga.prefix_splits;
    if (t.y == 0 || t.w == 0) return false;   // the merge looks at `first` and leaves the prefix out
    const int chunk = ((t.w + 31) / 32 + ga.prefix_splits - 1) / ga.prefix_splits * 32;
    w = {t.x, t.y, geo.block_table + (size_t)t.z * geo.max_pages_per_seq, min(split * chunk, t.w), min((split + 1) * chunk, t.w), t.w, -1, split};
    return true;
  }
  i -= n_prefix;
  const int split = i % ga.own_splits, tile = i / ga.own_splits % ga.own_tiles, s = i / (ga.own_splits * ga.own_tiles);
  const int len = max(geo.seq_lens[s], 0), n_tok = min(len + geo.block_size, geo.max_pages_per_seq * DF_PAGE), first = gt.first[s];
  const int chunk = ((n_tok - first + 31) / 32 + ga.own_splits - 1) / ga.own_splits * 32;
  w = {s * ga.rows + tile * kGroupTile, min(kGroupTile, ga.rows - tile * kGroupTile), geo.block_table + (size_t)s * geo.max_pages_per_seq,
       min(first + split * chunk, n_tok), min(first + (split + 1) * chunk, n_tok), n_tok, ga.causal ? len : -1, ga.prefix_splits + split};
  return true;
}

// Any storage type and head dim.  Four wavefronts of 16 rows each sweep the workgroup's keys, a pair of pages at a time straight from memory.
template <typename T, int HD>
__global__ __launch_bounds__(256, 2) void group_attn_kernel(const T* __restrict__ q, const T* __restrict__ pool, SeqGeom geo, GroupArgs ga, GroupTables gt,
                                                            float* __restrict__ part_o, float2* __restrict__ part_ml) {
  typedef PairFrags<T, HD> F;
  constexpr int DT = HD / 16;
  GroupWork w;
  int kvh;
  if (!group_work(w, kvh, geo, ga, gt)) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 15, g = lane >> 4;
  if (wave * 16 >= w.n_rows) return;
  const int group = ga.n_q_heads / ga.n_kv_heads;
  const bool valid = wave * 16 + n < w.n_rows;
  const int row = w.row0 + (valid ? wave * 16 + n : 0);
  const int s = row / ga.rows, slot = row % ga.rows / group, hq = kvh * group + row % group;   // rows is a multiple of the group
  const size_t m_hq = (size_t)(s * geo.block_size + slot) * ga.n_q_heads + hq;
  typename F::Query qf;
  F::query(qf, valid ? q + m_hq * HD : nullptr, lane);
  const int last = !valid ? -1 : (w.own_len >= 0 ? w.own_len + slot : w.n_tok - 1);

  float m_run = -INFINITY, l_run = 0.f;
  f32x4 acc[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) acc[dt] = (f32x4){0.f, 0.f, 0.f, 0.f};
  const float scale2 = ga.scale * 1.44269504088896341f;   // base-2 exponents

  for (int base = w.c0; base < w.c1; base += 32) {
    const int at = base / DF_PAGE;
    int pa = w.table[at], pb = base + DF_PAGE < w.c1 ? w.table[at + 1] : -1;
    const bool ok_a = pa >= 0 && pa < geo.n_pages, ok_b = pb >= 0 && pb < geo.n_pages;
    pa = ok_a ? pa : 0;   // a page that may be read; its keys weigh nothing
    pb = ok_b ? pb : pa;
    const T* ka = pool + kv_head_base(ga.layer, geo.n_pages, pa, ga.n_kv_heads, kvh, HD);
    const T* kb = pool + kv_head_base(ga.layer, geo.n_pages, pb, ga.n_kv_heads, kvh, HD);
    typename F::Keys kf;
    typename F::Values vf;
    F::keys(kf, ka, kb, lane);
    F::values(vf, ka, kb, lane);
    f32x4 sa, sb;
    F::scores(sa, sb, kf, qf);
    float v[8], p[8];
    bool there[8], all = true;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int pos = base + (i >> 2) * DF_PAGE + 4 * g + (i & 3);
      there[i] = (i < 4 ? ok_a : ok_b) && pos < w.c1;
      all = all && there[i];
      v[i] = there[i] && pos <= last ? (i < 4 ? sa[i & 3] : sb[i & 3]) * scale2 : -INFINITY;
    }
    if (!all) F::clear(vf, there);
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
    F::add(acc, vf, p);
  }
  const float l = quarter_sum(l_run);
  if (!valid) return;
  const size_t pr = m_hq * (ga.prefix_splits + ga.own_splits) + w.part;
  if (g == 0) part_ml[pr] = make_float2(m_run, l);
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
    *reinterpret_cast<float4*>(part_o + pr * HD + dt * 16 + 4 * g) = make_float4(acc[dt][0], acc[dt][1], acc[dt][2], acc[dt][3]);
}

// ---- bf16, head dim 64 or 128: wavefronts split the keys ------------------------------------------------------------------
// Eight wavefronts take every eighth pair of pages each for all RB blocks of 16 query rows, from a ring of their own in LDS: the pages go there
// directly (global_load_lds), K refilled as soon as a pair's scores are done and V as soon as its products are, so nothing in flight costs a
// register and no wavefront waits for another before the end, where their partial results are added in LDS.  The loads are counted by hand (NI per half page,
// in order): the compiler would wait for all of them ahead of every LDS read.
template <int HD>
struct KeySplit {
  static constexpr int KT = HD / 32, DT = HD / 16, NW = 8, LD = HD + 4;
  static constexpr int PART = DF_PAGE * HD * 2, NI = PART / 1024;   // bytes of the K or V part of a page, load instructions for it
  static constexpr int RING = NW * 4 * PART;                        // per wavefront: K of page A, of page B, V of page A, of page B
  static constexpr int bytes(int rb) { return (RING + rb * KT * 1024 > 4 * rb * 16 * LD * 4 ? RING + rb * KT * 1024 : 4 * rb * 16 * LD * 4); }
};

template <int HD, int RB>
__device__ __forceinline__ void group_sweep_keys(char* s_raw, float2 (*s_ml)[64], const GroupWork& w, int kvh, const bf16_t* __restrict__ q,
                                                 const bf16_t* __restrict__ pool, const SeqGeom& geo, const GroupArgs& ga, float* __restrict__ part_o,
                                                 float2* __restrict__ part_ml) {
  typedef KeySplit<HD> C;
  constexpr int KT = C::KT, DT = C::DT, NW = C::NW, LD = C::LD, PART = C::PART, NI = C::NI;
  float (*s_o)[RB * 16][LD] = reinterpret_cast<float (*)[RB * 16][LD]>(s_raw);   // overlays ring and queries in the end
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

  for (int k = 0; k < my_pairs; ++k) {
    const int base = w.c0 + (wave + NW * k) * 32;
    const bool more = k + 1 < my_pairs;
    if (more && ((k + 1) & 31) == 0) {
      ids = ids_next;
      if (k + 33 < my_pairs) ids_next = load_ids(k + 33);
    }
    Pair nxt = cur;
    if (more) nxt = pair_of(k + 1);

    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * NI) : "memory");   // this pair's K is there (its V still on the way)
    f32x4 sc[RB][2];
    {
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
    }
    __builtin_amdgcn_s_waitcnt(0xC07F);   // lgkmcnt(0): the K half has been read
    if (more) {
      fetch(nxt.a, 0);
      fetch(nxt.b, PART);
    }
    __builtin_amdgcn_sched_barrier(0);

    const bool tail = !cur.ok_a || !cur.ok_b || base + 32 > n_all;   // (n_all <= c1: keys behind the range as well)
    if (tail) {
      const int p0 = base + 4 * g;
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        const int upto = min(w.c1 - 1, last[rb]);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (!(cur.ok_a && p0 + i <= upto)) sc[rb][0][i] = -INFINITY;
          if (!(cur.ok_b && p0 + 16 + i <= upto)) sc[rb][1][i] = -INFINITY;
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
    u32x4 ph[RB], pl[RB];   // probabilities as hi + lo pairs
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
    if (more) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * NI) : "memory");   // V is there (the next pair's K may still be on its way)
    else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    u32x4 keep = {~0u, ~0u, ~0u, ~0u};   // V of rows that were never written and of foreign pages: 0 * whatever is there must stay 0
    if (base + 32 > w.c1 || !cur.ok_a || !cur.ok_b) {
      const int pos_a = base + 4 * g, pos_b = base + 16 + 4 * g;
      auto half = [&](bool ok, int p0) { return (ok && p0 < w.c1 ? 0x0000FFFFu : 0u) | (ok && p0 + 1 < w.c1 ? 0xFFFF0000u : 0u); };
      keep = (u32x4){half(cur.ok_a, pos_a), half(cur.ok_a, pos_a + 2), half(cur.ok_b, pos_b), half(cur.ok_b, pos_b + 2)};
    }
    {
      const uint2* va = reinterpret_cast<const uint2*>(my_ring + 2 * PART) + lane;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        const uint2 a = va[dt * 64], b = va[PART / 8 + dt * 64];
        const u32x4 vf = (u32x4){a.x, a.y, b.x, b.y} & keep;
#pragma unroll
        for (int rb = 0; rb < RB; ++rb)   // all hi products, then all lo products: two MFMAs on one accumulator are never back to back
          acc[rb][dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, vf), __builtin_bit_cast(bf16x8, ph[rb]), acc[rb][dt], 0, 0, 0);
#pragma unroll
        for (int rb = 0; rb < RB; ++rb)
          acc[rb][dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, vf), __builtin_bit_cast(bf16x8, pl[rb]), acc[rb][dt], 0, 0, 0);
      }
    }
    __builtin_amdgcn_s_waitcnt(0xC07F);   // lgkmcnt(0): the V half has been read
    if (more) {
      fetch(nxt.a + DF_PAGE * HD, 2 * PART);
      fetch(nxt.b + DF_PAGE * HD, 3 * PART);
    }
    cur = nxt;
  }

  // ---- the wavefronts' parts together: the upper four hand theirs to the lower four, then all rows leave
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    const float l = quarter_sum(l_run[rb]);
    if (g == 0) s_ml[wave][rb * 16 + n] = make_float2(m_run[rb], l);
  }
  __syncthreads();   // also: every wavefront is done with the ring and the queries that s_o overlays
  float mine[RB];
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    float m_all = -INFINITY;
#pragma unroll
    for (int v = 0; v < NW; ++v) m_all = fmaxf(m_all, s_ml[v][rb * 16 + n].x);
    mine[rb] = m_run[rb] == m_all ? 1.f : __builtin_amdgcn_exp2f(m_run[rb] - m_all);   // (no key: both are -inf)
  }
  auto slot = [&](int v, int rb, int dt) { return reinterpret_cast<float4*>(&s_o[v][rb * 16 + n][dt * 16 + 4 * g]); };
  if (wave >= 4) {
#pragma unroll
    for (int rb = 0; rb < RB; ++rb)
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
        *slot(wave - 4, rb, dt) = make_float4(acc[rb][dt][0] * mine[rb], acc[rb][dt][1] * mine[rb], acc[rb][dt][2] * mine[rb], acc[rb][dt][3] * mine[rb]);
  }
  __syncthreads();
  if (wave < 4) {
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
  for (int i = threadIdx.x; i < w.n_rows * (HD / 4); i += 64 * NW) {
    const int r = i / (HD / 4), d4 = i % (HD / 4), row = w.row0 + r;
    const int s = row / ga.rows, at = row % ga.rows;
    const size_t pr = ((size_t)(s * geo.block_size + at / group) * ga.n_q_heads + kvh * group + at % group) * parts + w.part;
    float4 o = *reinterpret_cast<const float4*>(&s_o[0][r][d4 * 4]);
#pragma unroll
    for (int v = 1; v < 4; ++v) {
      const float4 a = *reinterpret_cast<const float4*>(&s_o[v][r][d4 * 4]);
      o.x += a.x; o.y += a.y; o.z += a.z; o.w += a.w;
    }
    *reinterpret_cast<float4*>(part_o + pr * HD + d4 * 4) = o;
    if (d4 == 0) {
      float m_all = -INFINITY, l = 0.f;
#pragma unroll
      for (int v = 0; v < NW; ++v) m_all = fmaxf(m_all, s_ml[v][r].x);
#pragma unroll
      for (int v = 0; v < NW; ++v) {
        const float2 ml = s_ml[v][r];
        l += ml.y == 0.f ? 0.f : ml.y * (ml.x == m_all ? 1.f : __builtin_amdgcn_exp2f(ml.x - m_all));
      }
      part_ml[pr] = make_float2(m_all, l);
    }
  }
}

template <int HD, int RBP, int RBO>
__global__ __launch_bounds__(512, 2) void group_attn_keys_kernel(const bf16_t* __restrict__ q, const bf16_t* __restrict__ pool, SeqGeom geo, GroupArgs ga,
                                                                 GroupTables gt, float* __restrict__ part_o, float2* __restrict__ part_ml) {
  constexpr int RB = RBP > RBO ? RBP : RBO;
  __shared__ __attribute__((aligned(1024))) char s_raw[KeySplit<HD>::bytes(RB)];
  __shared__ float2 s_ml[8][64];
  GroupWork w;
  int kvh;
  if (!group_work(w, kvh, geo, ga, gt)) return;
  if (w.part < ga.prefix_splits) group_sweep_keys<HD, RBP>(s_raw, s_ml, w, kvh, q, pool, geo, ga, part_o, part_ml);
  else group_sweep_keys<HD, RBO>(s_raw, s_ml, w, kvh, q, pool, geo, ga, part_o, part_ml);
}

// Parts -> rows, a wavefront a row, two dims a lane.  A part without keys (its sum is exactly 0) is left out.  OPERAND: GEMM activation operand (Act<T>), else
// plain rows of the model's type.
template <typename T, bool OPERAND>
__global__ __launch_bounds__(256) void group_merge_kernel(const float* __restrict__ part_o, const float2* __restrict__ part_ml, T* __restrict__ out, GroupArgs ga,
                                                          const int32_t* __restrict__ first, int hd, int block, int n_rows) {
  const int lane = threadIdx.x & 63, row = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);   // m * n_q_heads + hq
  if (row >= n_rows) return;
  const int parts = ga.prefix_splits + ga.own_splits, m = row / ga.n_q_heads, hq = row % ga.n_q_heads;
  const int from = first[m / block] > 0 ? 0 : ga.prefix_splits;   // nothing in common: the prefix part was not computed
  const float2 ml = lane >= from && lane < parts ? part_ml[(size_t)row * parts + lane] : make_float2(-INFINITY, 0.f);
  const bool some = ml.y != 0.f;
  const float mx = wave_reduce_max(some ? ml.x : -INFINITY);
  const float wgt = some ? __builtin_amdgcn_exp2f(ml.x - (mx == -INFINITY ? 0.f : mx)) : 0.f;
  const unsigned long long live = __ballot(some);
  const float* po = part_o + (size_t)row * parts * hd + 2 * lane;
  float L = 0.f;
  float2 o = make_float2(0.f, 0.f);
  const bool mine = 2 * lane < hd;
  for (int i = from; i < parts; ++i)
    if (live >> i & 1) {
      const float w = lane_value(wgt, i);
      L += w * lane_value(ml.y, i);
      const float2 x = mine ? *reinterpret_cast<const float2*>(po + (size_t)i * hd) : make_float2(0.f, 0.f);
      o.x += w * x.x;
      o.y += w * x.y;
    }
  if (!mine) return;
  const float by = L != 0.f ? L : INFINITY;   // no visible key: zeros
  o.x /= by;
  o.y /= by;
  if constexpr (OPERAND) {
    Act<T>::store(out, m, hq * hd + 2 * lane, ga.n_q_heads * hd, o.x);
    Act<T>::store(out, m, hq * hd + 2 * lane + 1, ga.n_q_heads * hd, o.y);
  } else {
    T* to = out + (size_t)row * hd + 2 * lane;
    if constexpr (sizeof(T) == 2) *reinterpret_cast<uint32_t*>(to) = pack_bf16_pair(o.x, o.y);
    else *reinterpret_cast<float2*>(to) = o;
  }
}

template <typename T>
inline void group_attn_launch(hipStream_t st, const T* q, const T* pool, const SeqGeom& geo, const GroupArgs& ga, int hd, const GroupTables& gt, float* part_o,
                              float2* part_ml) {
  const dim3 grid((ga.max_tiles * ga.prefix_splits + ga.n_seqs * ga.own_tiles * ga.own_splits) * ga.n_kv_heads), block(256);
  if constexpr (sizeof(T) == 2) {
    const bool few = ga.rows <= 16, few_all = (long long)ga.n_seqs * ga.rows <= 16;
    auto keys = [&](auto c) {
      constexpr int HD = decltype(c)::value;
      if (few_all) hipLaunchKernelGGL((group_attn_keys_kernel<HD, 1, 1>), grid, dim3(512), 0, st, q, pool, geo, ga, gt, part_o, part_ml);
      else if (few) hipLaunchKernelGGL((group_attn_keys_kernel<HD, 4, 1>), grid, dim3(512), 0, st, q, pool, geo, ga, gt, part_o, part_ml);
      else hipLaunchKernelGGL((group_attn_keys_kernel<HD, 4, 4>), grid, dim3(512), 0, st, q, pool, geo, ga, gt, part_o, part_ml);
    };
    if (hd == 128) return keys(std::integral_constant<int, 128>{});
    if (hd == 64) return keys(std::integral_constant<int, 64>{});
  }
  auto go = [&](auto c) { hipLaunchKernelGGL((group_attn_kernel<T, decltype(c)::value>), grid, block, 0, st, q, pool, geo, ga, gt, part_o, part_ml); };
  switch (hd) {
    case 16: return go(std::integral_constant<int, 16>{});
    case 32: return go(std::integral_constant<int, 32>{});
    case 48: return go(std::integral_constant<int, 48>{});
    case 64: return go(std::integral_constant<int, 64>{});
    case 80: return go(std::integral_constant<int, 80>{});
    case 96: return go(std::integral_constant<int, 96>{});
    case 112: return go(std::integral_constant<int, 112>{});
    default: return go(std::integral_constant<int, 128>{});
  }
}
