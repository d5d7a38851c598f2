// Page ledger: which block-table row holds which page of the pools, and the copies that this asks for.
//
//   block_table[r][p] = page of tokens 16p .. 16p+15 of sequence r, -1 = none;  page_refs[i] = entries that hold page i, 0 = free
//
// Forking shares the parent's pages, reserving gives a row pages of its own for what it writes next (a copy of the page its last
// tokens stand in where another row holds that too), releasing gives pages back, compacting moves the pages in use to the lowest ids.
// Pages are taken in ascending order for rows in ascending order: what a call does depends on the ledger alone.
#pragma once
#include "common.h"

struct Ledger {
  int32_t *table, *seq_lens, *anchor, *refs;
  int32_t n_rows, mpps, n_pages;
  int32_t* status;
};

// rows of a call by value: a copy of the caller's host array that a captured graph keeps
constexpr int kRowsPerLaunch = 256;
struct RowPairs {
  int32_t a[kRowsPerLaunch], b[kRowsPerLaunch];
};
struct ForkRows {
  int32_t parent[kRowsPerLaunch], child[kRowsPerLaunch], count[kRowsPerLaunch];   // count: children of the parent in the launch, at the first of them; 0 at the others
};

// a value that another thread of the workgroup has just changed by an atomic, which the L1 does not see
__device__ __forceinline__ int agent_load(const int32_t* p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

__device__ __forceinline__ bool page_in(const Ledger& l, int id) { return id >= 0 && id < l.n_pages; }

// Children become what their parents are: one thread an entry.  Counts go up and down by integer atomics, whose order does not matter; a parent's pages are counted up once
// for all its children (60 children of four prompts of 8192 to 16384 tokens: 6.6 us with an atomic an entry, 3.2 so).  No child is a parent (checked on the host), so
// rows that are read are not written.
__global__ __launch_bounds__(256) void pages_fork_kernel(Ledger l, ForkRows rows) {
  const int from = rows.parent[blockIdx.y], to = rows.child[blockIdx.y], count = rows.count[blockIdx.y], p = blockIdx.x * 256 + threadIdx.x;
  const int n = l.seq_lens[from], held = n <= 0 ? 0 : (n - 1) / DF_PAGE + 1;   // (n + 15 need not fit)
  if (p == 0) {
    l.seq_lens[to] = n;
    l.anchor[to] = l.anchor[from];
    if (held > l.mpps) atomicOr(l.status, DF_STATUS_CAPACITY);
  }
  if (p >= l.mpps) return;
  int32_t* at = l.table + (size_t)to * l.mpps + p;
  const int old = *at, given = l.table[(size_t)from * l.mpps + p], id = p < held ? given : -1;
  if (page_in(l, old)) atomicSub(l.refs + old, 1);
  if (count > 0 && page_in(l, id)) atomicAdd(l.refs + id, count);
  *at = id;
  if (p < held && !page_in(l, id)) atomicOr(l.status, DF_STATUS_CAPACITY);
}

// Rows (a) give back what lies behind their first `keep` (b) tokens.  (60 rows of four prompts of 8192 to 16384 tokens 6.2 us; with a thread for an entry of sixteen
// rows, which counts a page down once for all of them, the same.)
__global__ __launch_bounds__(256) void pages_release_kernel(Ledger l, RowPairs rows) {
  const int r = rows.a[blockIdx.y], keep = rows.b[blockIdx.y], p = blockIdx.x * 256 + threadIdx.x;
  if (p == 0) l.seq_lens[r] = min(l.seq_lens[r], keep);
  if (p >= l.mpps || (long long)p * DF_PAGE < keep) return;
  int32_t* at = l.table + (size_t)r * l.mpps + p;
  const int id = *at;
  if (page_in(l, id)) atomicSub(l.refs + id, 1);
  if (id != -1) *at = -1;
}

// Inclusive sum over a workgroup of 1024 threads; *total: of all.  `s`: 17 words of LDS; ends behind a barrier, so that it may be called again.
__device__ __forceinline__ int block_sum(int v, int* s, int* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int o = __shfl_up(v, d, 64);
    if (lane >= d) v += o;
  }
  if (lane == 63) s[wave] = v;
  __syncthreads();
  int before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < 16; ++w) {
    const int x = s[w];
    if (w < wave) before += x;
    all += x;
  }
  __syncthreads();
  *total = all;
  return v + before;
}

// What one launch of the plan covers; rows beyond go to the next launch, which sees this one's counts.
constexpr int kReserveRows = 1024;

struct ReserveScratch {
  int4* copies;       // [kReserveRows] by row: from, to, rows to copy; from < 0: nothing
  unsigned long long* wants;   // a bit per asked-for entry that takes a page, 64 entries a word
  int32_t* free_ids;  // [n_pages] the lowest free pages, as many as are wanted
  int32_t* stuck;     // a row of this call did not fit: no row behind it takes pages
};

// Rows row0 .. row0 + n - 1 get pages for tokens[row] more tokens: one workgroup, a thread a row and then a thread an entry.  A chain of loads and
// barriers (32 rows of 405 to 643 tokens 6.9 us; 9.6 with the free ids through memory and a device-wide fence in front of the last look at the counts).
// The rule that a shared page's last asker keeps it: the k-th row of the call that asks for a page held c times gets a copy if k < c - 1.  Only the entry
// with a row's last tokens can be shared in a ledger that these calls have kept; one behind it is replaced whoever else holds it.
__global__ __launch_bounds__(1024) void pages_reserve_kernel(Ledger l, int row0, int n, const int32_t* __restrict__ tokens, int32_t* __restrict__ granted,
                                                             ReserveScratch sc) {
  __shared__ int s_id[kReserveRows], s_start[kReserveRows + 1], s_first[kReserveRows], s_cum[kReserveRows], s_base[kReserveRows], s_new[kReserveRows], s_sum[17];
  __shared__ int s_free[kReserveRows];   // the lowest of the free pages; those behind go through memory
  __shared__ unsigned char s_want[kReserveRows];
  const int t = threadIdx.x, row = row0 + t;
  int lowest[4];   // the counts of the first 4096 pages, of which the free ones are wanted below
#pragma unroll
  for (int i = 0; i < 4; ++i) lowest[i] = l.refs[min(4 * t + i, l.n_pages - 1)];
  int len = 0, first = 0, count = 0, id = -1 - t, c = 0;
  bool asks = false, refused = false;
  if (t < n) {
    len = l.seq_lens[row];
    const int more = tokens[row];
    asks = more > 0;
    first = max(len, 0) / DF_PAGE;
    const long long end = ((long long)len + more + DF_PAGE - 1) / DF_PAGE;
    refused = asks && (len < 0 || end > l.mpps);
    if (asks && !refused) {
      count = (int)end - first;
      const int held = l.table[(size_t)row * l.mpps + first];
      if (page_in(l, held)) {
        id = held;
        c = l.refs[held];
      }
    }
  }
  s_id[t] = id;
  s_first[t] = first;
  s_cum[t] = s_base[t] = 0;
  int n_entries;
  s_start[t] = block_sum(count, s_sum, &n_entries) - count;
  int rank = 0;
  if (count > 0 && id >= 0 && c > 1)
    for (int i = 0; i < t; ++i) rank += s_id[i] == id;
  const bool shared = count > 0 && id >= 0 && rank < c - 1, want_first = count > 0 && (id < 0 || shared);
  s_want[t] = want_first;
  if (t == 0) s_start[kReserveRows] = n_entries;
  __syncthreads();

  // ---- which entries take a page: 1024 at a time, thread by thread; what a single block of them found stays in registers
  auto row_of = [&](int e) {   // the last row whose entries start at or before e: one that has some
    int lo = 0, hi = kReserveRows;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (s_start[mid] <= e) lo = mid;
      else hi = mid;
    }
    return lo;
  };
  struct Entry {
    int32_t* at;
    int row, old;
    bool want;
  };
  auto look = [&](int e) {
    Entry x{nullptr, 0, -1, false};
    if (e >= n_entries) return x;
    x.row = row_of(e);
    const int k = e - s_start[x.row];
    x.at = l.table + (size_t)(row0 + x.row) * l.mpps + s_first[x.row] + k;
    if (k == 0) {
      x.old = s_id[x.row];   // (a missing page: below 0)
      x.want = s_want[x.row];
    } else {
      x.old = *x.at;
      x.want = !page_in(l, x.old) || l.refs[x.old] > 1;
    }
    return x;
  };
  int wanted = 0, upto = 0;
  Entry mine{nullptr, 0, -1, false};
  for (int e0 = 0; e0 < n_entries; e0 += 1024) {
    const int e = e0 + t;
    mine = look(e);
    if (n_entries > 1024) {
      const unsigned long long bits = __ballot(mine.want);
      if ((t & 63) == 0) sc.wants[e >> 6] = bits;
    }
    int in_block;
    upto = wanted + block_sum(mine.want ? 1 : 0, s_sum, &in_block);
    if (e < n_entries) {
      if (e == s_start[mine.row]) s_base[mine.row] = upto - mine.want;
      if (e + 1 == s_start[mine.row + 1]) s_cum[mine.row] = upto;
    }
    wanted += in_block;
  }
  // ---- the lowest free pages (the first block of counts has been on its way since the start)
  int found = 0;
  for (int p0 = 0; p0 < l.n_pages && found < wanted; p0 += 4096) {
    const int p = p0 + 4 * t;
    int free4 = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (p + i < l.n_pages && (p0 ? l.refs[p + i] : lowest[i]) == 0) free4 |= 1 << i;
    int in_block;
    int k = found + block_sum(__popc(free4), s_sum, &in_block) - __popc(free4);
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (free4 >> i & 1) {
        if (k < kReserveRows) s_free[k] = p + i;
        else if (k < wanted) sc.free_ids[k] = p + i;
        ++k;
      }
    found += in_block;
  }
  const bool stuck_before = row0 > 0 && *sc.stuck;
  __threadfence_block();
  __syncthreads();   // the words of `wants` and `free_ids` are there; the counts have been read
  if (t == 0) *sc.stuck = stuck_before || wanted > found;
  if (stuck_before) found = 0;

  // ---- taking them
  auto take = [&](const Entry& x, int k) {
    if (!x.want || s_cum[x.row] > found) return;
    const int page = k < kReserveRows ? s_free[k] : sc.free_ids[k];
    *x.at = page;
    if (x.at == l.table + (size_t)(row0 + x.row) * l.mpps + s_first[x.row]) s_new[x.row] = page;
    atomicAdd(l.refs + page, 1);
    if (page_in(l, x.old)) atomicSub(l.refs + x.old, 1);
  };
  if (n_entries <= 1024) {
    take(mine, upto - 1);
  } else {
    int given = 0;
    for (int e0 = 0; e0 < n_entries; e0 += 1024) {
      const int e = e0 + t;
      Entry x{nullptr, 0, -1, false};
      if (e < n_entries) {
        x.want = sc.wants[e >> 6] >> (e & 63) & 1;
        x.row = row_of(e);
        x.at = l.table + (size_t)(row0 + x.row) * l.mpps + s_first[x.row] + (e - s_start[x.row]);
        if (x.want) x.old = *x.at;
      }
      int in_block;
      const int k = given + block_sum(x.want ? 1 : 0, s_sum, &in_block) - 1;
      given += in_block;
      take(x, k);
    }
  }
  // the counts' atomics are done, in the L2 of this workgroup's XCD, before anybody looks at them again there (a device-wide fence would write that L2 back)
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  if (t >= n) return;
  const bool fits = s_cum[t] <= found;
  const int in_page = len % DF_PAGE;
  int4 copy = make_int4(-1, 0, 0, 0);
  bool ok = !refused;
  if (count > 0) {
    if (shared && fits && in_page > 0) copy = make_int4(id, s_new[t], (in_page + 3) & ~3, 0);
    // a row that takes nothing may still share its page with one that got no copy
    ok = s_cum[t] > s_base[t] ? fits : agent_load(l.refs + id) == 1;
  }
  sc.copies[t] = copy;
  if (granted) granted[row] = ok;
  if (!ok) atomicOr(l.status, DF_STATUS_CAPACITY);
}

// ---- copies ------------------------------------------------------------------------------------------------------------
// What a page is in both pools: layer l of the target is block l, layer l of the draft block n_layers + l.  Sizes in 16-byte units.
struct PageBlocks {
  u32x4 *target, *draft;
  int target_layers, layers;          // of the target, of both
  int target_units, draft_units;      // of a page in one layer
  int target_part, draft_part;        // of a K or V part (16 keys of one head)
  int n_pages, key_units;             // units of 8 dims of a key: 1 (bf16) or 2 (fp32)
};
struct PageBlock {
  u32x4* base;
  int units, part;
};
__device__ __forceinline__ PageBlock page_block(const PageBlocks& b, int layer) {
  if (layer < b.target_layers) return {b.target + (size_t)layer * b.n_pages * b.target_units, b.target_units, b.target_part};
  return {b.draft + (size_t)(layer - b.target_layers) * b.n_pages * b.draft_units, b.draft_units, b.draft_part};
}

// The first ROWS rows of a page: of every 8 dims of K the first ROWS keys, of every 16 dims of V the first ROWS / 4 quartets of keys.  Either is the
// first ROWS of 16 parts of a run of KU * 16 (K) or KU * 32 (V) units.
template <int ROWS, int KU>
__device__ __forceinline__ void copy_rows(u32x4* __restrict__ to, const u32x4* __restrict__ from, int units, int part) {
  constexpr int KR = KU * ROWS, VR = 2 * KU * ROWS;    // units copied of a run
  const int live = units / 16 * ROWS, live_part = part / 16 * ROWS;
  auto at = [&](int i) {
    const int p = i / live_part, k = i - p * live_part;
    return p * part + (p & 1 ? k / VR * (32 * KU) + k % VR : k / KR * (16 * KU) + k % KR);
  };
  for (int i = threadIdx.x; i < live; i += 4 * 256) {
    u32x4 v[4];
    int o[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      o[u] = at(min(i + 256 * u, live - 1));
      v[u] = from[o[u]];
    }
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (i + 256 * u < live) to[o[u]] = v[u];
  }
}
template <int KU>
__device__ __forceinline__ void copy_page_rows(u32x4* to, const u32x4* from, int units, int part, int rows) {
  if (rows == 4) copy_rows<4, KU>(to, from, units, part);
  else if (rows == 8) copy_rows<8, KU>(to, from, units, part);
  else if (rows == 12) copy_rows<12, KU>(to, from, units, part);
  else copy_rows<16, KU>(to, from, units, part);
}

// The copies of a plan: grid (layers, rows of the plan).
__global__ __launch_bounds__(256) void pages_copy_kernel(PageBlocks b, const int4* __restrict__ copies) {
  const int4 c = copies[blockIdx.y];
  if (c.x < 0) return;
  const PageBlock pb = page_block(b, blockIdx.x);
  u32x4* to = pb.base + (size_t)c.y * pb.units;
  const u32x4* from = pb.base + (size_t)c.x * pb.units;
  if (b.key_units == 1) copy_page_rows<1>(to, from, pb.units, pb.part, c.z);
  else copy_page_rows<2>(to, from, pb.units, pb.part, c.z);
}

// ---- compaction --------------------------------------------------------------------------------------------------------
struct CompactScratch {
  int32_t* head;    // pages in use, pages to move
  int2* moves;      // [n_pages / 2 + 1] from, to
  int32_t* to;      // [n_pages] where the pages behind the first head[0] ids go
  int32_t *src, *dst;   // [n_pages / 2 + 1] each
};

// One workgroup: with L pages in use, the k-th of them behind the ids below L goes to the k-th free page below L.
__global__ __launch_bounds__(1024) void pages_compact_kernel(Ledger l, CompactScratch sc, int32_t* __restrict__ n_live) {
  __shared__ int s_sum[17];
  const int t = threadIdx.x;
  int mine = 0, live;
  for (int p = t; p < l.n_pages; p += 1024) mine += l.refs[p] > 0;
  block_sum(mine, s_sum, &live);
  int moves = 0, holes = 0;
  for (int p0 = 0; p0 < l.n_pages; p0 += 1024) {
    const int p = p0 + t;
    const bool in = p < l.n_pages, used = in && l.refs[p] > 0;
    const bool move = used && p >= live, hole = in && !used && p < live;
    if (in && p >= live) sc.to[p] = p;
    int m, h;   // a block of ids lies on one side of L, but for one
    const int km = moves + block_sum(move, s_sum, &m) - 1, kh = holes + block_sum(hole, s_sum, &h) - 1;
    if (move) sc.src[km] = p;
    if (hole) sc.dst[kh] = p;
    moves += m;
    holes += h;
  }
  __threadfence_block();
  __syncthreads();
  for (int k = t; k < moves; k += 1024) {
    const int from = sc.src[k], to = sc.dst[k];
    sc.moves[k] = make_int2(from, to);
    sc.to[from] = to;
    l.refs[to] = l.refs[from];
    l.refs[from] = 0;
  }
  if (t == 0) {
    sc.head[0] = live;
    sc.head[1] = moves;
    if (n_live) *n_live = live;
  }
}

// The block table follows its pages (every workgroup a share), and the pages move: a workgroup takes a page of a layer at a time.
__global__ __launch_bounds__(256) void pages_move_kernel(Ledger l, PageBlocks b, CompactScratch sc) {
  const int live = sc.head[0], n = sc.head[1] * b.layers;
  const size_t entries = (size_t)l.n_rows * l.mpps;
  for (size_t e = (size_t)blockIdx.x * 256 + threadIdx.x; e < entries; e += (size_t)gridDim.x * 256) {
    const int id = l.table[e];
    if (id >= live && id < l.n_pages) l.table[e] = sc.to[id];
  }
  for (int i = blockIdx.x; i < n; i += gridDim.x) {
    const int2 m = sc.moves[i / b.layers];
    const PageBlock pb = page_block(b, i % b.layers);
    u32x4* to = pb.base + (size_t)m.y * pb.units;
    const u32x4* from = pb.base + (size_t)m.x * pb.units;
    for (int u = threadIdx.x; u < pb.units; u += 4 * 256) {
      u32x4 v[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) v[k] = from[min(u + 256 * k, pb.units - 1)];
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (u + 256 * k < pb.units) to[u + 256 * k] = v[k];
    }
  }
}
