// Pages of the cache: handed out, shared, copied, freed and moved.
//
// The bookkeeping (page tables, counts) is a few thousand integers, so one
// workgroup does it, in fixed order: the page ids it hands out depend on
// nothing but the tables.  The page data are moved by a second launch over
// the whole device, which reads the pairs and their number from memory.
// Bookkeeping is a chain of barriers and round trips (8 to 11 us for 32
// sequences over 700 pages), the copy runs at a large copy's rate.
#include "cache.h"

namespace dmoe {

namespace {

constexpr int kThreads = 512;
constexpr int kMaxSlots = 65536;
// Updates of up to this many entries over pools of up to this many pages keep
// entries and counts in LDS: an atomic there takes no trip to L2 (32 sequences
// over 700 pages: 20 us with both in memory, 8 to 11 us so).
constexpr int kLdsPages = 8192;
constexpr int kLdsEntries = 256;

// The pages' counts while an update changes them.
template <bool kLds>
struct Counts {
  int32_t* at;  // LDS, or the cache's own
  __device__ __forceinline__ int get(int p) const {
    // memory: atomics act in L2, so they are read past L1
    if constexpr (kLds) return at[p];
    return __hip_atomic_load(at + p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  __device__ __forceinline__ void add(int p, int d) const { atomicAdd(at + p, d); }
  __device__ __forceinline__ void set(int p, int v) const {
    if constexpr (kLds)
      at[p] = v;
    else
      __hip_atomic_store(at + p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  __device__ __forceinline__ void lower(int p, int v) const { atomicMin(at + p, v); }
  // what all threads did before is seen by all after
  __device__ __forceinline__ static void sync() {
    if constexpr (!kLds) __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0): stores and atomics have acted
    __syncthreads();
  }
};

// Page pairs to copy, in a workspace: their number, then from and to.
struct PairList {
  const int32_t* n;     // nullptr: all of `most`
  const int32_t* from;  // pair i: from[i * step], to[i * step]
  const int32_t* to;
  int step, most;
};

// What an update keeps of every entry between its phases.
struct Entry {
  int dst, src, keep, len;
  int full, count, had;  // shared pages; pages after and before the call
  int part;              // page kept in part, or -1
  int mine;              // the part stays where it is
  int fresh;             // first of its pages in the list of free ones
  int pad[2];
};

template <bool kLds>
__global__ __launch_bounds__(kThreads) void update_kernel(dmoe_cache c, const int32_t* dst, const int32_t* src, const int32_t* keep,
                                                          const int32_t* new_lens, int n, int32_t* status, int32_t* n_pairs,
                                                          Entry* entries_ws, int32_t* from, int32_t* to, int32_t* rows,
                                                          int32_t* free_list) {
  extern __shared__ int32_t lds_counts[];
  __shared__ Entry lds_entries[kLds ? kLdsEntries : 1];
  Entry* const entries = kLds ? lds_entries : entries_ws;
  __shared__ uint32_t seen[kMaxSlots / 32];
  __shared__ int waves[kThreads / 64];
  __shared__ int bad;
  const int tid = threadIdx.x, mp = c.max_pages, pt = c.page_tokens;
  const Counts<kLds> counts{kLds ? lds_counts : c.refs};
  if constexpr (kLds) {
    for (int p = tid; p < c.n_pages; p += kThreads) lds_counts[p] = c.refs[p];
  }
  auto pages = [&](int tokens) { return (tokens + pt - 1) / pt; };
  auto leave = [&](int outcome) {
    for (int i = tid; i < n && c.refused; i += kThreads)
      if (const int d = dst[i]; d >= 0 && d < c.n_slots) c.refused[d] = outcome;
    if (tid == 0 && status) *status = outcome;
  };
  for (int i = tid; i < (c.n_slots + 31) / 32; i += kThreads) seen[i] = 0;
  if (tid == 0) {
    bad = 0;
    *n_pairs = 0;
  }
  __syncthreads();
  bool ok = true;
  for (int i = tid; i < n; i += kThreads) {
    Entry e{};
    e.dst = dst[i];
    e.src = src ? src[i] : e.dst;
    e.len = new_lens[i];
    const bool in = e.dst >= 0 && e.dst < c.n_slots && e.src >= 0 && e.src < c.n_slots && e.len >= 0 && e.len <= mp * pt;
    ok = ok && in;
    if (in) {
      ok = ok && !(atomicOr(&seen[e.dst / 32], 1u << (e.dst % 32)) >> (e.dst % 32) & 1);
      const int held = c.lens[e.src], old = c.lens[e.dst];
      e.keep = keep ? keep[i] : min(held, e.len);
      ok = ok && held >= 0 && held <= mp * pt && old >= 0 && old <= mp * pt && e.keep >= 0 && e.keep <= min(held, e.len);
      if (ok) {
        e.full = e.keep / pt;
        e.count = pages(e.len);
        e.had = pages(old);
        e.part = -1;
        entries[i] = e;
      }
    }
  }
  if (!ok) atomicOr(&bad, 1);
  __syncthreads();
  if (bad) {
    leave(-1);
    return;
  }
  // the pages kept, as the tables stand
  const uint32_t cells = static_cast<uint32_t>(n) * mp;  // under 2^31
  for (uint32_t x = tid; x < cells; x += kThreads) {
    const int i = x / mp, j = x - i * mp;
    const Entry& e = entries[i];
    if (j < pages(e.keep)) {
      const int p = c.table[static_cast<long>(e.src) * mp + j];
      ok = ok && p >= 0 && p < c.n_pages;
      rows[x] = p;
    }
    if (j < e.had) {
      const int p = c.table[static_cast<long>(e.dst) * mp + j];
      ok = ok && p >= 0 && p < c.n_pages;
    }
  }
  if (!ok) atomicOr(&bad, 1);
  __syncthreads();
  if (bad) {
    leave(-1);
    return;
  }
  auto count_shared = [&](int sign) {
    for (uint32_t x = tid; x < cells; x += kThreads) {
      const int i = x / mp, j = x - i * mp;
      const Entry& e = entries[i];
      if (j < e.full) counts.add(rows[x], sign);
      if (j < e.had) counts.add(c.table[static_cast<long>(e.dst) * mp + j], -sign);
    }
  };
  count_shared(1);
  for (int i = tid; i < n; i += kThreads) {
    Entry& e = entries[i];
    if (e.keep % pt) e.part = rows[static_cast<uint32_t>(i) * mp + e.full];
  }
  counts.sync();
  // a part that nobody holds any more stays with the first entry that had it:
  // the entries that may keep it lower its count to their number less n
  for (int i = tid; i < n; i += kThreads) {
    Entry& e = entries[i];
    e.mine = e.part >= 0 && e.src == e.dst && counts.get(e.part) <= 0;
    if (e.mine) counts.lower(e.part, i - n);
  }
  counts.sync();
  for (int i = tid; i < n; i += kThreads) {
    Entry& e = entries[i];
    if (e.mine) e.mine = counts.get(e.part) == i - n;
  }
  counts.sync();
  for (int i = tid; i < n; i += kThreads)
    if (entries[i].mine) counts.set(entries[i].part, 0);
  counts.sync();
  // parts that stay are held by their entry, the others until they are copied
  for (int i = tid; i < n; i += kThreads)
    if (entries[i].part >= 0) counts.add(entries[i].part, 1);
  counts.sync();
  int need = 0, copies = 0;
  for (int i0 = 0; i0 < n; i0 += kThreads) {
    const int i = i0 + tid;
    int fresh = 0, copied = 0;
    if (i < n) {
      const Entry& e = entries[i];
      copied = e.part >= 0 && !e.mine;
      fresh = e.count - e.full - (e.part >= 0) + copied;
    }
    int total, ctotal;
    const int at = scan_exclusive<kThreads>(fresh, waves, &total);
    const int cat = scan_exclusive<kThreads>(copied, waves, &ctotal);
    if (i < n) {
      entries[i].fresh = need + at;
      if (copied) {
        from[copies + cat] = entries[i].part;
        to[copies + cat] = need + at;  // of the free list, below
      }
    }
    need += total;
    copies += ctotal;
  }
  // free pages, lowest first: a stretch of the counts per thread
  const int stretch = (c.n_pages + kThreads - 1) / kThreads;
  const int q0 = min(tid * stretch, c.n_pages), q1 = min(q0 + stretch, c.n_pages);
  int zeros = 0;
  for (int p = q0; p < q1; ++p) zeros += counts.get(p) == 0;
  int total;
  int at = scan_exclusive<kThreads>(zeros, waves, &total);
  if (need > total) {  // as it was
    if constexpr (!kLds) {
      count_shared(-1);
      for (int i = tid; i < n; i += kThreads)
        if (entries[i].part >= 0) counts.add(entries[i].part, -1);
    }
    leave(need - total);
    return;
  }
  for (int p = q0; p < q1 && at < need; ++p)
    if (counts.get(p) == 0) free_list[at++] = p;
  __syncthreads();
  for (int i = tid; i < copies; i += kThreads) {
    counts.add(from[i], -1);
    to[i] = free_list[to[i]];
  }
  for (int i = tid; i < need; i += kThreads) counts.add(free_list[i], 1);
  for (uint32_t x = tid; x < cells; x += kThreads) {
    const int i = x / mp, j = x - i * mp;
    const Entry& e = entries[i];
    if (j >= max(e.count, e.had)) continue;
    int p = -1;
    if (j < e.full || (e.mine && j == e.full))
      p = rows[x];
    else if (j < e.count)
      p = free_list[e.fresh + j - e.full - e.mine];
    c.table[static_cast<long>(e.dst) * mp + j] = p;
  }
  for (int i = tid; i < n; i += kThreads) c.lens[entries[i].dst] = entries[i].len;
  if (tid == 0) *n_pairs = copies;
  leave(0);
  if constexpr (kLds) {
    __syncthreads();
    for (int p = tid; p < c.n_pages; p += kThreads) c.refs[p] = lds_counts[p];
  }
}

// Live pages from n_live on move into the holes below it, lowest to lowest.
__global__ __launch_bounds__(kThreads) void compact_kernel(dmoe_cache c, int32_t* refs_out, int32_t* counts, int32_t* n_pairs,
                                                           int32_t* from, int32_t* to, int32_t* moved) {
  __shared__ int waves[kThreads / 64];
  const int tid = threadIdx.x, n = c.n_pages;
  const int stretch = (n + kThreads - 1) / kThreads;
  const int q0 = min(tid * stretch, n), q1 = min(q0 + stretch, n);
  int live = 0;
  for (int p = q0; p < q1; ++p) live += c.refs[p] > 0;
  int n_live;
  scan_exclusive<kThreads>(live, waves, &n_live);
  int holes = 0, movers = 0;
  for (int p = q0; p < q1; ++p) {
    const bool used = c.refs[p] > 0;
    holes += !used && p < n_live;
    movers += used && p >= n_live;
  }
  int n_holes, n_movers;  // equal
  int h = scan_exclusive<kThreads>(holes, waves, &n_holes);
  int m = scan_exclusive<kThreads>(movers, waves, &n_movers);
  for (int p = q0; p < q1; ++p) {
    const bool used = c.refs[p] > 0;
    if (!used && p < n_live) to[h++] = p;
    if (used && p >= n_live) from[m++] = p;
    moved[p] = p;
  }
  __syncthreads();
  for (int i = tid; i < n_movers; i += kThreads) moved[from[i]] = to[i];
  // refs_out may be refs: holes take their movers' counts before those go
  for (int p = q0; p < min(q1, n_live); ++p) {
    const int r = c.refs[p];
    if (r > 0) refs_out[p] = r;
  }
  for (int i = tid; i < n_movers; i += kThreads) refs_out[to[i]] = c.refs[from[i]];
  __syncthreads();
  for (int p = max(q0, n_live); p < q1; ++p) refs_out[p] = 0;
  if (tid == 0) {
    *n_pairs = n_movers;
    if (counts) {
      counts[0] = n_live;
      counts[1] = n_movers;
    }
  }
}

constexpr int kCopyThreads = 256;
constexpr int kUnroll = 4;
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
constexpr long kUnit = kCopyThreads * kUnroll;  // 16-byte pieces of a unit: 16 KiB
constexpr unsigned kCopyGrid = 4096;

// Units of 16 KiB: (pair, layer, keys or values, part of the page).  With
// `moved`, the table is rewritten too.  Non-temporal both ways: 586 MB of a
// compaction in 122 us against 130 through the caches (4.8 TB/s, the rate of a
// large copy).
__global__ __launch_bounds__(kCopyThreads) void copy_kernel(dmoe_cache c, PairList l, long page_len, const int32_t* moved,
                                                            int32_t* table_out) {
  const long gtid = static_cast<long>(blockIdx.x) * kCopyThreads + threadIdx.x;
  if (moved) {
    const long cells = static_cast<long>(c.n_slots) * c.max_pages;
    for (long x = gtid; x < cells; x += static_cast<long>(gridDim.x) * kCopyThreads) {
      const int p = c.table[x];
      table_out[x] = p >= 0 && p < c.n_pages ? moved[p] : p;
    }
  }
  const int n = l.n ? min(*l.n, l.most) : l.most;
  const long per_page = (page_len + kUnit - 1) / kUnit;
  const long units = n * static_cast<long>(c.n_layers) * 2 * per_page;
  for (long u = blockIdx.x; u < units; u += gridDim.x) {
    const long part = u % per_page, rest = u / per_page;
    const int kv = static_cast<int>(rest % 2), layer = static_cast<int>(rest / 2 % c.n_layers), i = static_cast<int>(rest / 2 / c.n_layers);
    const int a = l.from[static_cast<long>(i) * l.step], b = l.to[static_cast<long>(i) * l.step];
    if (a < 0 || a >= c.n_pages || b < 0 || b >= c.n_pages) continue;
    uint4* pool = static_cast<uint4*>(kv ? c.v : c.k) + static_cast<long>(layer) * c.n_pages * page_len;
    const u32x4* s = (const u32x4*)pool + a * page_len + part * kUnit;
    u32x4* d = (u32x4*)pool + b * page_len + part * kUnit;
    const long len = min(kUnit, page_len - part * kUnit);
    u32x4 x[kUnroll];
#pragma unroll
    for (int j = 0; j < kUnroll; ++j)
      if (threadIdx.x + j * kCopyThreads < len) x[j] = __builtin_nontemporal_load(s + threadIdx.x + j * kCopyThreads);
#pragma unroll
    for (int j = 0; j < kUnroll; ++j)
      if (threadIdx.x + j * kCopyThreads < len) __builtin_nontemporal_store(x[j], d + threadIdx.x + j * kCopyThreads);
  }
}

hipError_t copy_pages(const dmoe_cache& c, const PairList& l, const int32_t* moved, int32_t* table_out, hipStream_t s) {
  const long page_len = page_elems(c.page_tokens, c.n_kv_heads, c.head_dim) * static_cast<long>(dtype_bytes(c.dt)) / 16;
  const long units = l.most * static_cast<long>(c.n_layers) * 2 * ((page_len + kUnit - 1) / kUnit);
  const unsigned grid = units < static_cast<long>(kCopyGrid) ? static_cast<unsigned>(units) : kCopyGrid;
  copy_kernel<<<grid, kCopyThreads, 0, s>>>(c, l, page_len, moved, table_out);
  return hipGetLastError();
}

size_t align16(size_t b) { return (b + 15) & ~static_cast<size_t>(15); }

}  // namespace

// Workspace: pairs' number | entries | from | to | rows | free list.
size_t update_workspace_bytes(long n, long max_pages, long n_pages) {
  const long most = n * max_pages < n_pages ? n * max_pages : n_pages;  // pages handed out
  return 16 + align16(n * sizeof(Entry)) + 2 * align16(n * 4) + align16(n * max_pages * 4) + align16(most * 4);
}

hipError_t launch_update(const dmoe_cache& c, const int32_t* dst, const int32_t* src, const int32_t* keep,
                         const int32_t* new_lens, int n, int32_t* status, void* ws, hipStream_t s) {
  char* at = static_cast<char*>(ws);
  auto take = [&](size_t bytes) {
    char* p = at;
    at += align16(bytes);
    return reinterpret_cast<int32_t*>(p);
  };
  int32_t* n_pairs = take(16);
  Entry* entries = reinterpret_cast<Entry*>(take(n * sizeof(Entry)));
  int32_t* from = take(n * 4l);
  int32_t* to = take(n * 4l);
  int32_t* rows = take(static_cast<long>(n) * c.max_pages * 4);
  int32_t* free_list = take(0);
  if (c.n_pages <= kLdsPages && n <= kLdsEntries)
    update_kernel<true><<<1, kThreads, c.n_pages * 4l, s>>>(c, dst, src, keep, new_lens, n, status, n_pairs, entries, from, to,
                                                            rows, free_list);
  else
    update_kernel<false><<<1, kThreads, 0, s>>>(c, dst, src, keep, new_lens, n, status, n_pairs, entries, from, to, rows, free_list);
  hipError_t err = hipGetLastError();
  if (err != hipSuccess) return err;
  return copy_pages(c, PairList{n_pairs, from, to, 1, n}, nullptr, nullptr, s);
}

// Workspace: pairs' number | from | to | moved.
size_t compact_workspace_bytes(long n_pages) { return 16 + 3 * align16(n_pages * 4); }

hipError_t launch_compact(const dmoe_cache& c, int32_t* table_out, int32_t* refs_out, int32_t* counts, void* ws,
                          hipStream_t s) {
  int32_t* n_pairs = static_cast<int32_t*>(ws);
  const size_t step = align16(c.n_pages * 4l) / 4;
  int32_t* from = n_pairs + 4;
  int32_t* to = from + step;
  int32_t* moved = to + step;
  compact_kernel<<<1, kThreads, 0, s>>>(c, refs_out, counts, n_pairs, from, to, moved);
  hipError_t err = hipGetLastError();
  if (err != hipSuccess) return err;
  return copy_pages(c, PairList{n_pairs, from, to, 1, c.n_pages}, moved, table_out, s);
}

hipError_t launch_copy_pages(const dmoe_cache& c, const int32_t* pairs, int n, hipStream_t s) {
  return copy_pages(c, PairList{nullptr, pairs, pairs + 1, 2, n}, nullptr, nullptr, s);
}

}  // namespace dmoe
