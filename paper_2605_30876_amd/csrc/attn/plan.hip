// The attention's work items, made on the device: a step's lengths never
// visit the host, and every layer of the step uses the one plan.  One
// workgroup: prefix sums over sequences and row tiles, then an item per thread.
// 5.4 us for one sequence, 6.6 for 64: half of it the launch, the rest three
// round trips (offsets and slots, lengths, page ids) and the barriers; 1024
// threads took 2.7 more.
#include "cache.h"

namespace dmoe {

namespace {

constexpr int kThreads = 256;
constexpr int kMaxSeqs = 4096;
constexpr int kKeptSeqs = 512;  // sequences kept in LDS; further ones are read again
// Items that splitting aims at, all kv heads together, and their key tiles at least.
constexpr int kSplitRows = 512;   // items of 32 rows
constexpr int kSplitBlock = 512;  // items of 128 rows: as many workgroups as the device holds at once
constexpr int kMinRows = 8;   // two a wave
constexpr int kMinTwo = 6;    // 64 rows: three a wave
constexpr int kMinBlock = 4;
constexpr int kMinWide = 8;
// Pieces that even out row tiles of 128, key tiles: long enough not to notice their partial results.
constexpr int kEvenBf16 = 48;
constexpr int kEvenF32 = 16;
constexpr long kFewTiles = 16, kFewKeys = 2048;

// Largest i with a[i] <= x, for a[0] = 0 <= x < a[n].
__device__ __forceinline__ int find(const int* a, int n, int x) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (a[mid] <= x)
      lo = mid;
    else
      hi = mid;
  }
  return lo;
}

// A row tile's sequence and its key tiles.
struct Tile {
  Seq q;
  int first, rows, kt;
};

__global__ __launch_bounds__(kThreads) void plan_kernel(dmoe_cache c, dmoe_batch b, AttnShape sh, int mask_block, int32_t* plan) {
  __shared__ int tiles[kMaxSeqs + 1];  // row tiles before each sequence
  __shared__ Seq seqs[kKeptSeqs];
  __shared__ Tile tile[kThreads];
  __shared__ int items[kThreads + 1];  // items before each row tile of a pass
  __shared__ int parts[kThreads];
  __shared__ int iwaves[kThreads / 64];
  __shared__ long lwaves[kThreads / 64];
  __shared__ int longest;  // key tiles of a row tile at most
  const int tid = threadIdx.x;
  if (tid == 0) longest = 0;
  int n_tiles = 0;
  for (int i0 = 0; i0 < b.n_seqs; i0 += kThreads) {
    const int i = i0 + tid;
    int n = 0;
    if (i < b.n_seqs) {
      const Seq q = load_seq(c, b, i);
      if (i < kKeptSeqs) seqs[i] = q;
      n = static_cast<int>((static_cast<long>(q.n) * sh.group + sh.tile_rows - 1) / sh.tile_rows);
    }
    // Offsets that are not sorted could make more row tiles than the arrays
    // hold, or an int: cut after each pass, whose own stay below 2^31 (rises
    // of at most 2^30 rows, 128 to a tile, between at most 128 falls).
    int total;
    const int at = scan_exclusive<kThreads>(n, iwaves, &total), most_tiles = static_cast<int>(sh.max_tiles);
    if (i < b.n_seqs) tiles[i] = min(n_tiles + at, most_tiles);
    n_tiles = min(n_tiles + total, most_tiles);
  }
  if (tid == 0) tiles[b.n_seqs] = n_tiles;
  __syncthreads();
  // longest rows first under a causal mask: the last tiles see the most keys
  auto load_tile = [&](int t) {
    Tile r{};
    if (t >= n_tiles) return r;
    t = n_tiles - 1 - t;
    const int i = find(tiles, b.n_seqs, t);
    r.q = i < kKeptSeqs ? seqs[i] : load_seq(c, b, i);
    r.rows = r.q.n * sh.group;
    r.first = (t - tiles[i]) * sh.tile_rows;
    const int last = min(r.first + sh.tile_rows, r.rows) - 1;
    r.kt = (visible_end(r.q.pos0 + last / sh.group, r.q.len, mask_block) + kTileTokens - 1) / kTileTokens;
    return r;
  };
  Tile r = load_tile(tid);
  long keys = r.kt;
  int most = r.kt;
  for (int t = tid + kThreads; t < n_tiles; t += kThreads) {
    const int kt = load_tile(t).kt;
    keys += kt;
    most = max(most, kt);
  }
  const long split = sh.aim;
  const bool many = n_tiles > split / 2;
  if (sh.tile_rows == 128 && many) {
#pragma unroll
    for (int d = 32; d >= 1; d /= 2) most = max(most, __shfl_xor(most, d));
    if ((tid & 63) == 0) atomicMax(&longest, most);
  }
  long all;
  scan_exclusive<kThreads>(keys, lwaves, &all);
  // Pieces of `chunk` key tiles: sum ceil(kt / chunk) <= n_tiles + all / chunk,
  // and all / chunk <= split_items, which the arrays' sizes count on.
  // Items of 128 rows leave partial results of 64 KiB: they fill one round of
  // workgroups but do not pass it, and row tiles of about one length that are more
  // than half of the aim are not split.  Of uneven lengths they are, into two
  // rounds, in pieces that are long beside their partial results: 60 blocks of up
  // to 16k, 12 query and 3 kv heads of 32: 93 -> 67 us; 48 of up to 8k, 64 and 8 of 128: 285 -> 245;
  // fp32, 73 of 24 tokens of up to 5k, 10 and 2 of 96: 240 -> 196.  With fewer row tiles it costs
  // more than it evens out: 32 blocks of up to 16k, 16 and 4 of 128: 66 -> 74.
  // Items of 32 rows are cheap to join: pieces of the average length even the
  // sequences out, of half of it where there are many sequences (64 of up to 16k tokens:
  // 191 -> 181 us).
  const long room = sh.tile_rows <= 64 ? (many && sh.tile_rows == 32 ? sh.split_items : split) : max(max(split - n_tiles, split / 2), 1l);
  long len = max(static_cast<long>(sh.min_tiles), (all + room - 1) / room);
  if (sh.tile_rows == 128 && many && 10l * longest * n_tiles > 13 * all)
    len = min(len, max(static_cast<long>(sh.even_tiles), (all + 2 * split - 1) / (2 * split)));
  const int chunk = static_cast<int>(len);

  AttnPlanHead* head = reinterpret_cast<AttnPlanHead*>(plan);
  AttnItem* out = reinterpret_cast<AttnItem*>(head + 1);
  AttnMerge* merges = reinterpret_cast<AttnMerge*>(out + sh.max_items());
  int n_items = 0, n_parts = 0, n_merges = 0;
  for (int t0 = 0; t0 < n_tiles; t0 += kThreads) {
    if (t0 > 0) r = load_tile(t0 + tid);
    const int pieces = t0 + tid < n_tiles ? max(1, (r.kt + chunk - 1) / chunk) : 0;
    tile[tid] = r;
    // three sums at once, 21 bits each: a pass has at most kThreads + split items
    const long mine = pieces | (pieces > 1 ? static_cast<long>(pieces) << 21 | 1l << 42 : 0);
    long sum;
    const long at = scan_exclusive<kThreads>(mine, lwaves, &sum);
    constexpr long kBits = (1 << 21) - 1;
    const int total = static_cast<int>(sum & kBits);
    const int part = n_parts + static_cast<int>(at >> 21 & kBits);
    items[tid] = static_cast<int>(at & kBits);
    parts[tid] = pieces > 1 ? part : -1;
    if (pieces > 1) merges[n_merges + (at >> 42)] = AttnMerge{r.q.row0, r.first, r.rows, part, pieces, {0, 0, 0}};
    if (tid == 0) items[kThreads] = total;
    __syncthreads();
    for (int x = tid; x < total; x += kThreads) {
      const int j = find(items, kThreads, x);
      const Tile& u = tile[j];
      const int p = x - items[j], n = max(1, (u.kt + chunk - 1) / chunk);
      AttnItem it{u.q.slot, u.q.row0, u.q.n, u.q.len, u.first, u.rows, 0, 0, parts[j] < 0 ? -1 : parts[j] + p, {}, 0};
      const long units = (u.kt + sh.unit - 1) / sh.unit;
      it.kt0 = static_cast<int>(units * p / n) * sh.unit;
      it.kt1 = min(static_cast<int>(units * (p + 1) / n) * sh.unit, u.kt);
      const int mid = item_middle(it.kt0, it.kt1);
#pragma unroll
      for (int i = 0; i < 6; ++i) {
        const int kt = i < 4 ? it.kt0 + i : mid + i - 4;
        it.page[i] = kt < it.kt1 ? c.table[static_cast<long>(u.q.slot) * c.max_pages + kt * kTileTokens / c.page_tokens] : -1;
      }
      out[n_items + x] = it;
    }
    n_items += total;
    n_parts += static_cast<int>(sum >> 21 & kBits);
    n_merges += static_cast<int>(sum >> 42);
    __syncthreads();
  }
  if (tid == 0) {
    head->n_items = n_items;
    head->n_merges = n_merges;
  }
}

}  // namespace

namespace {

long most_rows(int T, int max_new, int group) { return static_cast<long>(max_new < T ? max_new : T) * group; }

AttnShape shape_of(int tile_rows, int n_seqs, int T, int max_new, int n_heads, int n_kv_heads) {
  AttnShape s;
  s.group = n_heads / n_kv_heads;
  s.tile_rows = tile_rows;
  const long by_seq = n_seqs * ((most_rows(T, max_new, s.group) + tile_rows - 1) / tile_rows);
  const long by_rows = static_cast<long>(T) * s.group / tile_rows + n_seqs;
  s.max_tiles = by_seq < by_rows ? by_seq : by_rows;
  const int aim = (tile_rows <= 64 ? kSplitRows : kSplitBlock) / n_kv_heads;
  s.aim = aim > 1 ? aim : 1;
  // twice the aim where the plan may go for it: always with 32 rows, with 128 where it may find many row tiles
  s.split_items = tile_rows == 32 || (tile_rows == 128 && s.max_tiles > s.aim / 2) ? 2 * s.aim : s.aim;
  s.min_tiles = tile_rows == 32 ? kMinRows : tile_rows == 64 ? kMinTwo : kMinBlock;
  s.even_tiles = 0;
  s.wide = false;
  s.unit = 1;
  return s;
}

}  // namespace

AttnShape attn_shape(const dmoe_cache& c, const dmoe_batch& b, int n_heads) {
  const long most = most_rows(b.T, b.max_new, n_heads / c.n_kv_heads);
  auto shape = [&](int rows) { return shape_of(rows, b.n_seqs, b.T, b.max_new, n_heads, c.n_kv_heads); };
  if (most <= 32) return shape(32);
  // More than 64 rows a sequence: 128 to a workgroup read the cache once where
  // 64 read it twice, but a workgroup of 64 starts sooner and there are twice as
  // many.  64 where little is read: under kFewTiles row tiles of all kv heads, or kFewKeys
  // (row tile, key tile) pairs at the sequences' longest.  A step of one sequence,
  // 128 rows of four kv heads: 12.5 against 16.7 us a layer at 400 tokens, 17.1 against 18.9 at 4096, 26.7
  // against 25.3 at 16000; of eight: 16.4 against 19.1 at 400, 31.8 against 30.2 at 4096.
  const AttnShape two = shape(64);
  const long tiles = two.max_tiles * c.n_kv_heads, keys = static_cast<long>(c.max_pages) * c.page_tokens / kTileTokens;
  if (most <= 64 || tiles <= kFewTiles || tiles * keys <= kFewKeys) return two;
  AttnShape s = shape(128);
  // one workgroup a CU: where a wave needs more than half of a SIMD's
  // registers, and where eight waves work on an item, which they do if the
  // batch's row tiles alone do not fill the device
  const bool half = two_per_cu(c.dt, padded_dim(c.head_dim));
  s.wide = half && s.max_tiles * c.n_kv_heads < kSplitBlock / 2;
  if (!half || s.wide) s.aim = s.aim > 1 ? s.aim / 2 : 1;
  if (s.wide) s.min_tiles = kMinWide;
  s.even_tiles = c.dt == DMOE_F32 ? kEvenF32 : kEvenBf16;
  s.unit = stage_tiles(c.dt, padded_dim(c.head_dim));
  return s;
}

size_t plan_ints(int n_seqs, int T, int max_new, int n_heads, int n_kv_heads) {
  size_t n = 0;
  for (int rows : {32, 64, 128}) {
    const size_t m = plan_ints(shape_of(rows, n_seqs, T, max_new, n_heads, n_kv_heads));
    n = m > n && (rows > 32 || most_rows(T, max_new, n_heads / n_kv_heads) <= 32) ? m : n;
  }
  return n;
}

size_t attn_workspace_bytes(int n_seqs, int T, int max_new, int n_heads, int n_kv_heads, int dp) {
  const long most = most_rows(T, max_new, n_heads / n_kv_heads);
  const int rows = most <= 32 ? 32 : most <= 64 ? 64 : 128;
  return attn_workspace_bytes(shape_of(rows, n_seqs, T, max_new, n_heads, n_kv_heads), n_kv_heads, dp);
}

hipError_t launch_attention_plan(const dmoe_cache& c, const dmoe_batch& b, const AttnShape& sh, int mask_block,
                                 int32_t* plan, hipStream_t s) {
  plan_kernel<<<1, kThreads, 0, s>>>(c, b, sh, mask_block, plan);
  return hipGetLastError();
}

}  // namespace dmoe
