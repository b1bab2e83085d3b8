// The attention's work items, made on the device: a step's lengths never
// visit the host, and every layer of the step uses the one plan.  One
// workgroup: prefix sums over sequences and row tiles, then an item per thread.
// 5.4 us for one sequence, 6.6 for 64: half of it the launch, the rest three
// round trips (offsets and slots, lengths, page ids) and the barriers; 1024
// threads took 2.7 more.
#include <algorithm>

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
constexpr int kSplitWide = 256;   // items of eight waves: one a CU
// Their key tiles: one or two a wave (a block over 4096 tokens, eight layers: 118.7 us with 12, 121.5 with 10, 122.7 with 16), but
// up to kWholeEight stay with one (a block over 400: 20.0 us in two pieces, which have to be joined, 17.1 in one).
constexpr int kMinEight = 12, kWholeEight = 20;
constexpr long kFewTiles32 = 128, kFewKeys32 = 20000, kFewWork32 = 28000;
constexpr long kFewTiles16 = 64, kFewKeys16 = 256;
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
  const long room = sh.tile_rows == 32 && many   ? sh.split_items
                    : sh.tile_rows <= 64 && !sh.wide ? split
                                                     : max(max(split - n_tiles, split / 2), 1l);
  long len = max(static_cast<long>(sh.min_tiles), (all + room - 1) / room);
  if (sh.tile_rows == 128 && many && 10l * longest * n_tiles > 13 * all)
    len = min(len, max(static_cast<long>(sh.even_tiles), (all + 2 * split - 1) / (2 * split)));
  const int chunk = static_cast<int>(len);
  auto pieces_of = [&](int kt) { return kt <= sh.whole_tiles ? 1 : (kt + chunk - 1) / chunk; };

  AttnPlanHead* head = reinterpret_cast<AttnPlanHead*>(plan);
  AttnItem* out = reinterpret_cast<AttnItem*>(head + 1);
  AttnMerge* merges = reinterpret_cast<AttnMerge*>(out + sh.max_items());
  int n_items = 0, n_parts = 0, n_merges = 0;
  for (int t0 = 0; t0 < n_tiles; t0 += kThreads) {
    if (t0 > 0) r = load_tile(t0 + tid);
    const int pieces = t0 + tid < n_tiles ? pieces_of(r.kt) : 0;
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
      const int p = x - items[j], n = pieces_of(u.kt);
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
  s.whole_tiles = s.min_tiles;
  s.even_tiles = 0;
  s.wide = false;
  s.unit = 1;
  return s;
}

}  // namespace

AttnShape attn_shape(const dmoe_cache& c, const dmoe_batch& b, int n_heads) {
  const long most = most_rows(b.T, b.max_new, n_heads / c.n_kv_heads);
  auto shape = [&](int rows) { return shape_of(rows, b.n_seqs, b.T, b.max_new, n_heads, c.n_kv_heads); };
  const bool few = c.format != DMOE_KV_PLAIN;  // bits: bf16 products, whatever the rows
  if (few) {
    AttnShape s = shape(32);
    const long tiles = s.max_tiles * c.n_kv_heads, keys = static_cast<long>(c.max_pages) * c.page_tokens / kTileTokens;
    // 32 rows to eight waves start sooner than 128 to four and are split further, but read the cache four times as often: they
    // take sequences of up to 64 rows (8 query and 4 kv heads of 128, us of 32 and of 128: 64 blocks of 32 tokens of up to 8192 in 4
    // bits 65/98, in 8 bits 78/96, fp32 in 4 bits 134/223; one over 100,000 40/53), and few row tiles of all kv heads over few
    // keys, fewer where one costs more (kFewWork32: by dp and the bf16 parts of a row).  us of 32 and of 128, 4 kv heads in 4 bits over
    // 3000 tokens, 32, 64, 96 row tiles: bf16 128 elements 21.3/22.8, 23.8/28.0, 26.6/30.5; 256 elements 27.9/31.6, 32.7/35.8,
    // 38.8/41.1, 128 of them 42.6/39.9; fp32 128 elements 26.4/29.0, 32.8/35.4, 38.8/38.7, 128 of them 44.1/38.8; 256 elements
    // 48.5/53.9, 70.5/68.1, 89.5/82.7.  16 tiles over 4096 tokens in 8 bits, a layer: 14.9/18.8; 256 over up to 8192: 39/33.
    // `keys` is what the tables have room for (lengths are the device's), in these measurements hardly more than the sequences held.
    // Where there is room for far more, few rows over short sequences get the form of long ones: one block of 32 tokens in 8 bits, 16
    // and 4 heads of 128, a layer of eight, with room for just the sequence and for 131,072 tokens: over 400 10.3/12.9, 4096
    // 14.8/18.7, 16,384 20.7/30.3; two blocks over 4096 16.6/23.0, four 20.7/26.4, eight 32.4/31.8.  One token: no difference.
    // 16 rows: to four waves, or to eight, which have half of the partial results to join but start later, where row tiles are few
    // and may be long.  us of four and of eight, 4 bits, 32 and 8 heads of 128, in a graph: one token over 1000 keys 19.4/20.3, 4096
    // 20.5/20.9, 16,000 25.3/23.2, 32,000 28.5/26.3, 131,000 38.8/36.8 (not a graph); 8 over 8192 22.7/21.8, 16 32.6/33.9; 16 and 4
    // heads of 256 over 32,000 42.7/34.4.  Where eight do not fit (quant_rows_waves), four: 73.1/74.4.
    const int parts = c.dt == DMOE_F32 ? 3 : 1, dp = padded_dim(c.head_dim);
    const bool few16 = tiles <= kFewTiles16 && keys >= kFewKeys16 && quant_rows_waves(parts, dp, key_bits(c.format) + value_bits(c.format), 16) == 2;
    const long work = tiles * dp * parts;
    if (most <= 16 ? few16 : most <= 64 || (tiles <= kFewTiles32 && work <= kFewWork32 && tiles * keys <= kFewKeys32)) {
      s.wide = true;
      s.aim = kSplitWide / c.n_kv_heads > 1 ? kSplitWide / c.n_kv_heads : 1;
      s.split_items = 2 * s.aim;
      s.min_tiles = kMinEight;
      s.whole_tiles = kWholeEight;
      return s;
    }
  }
  if (most <= 32) return shape(32);
  // More than 64 rows a sequence: 128 to a workgroup read the cache once where
  // 64 read it twice, but a workgroup of 64 starts sooner and there are twice as
  // many.  64 where little is read: under kFewTiles row tiles of all kv heads, or kFewKeys
  // (row tile, key tile) pairs at the sequences' longest.  A step of one sequence,
  // 128 rows of four kv heads: 12.5 against 16.7 us a layer at 400 tokens, 17.1 against 18.9 at 4096, 26.7
  // against 25.3 at 16000; of eight: 16.4 against 19.1 at 400, 31.8 against 30.2 at 4096.
  const AttnShape two = shape(64);
  const long tiles = two.max_tiles * c.n_kv_heads, keys = static_cast<long>(c.max_pages) * c.page_tokens / kTileTokens;
  if (!few && (most <= 64 || tiles <= kFewTiles || tiles * keys <= kFewKeys)) return two;
  AttnShape s = shape(128);
  // one workgroup a CU: where a wave needs more than half of a SIMD's
  // registers, and where eight waves work on an item, which they do if the
  // batch's row tiles alone do not fill the device
  const int dp = padded_dim(c.head_dim);
  const bool half = few ? quant_two_per_cu(c.dt, dp) : two_per_cu(c.dt, dp);
  s.wide = !few && half && s.max_tiles * c.n_kv_heads < kSplitBlock / 2;
  if (!half || s.wide) s.aim = s.aim > 1 ? s.aim / 2 : 1;
  if (s.wide) s.min_tiles = s.whole_tiles = kMinWide;
  s.even_tiles = c.dt == DMOE_F32 && !few ? kEvenF32 : kEvenBf16;
  s.unit = stage_tiles(few ? DMOE_BF16 : c.dt, dp);
  return s;
}

size_t plan_ints(int n_seqs, int T, int max_new, int n_heads, int n_kv_heads) {
  size_t n = 0;
  for (int rows : {32, 64, 128}) {
    const size_t m = plan_ints(shape_of(rows, n_seqs, T, max_new, n_heads, n_kv_heads));
    n = m > n && (rows > 32 || most_rows(T, max_new, n_heads / n_kv_heads) <= 64) ? m : n;
  }
  // 32 rows to an item also where there are more of them, but few (attn_shape)
  AttnShape few = shape_of(32, n_seqs, T, max_new, n_heads, n_kv_heads);
  few.max_tiles = std::min(few.max_tiles, kFewTiles32 / n_kv_heads);
  n = plan_ints(few) > n ? plan_ints(few) : n;
  return n;
}

size_t attn_workspace_bytes(int n_seqs, int T, int max_new, int n_heads, int n_kv_heads, int dp) {
  const long most = most_rows(T, max_new, n_heads / n_kv_heads);
  // what a cache of few bits has of 32 rows where others have 64 or 128 (attn_shape) leaves no more to join
  const int rows = most <= 32 ? 32 : most <= 64 ? 64 : 128;
  return attn_workspace_bytes(shape_of(rows, n_seqs, T, max_new, n_heads, n_kv_heads), n_kv_heads, dp);
}

hipError_t launch_attention_plan(const dmoe_cache& c, const dmoe_batch& b, const AttnShape& sh, int mask_block,
                                 int32_t* plan, hipStream_t s) {
  plan_kernel<<<1, kThreads, 0, s>>>(c, b, sh, mask_block, plan);
  return hipGetLastError();
}

}  // namespace dmoe
