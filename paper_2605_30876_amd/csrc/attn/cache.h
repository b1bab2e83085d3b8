// The paged key/value cache as the kernels see it: layout, batch and work
// items, and the launchers behind the entry points of the attention section
// of dmoe.h.
#pragma once

#include "dmoe_common.h"

namespace dmoe {

constexpr int kTileTokens = 32;  // tokens of one tile of a page: the matrix instruction's rows

// Head dimension as the cache holds it: the next size there are kernels for.
__host__ __device__ constexpr int padded_dim(int head_dim) {
  return head_dim <= 32 ? 32 : head_dim <= 64 ? 64 : head_dim <= 96 ? 96 : head_dim <= 128 ? 128 : head_dim <= 192 ? 192 : 256;
}

inline long page_elems(int page_tokens, int n_kv_heads, int head_dim) {
  return static_cast<long>(page_tokens) * n_kv_heads * padded_dim(head_dim);
}

// A cache in few bits: bits of an element of its keys and values (0: plain),
// elements that share a scale, scale bytes of a token's head (a power of two), bytes of a tile.
__host__ __device__ constexpr int key_bits(dmoe_kv_format f) { return f == DMOE_KV_PLAIN ? 0 : f == DMOE_KV_FP4 ? 4 : 8; }
__host__ __device__ constexpr int value_bits(dmoe_kv_format f) { return f == DMOE_KV_PLAIN ? 0 : f == DMOE_KV_FP8 ? 8 : 4; }
constexpr int kGroup = 32;
__host__ __device__ constexpr int scale_row(int dp) { return dp <= 32 ? 1 : dp <= 64 ? 2 : dp <= 128 ? 4 : 8; }
__host__ __device__ constexpr int quant_tile(int bits, int dp) { return dp * 4 * bits + kTileTokens * scale_row(dp); }
// Bytes from the start of a tile to the code of token r's element d (4 bits: of an even one and the next) and to its scales.
template <int kBits>
__host__ __device__ constexpr int code_at(int r, int d) {
  constexpr int per = 128 / kBits;  // elements of a 16-byte chunk
  return (d / per * kTileTokens + r) * 16 + d % per * kBits / 8;
}
template <int kBits>
__host__ __device__ constexpr int scale_at(int dp, int r) {
  return dp * 4 * kBits + r * scale_row(dp);
}
// Bytes of a page of keys, or of values.
inline long page_bytes(dmoe_dtype dt, int bits, int page_tokens, int n_kv_heads, int head_dim) {
  if (bits == 0) return page_elems(page_tokens, n_kv_heads, head_dim) * static_cast<long>(dtype_bytes(dt));
  return static_cast<long>(page_tokens / kTileTokens) * n_kv_heads * quant_tile(bits, padded_dim(head_dim));
}

// Elements from the start of a tile's keys (values) to one 16-byte chunk of
// c values.  Keys: chunk of token r, elements c*j .. c*j + c-1.  Values: chunk
// of element d, tokens 2c*s + 8j + 4h + t for j < c/4, t < 4.
template <int c>
__host__ __device__ constexpr int key_chunk(int r, int j) {
  return (j * kTileTokens + r) * c;
}
template <int c>
__host__ __device__ constexpr int value_chunk(int d, int s, int h) {
  return ((((d / 32) * (16 / c) + s) * 2 + h) * 32 + d % 32) * c;
}

// The new tokens of one sequence of a batch, everything cut to its range.
struct Seq {
  int slot;   // row of the page table
  int row0;   // first row of the step's tensors
  int n;      // new tokens (0: nothing to do)
  int len;    // tokens in the cache, the new ones included
  int pos0;   // position of the first new token (negative if n > len)
};

__device__ __forceinline__ Seq load_seq(const dmoe_cache& c, const dmoe_batch& b, int i) {
  Seq s;
  s.row0 = min(max(b.q_offsets[i], 0), b.T);
  const int row1 = min(max(b.q_offsets[i + 1], 0), b.T);
  s.n = min(max(row1 - s.row0, 0), b.max_new);
  s.slot = b.slots ? b.slots[i] : i;
  const bool known = s.slot >= 0 && s.slot < c.n_slots;
  s.slot = known ? s.slot : 0;
  // both loads on their way together
  const int32_t* marks = c.refused ? c.refused : c.lens;
  const int mark = marks[s.slot], len = c.lens[s.slot];
  s.len = known ? min(max(len, 0), c.max_pages * c.page_tokens) : 0;
  if (!known || (c.refused && mark != 0)) s.n = 0;
  s.pos0 = s.len - s.n;
  return s;
}

// Exclusive prefix sums over a workgroup's kThreads threads, waves[kThreads/64]
// in LDS; *total is their sum.
template <int kThreads, typename V>
__device__ __forceinline__ V scan_exclusive(V v, V* waves, V* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  V x = v;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const V y = __shfl_up(x, d);
    if (lane >= d) x += y;
  }
  if (lane == 63) waves[wave] = x;
  __syncthreads();
  V base = 0, sum = 0;
#pragma unroll
  for (int i = 0; i < kThreads / 64; ++i) {
    base += i < wave ? waves[i] : 0;
    sum += waves[i];
  }
  __syncthreads();
  *total = sum;
  return base + x - v;
}

// Keys that the token at position p sees (a prefix of the sequence).
__host__ __device__ __forceinline__ int visible_end(int p, int len, int mask_block) {
  if (p < 0) return 0;
  if (mask_block <= 0) return len;
  const long e = (static_cast<long>(p / mask_block) + 1) * mask_block;
  return e < len ? static_cast<int>(e) : len;
}

// Division of whole numbers below 2^30 by one that the host knows: three instructions, where the general one
// takes thirty and their place in the instruction cache.  n / d = n m >> s, m = ceil(2^s / d), 2^(s - 30) >= d: the
// product's excess over n 2^s / d is below 2^s / d.
struct FastDiv {
  uint32_t m;
  int s;
  __host__ __device__ __forceinline__ int of(int n) const { return static_cast<int>(static_cast<uint64_t>(static_cast<uint32_t>(n)) * m >> s); }
};
inline FastDiv fast_div(int d) {
  int s = 30;
  while ((1l << (s - 30)) < d) ++s;
  return FastDiv{static_cast<uint32_t>(((1ul << s) + d - 1) / d), s};
}

// ---- work items of the attention -------------------------------------------
// Rows of one kv head are (token, query head of the group) pairs, the head
// fastest.  An item is one row tile over a range of key tiles; a row tile cut
// into several items has its partial results merged by a second kernel.
struct AttnItem {
  int slot, row0, n, len;     // the sequence (load_seq)
  int first, rows;            // first row of the tile, rows of the sequence
  int kt0, kt1;               // key tiles of 32 tokens
  int part;                   // partial result, or -1: the only item of its rows
  // Pages of the first four key tiles and of two from item_middle on (-1:
  // none) as the table stood for the plan: loads start from them while the
  // table is read, and are made again where it says otherwise (pages move, by
  // a compaction, while a plan goes by lengths alone).
  int page[6];
  int pad;
};
// Where the second half of an item's key tiles starts: the first has as many
// pairs of tiles, or one more.
__host__ __device__ constexpr int item_middle(int kt0, int kt1) {
  const int first = ((kt1 - kt0 + 1) / 2 + 1) / 2 * 2;
  return first < kt1 - kt0 ? kt0 + first : kt1;
}
struct AttnMerge {
  int row0, first, rows;      // as above
  int part, pieces;           // partial results part .. part + pieces-1
  int pad[3];
};
struct AttnPlanHead {
  int n_items, n_merges, pad[2];
};
static_assert(sizeof(AttnItem) == 64 && sizeof(AttnMerge) == 32 && sizeof(AttnPlanHead) == 16);

// What the host knows of a plan: the kernel's row tile and the bounds that
// size its arrays and grids.
struct AttnShape {
  int group;       // query heads of a kv head
  int tile_rows;   // rows of an item
  int min_tiles;   // key tiles of an item at least, where rows are split
  int whole_tiles; // key tiles that are not split
  long max_tiles;  // row tiles of the batch at most
  long split_items;  // items that splitting along the keys may add, and merges, at most
  int aim;           // items that splitting aims at: at most split_items
  int even_tiles;    // 128 rows: key tiles of a piece at least, where pieces even out lengths
  bool wide;         // block kernel: two halves of an item's keys per workgroup
  int unit;          // key tiles that an item's range is a multiple of (stage_tiles)
  __host__ __device__ long max_items() const { return max_tiles + split_items; }
  __host__ __device__ long max_parts() const { return 2 * split_items; }
};
// Key tiles of a stage of the block kernel: up to 16 KiB of keys, or one tile.
constexpr int stage_tiles(dmoe_dtype dt, int dp) { return dp * (dt == DMOE_F32 ? 4 : 2) * kTileTokens <= 8192 ? 2 : 1; }
// What any cache needs for these sizes.
size_t plan_ints(int n_seqs, int T, int max_new, int n_heads, int n_kv_heads);
size_t attn_workspace_bytes(int n_seqs, int T, int max_new, int n_heads, int n_kv_heads, int dp);
// Two workgroups of the block kernel fit a CU where a wave's registers fit half of a SIMD's.
constexpr bool two_per_cu(dmoe_dtype dt, int dp) { return dp * (dt == DMOE_F32 ? 4 : 2) <= 256; }
// and in a cache of few bits, whose products are bf16 and whose fp32 queries take three registers for one
constexpr bool quant_two_per_cu(dmoe_dtype dt, int dp) { return dp <= (dt == DMOE_F32 ? 64 : 128); }
// Waves of a SIMD in the kernel of few rows of such a cache: two where a lane's queries (in so many bf16 parts), sums and codes leave
// room for the rest in half of the registers, or nearly.  64 single tokens of up to 16k, 16 and 4 heads of 256 in 4 bits: 86 us
// with two, 103 with one; of up to 8k in 8 bits, which are far from fitting: 205 (spilled) and 96.  Forms of 16 rows that spill some
// bytes a lane with two, 64 tokens of up to 8k, 16 and 4 heads: fp32 192 elements in 4 bits (84 bytes) 78 us, 91 with one; with keys in 8 (80
// bytes) 79 and 84; bf16 256 elements, keys in 8 and values in 4 (36 bytes), 72 and 75; a token over 16,000 31, 31 and 32 with
// two, 31, 32 and 33 with one.  Three, where they fit, measured as two.  fp32, 256 elements, 32 rows do not fit one wave either: 440 to 484
// bytes a lane spill.
constexpr int quant_rows_waves(int parts, int dp, int bits, int rows) {
  return parts * dp * rows / 128 + dp * rows / 64 + dp * bits / 64 < 160 ? 2 : 1;
}
AttnShape attn_shape(const dmoe_cache& c, const dmoe_batch& b, int n_heads);

inline size_t plan_ints(const AttnShape& s) {
  return (sizeof(AttnPlanHead) + static_cast<size_t>(s.max_items()) * sizeof(AttnItem) +
          static_cast<size_t>(s.split_items) * sizeof(AttnMerge)) / sizeof(int);
}
__host__ __device__ inline const AttnItem* plan_items(const int32_t* plan) {
  return reinterpret_cast<const AttnItem*>(plan + sizeof(AttnPlanHead) / sizeof(int));
}
// Partial results of max_parts row tiles of every kv head: [part][kv head] of
// tile_rows x dp sums in the order in which the lanes hold them (partial_at),
// then as many (maximum, sum) pairs.
inline size_t attn_workspace_bytes(const AttnShape& s, int n_kv_heads, int dp) {
  return static_cast<size_t>(s.max_parts()) * n_kv_heads * s.tile_rows * (dp + 2) * sizeof(float);
}

// Floats from the start of a row tile's sums to the four of row r, elements
// d .. d+3: the waves' 32 rows one after another, each stored as it lies in
// the registers, 16 bytes a lane, so that a store is one contiguous KiB.
__host__ __device__ constexpr int partial_at(int dp, int r, int d) {
  return r / 32 * (32 * dp) + (d / 8 * 64 + d / 4 % 2 * 32 + r % 32) * 4;
}

// What the attention's kernels know of a cache: the format is in their names.  (Arguments of 8 bytes more move
// others into another line: 0.2 us of a launch of 9.7.)
struct AttnCache {
  void *k, *v;
  int32_t *table, *lens, *refs;
  dmoe_dtype dt;
  int n_layers, n_pages, page_tokens, n_kv_heads, head_dim, n_slots, max_pages;
  int32_t* refused;
};
inline AttnCache attn_cache(const dmoe_cache& c) {
  return AttnCache{c.k, c.v, c.table, c.lens, c.refs, c.dt, c.n_layers, c.n_pages, c.page_tokens, c.n_kv_heads, c.head_dim, c.n_slots, c.max_pages,
                   c.refused};
}
struct AttnArgs {
  AttnCache cache;
  int layer;
  dmoe_batch batch;
  int n_heads, mask_block;
  const void* q;
  long q_stride;
  float scale;
  const int32_t* plan;
  void* out;
  long out_stride;
  float* lse;
  void* workspace;
};
hipError_t launch_attention_bf16(const AttnArgs& a, const AttnShape& sh, hipStream_t s);
hipError_t launch_attention_f32(const AttnArgs& a, const AttnShape& sh, hipStream_t s);
// T: the rows' type; bits of keys and of values
template <typename T, int kKB, int kVB>
hipError_t launch_attention_quant(const AttnArgs& a, const AttnShape& sh, hipStream_t s);
hipError_t launch_attention_plan(const dmoe_cache& c, const dmoe_batch& b, const AttnShape& sh, int mask_block,
                                 int32_t* plan, hipStream_t s);

hipError_t launch_rope(const void* x, long x_stride, void* out, long out_stride, dmoe_dtype dt, int T, int n_heads,
                       int head_dim, const int32_t* positions, const dmoe_rotary& rope, bool inverse, hipStream_t s);
struct AppendArgs {
  dmoe_cache cache;
  int layer;
  dmoe_batch batch;
  const void* k;
  long k_stride;
  const void* v;
  long v_stride;
  const void* q;  // or nullptr
  long q_stride;
  void* q_out;
  long q_out_stride;
  int n_heads;
  dmoe_rotary rope;  // turns nullptr: no rotation
};
hipError_t launch_append(const AppendArgs& a, hipStream_t s);
hipError_t launch_append_quant(const AppendArgs& a, hipStream_t s);
struct ReadArgs {
  dmoe_cache cache;
  int layer;
  dmoe_batch batch;
  const int32_t* starts;  // or nullptr: the last tokens
  void* k;                // either may be nullptr
  long k_stride;
  void* v;
  long v_stride;
};
hipError_t launch_read(const ReadArgs& a, hipStream_t s);

size_t update_workspace_bytes(long n, long max_pages, long n_pages);
hipError_t launch_update(const dmoe_cache& c, const int32_t* dst, const int32_t* src, const int32_t* keep,
                         const int32_t* new_lens, int n, int32_t* status, void* ws, hipStream_t s);
size_t compact_workspace_bytes(long n_pages);
hipError_t launch_compact(const dmoe_cache& c, int32_t* table_out, int32_t* refs_out, int32_t* counts, void* ws,
                          hipStream_t s);
hipError_t launch_copy_pages(const dmoe_cache& c, const int32_t* pairs, int n, hipStream_t s);

}  // namespace dmoe
