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

struct AttnArgs {
  dmoe_cache cache;
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

size_t update_workspace_bytes(long n, long max_pages, long n_pages);
hipError_t launch_update(const dmoe_cache& c, const int32_t* dst, const int32_t* src, const int32_t* keep,
                         const int32_t* new_lens, int n, int32_t* status, void* ws, hipStream_t s);
size_t compact_workspace_bytes(long n_pages);
hipError_t launch_compact(const dmoe_cache& c, int32_t* table_out, int32_t* refs_out, int32_t* counts, void* ws,
                          hipStream_t s);
hipError_t launch_copy_pages(const dmoe_cache& c, const int32_t* pairs, int n, hipStream_t s);

}  // namespace dmoe
