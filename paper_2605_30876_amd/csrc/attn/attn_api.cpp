// C ABI of the attention section of dmoe.h: argument validation on the host,
// then the launchers.
#include <algorithm>
#include <cmath>

#include "attn/cache.h"
#include "host/checks.h"

namespace {

using namespace dmoe::host;

constexpr int kMaxSeqs = 4096;
constexpr int kMaxSlots = 65536;
constexpr int kMaxKvHeads = 256;
constexpr int kMaxGroup = 1024;
constexpr int kMaxPageTokens = 1024;
constexpr int kMaxEntries = 4096;
constexpr long kMaxTokens = 1 << 30;  // of a sequence: a tile beyond the last still fits int32
constexpr int kMaxRows = 1 << 26;    // rows of a step's tensors: grids stay below 2^32 threads
constexpr long kMaxHeadRows = 1 << 30;  // (row, head) pairs: a tile beyond the last still fits int32

bool valid_head_dim(int d) { return d >= 8 && d <= 256 && d % 8 == 0; }
bool valid_page(int page_tokens, int n_kv_heads, int head_dim) {
  return page_tokens >= 32 && page_tokens <= kMaxPageTokens && page_tokens % 32 == 0 && n_kv_heads >= 1 &&
         n_kv_heads <= kMaxKvHeads && valid_head_dim(head_dim);
}
bool valid_format(dmoe_kv_format f) { return f >= DMOE_KV_PLAIN && f <= DMOE_KV_FP8_FP4; }
bool misaligned_to(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n != 0; }

#define ALIGNED_TO(p, n) REQUIRE(!misaligned_to(p, n), #p " is not " #n "-byte aligned")
// A step's tensor: rows `stride` elements apart that hold `width` elements.
#define ROWS(p, stride, width, dt)                                                                              \
  do {                                                                                                          \
    ALIGNED(p);                                                                                                 \
    REQUIRE((stride) >= (width) && (stride) % dmoe::chunk_elems(dt) == 0 && (stride) <= kIntLimit,              \
            #stride "=%ld must be at least %ld and a multiple of 16 bytes", static_cast<long>(stride),          \
            static_cast<long>(width));                                                                          \
  } while (0)
#define FORWARD(expr)                 \
  do {                                \
    const dmoe_status st_ = (expr);   \
    if (st_ != DMOE_OK) return st_;   \
  } while (0)

#undef DMOE_FN
#define DMOE_FN fn

dmoe_status check_cache(const char* fn, const dmoe_cache* c, bool refs) {
  REQUIRE(c, "cache must not be NULL");
  REQUIRE(c->k && c->v && c->table && c->lens, "the cache's k, v, table and lens must not be NULL");
  REQUIRE(!refs || c->refs, "the cache's refs must not be NULL");
  REQUIRE(valid_dtype(c->dt), "unknown dtype %d", static_cast<int>(c->dt));
  REQUIRE(valid_format(c->format), "unknown cache format %d", static_cast<int>(c->format));
  REQUIRE(c->n_layers >= 1 && c->n_pages >= 1 && c->n_slots >= 1 && c->max_pages >= 1,
          "n_layers=%d, n_pages=%d, n_slots=%d and max_pages=%d must be >= 1", c->n_layers, c->n_pages, c->n_slots, c->max_pages);
  REQUIRE(valid_page(c->page_tokens, c->n_kv_heads, c->head_dim),
          "page_tokens=%d must be a multiple of 32 up to %d, n_kv_heads=%d in [1, %d], head_dim=%d a multiple of 8 in [8, 256]",
          c->page_tokens, kMaxPageTokens, c->n_kv_heads, kMaxKvHeads, c->head_dim);
  REQUIRE(static_cast<long>(c->max_pages) * c->page_tokens <= kMaxTokens, "max_pages*page_tokens must be at most %ld", kMaxTokens);
  SUPPORT(c->n_slots <= kMaxSlots, "n_slots=%d must be at most %d", c->n_slots, kMaxSlots);
  REQUIRE(!misaligned(c->k) && !misaligned(c->v), "the cache's k and v must be 16-byte aligned");
  REQUIRE(!misaligned_to(c->table, 4) && !misaligned_to(c->lens, 4) && !misaligned_to(c->refs, 4) && !misaligned_to(c->refused, 4),
          "the cache's table, lens, refs and refused must be 4-byte aligned");
  return DMOE_OK;
}

dmoe_status check_batch(const char* fn, const dmoe_cache* c, const dmoe_batch& b) {
  REQUIRE(b.q_offsets, "q_offsets must not be NULL");
  REQUIRE(b.n_seqs >= 1 && b.T >= 1 && b.max_new >= 1, "n_seqs=%d, T=%d and max_new=%d must be >= 1", b.n_seqs, b.T, b.max_new);
  REQUIRE(b.slots || b.n_seqs <= c->n_slots, "without slots n_seqs=%d must be at most n_slots=%d", b.n_seqs, c->n_slots);
  SUPPORT(b.n_seqs <= kMaxSeqs, "n_seqs=%d must be at most %d", b.n_seqs, kMaxSeqs);
  SUPPORT(b.T <= kMaxRows, "T=%d must be at most %d", b.T, kMaxRows);
  ALIGNED_TO(b.q_offsets, 4);
  ALIGNED_TO(b.slots, 4);
  return DMOE_OK;
}

dmoe_status check_heads(const char* fn, int T, int n_heads, int n_kv_heads) {
  REQUIRE(n_heads >= 1 && n_heads % n_kv_heads == 0, "n_heads=%d must be a multiple of n_kv_heads=%d", n_heads, n_kv_heads);
  SUPPORT(n_heads / n_kv_heads <= kMaxGroup, "n_heads / n_kv_heads = %d must be at most %d", n_heads / n_kv_heads, kMaxGroup);
  SUPPORT(static_cast<long>(T) * n_heads <= kMaxHeadRows, "T*n_heads must be at most %ld", kMaxHeadRows);
  return DMOE_OK;
}

dmoe_status check_rope(const char* fn, const dmoe_rotary& r, int head_dim) {
  REQUIRE(r.rot_dim >= 2 && r.rot_dim % 2 == 0 && r.rot_dim <= head_dim, "rot_dim=%d must be even and in [2, head_dim=%d]",
          r.rot_dim, head_dim);
  REQUIRE(std::isfinite(r.scale), "the rotation's scale must be finite");
  ALIGNED_TO(r.turns, 8);
  return DMOE_OK;
}

#undef DMOE_FN
#define DMOE_FN __func__

bool overlap(const void* a, size_t na, const void* b, size_t nb) {
  const char* pa = static_cast<const char*>(a);
  const char* pb = static_cast<const char*>(b);
  return pa < pb + nb && pb < pa + na;
}
// Whether two step's tensors share an element.  With one stride they may be
// columns of one wider tensor; with two, their spans tell.
bool rows_overlap(const void* a, long a_stride, const void* b, long b_stride, long rows, long width, dmoe_dtype dt) {
  const size_t e = dmoe::dtype_bytes(dt), w = width * e, pitch = a_stride * e;
  if (!overlap(a, ((rows - 1) * a_stride + width) * e, b, ((rows - 1) * b_stride + width) * e)) return false;
  const uintptr_t pa = reinterpret_cast<uintptr_t>(a), pb = reinterpret_cast<uintptr_t>(b);
  const size_t off = (pa < pb ? pb - pa : pa - pb) % pitch;
  return a_stride != b_stride || off < w || pitch - off < w;
}

template <typename T>
hipError_t attend(dmoe_kv_format format, const dmoe::AttnArgs& a, const dmoe::AttnShape& sh, hipStream_t s) {
  switch (format) {
    case DMOE_KV_FP8: return dmoe::launch_attention_quant<T, 8, 8>(a, sh, s);
    case DMOE_KV_FP4: return dmoe::launch_attention_quant<T, 4, 4>(a, sh, s);
    case DMOE_KV_FP8_FP4: return dmoe::launch_attention_quant<T, 8, 4>(a, sh, s);
    default: return sizeof(T) == 4 ? dmoe::launch_attention_f32(a, sh, s) : dmoe::launch_attention_bf16(a, sh, s);
  }
}

bool valid_shape(int n_seqs, int T, int max_new, int n_heads, int n_kv_heads) {
  return n_seqs >= 1 && n_seqs <= kMaxSeqs && T >= 1 && T <= kMaxRows && max_new >= 1 && n_kv_heads >= 1 && n_kv_heads <= kMaxKvHeads &&
         n_heads >= 1 && n_heads % n_kv_heads == 0 && n_heads / n_kv_heads <= kMaxGroup &&
         static_cast<long>(T) * n_heads <= kMaxHeadRows;
}

}  // namespace

extern "C" {

dmoe_status dmoe_rope_turns(int rot_dim, double base, dmoe_rope_scaling scaling, double factor, double original,
                            double* turns, float* scale) {
  REQUIRE(turns && scale, "turns and scale must not be NULL");
  REQUIRE(rot_dim >= 2 && rot_dim % 2 == 0, "rot_dim=%d must be even and >= 2", rot_dim);
  REQUIRE(base > 1.0 && std::isfinite(base), "base=%g must be above 1", base);
  REQUIRE(scaling >= DMOE_ROPE_NONE && scaling <= DMOE_ROPE_YARN, "unknown scaling %d", static_cast<int>(scaling));
  REQUIRE(factor >= 1.0 && std::isfinite(factor) && (scaling != DMOE_ROPE_NONE || factor == 1.0),
          "factor=%g must be >= 1, and 1 without scaling", factor);
  REQUIRE(scaling != DMOE_ROPE_YARN || (original >= 1.0 && std::isfinite(original)), "original=%g must be >= 1", original);
  constexpr double kTwoPi = 6.283185307179586476925;
  constexpr double kFast = 32.0, kSlow = 1.0;  // turns within `original` positions at which the ramp starts and ends
  if (scaling == DMOE_ROPE_NTK && rot_dim > 2) base *= std::pow(factor, rot_dim / (rot_dim - 2.0));
  double lo = 0.0, hi = 0.0;
  if (scaling == DMOE_ROPE_YARN) {
    auto pair = [&](double t) { return rot_dim * std::log(original / (t * kTwoPi)) / (2.0 * std::log(base)); };
    lo = std::fmax(std::floor(pair(kFast)), 0.0);
    hi = std::fmin(std::ceil(pair(kSlow)), rot_dim - 1.0);
  }
  for (int i = 0; i < rot_dim / 2; ++i) {
    double f = std::pow(base, -2.0 * i / rot_dim) / kTwoPi;
    if (scaling == DMOE_ROPE_LINEAR) f /= factor;
    if (scaling == DMOE_ROPE_YARN) {
      // ends that were cut to the pairs and met or crossed: every pair is slow, or every pair is fast
      const double ramp = hi > lo ? std::fmin(std::fmax((i - lo) / (hi - lo), 0.0), 1.0) : hi <= 0.0 ? 1.0 : 0.0;
      f = f / factor * ramp + f * (1.0 - ramp);
    }
    turns[i] = f;
  }
  *scale = scaling == DMOE_ROPE_YARN ? static_cast<float>(0.1 * std::log(factor) + 1.0) : 1.f;
  return ok();
}

dmoe_status dmoe_rope(const void* x, long x_stride, void* out, long out_stride, dmoe_dtype dt, int T, int n_heads,
                      int head_dim, const int32_t* positions, dmoe_rotary rope, int inverse, void* stream) {
  REQUIRE(x && out && positions && rope.turns, "x, out, positions and rope.turns must not be NULL");
  REQUIRE(valid_dtype(dt), "unknown dtype %d", static_cast<int>(dt));
  REQUIRE(T >= 1 && n_heads >= 1, "T=%d and n_heads=%d must be >= 1", T, n_heads);
  REQUIRE(valid_head_dim(head_dim), "head_dim=%d must be a multiple of 8 in [8, 256]", head_dim);
  const long width = static_cast<long>(n_heads) * head_dim;
  REQUIRE(width <= kIntLimit, "n_heads*head_dim must fit in int32");
  SUPPORT(n_heads <= 65535, "n_heads=%d must be at most 65535", n_heads);
  SUPPORT(T <= kMaxRows, "T=%d must be at most %d", T, kMaxRows);
  FORWARD(check_rope(__func__, rope, head_dim));
  ROWS(x, x_stride, width, dt);
  ROWS(out, out_stride, width, dt);
  ALIGNED_TO(positions, 4);
  REQUIRE((x == out && x_stride == out_stride) || !rows_overlap(x, x_stride, out, out_stride, T, width, dt),
          "out must be x with the same stride or not overlap it");
  return hip_status(dmoe::launch_rope(x, x_stride, out, out_stride, dt, T, n_heads, head_dim, positions, rope, inverse != 0,
                                      static_cast<hipStream_t>(stream)),
                    __func__);
}

size_t dmoe_cache_page_bytes(dmoe_dtype dt, int page_tokens, int n_kv_heads, int head_dim) {
  if (!valid_dtype(dt) || !valid_page(page_tokens, n_kv_heads, head_dim)) return 0;
  return static_cast<size_t>(dmoe::page_elems(page_tokens, n_kv_heads, head_dim)) * dmoe::dtype_bytes(dt);
}

size_t dmoe_cache_key_page_bytes(dmoe_dtype dt, dmoe_kv_format format, int page_tokens, int n_kv_heads, int head_dim) {
  if (!valid_dtype(dt) || !valid_format(format) || !valid_page(page_tokens, n_kv_heads, head_dim)) return 0;
  return static_cast<size_t>(dmoe::page_bytes(dt, dmoe::key_bits(format), page_tokens, n_kv_heads, head_dim));
}

size_t dmoe_cache_value_page_bytes(dmoe_dtype dt, dmoe_kv_format format, int page_tokens, int n_kv_heads, int head_dim) {
  if (!valid_dtype(dt) || !valid_format(format) || !valid_page(page_tokens, n_kv_heads, head_dim)) return 0;
  return static_cast<size_t>(dmoe::page_bytes(dt, dmoe::value_bits(format), page_tokens, n_kv_heads, head_dim));
}

dmoe_status dmoe_cache_append(const dmoe_cache* cache, int layer, dmoe_batch batch, const void* k, long k_stride,
                              const void* v, long v_stride, const void* q, long q_stride, void* q_out,
                              long q_out_stride, int n_heads, dmoe_rotary rope, void* stream) {
  FORWARD(check_cache(__func__, cache, false));
  FORWARD(check_batch(__func__, cache, batch));
  REQUIRE(layer >= 0 && layer < cache->n_layers, "layer=%d must be in [0, %d)", layer, cache->n_layers);
  REQUIRE(k && v, "k and v must not be NULL");
  REQUIRE((q != nullptr) == (q_out != nullptr), "q and q_out must both be set or both be NULL");
  const long kv_width = static_cast<long>(cache->n_kv_heads) * cache->head_dim;
  ROWS(k, k_stride, kv_width, cache->dt);
  ROWS(v, v_stride, kv_width, cache->dt);
  if (rope.turns)
    FORWARD(check_rope(__func__, rope, cache->head_dim));
  else
    rope.rot_dim = 0;
  if (q) {
    FORWARD(check_heads(__func__, batch.T, n_heads, cache->n_kv_heads));
    const long width = static_cast<long>(n_heads) * cache->head_dim;
    SUPPORT(n_heads <= 8192, "n_heads=%d must be at most 8192", n_heads);
    ROWS(q, q_stride, width, cache->dt);
    ROWS(q_out, q_out_stride, width, cache->dt);
    REQUIRE((q == q_out && q_stride == q_out_stride) ||
                !rows_overlap(q, q_stride, q_out, q_out_stride, batch.T, width, cache->dt),
            "q_out must be q with the same stride or not overlap it");
  }
  dmoe::AppendArgs a{*cache, layer, batch, k, k_stride, v, v_stride, q, q_stride, q_out, q_out_stride, n_heads, rope};
  const hipStream_t s = static_cast<hipStream_t>(stream);
  return hip_status(cache->format == DMOE_KV_PLAIN ? dmoe::launch_append(a, s) : dmoe::launch_append_quant(a, s), __func__);
}

dmoe_status dmoe_cache_read(const dmoe_cache* cache, int layer, dmoe_batch batch, const int32_t* starts, void* k,
                            long k_stride, void* v, long v_stride, void* stream) {
  FORWARD(check_cache(__func__, cache, false));
  FORWARD(check_batch(__func__, cache, batch));
  REQUIRE(layer >= 0 && layer < cache->n_layers, "layer=%d must be in [0, %d)", layer, cache->n_layers);
  REQUIRE(k || v, "k and v must not both be NULL");
  const long width = static_cast<long>(cache->n_kv_heads) * cache->head_dim;
  if (k) ROWS(k, k_stride, width, cache->dt);
  if (v) ROWS(v, v_stride, width, cache->dt);
  REQUIRE(!k || !v || !rows_overlap(k, k_stride, v, v_stride, batch.T, width, cache->dt), "k and v must not overlap");
  ALIGNED_TO(starts, 4);
  dmoe::ReadArgs a{*cache, layer, batch, starts, k, k_stride, v, v_stride};
  return hip_status(dmoe::launch_read(a, static_cast<hipStream_t>(stream)), __func__);
}

size_t dmoe_attention_plan_ints(int n_seqs, int T, int max_new, int n_heads, int n_kv_heads) {
  if (!valid_shape(n_seqs, T, max_new, n_heads, n_kv_heads)) return 0;
  return dmoe::plan_ints(n_seqs, T, max_new, n_heads, n_kv_heads);
}

size_t dmoe_attention_workspace_size(dmoe_dtype dt, int n_seqs, int T, int max_new, int n_heads, int n_kv_heads,
                                     int head_dim) {
  if (!valid_dtype(dt) || !valid_shape(n_seqs, T, max_new, n_heads, n_kv_heads) || !valid_head_dim(head_dim)) return 0;
  return dmoe::attn_workspace_bytes(n_seqs, T, max_new, n_heads, n_kv_heads, dmoe::padded_dim(head_dim));
}

dmoe_status dmoe_attention_plan(const dmoe_cache* cache, dmoe_batch batch, int n_heads, int mask_block, int32_t* plan,
                                size_t plan_ints, void* stream) {
  FORWARD(check_cache(__func__, cache, false));
  FORWARD(check_batch(__func__, cache, batch));
  FORWARD(check_heads(__func__, batch.T, n_heads, cache->n_kv_heads));
  REQUIRE(plan, "plan must not be NULL");
  ALIGNED(plan);
  REQUIRE(mask_block >= 0, "mask_block=%d must be >= 0", mask_block);
  const dmoe::AttnShape sh = dmoe::attn_shape(*cache, batch, n_heads);
  const size_t ints = std::max(dmoe::plan_ints(batch.n_seqs, batch.T, batch.max_new, n_heads, cache->n_kv_heads), dmoe::plan_ints(sh));
  REQUIRE(plan_ints >= ints, "a plan of %zu ints is smaller than the %zu needed", plan_ints, ints);
  return hip_status(dmoe::launch_attention_plan(*cache, batch, sh, mask_block, plan, static_cast<hipStream_t>(stream)), __func__);
}

dmoe_status dmoe_attention(const dmoe_cache* cache, int layer, dmoe_batch batch, int n_heads, int mask_block,
                           const void* q, long q_stride, float scale, const int32_t* plan, size_t plan_ints, void* out,
                           long out_stride, float* lse, void* workspace, size_t ws_bytes, void* stream) {
  FORWARD(check_cache(__func__, cache, false));
  FORWARD(check_batch(__func__, cache, batch));
  FORWARD(check_heads(__func__, batch.T, n_heads, cache->n_kv_heads));
  REQUIRE(layer >= 0 && layer < cache->n_layers, "layer=%d must be in [0, %d)", layer, cache->n_layers);
  REQUIRE(q && plan && out && workspace, "q, plan, out and workspace must not be NULL");
  REQUIRE(mask_block >= 0, "mask_block=%d must be >= 0", mask_block);
  REQUIRE(scale > 0.f && std::isfinite(scale * 1.44269504f), "scale=%g must be above 0 and scale * log2(e) finite",
          static_cast<double>(scale));
  const long width = static_cast<long>(n_heads) * cache->head_dim;
  ROWS(q, q_stride, width, cache->dt);
  ROWS(out, out_stride, width, cache->dt);
  REQUIRE(!rows_overlap(q, q_stride, out, out_stride, batch.T, width, cache->dt), "out must not overlap q");
  ALIGNED(plan);
  ALIGNED(workspace);
  ALIGNED_TO(lse, 4);
  const dmoe::AttnShape sh = dmoe::attn_shape(*cache, batch, n_heads);
  const size_t ints = std::max(dmoe::plan_ints(batch.n_seqs, batch.T, batch.max_new, n_heads, cache->n_kv_heads), dmoe::plan_ints(sh));
  REQUIRE(plan_ints >= ints, "a plan of %zu ints is smaller than the %zu needed", plan_ints, ints);
  const int dp = dmoe::padded_dim(cache->head_dim);
  const size_t need = std::max(dmoe::attn_workspace_bytes(batch.n_seqs, batch.T, batch.max_new, n_heads, cache->n_kv_heads, dp),
                               dmoe::attn_workspace_bytes(sh, cache->n_kv_heads, dp));
  REQUIRE(ws_bytes >= need, "workspace of %zu bytes is smaller than the %zu bytes needed", ws_bytes, need);
  dmoe::AttnArgs a{dmoe::attn_cache(*cache), layer, batch, n_heads, mask_block, q, q_stride, scale, plan, out, out_stride, lse, workspace};
  const hipStream_t s = static_cast<hipStream_t>(stream);
  return hip_status(cache->dt == DMOE_BF16 ? attend<dmoe::bf16_t>(cache->format, a, sh, s) : attend<float>(cache->format, a, sh, s), __func__);
}

size_t dmoe_cache_update_workspace_size(int n, int max_pages, int n_pages) {
  if (n < 1 || n > kMaxEntries || max_pages < 1 || n_pages < 1 || static_cast<long>(n) * max_pages > kIntLimit) return 0;
  return dmoe::update_workspace_bytes(n, max_pages, n_pages);
}

dmoe_status dmoe_cache_update(const dmoe_cache* cache, const int32_t* dst, const int32_t* src, const int32_t* keep,
                              const int32_t* new_lens, int n, int32_t* status, void* workspace, size_t ws_bytes,
                              void* stream) {
  FORWARD(check_cache(__func__, cache, true));
  REQUIRE(dst && new_lens && workspace, "dst, new_lens and workspace must not be NULL");
  REQUIRE(n >= 1, "n=%d must be >= 1", n);
  SUPPORT(n <= kMaxEntries, "n=%d must be at most %d", n, kMaxEntries);
  REQUIRE(static_cast<long>(n) * cache->max_pages <= kIntLimit, "n*max_pages must fit in int32");
  ALIGNED_TO(dst, 4);
  ALIGNED_TO(src, 4);
  ALIGNED_TO(keep, 4);
  ALIGNED_TO(new_lens, 4);
  ALIGNED_TO(status, 4);
  ALIGNED(workspace);
  const size_t need = dmoe::update_workspace_bytes(n, cache->max_pages, cache->n_pages);
  REQUIRE(ws_bytes >= need, "workspace of %zu bytes is smaller than the %zu bytes needed", ws_bytes, need);
  return hip_status(dmoe::launch_update(*cache, dst, src, keep, new_lens, n, status, workspace, static_cast<hipStream_t>(stream)),
                    __func__);
}

size_t dmoe_cache_compact_workspace_size(int n_pages) { return n_pages < 1 ? 0 : dmoe::compact_workspace_bytes(n_pages); }

dmoe_status dmoe_cache_compact(const dmoe_cache* cache, int32_t* table_out, int32_t* refs_out, int32_t* counts,
                               void* workspace, size_t ws_bytes, void* stream) {
  FORWARD(check_cache(__func__, cache, true));
  REQUIRE(table_out && refs_out && workspace, "table_out, refs_out and workspace must not be NULL");
  ALIGNED_TO(table_out, 4);
  ALIGNED_TO(refs_out, 4);
  ALIGNED_TO(counts, 4);
  ALIGNED(workspace);
  const size_t tb = static_cast<size_t>(cache->n_slots) * cache->max_pages * 4, rb = static_cast<size_t>(cache->n_pages) * 4;
  REQUIRE(table_out == cache->table || !overlap(table_out, tb, cache->table, tb), "table_out must be the table or not overlap it");
  REQUIRE(refs_out == cache->refs || !overlap(refs_out, rb, cache->refs, rb), "refs_out must be refs or not overlap it");
  const size_t need = dmoe::compact_workspace_bytes(cache->n_pages);
  REQUIRE(ws_bytes >= need, "workspace of %zu bytes is smaller than the %zu bytes needed", ws_bytes, need);
  return hip_status(dmoe::launch_compact(*cache, table_out, refs_out, counts, workspace, static_cast<hipStream_t>(stream)), __func__);
}

dmoe_status dmoe_cache_copy_pages(const dmoe_cache* cache, const int32_t* pairs, int n, void* stream) {
  FORWARD(check_cache(__func__, cache, false));
  REQUIRE(pairs, "pairs must not be NULL");
  REQUIRE(n >= 1, "n=%d must be >= 1", n);
  ALIGNED_TO(pairs, 4);
  return hip_status(dmoe::launch_copy_pages(*cache, pairs, n, static_cast<hipStream_t>(stream)), __func__);
}

}  // extern "C"
