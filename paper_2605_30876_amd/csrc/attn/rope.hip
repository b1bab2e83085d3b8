// Rotary positions, and the store of a step's keys and values into the paged
// cache with the rotation fused in.
//
// A thread takes the same two 16-byte chunks (a row's pairs lie in chunks that
// belong together) of one token in one head after another, so that a pair's
// cos and sin are formed once, in registers, for all of its heads; no two
// lanes load the same bytes and nothing passes through LDS.  The work is
// bytes: every element is read and written once.  bf16, 32 query and 8 kv heads
// of 128: 8000 prompt tokens in 60 us (217 MB, 3.6 TB/s; the values' turn through LDS
// is 11 us of it, a large copy runs at 4.9 TB/s); fp32, 4096 rows of 12 heads of 96: 8.5 us
// (38 MB, 4.4 TB/s).  A block of 32 tokens takes 4.4 us, three round trips to memory and the launch.
#include "rotate.h"

namespace dmoe {

namespace {

using namespace rotary;

template <typename T, bool kAligned>
__global__ __launch_bounds__(kThreads) void rope_kernel(const T* x, long x_stride, T* out, long out_stride, int T_, int n_heads,
                                                        int heads, int dim, const int32_t* positions, dmoe_rotary r, bool inverse) {
  const int t0 = blockIdx.x * kTokens, n = min(kTokens, T_ - t0);
  const int h0 = blockIdx.y * heads;
  rotate_rows<T, kAligned>(
      n, min(heads, n_heads - h0), dim, dim, r, inverse, [&](int i) { return positions[t0 + i]; },
      [&](int i, int h) { return x + (t0 + i) * x_stride + (h0 + h) * dim; },
      [&](int i, int h, int j) { return out + (t0 + i) * out_stride + (h0 + h) * dim + j * Chunk<T>::c; });
}

// blockIdx.x: tile of 32 positions.  blockIdx.y: the values of one
// kv head each, then (8 of the tile's new tokens, group of `heads` heads) of the
// queries and keys.
template <typename T, bool kAligned>
__global__ __launch_bounds__(kThreads) void append_kernel(AppendArgs a, int tiles, int heads, int groups) {
  constexpr int c = Chunk<T>::c;
  extern __shared__ float4 lds[];
  const int hkv = a.cache.n_kv_heads, dim = a.cache.head_dim;
  int tile0;
  const Seq q = find_tile<false>(a.batch.n_seqs, blockIdx.x, tiles, tile0, [&](int i) { return load_seq(a.cache, a.batch, i); });
  const int start = max(q.pos0, 0);
  const int y = static_cast<int>(blockIdx.y) - hkv;
  const int end = min(q.len, tile0 + kTileTokens);
  const int p0 = max(start, tile0) + (y < 0 ? 0 : y / groups * kTokens), p1 = y < 0 ? end : min(end, p0 + kTokens), n = p1 - p0;
  if (n <= 0) return;
  const long t0 = q.row0 + (p0 - q.pos0);
  const int dp = padded_dim(dim), pt = a.cache.page_tokens;
  const int page = a.cache.table[static_cast<long>(q.slot) * a.cache.max_pages + p0 / pt];
  const bool held = page >= 0 && page < a.cache.n_pages;
  // the tile of kv head 0
  const long at = ((static_cast<long>(a.layer) * a.cache.n_pages + page) * hkv * pt + p0 % pt / kTileTokens * kTileTokens) * dp;
  if (y >= 0) {
    const int nq = a.q ? a.n_heads : 0, h0 = y % groups * heads;
    rotate_rows<T, kAligned>(
        n, min(heads, nq + hkv - h0), dim, dp, a.rope, false, [&](int i) { return p0 + i; },
        [&](int i, int h) {
          h += h0;
          return h < nq ? static_cast<const T*>(a.q) + (t0 + i) * a.q_stride + h * dim
                        : static_cast<const T*>(a.k) + (t0 + i) * a.k_stride + (h - nq) * dim;
        },
        [&](int i, int h, int j) -> T* {
          h += h0;
          if (h < nq) return j * c < dim ? static_cast<T*>(a.q_out) + (t0 + i) * a.q_out_stride + h * dim + j * c : nullptr;
          return held ? static_cast<T*>(a.cache.k) + at + static_cast<long>(h - nq) * pt * dp + key_chunk<c>((p0 + i) % kTileTokens, j)
                      : nullptr;
        });
    return;
  }
  if (!held) return;
  // values: a chunk holds c tokens of one element, so the tile is turned in LDS
  const int hk = blockIdx.y, r0 = p0 % kTileTokens;
  T* tile = reinterpret_cast<T*>(lds);
  const T* vin = static_cast<const T*>(a.v) + t0 * a.v_stride + static_cast<long>(hk) * dim;
  for (int x = threadIdx.x; x < n * (dim / c); x += kThreads) {
    const int i = x / (dim / c), j = x - i * (dim / c);
    *reinterpret_cast<Chunk<T>*>(tile + (r0 + i) * dp + j * c) = *reinterpret_cast<const Chunk<T>*>(vin + i * a.v_stride + j * c);
  }
  __syncthreads();
  T* vp = static_cast<T*>(a.cache.v) + at + static_cast<long>(hk) * pt * dp;
  for (int x = threadIdx.x; x < dp * (32 / c); x += kThreads) {
    const int d = x / 32 / (32 / c) * 32 + x % 32, sh = x / 32 % (32 / c), s = sh / 2, h = sh % 2;
    Chunk<T> w;
    bool all = true;
    uint32_t have = 0;
#pragma unroll
    for (int e = 0; e < c; ++e) {
      const int r = 2 * c * s + 8 * (e / 4) + 4 * h + e % 4;
      const bool in = r >= r0 && r < r0 + n;
      all = all && in;
      have |= static_cast<uint32_t>(in) << e;
      w.v[e] = in && d < dim ? tile[r * dp + d] : T(0);
    }
    T* to = vp + value_chunk<c>(d, s, h);
    if (all) {
      *reinterpret_cast<Chunk<T>*>(to) = w;
    } else {
#pragma unroll
      for (int e = 0; e < c; ++e)
        if (have >> e & 1) to[e] = w.v[e];
    }
  }
}

template <typename T>
hipError_t append(const AppendArgs& a, hipStream_t s) {
  const int most = a.batch.max_new < a.batch.T ? a.batch.max_new : a.batch.T;
  const int turned = a.cache.n_kv_heads + (a.q ? a.n_heads : 0), dp = padded_dim(a.cache.head_dim);
  const size_t lds = static_cast<size_t>(kTileTokens) * dp * sizeof(T);
  const TileGrid tg = tile_grid(a.batch);
  // at most `most` of a tile's positions are new
  const int sub = ((most < kTileTokens ? most : kTileTokens) + kTokens - 1) / kTokens;
  const int heads = heads_of_workgroup(tg.tiles * sub, (a.batch.T + kTokens - 1) / kTokens, turned, dp / Chunk<T>::c);
  const int groups = (turned + heads - 1) / heads;
  const dim3 grid(static_cast<unsigned>(tg.tiles), a.cache.n_kv_heads + sub * groups);
  if (aligned_pairs(a.rope, Chunk<T>::c))
    append_kernel<T, true><<<grid, kThreads, lds, s>>>(a, tg.each, heads, groups);
  else
    append_kernel<T, false><<<grid, kThreads, lds, s>>>(a, tg.each, heads, groups);
  return hipGetLastError();
}

template <typename T>
hipError_t rope(const void* x, long x_stride, void* out, long out_stride, int T_, int n_heads, int dim, const int32_t* positions,
                const dmoe_rotary& r, bool inverse, hipStream_t s) {
  const int groups = (T_ + kTokens - 1) / kTokens;
  const int heads = heads_of_workgroup(groups, groups, n_heads, dim / Chunk<T>::c);
  const dim3 grid(groups, (n_heads + heads - 1) / heads);
  auto run = [&](auto kernel) {
    kernel<<<grid, kThreads, 0, s>>>(static_cast<const T*>(x), x_stride, static_cast<T*>(out), out_stride, T_, n_heads, heads, dim, positions,
                                     r, inverse);
  };
  if (aligned_pairs(r, Chunk<T>::c))
    run(rope_kernel<T, true>);
  else
    run(rope_kernel<T, false>);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rope(const void* x, long x_stride, void* out, long out_stride, dmoe_dtype dt, int T, int n_heads,
                       int head_dim, const int32_t* positions, const dmoe_rotary& r, bool inverse, hipStream_t s) {
  return dt == DMOE_BF16 ? rope<bf16_t>(x, x_stride, out, out_stride, T, n_heads, head_dim, positions, r, inverse, s)
                         : rope<float>(x, x_stride, out, out_stride, T, n_heads, head_dim, positions, r, inverse, s);
}

hipError_t launch_append(const AppendArgs& a, hipStream_t s) {
  return a.cache.dt == DMOE_BF16 ? append<bf16_t>(a, s) : append<float>(a, s);
}

}  // namespace dmoe
