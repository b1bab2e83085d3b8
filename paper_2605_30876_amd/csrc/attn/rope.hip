// Rotary positions, and the store of a step's keys and values into the paged
// cache with the rotation fused in.
//
// A workgroup takes 32 tokens of one kv head or of a few query heads: it
// forms cos and sin of (token, pair) once in LDS and uses them for all of its
// heads.  The work is bytes: every element is read and written once, in
// 16-byte chunks.
#include "cache.h"

namespace dmoe {

namespace {

constexpr int kThreads = 256;
constexpr int kTokens = 32;
constexpr int kQueryHeads = 4;  // query heads of a workgroup

template <typename T>
struct alignas(16) Chunk {
  static constexpr int c = 16 / sizeof(T);
  T v[c];
};

// cos and sin, times the scale, of every pair of `n` tokens; pos(i): position
// of token i.
template <typename Pos>
__device__ __forceinline__ void form_angles(float2* cs, const dmoe_rotary& r, int n, bool inverse, Pos pos) {
  const int pairs = r.rot_dim / 2;
  for (int x = threadIdx.x; x < n * pairs; x += kThreads) {
    const int i = x / pairs, f = x - i * pairs;
    double turn = static_cast<double>(pos(i)) * r.turns[f];
    turn -= rint(turn);  // [-1/2, 1/2]: the float32 below is off by 2^-26 turns at most
    float s, co;
    sincospif(2.f * static_cast<float>(turn), &s, &co);
    cs[x] = make_float2(co * r.scale, (inverse ? -s : s) * r.scale);
  }
}

// One chunk of a head, elements d0 .. d0 + c-1, rotated: `x` holds the head.
// Everything is loaded before the caller stores, so x may be the output.
template <typename T>
__device__ __forceinline__ Chunk<T> rotated(const T* x, int d0, const float2* cs, int rot, bool interleaved) {
  constexpr int c = Chunk<T>::c;
  Chunk<T> a = *reinterpret_cast<const Chunk<T>*>(x + d0);
  if (d0 >= rot) return a;
  if (interleaved) {
#pragma unroll
    for (int e = 0; e < c; e += 2) {
      if (d0 + e >= rot) break;
      const float2 t = cs[(d0 + e) / 2];
      const float x1 = load_as_f32<T>(&a.v[e]), x2 = load_as_f32<T>(&a.v[e + 1]);
      store_from_f32<T>(&a.v[e], x1 * t.x - x2 * t.y);
      store_from_f32<T>(&a.v[e + 1], x2 * t.x + x1 * t.y);
    }
    return a;
  }
  const int hr = rot / 2;
  Chunk<T> b;
  if (hr % c == 0) {
    b = *reinterpret_cast<const Chunk<T>*>(x + (d0 < hr ? d0 + hr : d0 - hr));
  } else {
#pragma unroll
    for (int e = 0; e < c; ++e)
      if (d0 + e < rot) b.v[e] = x[d0 + e < hr ? d0 + e + hr : d0 + e - hr];
  }
#pragma unroll
  for (int e = 0; e < c; ++e) {
    const int d = d0 + e;
    if (d < rot) {
      const float2 t = cs[d < hr ? d : d - hr];
      const float u = load_as_f32<T>(&a.v[e]), w = load_as_f32<T>(&b.v[e]);
      store_from_f32<T>(&a.v[e], d < hr ? u * t.x - w * t.y : u * t.x + w * t.y);
    }
  }
  return a;
}

// `heads` heads of n tokens from in to out; a head's chunks lie in one wave,
// whose loads are all done when it stores: in place is safe.
template <typename T>
__device__ __forceinline__ void rotate_heads(const T* in, long in_stride, T* out, long out_stride, int n, int heads,
                                             int dim, const float2* cs, int pairs, const dmoe_rotary& r) {
  constexpr int c = Chunk<T>::c;
  const int chunks = dim / c;
  int width = 1;
  while (width < chunks) width *= 2;  // lanes of a head, at most 64
  const int j = threadIdx.x & (width - 1);
  for (int x = threadIdx.x / width; x < n * heads; x += kThreads / width) {
    const int i = x / heads, h = x - i * heads;
    if (j < chunks) {
      const Chunk<T> y = rotated<T>(in + i * in_stride + h * dim, j * c, cs + i * pairs, r.turns ? r.rot_dim : 0, r.interleaved);
      *reinterpret_cast<Chunk<T>*>(out + i * out_stride + h * dim + j * c) = y;
    }
  }
}

template <typename T>
__global__ __launch_bounds__(kThreads) void rope_kernel(const T* x, long x_stride, T* out, long out_stride, int T_, int heads,
                                                        int dim, const int32_t* positions, dmoe_rotary r, bool inverse) {
  extern __shared__ float2 cs[];
  const int t0 = blockIdx.x * kTokens, n = min(kTokens, T_ - t0);
  const int h0 = blockIdx.y * kQueryHeads;
  form_angles(cs, r, n, inverse, [&](int i) { return positions[t0 + i]; });
  __syncthreads();
  rotate_heads<T>(x + t0 * x_stride + h0 * dim, x_stride, out + t0 * out_stride + h0 * dim, out_stride, n,
                  min(kQueryHeads, heads - h0), dim, cs, r.rot_dim / 2, r);
}

// blockIdx.x: (sequence, tile of 32 positions); blockIdx.y: kv heads, then
// groups of query heads.
template <typename T>
__global__ __launch_bounds__(kThreads) void append_kernel(AppendArgs a, int tiles) {
  constexpr int c = Chunk<T>::c;
  extern __shared__ float2 cs[];
  const int si = blockIdx.x / tiles, hkv = a.cache.n_kv_heads, dim = a.cache.head_dim;
  const Seq q = load_seq(a.cache, a.batch, si);
  const int start = max(q.pos0, 0);
  const int p0 = max(start, (start / kTokens + static_cast<int>(blockIdx.x % tiles)) * kTokens);
  const int p1 = min(q.len, (p0 / kTokens + 1) * kTokens);
  const int n = p1 - p0;
  if (n <= 0) return;
  const long t0 = q.row0 + (p0 - q.pos0);
  const int pairs = a.rope.rot_dim / 2;
  if (a.rope.turns) form_angles(cs, a.rope, n, false, [&](int i) { return p0 + i; });
  __syncthreads();
  if (static_cast<int>(blockIdx.y) >= hkv) {
    const int h0 = (blockIdx.y - hkv) * kQueryHeads;
    rotate_heads<T>(static_cast<const T*>(a.q) + t0 * a.q_stride + h0 * dim, a.q_stride,
                    static_cast<T*>(a.q_out) + t0 * a.q_out_stride + h0 * dim, a.q_out_stride, n,
                    min(kQueryHeads, a.n_heads - h0), dim, cs, pairs, a.rope);
    return;
  }
  const int hk = blockIdx.y, dp = padded_dim(dim), pt = a.cache.page_tokens;
  const int page = a.cache.table[static_cast<long>(q.slot) * a.cache.max_pages + p0 / pt];
  if (page < 0 || page >= a.cache.n_pages) return;
  const long at = (((static_cast<long>(a.layer) * a.cache.n_pages + page) * hkv + hk) * pt + p0 % pt / kTokens * kTokens) * dp;
  const int r0 = p0 % kTokens;
  const T* kin = static_cast<const T*>(a.k) + t0 * a.k_stride + static_cast<long>(hk) * dim;
  T* kp = static_cast<T*>(a.cache.k) + at;
  const int chunks = dp / c;
  for (int x = threadIdx.x; x < n * chunks; x += kThreads) {
    const int i = x % n, j = x / n;  // neighbouring tokens of a chunk are neighbours in the page
    Chunk<T> y{};
    if (j * c < dim) y = rotated<T>(kin + i * a.k_stride, j * c, cs + i * pairs, a.rope.turns ? a.rope.rot_dim : 0, a.rope.interleaved);
    *reinterpret_cast<Chunk<T>*>(kp + key_chunk<c>(r0 + i, j)) = y;
  }
  // values: a chunk holds 2c/2 tokens of one element, so the tile is turned in LDS
  __syncthreads();
  T* tile = reinterpret_cast<T*>(cs);
  const T* vin = static_cast<const T*>(a.v) + t0 * a.v_stride + static_cast<long>(hk) * dim;
  for (int x = threadIdx.x; x < n * (dim / c); x += kThreads) {
    const int i = x / (dim / c), j = x - i * (dim / c);
    *reinterpret_cast<Chunk<T>*>(tile + (r0 + i) * dp + j * c) = *reinterpret_cast<const Chunk<T>*>(vin + i * a.v_stride + j * c);
  }
  __syncthreads();
  T* vp = static_cast<T*>(a.cache.v) + at;
  for (int x = threadIdx.x; x < dp * (32 / c); x += kThreads) {
    const int d = x / 32 / (32 / c) * 32 + x % 32, sh = x / 32 % (32 / c), s = sh / 2, h = sh % 2;
    Chunk<T> y;
    bool all = true;
    uint32_t have = 0;
#pragma unroll
    for (int e = 0; e < c; ++e) {
      const int r = 2 * c * s + 8 * (e / 4) + 4 * h + e % 4;
      const bool in = r >= r0 && r < r0 + n;
      all = all && in;
      have |= static_cast<uint32_t>(in) << e;
      y.v[e] = in && d < dim ? tile[r * dp + d] : T(0);
    }
    T* to = vp + value_chunk<c>(d, s, h);
    if (all) {
      *reinterpret_cast<Chunk<T>*>(to) = y;
    } else {
#pragma unroll
      for (int e = 0; e < c; ++e)
        if (have >> e & 1) to[e] = y.v[e];
    }
  }
}

template <typename T>
hipError_t append(const AppendArgs& a, hipStream_t s) {
  const int most = a.batch.max_new < a.batch.T ? a.batch.max_new : a.batch.T;
  const int tiles = (most + kTokens - 2) / kTokens + 1;
  const unsigned y = a.cache.n_kv_heads + (a.q ? (a.n_heads + kQueryHeads - 1) / kQueryHeads : 0);
  const size_t angles = a.rope.turns ? static_cast<size_t>(kTokens) * (a.rope.rot_dim / 2) * sizeof(float2) : 0;
  const size_t turn = static_cast<size_t>(kTokens) * padded_dim(a.cache.head_dim) * sizeof(T);
  append_kernel<T><<<dim3(static_cast<unsigned>(a.batch.n_seqs) * tiles, y), kThreads, angles > turn ? angles : turn, s>>>(a, tiles);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rope(const void* x, long x_stride, void* out, long out_stride, dmoe_dtype dt, int T, int n_heads,
                       int head_dim, const int32_t* positions, const dmoe_rotary& r, bool inverse, hipStream_t s) {
  const dim3 grid((T + kTokens - 1) / kTokens, (n_heads + kQueryHeads - 1) / kQueryHeads);
  const size_t lds = static_cast<size_t>(kTokens) * (r.rot_dim / 2) * sizeof(float2);
  if (dt == DMOE_BF16)
    rope_kernel<bf16_t><<<grid, kThreads, lds, s>>>(static_cast<const bf16_t*>(x), x_stride, static_cast<bf16_t*>(out),
                                                    out_stride, T, n_heads, head_dim, positions, r, inverse);
  else
    rope_kernel<float><<<grid, kThreads, lds, s>>>(static_cast<const float*>(x), x_stride, static_cast<float*>(out),
                                                   out_stride, T, n_heads, head_dim, positions, r, inverse);
  return hipGetLastError();
}

hipError_t launch_append(const AppendArgs& a, hipStream_t s) {
  return a.cache.dt == DMOE_BF16 ? append<bf16_t>(a, s) : append<float>(a, s);
}

}  // namespace dmoe
