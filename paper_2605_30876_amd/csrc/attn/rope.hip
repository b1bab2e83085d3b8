// Rotary positions, and the store of a step's keys and values into the paged
// cache with the rotation fused in.
//
// A workgroup takes 8 tokens of a few heads: it forms cos and sin of (token,
// pair) once in LDS and uses them for all of its heads, a 16-byte chunk per
// thread and row, the loads of several rows in flight together.  The work is
// bytes: every element is read and written once.
#include "cache.h"

namespace dmoe {

namespace {

constexpr int kThreads = 256;
constexpr int kTokens = 8;      // of a workgroup that rotates
constexpr int kInFlight = 4;    // rows a thread loads before it stores

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

// A chunk's values in float32, and rounded back (to nearest even, by the
// conversion instruction).
__device__ __forceinline__ void widen(const Chunk<float>& x, float (&f)[4]) {
#pragma unroll
  for (int e = 0; e < 4; ++e) f[e] = x.v[e];
}
__device__ __forceinline__ void widen(const Chunk<bf16_t>& x, float (&f)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) f[e] = bf16_to_f32(x.v[e]);
}
__device__ __forceinline__ Chunk<float> narrow(const float (&f)[4]) { return Chunk<float>{{f[0], f[1], f[2], f[3]}}; }
__device__ __forceinline__ Chunk<bf16_t> narrow(const float (&f)[8]) {
  bf16x8 v;
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = static_cast<__bf16>(f[e]);
  return __builtin_bit_cast(Chunk<bf16_t>, v);
}

// One chunk of a head, elements d0 .. d0 + c-1, rotated: `x` holds the head.
// Everything is loaded before the caller stores, so x may be the output.
template <typename T>
__device__ __forceinline__ Chunk<T> rotated(const T* x, int d0, const float2* cs, int rot, bool interleaved) {
  constexpr int c = Chunk<T>::c;
  const Chunk<T> a = *reinterpret_cast<const Chunk<T>*>(x + d0);
  if (d0 >= rot) return a;
  float u[c];
  widen(a, u);
  if (interleaved) {
#pragma unroll
    for (int e = 0; e < c; e += 2) {
      const bool in = d0 + e < rot;  // rot is even: a pair is in or out
      const float2 t = cs[in ? (d0 + e) / 2 : 0];
      const float x1 = u[e], x2 = u[e + 1];
      u[e] = in ? x1 * t.x - x2 * t.y : x1;
      u[e + 1] = in ? x2 * t.x + x1 * t.y : x2;
    }
    return narrow(u);
  }
  const int hr = rot / 2;
  float w[c];
  if (hr % c == 0) {
    // a chunk lies in one half, its partner is a chunk
    const bool low = d0 < hr;
    widen(*reinterpret_cast<const Chunk<T>*>(x + (low ? d0 + hr : d0 - hr)), w);
    const float2* t = cs + (low ? d0 : d0 - hr);
#pragma unroll
    for (int e = 0; e < c; ++e) u[e] = u[e] * t[e].x + (low ? -w[e] : w[e]) * t[e].y;
    return narrow(u);
  }
#pragma unroll
  for (int e = 0; e < c; ++e) {
    const int d = d0 + e;
    if (d < rot) {
      const float2 t = cs[d < hr ? d : d - hr];
      w[e] = load_as_f32<T>(x + (d < hr ? d + hr : d - hr));
      u[e] = u[e] * t.x + (d < hr ? -w[e] : w[e]) * t.y;
    }
  }
  return narrow(u);
}

// n tokens of `heads` heads through the rotation; in(i, h) and out(i, h, j):
// a head's elements, and where its chunk j goes (nullptr: nowhere).  A row's
// chunks lie in one wave, whose loads of them are done when it stores: in
// place is safe.  Chunks from dim on, up to `padded`, are 0.
template <typename T, typename In, typename Out>
__device__ __forceinline__ void rotate_rows(int n, int heads, int dim, int padded, const float2* cs, const dmoe_rotary& r, In in, Out out) {
  constexpr int c = Chunk<T>::c;
  const int chunks = padded / c, pairs = r.rot_dim / 2;
  const int log = chunks > 1 ? 32 - __builtin_clz(chunks - 1) : 0;  // lanes of a row: 2^log, at most 64
  const int j = threadIdx.x & ((1 << log) - 1), step = kThreads >> log, rows = n * heads;
  for (int x0 = threadIdx.x >> log; x0 < rows; x0 += step * kInFlight) {
    Chunk<T> y[kInFlight];
#pragma unroll
    for (int u = 0; u < kInFlight; ++u) {
      const int x = x0 + u * step;
      y[u] = Chunk<T>{};
      if (x < rows && j * c < dim) {
        const int h = x / n, i = x - h * n;
        y[u] = rotated<T>(in(i, h), j * c, cs + i * pairs, r.turns ? r.rot_dim : 0, r.interleaved);
      }
    }
#pragma unroll
    for (int u = 0; u < kInFlight; ++u) {
      const int x = x0 + u * step;
      if (x < rows && j < chunks) {
        const int h = x / n, i = x - h * n;
        if (T* to = out(i, h, j)) *reinterpret_cast<Chunk<T>*>(to) = y[u];
      }
    }
  }
}

template <typename T>
__global__ __launch_bounds__(kThreads) void rope_kernel(const T* x, long x_stride, T* out, long out_stride, int T_, int n_heads,
                                                        int heads, int dim, const int32_t* positions, dmoe_rotary r, bool inverse) {
  extern __shared__ float2 cs[];
  const int t0 = blockIdx.x * kTokens, n = min(kTokens, T_ - t0);
  const int h0 = blockIdx.y * heads;
  form_angles(cs, r, n, inverse, [&](int i) { return positions[t0 + i]; });
  __syncthreads();
  rotate_rows<T>(
      n, min(heads, n_heads - h0), dim, dim, cs, r, [&](int i, int h) { return x + (t0 + i) * x_stride + (h0 + h) * dim; },
      [&](int i, int h, int j) { return out + (t0 + i) * out_stride + (h0 + h) * dim + j * Chunk<T>::c; });
}

// The x-th tile of 32 positions that a batch's new tokens lie in, and its
// sequence.  `tiles` > 0: every sequence has that many, some of them empty;
// else those there are, counted by each wave, 64 sequences at a time.
__device__ __forceinline__ Seq find_tile(const AppendArgs& a, int x, int tiles, int& tile0) {
  Seq q;
  if (tiles > 0) {
    q = load_seq(a.cache, a.batch, x / tiles);
    tile0 = (max(q.pos0, 0) / kTileTokens + x % tiles) * kTileTokens;
    return q;
  }
  const int lane = threadIdx.x & 63;
  for (int i0 = 0; i0 < a.batch.n_seqs; i0 += 64) {
    q = Seq{0, 0, 0, 0, 0};
    if (i0 + lane < a.batch.n_seqs) q = load_seq(a.cache, a.batch, i0 + lane);
    const int first = max(q.pos0, 0) / kTileTokens, n = q.len > max(q.pos0, 0) ? (q.len - 1) / kTileTokens - first + 1 : 0;
    int upto = n;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const int y = __shfl_up(upto, d);
      if (lane >= d) upto += y;
    }
    const uint64_t behind = __ballot(upto > x);
    if (behind) {
      const int l = __builtin_ctzll(behind);
      tile0 = (__shfl(first, l) + x - __shfl(upto - n, l)) * kTileTokens;
      return Seq{__shfl(q.slot, l), __shfl(q.row0, l), __shfl(q.n, l), __shfl(q.len, l), __shfl(q.pos0, l)};
    }
    x -= __shfl(upto, 63);
  }
  tile0 = 0;
  return Seq{0, 0, 0, 0, 0};
}

// blockIdx.x: tile of 32 positions.  blockIdx.y: the values of one
// kv head each, then (8 tokens, group of `heads` heads) of the queries and keys.
template <typename T>
__global__ __launch_bounds__(kThreads) void append_kernel(AppendArgs a, int tiles, int heads, int groups) {
  constexpr int c = Chunk<T>::c;
  extern __shared__ float2 cs[];
  const int hkv = a.cache.n_kv_heads, dim = a.cache.head_dim;
  int tile0;
  const Seq q = find_tile(a, blockIdx.x, tiles, tile0);
  const int start = max(q.pos0, 0);
  const int y = static_cast<int>(blockIdx.y) - hkv;
  const int from = y < 0 ? tile0 : tile0 + y / groups * kTokens;
  const int p0 = max(start, from), p1 = min(q.len, from + (y < 0 ? kTileTokens : kTokens)), n = p1 - p0;
  if (n <= 0) return;
  const long t0 = q.row0 + (p0 - q.pos0);
  const int dp = padded_dim(dim), pt = a.cache.page_tokens;
  const int page = a.cache.table[static_cast<long>(q.slot) * a.cache.max_pages + p0 / pt];
  const bool held = page >= 0 && page < a.cache.n_pages;
  // the tile of kv head 0
  const long at = ((static_cast<long>(a.layer) * a.cache.n_pages + page) * hkv * pt + p0 % pt / kTileTokens * kTileTokens) * dp;
  if (y >= 0) {
    const int nq = a.q ? a.n_heads : 0, h0 = y % groups * heads;
    if (a.rope.turns) form_angles(cs, a.rope, n, false, [&](int i) { return p0 + i; });
    __syncthreads();
    rotate_rows<T>(
        n, min(heads, nq + hkv - h0), dim, dp, cs, a.rope,
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
  T* tile = reinterpret_cast<T*>(cs);
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

// Heads of a workgroup that rotates: as many as keep kGroups workgroups, so
// that their angles are formed for as many heads as possible.
constexpr long kGroups = 2048;
int heads_of_workgroup(long token_groups, int n_heads) {
  int heads = 1;
  while (heads < n_heads && token_groups * ((n_heads + 2 * heads - 1) / (2 * heads)) >= kGroups) heads *= 2;
  return heads < n_heads ? heads : n_heads;
}

template <typename T>
hipError_t append(const AppendArgs& a, hipStream_t s) {
  constexpr int kSub = kTileTokens / kTokens;
  const int most = a.batch.max_new < a.batch.T ? a.batch.max_new : a.batch.T;
  const int tiles = (most + kTileTokens - 2) / kTileTokens + 1;
  const int turned = a.cache.n_kv_heads + (a.q ? a.n_heads : 0), dp = padded_dim(a.cache.head_dim);
  const int heads = heads_of_workgroup((a.batch.T + kTokens - 1) / kTokens, turned);
  const int groups = (turned + heads - 1) / heads;
  const size_t angles = a.rope.turns ? static_cast<size_t>(kTokens) * (a.rope.rot_dim / 2) * sizeof(float2) : 0;
  const size_t turn = static_cast<size_t>(kTileTokens) * dp * sizeof(T);
  // n tokens lie in at most n / 32 + 2 tiles
  const long each = static_cast<long>(a.batch.n_seqs) * tiles, counted = a.batch.T / kTileTokens + 2l * a.batch.n_seqs;
  append_kernel<T><<<dim3(static_cast<unsigned>(each < counted ? each : counted), a.cache.n_kv_heads + kSub * groups), kThreads,
                     angles > turn ? angles : turn, s>>>(a, each <= counted ? tiles : 0, heads, groups);
  return hipGetLastError();
}

template <typename T>
hipError_t rope(const void* x, long x_stride, void* out, long out_stride, int T_, int n_heads, int dim, const int32_t* positions,
                const dmoe_rotary& r, bool inverse, hipStream_t s) {
  const int groups = (T_ + kTokens - 1) / kTokens;
  const int heads = heads_of_workgroup(groups, n_heads);
  const size_t lds = static_cast<size_t>(kTokens) * (r.rot_dim / 2) * sizeof(float2);
  rope_kernel<T><<<dim3(groups, (n_heads + heads - 1) / heads), kThreads, lds, s>>>(
      static_cast<const T*>(x), x_stride, static_cast<T*>(out), out_stride, T_, n_heads, heads, dim, positions, r, inverse);
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
