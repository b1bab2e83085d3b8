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
#include "cache.h"

namespace dmoe {

namespace {

constexpr int kThreads = 256;
constexpr int kTokens = 8;    // of a workgroup that rotates: 128 bytes of a page's keys
constexpr int kInFlight = 2;  // heads a thread loads before it stores (4: 67 against 59 us for 8000 prompt tokens)

template <typename T>
struct alignas(16) Chunk {
  static constexpr int c = 16 / sizeof(T);
  T v[c];
};

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

// A thread's share of a row: two chunks and what their elements are turned by.
// kAligned: interleaved pairs, or halves of whole chunks: element e of the one
// chunk pairs with element e of the other (interleaved: 2c consecutive
// elements, pairs within).  Otherwise the halves' border lies within a chunk,
// and an element's partner is read by itself.
template <typename T, bool kAligned>
struct Unit {
  static constexpr int c = Chunk<T>::c;
  static constexpr int kPairs = kAligned ? c : 2 * c;  // cos and sin kept: per pair, or per element
  int c0, c1;       // chunks of the row
  bool turned;      // some element of them is rotated
  float co[kPairs], si[kPairs];

  __device__ __forceinline__ Unit(int u, const dmoe_rotary& r) {
    const int hr = r.rot_dim / 2, n = hr / c;
    const bool halves = kAligned && !r.interleaved;
    c0 = halves && u < n ? u : 2 * u;
    c1 = halves && u < n ? u + n : 2 * u + 1;
    turned = r.turns && (halves ? u < n : 2 * c * u < r.rot_dim);
  }
  // pair (aligned) or element (otherwise) e's frequency; -1: not rotated
  __device__ __forceinline__ int pair_of(int e, const dmoe_rotary& r) const {
    const int hr = r.rot_dim / 2;
    if constexpr (kAligned) return r.interleaved ? (c * (c0 / 2) + e < hr ? c * (c0 / 2) + e : -1) : c * c0 + e;
    const int d = c * c0 + e;
    return d < hr ? d : d < 2 * hr ? d - hr : -1;
  }
  __device__ __forceinline__ void form(int position, const dmoe_rotary& r, bool inverse) {
    if (!turned) return;
    double f[kPairs];  // all on their way together
#pragma unroll
    for (int e = 0; e < kPairs; ++e) f[e] = r.turns[max(pair_of(e, r), 0)];
#pragma unroll
    for (int e = 0; e < kPairs; ++e) {
      double turn = static_cast<double>(position) * f[e];
      turn -= rint(turn);  // [-1/2, 1/2]: the float32 below is off by 2^-26 turns at most
      float s, q;
      sincospif(2.f * static_cast<float>(turn), &s, &q);
      co[e] = q * r.scale;
      si[e] = (inverse ? -s : s) * r.scale;
    }
  }
  struct Loaded {
    Chunk<T> a, b;
    T partner[kAligned ? 1 : 2 * c];
  };
  __device__ __forceinline__ Loaded load(const T* x, int chunks, const dmoe_rotary& r) const {
    Loaded l;
    l.a = c0 < chunks ? *reinterpret_cast<const Chunk<T>*>(x + c0 * c) : Chunk<T>{};
    l.b = c1 < chunks ? *reinterpret_cast<const Chunk<T>*>(x + c1 * c) : Chunk<T>{};
    if constexpr (!kAligned) {
      const int hr = r.rot_dim / 2;
#pragma unroll
      for (int e = 0; e < 2 * c; ++e) {
        const int d = c * c0 + e;
        l.partner[e] = T(0);
        if (turned && d < 2 * hr) l.partner[e] = x[d < hr ? d + hr : d - hr];
      }
    }
    return l;
  }
  __device__ __forceinline__ void turn(Loaded& l, const dmoe_rotary& r) const {
    if (!turned) return;
    float x[c], y[c];
    widen(l.a, x);
    widen(l.b, y);
    if constexpr (!kAligned) {
      const int hr = r.rot_dim / 2;
#pragma unroll
      for (int e = 0; e < 2 * c; ++e) {
        const int d = c * c0 + e;
        const float p = load_as_f32<T>(&l.partner[e]);
        float& v = e < c ? x[e] : y[e - c];
        v = d < 2 * hr ? v * co[e] + (d < hr ? -p : p) * si[e] : v;
      }
    } else if (r.interleaved) {
#pragma unroll
      for (int e = 0; e < c; ++e) {
        float* v = e < c / 2 ? x + 2 * e : y + 2 * e - c;
        const float v1 = v[0], v2 = v[1];
        const bool in = pair_of(e, r) >= 0;
        v[0] = in ? v1 * co[e] - v2 * si[e] : v1;
        v[1] = in ? v2 * co[e] + v1 * si[e] : v2;
      }
    } else {
#pragma unroll
      for (int e = 0; e < c; ++e) {
        const float v1 = x[e], v2 = y[e];
        x[e] = v1 * co[e] - v2 * si[e];
        y[e] = v2 * co[e] + v1 * si[e];
      }
    }
    l.a = narrow(x);
    l.b = narrow(y);
  }
};

bool aligned_pairs(const dmoe_rotary& r, int c) { return r.interleaved || !r.turns || r.rot_dim / 2 % c == 0; }

// n tokens of `heads` heads through the rotation; in(i, h) and out(i, h, j): a
// head's elements, and where its chunk j goes (nullptr: nowhere).  A row's
// chunks lie in one wave, whose loads of them are done when it stores: in
// place is safe.  Chunks from dim on, up to `padded`, are 0.
template <typename T, bool kAligned, typename Pos, typename In, typename Out>
__device__ __forceinline__ void rotate_rows(int n, int heads, int dim, int padded, const dmoe_rotary& r, bool inverse, Pos pos, In in, Out out) {
  constexpr int c = Chunk<T>::c;
  const int chunks = padded / c, units = (chunks + 1) / 2;
  const int log = units > 1 ? 32 - __builtin_clz(units - 1) : 0;  // lanes of a row: 2^log, at most 32
  const int row = threadIdx.x >> log, i = row % kTokens, step = (kThreads >> log) / kTokens;
  Unit<T, kAligned> u(threadIdx.x & ((1 << log) - 1), r);
  if (i >= n || u.c0 >= chunks) return;
  for (int h0 = row / kTokens; h0 < heads; h0 += step * kInFlight) {
    typename Unit<T, kAligned>::Loaded l[kInFlight];
#pragma unroll
    for (int y = 0; y < kInFlight; ++y) {
      const int h = h0 + y * step;
      if (h < heads) l[y] = u.load(in(i, h), dim / c, r);
    }
    if (h0 == row / kTokens) u.form(pos(i), r, inverse);  // while the first heads are on their way
#pragma unroll
    for (int y = 0; y < kInFlight; ++y) {
      const int h = h0 + y * step;
      if (h < heads) {
        u.turn(l[y], r);
        if (T* to = out(i, h, u.c0)) *reinterpret_cast<Chunk<T>*>(to) = l[y].a;
        if (u.c1 < chunks)
          if (T* to = out(i, h, u.c1)) *reinterpret_cast<Chunk<T>*>(to) = l[y].b;
      }
    }
  }
}

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
// kv head each, then (8 of the tile's new tokens, group of `heads` heads) of the
// queries and keys.
template <typename T, bool kAligned>
__global__ __launch_bounds__(kThreads) void append_kernel(AppendArgs a, int tiles, int heads, int groups) {
  constexpr int c = Chunk<T>::c;
  extern __shared__ float4 lds[];
  const int hkv = a.cache.n_kv_heads, dim = a.cache.head_dim;
  int tile0;
  const Seq q = find_tile(a, blockIdx.x, tiles, tile0);
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

// Heads of a workgroup that rotates.  One where that leaves few workgroups (a
// block of 32 tokens, 20 heads: 0.3 us less than with four); else as many as its lanes
// take at once (64 single tokens: 8.1 us with one, 6.2 with four; 46 sequences of 2, 24 heads of
// 32: 15.5 with one, 6.1), and as keep kGroups workgroups, so that angles are formed for
// as many heads as possible.  launched: token groups of the grid, some empty.
constexpr long kFill = 512, kGroups = 1024;
int heads_of_workgroup(long launched, long token_groups, int n_heads, int chunks) {
  int lanes = 1;  // of a row, as in rotate_rows
  while (lanes < (chunks + 1) / 2) lanes *= 2;
  int heads = 1;
  while (heads < n_heads && heads * lanes * kTokens < kThreads && launched * ((n_heads + heads - 1) / heads) > kFill) heads *= 2;
  while (heads < n_heads && token_groups * ((n_heads + 2 * heads - 1) / (2 * heads)) >= kGroups) heads *= 2;
  return heads < n_heads ? heads : n_heads;
}

template <typename T>
hipError_t append(const AppendArgs& a, hipStream_t s) {
  const int most = a.batch.max_new < a.batch.T ? a.batch.max_new : a.batch.T;
  const int tiles = (most + kTileTokens - 2) / kTileTokens + 1;
  const int turned = a.cache.n_kv_heads + (a.q ? a.n_heads : 0), dp = padded_dim(a.cache.head_dim);
  const size_t lds = static_cast<size_t>(kTileTokens) * dp * sizeof(T);
  // n tokens lie in at most n / 32 + 2 tiles, and at most `most` of a tile's positions are new
  const long each = static_cast<long>(a.batch.n_seqs) * tiles, counted = a.batch.T / kTileTokens + 2l * a.batch.n_seqs;
  const long grid_tiles = each < counted ? each : counted;
  const int sub = ((most < kTileTokens ? most : kTileTokens) + kTokens - 1) / kTokens;
  const int heads = heads_of_workgroup(grid_tiles * sub, (a.batch.T + kTokens - 1) / kTokens, turned, dp / Chunk<T>::c);
  const int groups = (turned + heads - 1) / heads;
  const dim3 grid(static_cast<unsigned>(grid_tiles), a.cache.n_kv_heads + sub * groups);
  if (aligned_pairs(a.rope, Chunk<T>::c))
    append_kernel<T, true><<<grid, kThreads, lds, s>>>(a, each <= counted ? tiles : 0, heads, groups);
  else
    append_kernel<T, false><<<grid, kThreads, lds, s>>>(a, each <= counted ? tiles : 0, heads, groups);
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
