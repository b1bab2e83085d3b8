// Device code of the kernels that rotate rows of heads, and of those that walk
// a batch's tokens by the tiles of 32 positions they lie in.
#pragma once

#include "cache.h"

namespace dmoe {
namespace rotary {

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

inline bool aligned_pairs(const dmoe_rotary& r, int c) { return r.interleaved || !r.turns || r.rot_dim / 2 % c == 0; }

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

// The x-th tile of 32 positions that a batch's tokens lie in, and its
// sequence, which load(i) tells: tokens from pos0 up to len (kBelow: those before position 0
// too).  `tiles` > 0: every sequence has that many, some of them empty;
// else those there are, counted by each wave, 64 sequences at a time.
template <bool kBelow, typename Load>
__device__ __forceinline__ Seq find_tile(int n_seqs, int x, int tiles, int& tile0, Load load) {
  Seq q;
  auto first_tile = [](const Seq& q) { return (kBelow ? q.pos0 : max(q.pos0, 0)) >> 5; };
  if (tiles > 0) {
    q = load(x / tiles);
    tile0 = (first_tile(q) + x % tiles) * kTileTokens;
    return q;
  }
  const int lane = threadIdx.x & 63;
  for (int i0 = 0; i0 < n_seqs; i0 += 64) {
    q = Seq{0, 0, 0, 0, 0};
    if (i0 + lane < n_seqs) q = load(i0 + lane);
    const int first = first_tile(q), n = q.len > (kBelow ? q.pos0 : max(q.pos0, 0)) ? ((q.len - 1) >> 5) - first + 1 : 0;
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

// Tiles of a grid that covers them: n tokens lie in at most n / 32 + 2, so every sequence has `each` at most, and all
// together `counted`.
struct TileGrid {
  long tiles;
  int each;  // find_tile's `tiles`
};
inline TileGrid tile_grid(const dmoe_batch& b) {
  const int most = b.max_new < b.T ? b.max_new : b.T;
  const int tiles = (most + kTileTokens - 2) / kTileTokens + 1;
  const long each = static_cast<long>(b.n_seqs) * tiles, counted = b.T / kTileTokens + 2l * b.n_seqs;
  return each <= counted ? TileGrid{each, tiles} : TileGrid{counted, 0};
}

// Heads of a workgroup that rotates.  One where that leaves few workgroups (a
// block of 32 tokens, 20 heads: 0.3 us less than with four); else as many as its lanes
// take at once (64 single tokens: 8.1 us with one, 6.2 with four; 46 sequences of 2, 24 heads of
// 32: 15.5 with one, 6.1), and as keep kGroups workgroups, so that angles are formed for
// as many heads as possible.  launched: token groups of the grid, some empty.
constexpr long kFill = 512, kGroups = 1024;
inline int heads_of_workgroup(long launched, long token_groups, int n_heads, int chunks) {
  int lanes = 1;  // of a row, as in rotate_rows
  while (lanes < (chunks + 1) / 2) lanes *= 2;
  int heads = 1;
  while (heads < n_heads && heads * lanes * kTokens < kThreads && launched * ((n_heads + heads - 1) / heads) > kFill) heads *= 2;
  while (heads < n_heads && token_groups * ((n_heads + 2 * heads - 1) / (2 * heads)) >= kGroups) heads *= 2;
  return heads < n_heads ? heads : n_heads;
}

}  // namespace rotary
}  // namespace dmoe
