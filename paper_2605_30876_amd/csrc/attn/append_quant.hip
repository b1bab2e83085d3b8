// The store of a step's keys and values into a cache of few bits, with the
// rotation and the quantisation fused, and the way back: rows of tokens as a
// cache of any format holds them.
//
// A lane takes eight consecutive elements of a token's head, so four lanes hold
// the 32 that share a scale: its maximum is two exchanges within them, loads of
// rows are contiguous and a quad's codes are one 16-byte chunk (or two) of the page.
// Keys and values lie in the page alike, token by token, so nothing is turned.
// Both ways are bound by memory: prompts of 11753 tokens (32 heads of 128 with queries, 8 of keys in 8 bits and values
// in 4) are stored and read back in 73 us (326 MB, 4.5 TB/s), 48 sequences of 89,941 tokens and 8 heads read back from 4 bits in 104
// us (466 MB, 4.5 TB/s), where a large copy reaches 5.2.  A block of 32 tokens is bound by its latency: 4.5 and 3.5 us alone, 7.0
// together in a graph.  Further from the bytes: rotated halves in the store (Turn8), 90 us for prompts of 263 MB; rows of
// float32 read from 4 bits, 336 for 743 MB; a plain cache's values, whose elements lie apart and are loaded one by one, with its
// keys 330 for 972 MB of bf16, 549 for 2.1 GB of float32.
#include "quant.h"
#include "rotate.h"

namespace dmoe {

namespace {

using namespace rotary;
using namespace quant;

// Eight elements of a row, in float32.
__device__ __forceinline__ void load8(const float* p, float (&f)[8]) {
  const f32x4 a = *reinterpret_cast<const f32x4*>(p), b = *reinterpret_cast<const f32x4*>(p + 4);
#pragma unroll
  for (int e = 0; e < 4; ++e) f[e] = a[e], f[4 + e] = b[e];
}
__device__ __forceinline__ void load8(const bf16_t* p, float (&f)[8]) { widen(*reinterpret_cast<const Chunk<bf16_t>*>(p), f); }
__device__ __forceinline__ void round8(float (&)[8], const float*) {}
__device__ __forceinline__ void round8(float (&f)[8], const bf16_t*) {
  const Chunk<bf16_t> c = narrow(f);
  widen(c, f);
}

// The largest of the four lanes of a quad.
__device__ __forceinline__ uint32_t quad_max(uint32_t v) {
  v = max(v, static_cast<uint32_t>(__builtin_amdgcn_mov_dpp(v, 0xB1, 0xF, 0xF, true)));  // lanes 1, 0, 3, 2
  return max(v, static_cast<uint32_t>(__builtin_amdgcn_mov_dpp(v, 0x4E, 0xF, 0xF, true)));  // lanes 2, 3, 0, 1
}

// Elements d .. d+7 of a head at x, f, rotated with the token's (cos, sin) of every pair: own cos -+ partner sin.  Queries
// in float32, as rope.hip does; keys in binary64, rounded to float32 and from there to T: which of two codes a key next to
// their border takes does not depend on how a product was summed.  Halves cost more than adjacent pairs: the partners are loaded
// again, and a lane holds eight angles instead of four (177 registers for bf16 against 95: two waves a SIMD, not five).
enum Pairs { kNoPairs, kAdjacent, kHalves, kAnyHalves };  // kHalves: eight elements are of one half
template <typename T, typename A, Pairs kPairs>
struct Turn8 {
  static constexpr int kAngles = kPairs == kNoPairs ? 1 : kPairs == kAdjacent ? 4 : 8;
  A c[kAngles], s[kAngles];
  float p[8];  // partners, negated in the first half
  // loads only; angle: pairs of (cos, sin) of the token
  __device__ __forceinline__ void load(const T* x, int d, int rot, const A* angle) {
    const int hr = rot / 2;
    if (kPairs == kNoPairs || d >= rot) return;
#pragma unroll
    for (int e = 0; e < kAngles; ++e) {
      int i = kPairs == kAdjacent ? d / 2 + e : d + e;
      if (kPairs != kAdjacent) i = i < hr ? i : i - hr;
      if (kPairs != kHalves) i = min(i, hr - 1);
      c[e] = angle[2 * i];
      s[e] = angle[2 * i + 1];
    }
    if constexpr (kPairs == kHalves) {
      load8(x + (d < hr ? d + hr : d - hr), p);
#pragma unroll
      for (int e = 0; e < 8; ++e) s[e] = d < hr ? -s[e] : s[e];
    } else if constexpr (kPairs == kAnyHalves) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int i = min(d + e, rot - 1);
        p[e] = load_as_f32<T>(x + (i < hr ? i + hr : i - hr));
        s[e] = i < hr ? -s[e] : s[e];
      }
    }
  }
  static __device__ __forceinline__ float one(A x, A c, A y, A s) {
#pragma clang fp contract(off)  // else the rounding to float32 and the one to T that follows may become one
    return static_cast<float>(fma(x, c, y * s));
  }
  __device__ __forceinline__ void turn(float (&f)[8], int d, int rot) const {
    if (kPairs == kNoPairs || d >= rot) return;
    if constexpr (kPairs == kAdjacent) {
#pragma unroll
      for (int e = 0; e < 8; e += 2) {
        const A x1 = f[e], x2 = f[e + 1];
        const bool in = d + e < rot;
        const float y1 = one(x1, c[e / 2], -x2, s[e / 2]), y2 = one(x2, c[e / 2], x1, s[e / 2]);
        f[e] = in ? y1 : f[e];
        f[e + 1] = in ? y2 : f[e + 1];
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float y = one(f[e], c[e], p[e], s[e]);
        f[e] = kPairs == kHalves || d + e < rot ? y : f[e];
      }
    }
    round8(f, static_cast<const T*>(nullptr));
  }
};

// Eight elements of a group into the tile at `to`.
template <int kBits>
__device__ __forceinline__ void put8(uint8_t* to, int dp, int r, int d, const float (&f)[8]) {
  uint32_t top = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(f[e]) & 0x7fffffffu);
  const int b = scale_byte<kBits>(quad_max(top));
  const Codes<kBits> c = encode<kBits>(f, b);
  *reinterpret_cast<Codes<kBits>*>(to + code_at<kBits>(r, d)) = c;
  if (d % kGroup == 0) to[scale_at<kBits>(dp, r) + d / kGroup] = static_cast<uint8_t>(b);
}

// Rows that are written once go past the caches: through them the prompts' store and read took 83 us, so 73, the read of 48
// sequences 110, so 101.  Codes go through them: a page's chunks of 16 bytes are written by many lanes (past them the store alone 59.5 us, so 44, with
// the rows in the memory-side cache).
template <typename V>
__device__ __forceinline__ void store_past(const V& x, V* p) {
  __builtin_nontemporal_store(x, p);
}
__device__ __forceinline__ void store_row8(float* p, const float (&f)[8]) {
  store_past(f32x4{f[0], f[1], f[2], f[3]}, reinterpret_cast<f32x4*>(p));
  store_past(f32x4{f[4], f[5], f[6], f[7]}, reinterpret_cast<f32x4*>(p + 4));
}
__device__ __forceinline__ void store_row8(bf16_t* p, const float (&f)[8]) {
  store_past(__builtin_bit_cast(bf16x8, narrow(f)), reinterpret_cast<bf16x8*>(p));
}

// What a workgroup takes of 8 tokens: `heads` heads of the queries, or the keys and values of `kv_heads`.
struct AppendShape {
  int tiles;                       // find_tile's
  int heads, groups, kv_heads, kv_groups;
  int log;                         // lanes of a row of a head: 2^log, eight elements each
  FastDiv by_heads, by_kv_heads;
};

// blockIdx.x: tile of 32 positions.  blockIdx.y: 8 of the tile's new tokens, and of those the keys and values, or
// queries, of some heads.  The angles' cos and sin are formed once a workgroup, in LDS (in binary64 for keys, where they cost more
// than the row: with one in each lane's registers and rows taken by head, the prompts' store took 77 us, so 44, with their
// rows in the memory-side cache; 58 without); rows are taken in the order they lie in.  Loading the first of them before the angles
// are formed took registers, and longer: 76 us with the read, so 74; a block 57.8, so 56.1.
template <typename T, int kK, int kV, Pairs kPairs>
__global__ __launch_bounds__(kThreads) void append_quant_kernel(AppendArgs a, AppendShape sh) {
  extern __shared__ double angles[];  // [kTokens][rot_dim / 2][2]: cos and sin (floats for queries)
  const int hkv = a.cache.n_kv_heads, dim = a.cache.head_dim;
  int tile0;
  const Seq q = find_tile<false>(a.batch.n_seqs, blockIdx.x, sh.tiles, tile0, [&](int i) { return load_seq(a.cache, a.batch, i); });
  const int sub = blockIdx.y / (sh.kv_groups + sh.groups), y = blockIdx.y - sub * (sh.kv_groups + sh.groups);
  const int p0 = max(max(q.pos0, 0), tile0) + sub * kTokens, p1 = min(min(q.len, tile0 + kTileTokens), p0 + kTokens), n = p1 - p0;
  if (n <= 0) return;
  const long t0 = q.row0 + (p0 - q.pos0);
  const dmoe_rotary& r = a.rope;
  const int rot = kPairs == kNoPairs ? 0 : r.rot_dim, hr = rot / 2;
  const bool queries = y >= sh.kv_groups;
  const int pt = a.cache.page_tokens, dp = padded_dim(dim), tpp = pt / kTileTokens;
  int page = 0;
  if (!queries) {
    page = a.cache.table[static_cast<long>(q.slot) * a.cache.max_pages + p0 / pt];
    if (page < 0 || page >= a.cache.n_pages) return;
  }
  float* fangles = reinterpret_cast<float*>(angles);
  for (int x = threadIdx.x; kPairs != kNoPairs && x < n * hr; x += kThreads) {
    const int i = x / max(hr, 1);
    double turn = static_cast<double>(p0 + i) * r.turns[x - i * hr];
    turn -= rint(turn);
    if (queries) {  // as rope.hip forms them
      float s, c;
      sincospif(2.f * static_cast<float>(turn), &s, &c);
      fangles[2 * x] = c * r.scale;
      fangles[2 * x + 1] = s * r.scale;
    } else {
      double s, c;
      sincospi(2.0 * turn, &s, &c);
      angles[2 * x] = c * static_cast<double>(r.scale);
      angles[2 * x + 1] = s * static_cast<double>(r.scale);
    }
  }
  __syncthreads();
  // rows of queries a thread loads before it stores (bf16, 11753 prompt tokens: 62 us with one, 58.5 with two, 56.4 with
  // four; fp32, 1601: 11 with two, 15 with four, for the registers)
  constexpr int kFly = sizeof(T) == 2 ? 4 : 2;
  const int d = (threadIdx.x & ((1 << sh.log) - 1)) * 8, first = threadIdx.x >> sh.log, step = kThreads >> sh.log;
  if (queries) {
    if (d >= dim) return;
    const int h0 = (y - sh.kv_groups) * sh.heads, hs = min(sh.heads, a.n_heads - h0);
    const bool even = hs == sh.heads;  // the last group of heads may be smaller
    const T* in = static_cast<const T*>(a.q) + t0 * a.q_stride + static_cast<long>(h0) * dim + d;
    T* out = static_cast<T*>(a.q_out) + t0 * a.q_out_stride + static_cast<long>(h0) * dim + d;
    const int rows = n * hs;
    for (int row = first; row < rows; row += step * kFly) {
      float f[kFly][8];
      Turn8<T, float, kPairs> t[kFly];
#pragma unroll
      for (int x = 0; x < kFly; ++x) {
        const int rx = min(row + x * step, rows - 1), i = even ? sh.by_heads.of(rx) : rx / hs, h = rx - i * hs;
        const T* p = in + i * a.q_stride + h * dim;
        load8(p, f[x]);
        t[x].load(p - d, d, rot, fangles + 2 * i * hr);
      }
#pragma unroll
      for (int x = 0; x < kFly; ++x) {
        const int rx = row + x * step, i = even ? sh.by_heads.of(rx) : rx / hs, h = rx - i * hs;
        if (rx >= rows) break;
        t[x].turn(f[x], d, rot);
        store_row8(out + i * a.q_out_stride + h * dim, f[x]);
      }
    }
    return;
  }
  if (d >= dp) return;
  const int h0 = y * sh.kv_heads, hs = min(sh.kv_heads, hkv - h0);
  const bool even = hs == sh.kv_heads;
  // the tile of the first head
  const long tile = ((static_cast<long>(a.layer) * a.cache.n_pages + page) * hkv + h0) * tpp + p0 % pt / kTileTokens;
  uint8_t* kt = static_cast<uint8_t*>(a.cache.k) + tile * quant_tile(kK, dp);
  uint8_t* vt = static_cast<uint8_t*>(a.cache.v) + tile * quant_tile(kV, dp);
  const T* kin = static_cast<const T*>(a.k) + t0 * a.k_stride + static_cast<long>(h0) * dim + d;
  const T* vin = static_cast<const T*>(a.v) + t0 * a.v_stride + static_cast<long>(h0) * dim + d;
  for (int row = first; row < n * hs; row += step) {
    const int i = even ? sh.by_kv_heads.of(row) : row / hs, h = row - i * hs, at = (p0 + i) % kTileTokens;
    float k[8] = {}, v[8] = {};
    Turn8<T, double, kPairs> t;
    if (d < dim) {
      const T* p = kin + i * a.k_stride + h * dim;
      load8(p, k);
      load8(vin + i * a.v_stride + h * dim, v);
      t.load(p - d, d, rot, angles + 2 * i * hr);
      t.turn(k, d, rot);
    }
    put8<kK>(kt + static_cast<long>(h * tpp) * quant_tile(kK, dp), dp, at, d, k);
    put8<kV>(vt + static_cast<long>(h * tpp) * quant_tile(kV, dp), dp, at, d, v);
  }
}

// Heads of a workgroup: one where that leaves few workgroups, else as many as leave kFill, so that angles serve many heads.
int heads_each(long launched, int n_heads) {
  int heads = 1;
  while (heads < n_heads && launched * ((n_heads + heads - 1) / heads) > kFill) heads *= 2;
  return heads < n_heads ? heads : n_heads;
}

template <typename T, int kK, int kV>
hipError_t append_quant(const AppendArgs& a, hipStream_t s) {
  const int most = a.batch.max_new < a.batch.T ? a.batch.max_new : a.batch.T;
  const int dp = padded_dim(a.cache.head_dim), hkv = a.cache.n_kv_heads, nq = a.q ? a.n_heads : 0;
  const TileGrid tg = tile_grid(a.batch);
  const int sub = ((most < kTileTokens ? most : kTileTokens) + kTokens - 1) / kTokens;
  AppendShape sh;
  sh.tiles = tg.each;
  sh.heads = nq ? heads_each(tg.tiles * sub, nq) : 1;
  sh.groups = (nq + sh.heads - 1) / sh.heads;
  sh.kv_heads = heads_each(tg.tiles * sub, hkv);
  sh.kv_groups = (hkv + sh.kv_heads - 1) / sh.kv_heads;
  sh.log = dp <= 32 ? 2 : dp <= 64 ? 3 : dp <= 128 ? 4 : 5;
  sh.by_heads = fast_div(sh.heads);
  sh.by_kv_heads = fast_div(sh.kv_heads);
  const dim3 grid(static_cast<unsigned>(tg.tiles), sub * (sh.kv_groups + sh.groups));
  const size_t lds = a.rope.turns ? static_cast<size_t>(kTokens) * a.rope.rot_dim * sizeof(double) : 0;
  auto run = [&](auto kernel) { kernel<<<grid, kThreads, lds, s>>>(a, sh); };
  if (!a.rope.turns)
    run(append_quant_kernel<T, kK, kV, kNoPairs>);
  else if (a.rope.interleaved)
    run(append_quant_kernel<T, kK, kV, kAdjacent>);
  else if (a.rope.rot_dim % 16 == 0)
    run(append_quant_kernel<T, kK, kV, kHalves>);
  else
    run(append_quant_kernel<T, kK, kV, kAnyHalves>);
  return hipGetLastError();
}

template <typename T>
hipError_t append_quant_type(const AppendArgs& a, hipStream_t s) {
  switch (a.cache.format) {
    case DMOE_KV_FP8: return append_quant<T, 8, 8>(a, s);
    case DMOE_KV_FP4: return append_quant<T, 4, 4>(a, s);
    default: return append_quant<T, 8, 4>(a, s);
  }
}

// ---- reading back -----------------------------------------------------------

__device__ __forceinline__ void store8(float* p, const bf16x8& x) {
#pragma unroll
  for (int i = 0; i < 8; i += 4)
    store_past(f32x4{static_cast<float>(x[i]), static_cast<float>(x[i + 1]), static_cast<float>(x[i + 2]), static_cast<float>(x[i + 3])}, reinterpret_cast<f32x4*>(p + i));
}
__device__ __forceinline__ void store8(bf16_t* p, const bf16x8& x) { store_past(x, reinterpret_cast<bf16x8*>(p)); }

// Elements d .. d+7 of token r of a tile, kept in the layout of keys (kValues: of values)
// with kBits bits (0: as T): loaded, then stored to a row.
template <typename T, int kBits, bool kValues>
struct Get8 {
  Codes<kBits> c;
  uint8_t s;
  __device__ __forceinline__ void load(const uint8_t* tile, int dp, int r, int d) {
    c = *reinterpret_cast<const Codes<kBits>*>(tile + code_at<kBits>(r, d));
    s = tile[scale_at<kBits>(dp, r) + d / kGroup];
  }
  __device__ __forceinline__ void store(T* to, bool there) const {
    const bf16x8 x = decode<kBits>(c.w, scale_of(s));
    store8(to, there ? x : bf16x8{});
  }
};
template <typename T, bool kValues>
struct Get8<T, 0, kValues> {
  static constexpr int c = Chunk<T>::c;
  typedef T Vec __attribute__((ext_vector_type(16 / sizeof(T))));
  Vec v[8 / c];
  __device__ __forceinline__ void load(const uint8_t* tile, int, int r, int d) {
    const T* t = reinterpret_cast<const T*>(tile);
#pragma unroll
    for (int x = 0; x < 8 / c; ++x) {
      if constexpr (!kValues) {
        v[x] = *reinterpret_cast<const Vec*>(t + key_chunk<c>(r, d / c + x));
      } else {
#pragma unroll
        for (int e = 0; e < c; ++e) v[x][e] = t[value_chunk<c>(d + c * x + e, r / (2 * c), r / 4 % 2) + r % (2 * c) / 8 * 4 + r % 4];
      }
    }
  }
  __device__ __forceinline__ void store(T* to, bool there) const {
#pragma unroll
    for (int x = 0; x < 8 / c; ++x) store_past(there ? v[x] : Vec{}, reinterpret_cast<Vec*>(to) + x);
  }
};

// What a workgroup of the read takes: `heads` heads of a tile's tokens.
struct ReadShape {
  int tiles, heads, groups;  // tiles: find_tile's
  int log;                   // lanes of a row of a head: 2^log, eight elements each
  FastDiv by_heads, by_last; // by_last: of the last group, which may be smaller
};

// blockIdx.x: tile of 32 positions.  blockIdx.y: keys or values, some heads of them.  Rows are written in the order they lie in.
template <typename T, int kK, int kV>
__global__ __launch_bounds__(kThreads) void read_kernel(ReadArgs a, ReadShape sh) {
  const int hkv = a.cache.n_kv_heads, dim = a.cache.head_dim;
  auto load = [&](int i) {
    Seq s = load_seq(a.cache, a.batch, i);
    if (a.starts) s.pos0 = min(max(a.starts[i], 0), a.cache.max_pages * a.cache.page_tokens);
    s.len = s.pos0 + s.n;  // the end of what is read
    return s;
  };
  int tile0;
  const Seq q = find_tile<true>(a.batch.n_seqs, blockIdx.x, sh.tiles, tile0, load);
  const int p0 = max(q.pos0, tile0), p1 = min(q.len, tile0 + kTileTokens), n = p1 - p0;
  const int d = (threadIdx.x & ((1 << sh.log) - 1)) * 8, first = threadIdx.x >> sh.log, step = kThreads >> sh.log;
  if (n <= 0 || d >= dim) return;
  const long t0 = q.row0 + (p0 - q.pos0);
  const bool values = a.k == nullptr || (a.v != nullptr && static_cast<int>(blockIdx.y) >= sh.groups);
  const int y = static_cast<int>(blockIdx.y) - (values && a.k ? sh.groups : 0);
  const int h0 = y * sh.heads, hs = min(sh.heads, hkv - h0);
  const FastDiv by = hs == sh.heads ? sh.by_heads : sh.by_last;
  const int pt = a.cache.page_tokens, dp = padded_dim(dim), tpp = pt / kTileTokens;
  const int len = min(max(a.cache.lens[q.slot], 0), a.cache.max_pages * pt);  // tokens from here on are not there
  int page = p0 >= 0 && p0 < len ? a.cache.table[static_cast<long>(q.slot) * a.cache.max_pages + p0 / pt] : -1;
  const bool held = page >= 0 && page < a.cache.n_pages;
  page = held ? page : 0;  // of no page: some tile of the pool, and 0
  // the tile of the first head
  const long tile = ((static_cast<long>(a.layer) * a.cache.n_pages + page) * hkv + h0) * tpp + max(p0, 0) % pt / kTileTokens;
  const int rows = n * hs;
  auto copy = [&](const uint8_t* pool, T* out, long stride, auto bits, auto is_value) {
    constexpr int kBits = decltype(bits)::value;
    // rows a thread loads before it stores (4 bits, 48 sequences: 119 us with one, 109 with two, 101 with four, 102 with eight)
    constexpr int kFly = kBits ? 4 : decltype(is_value)::value ? 1 : 2;
    const int size = kBits ? quant_tile(kBits, dp) : kTileTokens * dp * static_cast<int>(sizeof(T));
    const uint8_t* from = pool + tile * size;
    T* to = out + t0 * stride + static_cast<long>(h0) * dim + d;
    for (int row = first; row < rows; row += step * kFly) {
      Get8<T, kBits, decltype(is_value)::value> x[kFly];
#pragma unroll
      for (int j = 0; j < kFly; ++j) {
        const int rj = min(row + j * step, rows - 1), i = by.of(rj);
        x[j].load(from + static_cast<long>((rj - i * hs) * tpp) * size, dp, (p0 + i) & 31, d);
      }
#pragma unroll
      for (int j = 0; j < kFly; ++j) {
        const int rj = row + j * step, i = by.of(rj);
        if (rj < rows) x[j].store(to + i * stride + (rj - i * hs) * dim, held && p0 + i < len);
      }
    }
  };
  if (values)
    copy(static_cast<const uint8_t*>(a.cache.v), static_cast<T*>(a.v), a.v_stride, std::integral_constant<int, kV>(), std::true_type());
  else
    copy(static_cast<const uint8_t*>(a.cache.k), static_cast<T*>(a.k), a.k_stride, std::integral_constant<int, kK>(), std::false_type());
}

template <typename T, int kK, int kV>
hipError_t read(const ReadArgs& a, hipStream_t s) {
  const TileGrid tg = tile_grid(a.batch);
  const int hkv = a.cache.n_kv_heads, dp = padded_dim(a.cache.head_dim);
  ReadShape sh;
  sh.tiles = tg.each;
  sh.heads = heads_each(tg.tiles, hkv);
  sh.groups = (hkv + sh.heads - 1) / sh.heads;
  sh.log = dp <= 32 ? 2 : dp <= 64 ? 3 : dp <= 128 ? 4 : 5;
  sh.by_heads = fast_div(sh.heads);
  sh.by_last = fast_div(hkv - (sh.groups - 1) * sh.heads);
  const dim3 grid(static_cast<unsigned>(tg.tiles), sh.groups * (a.k && a.v ? 2 : 1));
  read_kernel<T, kK, kV><<<grid, kThreads, 0, s>>>(a, sh);
  return hipGetLastError();
}

template <typename T>
hipError_t read_type(const ReadArgs& a, hipStream_t s) {
  switch (a.cache.format) {
    case DMOE_KV_PLAIN: return read<T, 0, 0>(a, s);
    case DMOE_KV_FP8: return read<T, 8, 8>(a, s);
    case DMOE_KV_FP4: return read<T, 4, 4>(a, s);
    default: return read<T, 8, 4>(a, s);
  }
}

}  // namespace

hipError_t launch_append_quant(const AppendArgs& a, hipStream_t s) {
  return a.cache.dt == DMOE_BF16 ? append_quant_type<bf16_t>(a, s) : append_quant_type<float>(a, s);
}

hipError_t launch_read(const ReadArgs& a, hipStream_t s) {
  return a.cache.dt == DMOE_BF16 ? read_type<bf16_t>(a, s) : read_type<float>(a, s);
}

}  // namespace dmoe
