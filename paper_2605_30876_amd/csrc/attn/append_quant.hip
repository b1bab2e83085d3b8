// The store of a step's keys and values into a cache of few bits, with the
// rotation and the quantisation fused, and the way back: rows of tokens as a
// cache of any format holds them.
//
// A lane takes eight consecutive elements of a token's head, so four lanes hold
// the 32 that share a scale: its maximum is two exchanges within them, loads of
// rows are contiguous and a quad's codes are one 16-byte chunk (or two) of the page.
// Keys and values lie in the page alike, token by token, so nothing is turned.
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

// Elements d .. d+7 of a head at x, rotated in binary64 with the token's (cos, sin) of
// every pair, rounded to float32 and from there to T: which of two codes a key next to their
// border takes does not depend on how a product was summed.
template <typename T>
__device__ __forceinline__ void rotate8(const T* x, int d, const dmoe_rotary& r, const double2* angle, float (&f)[8]) {
  const int rot = r.rot_dim, hr = rot / 2;
  if (d >= rot) return;
  if (r.interleaved) {
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
      if (d + e >= rot) continue;
      const double2 a = angle[(d + e) / 2];
      const double x1 = f[e], x2 = f[e + 1];
      f[e] = static_cast<float>(x1 * a.x - x2 * a.y);
      f[e + 1] = static_cast<float>(x2 * a.x + x1 * a.y);
    }
  } else if (hr % 8 == 0) {  // the eight are of one half
    const bool first = d < hr;
    float p[8];
    load8(x + (first ? d + hr : d - hr), p);
    const double2* a = angle + (first ? d : d - hr);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const double s = first ? -a[e].y : a[e].y;
      f[e] = static_cast<float>(static_cast<double>(f[e]) * a[e].x + static_cast<double>(p[e]) * s);
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int i = d + e;
      if (i >= rot) continue;
      const double2 a = angle[i < hr ? i : i - hr];
      const double p = load_as_f32<T>(x + (i < hr ? i + hr : i - hr));
      f[e] = static_cast<float>(static_cast<double>(f[e]) * a.x + p * (i < hr ? -a.y : a.y));
    }
  }
  round8(f, x);
}

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

// blockIdx.x: tile of 32 positions.  blockIdx.y: 8 of the tile's new tokens, and
// of those the keys and values of `kv_heads` heads, or `heads` heads of the queries.
template <typename T, int kK, int kV, bool kAligned>
__global__ __launch_bounds__(kThreads) void append_quant_kernel(AppendArgs a, int tiles, int heads, int groups, int kv_heads, int kv_groups) {
  extern __shared__ double2 angle[];  // [kTokens][rot_dim / 2]: cos and sin
  const int hkv = a.cache.n_kv_heads, dim = a.cache.head_dim;
  int tile0;
  const Seq q = find_tile<false>(a.batch.n_seqs, blockIdx.x, tiles, tile0, [&](int i) { return load_seq(a.cache, a.batch, i); });
  const int sub = blockIdx.y / (kv_groups + groups), y = blockIdx.y - sub * (kv_groups + groups);
  const int p0 = max(max(q.pos0, 0), tile0) + sub * kTokens, p1 = min(min(q.len, tile0 + kTileTokens), p0 + kTokens), n = p1 - p0;
  if (n <= 0) return;
  const long t0 = q.row0 + (p0 - q.pos0);
  const dmoe_rotary r = a.rope;
  if (y >= kv_groups) {
    const int h0 = (y - kv_groups) * heads;
    rotate_rows<T, kAligned>(
        n, min(heads, a.n_heads - h0), dim, dim, r, false, [&](int i) { return p0 + i; },
        [&](int i, int h) { return static_cast<const T*>(a.q) + (t0 + i) * a.q_stride + (h0 + h) * dim; },
        [&](int i, int h, int j) { return static_cast<T*>(a.q_out) + (t0 + i) * a.q_out_stride + (h0 + h) * dim + j * Chunk<T>::c; });
    return;
  }
  const int pt = a.cache.page_tokens, dp = padded_dim(dim), tpp = pt / kTileTokens;
  const int page = a.cache.table[static_cast<long>(q.slot) * a.cache.max_pages + p0 / pt];
  if (page < 0 || page >= a.cache.n_pages) return;
  const int hr = r.turns ? r.rot_dim / 2 : 0;
  for (int x = threadIdx.x; x < n * hr; x += kThreads) {
    const int i = x / hr;
    double turn = static_cast<double>(p0 + i) * r.turns[x - i * hr], s, c;
    turn -= rint(turn);
    sincospi(2.0 * turn, &s, &c);
    angle[x] = make_double2(c * static_cast<double>(r.scale), s * static_cast<double>(r.scale));
  }
  __syncthreads();
  const int h0 = y * kv_heads, hs = min(kv_heads, hkv - h0), lanes = dp / 8;
  // the tile of kv head 0
  const long tile = ((static_cast<long>(a.layer) * a.cache.n_pages + page) * hkv) * tpp + p0 % pt / kTileTokens;
  const int each = n * hs * lanes;
  for (int x = threadIdx.x; x < 2 * each; x += kThreads) {
    const bool values = x >= each;
    const int u = values ? x - each : x, d = u % lanes * 8, h = h0 + u / lanes % hs, i = u / lanes / hs;
    const T* row = (values ? static_cast<const T*>(a.v) + (t0 + i) * a.v_stride : static_cast<const T*>(a.k) + (t0 + i) * a.k_stride) +
                   static_cast<long>(h) * dim;
    float f[8] = {};
    if (d < dim) load8(row + d, f);
    const int at = (p0 + i) % kTileTokens;
    const long place = tile + static_cast<long>(h) * tpp;
    if (values) {
      put8<kV>(static_cast<uint8_t*>(a.cache.v) + place * quant_tile(kV, dp), dp, at, d, f);
    } else {
      if (hr > 0 && d < dim) rotate8(row, d, r, angle + i * hr, f);
      put8<kK>(static_cast<uint8_t*>(a.cache.k) + place * quant_tile(kK, dp), dp, at, d, f);
    }
  }
}

template <typename T, int kK, int kV>
hipError_t append_quant(const AppendArgs& a, hipStream_t s) {
  const int most = a.batch.max_new < a.batch.T ? a.batch.max_new : a.batch.T;
  const int dp = padded_dim(a.cache.head_dim), hkv = a.cache.n_kv_heads, nq = a.q ? a.n_heads : 0;
  const TileGrid tg = tile_grid(a.batch);
  const int sub = ((most < kTileTokens ? most : kTileTokens) + kTokens - 1) / kTokens;
  const int heads = nq ? heads_of_workgroup(tg.tiles * sub, (a.batch.T + kTokens - 1) / kTokens, nq, dp / Chunk<T>::c) : 1;
  const int groups = (nq + heads - 1) / heads;
  // as many heads to one set of angles as leave workgroups for the device
  int kv_heads = 1;
  while (kv_heads < hkv && tg.tiles * sub * ((hkv + kv_heads - 1) / kv_heads) > kFill) kv_heads *= 2;
  kv_heads = kv_heads < hkv ? kv_heads : hkv;
  const int kv_groups = (hkv + kv_heads - 1) / kv_heads;
  const dim3 grid(static_cast<unsigned>(tg.tiles), sub * (kv_groups + groups));
  const size_t lds = a.rope.turns ? static_cast<size_t>(kTokens) * (a.rope.rot_dim / 2) * sizeof(double2) : 0;
  if (aligned_pairs(a.rope, Chunk<T>::c))
    append_quant_kernel<T, kK, kV, true><<<grid, kThreads, lds, s>>>(a, tg.each, heads, groups, kv_heads, kv_groups);
  else
    append_quant_kernel<T, kK, kV, false><<<grid, kThreads, lds, s>>>(a, tg.each, heads, groups, kv_heads, kv_groups);
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
    *reinterpret_cast<f32x4*>(p + i) = f32x4{static_cast<float>(x[i]), static_cast<float>(x[i + 1]), static_cast<float>(x[i + 2]), static_cast<float>(x[i + 3])};
}
__device__ __forceinline__ void store8(bf16_t* p, const bf16x8& x) { *reinterpret_cast<bf16x8*>(p) = x; }

// Elements d .. d+7 of token r of a tile, kept in the layout of keys (kValues: of values)
// with kBits bits (0: as T), to a row.
template <typename T, int kBits, bool kValues>
__device__ __forceinline__ void get8(const uint8_t* tile, int dp, int r, int d, T* to) {
  if constexpr (kBits > 0) {
    const Codes<kBits> c = *reinterpret_cast<const Codes<kBits>*>(tile + code_at<kBits>(r, d));
    store8(to, decode<kBits>(c.w, scale_of(tile[scale_at<kBits>(dp, r) + d / kGroup])));
  } else {
    constexpr int c = Chunk<T>::c;
    const T* t = reinterpret_cast<const T*>(tile);
#pragma unroll
    for (int x = 0; x < 8; x += c) {
      Chunk<T> v;
      if constexpr (!kValues) {
        v = *reinterpret_cast<const Chunk<T>*>(t + key_chunk<c>(r, (d + x) / c));
      } else {
#pragma unroll
        for (int e = 0; e < c; ++e) v.v[e] = t[value_chunk<c>(d + x + e, r / (2 * c), r / 4 % 2) + r % (2 * c) / 8 * 4 + r % 4];
      }
      *reinterpret_cast<Chunk<T>*>(to + x) = v;
    }
  }
}

// blockIdx.x: tile of 32 positions.  blockIdx.y: keys or values, `heads` heads of them.
template <typename T, int kK, int kV>
__global__ __launch_bounds__(kThreads) void read_kernel(ReadArgs a, int tiles, int heads, int groups) {
  const int hkv = a.cache.n_kv_heads, dim = a.cache.head_dim;
  auto load = [&](int i) {
    Seq s = load_seq(a.cache, a.batch, i);
    if (a.starts) s.pos0 = min(max(a.starts[i], 0), a.cache.max_pages * a.cache.page_tokens);
    s.len = s.pos0 + s.n;  // the end of what is read
    return s;
  };
  int tile0;
  const Seq q = find_tile<true>(a.batch.n_seqs, blockIdx.x, tiles, tile0, load);
  const int p0 = max(q.pos0, tile0), p1 = min(q.len, tile0 + kTileTokens), n = p1 - p0;
  if (n <= 0) return;
  const long t0 = q.row0 + (p0 - q.pos0);
  const bool values = a.k == nullptr || (a.v != nullptr && static_cast<int>(blockIdx.y) >= groups);
  const int h0 = static_cast<int>(blockIdx.y) % groups * heads, hs = min(heads, hkv - h0), lanes = dim / 8;
  const int pt = a.cache.page_tokens, dp = padded_dim(dim), tpp = pt / kTileTokens;
  const int len = min(max(a.cache.lens[q.slot], 0), a.cache.max_pages * pt);  // tokens from here on are not there
  const int page = p0 >= 0 && p0 < len ? a.cache.table[static_cast<long>(q.slot) * a.cache.max_pages + p0 / pt] : -1;
  const bool held = page >= 0 && page < a.cache.n_pages;
  const long tile = ((static_cast<long>(a.layer) * a.cache.n_pages + page) * hkv) * tpp + max(p0, 0) % pt / kTileTokens;
  auto copy = [&](const uint8_t* pool, T* out, long stride, auto bits, auto is_value) {
    constexpr int kBits = decltype(bits)::value;
    const int size = kBits ? quant_tile(kBits, dp) : kTileTokens * dp * static_cast<int>(sizeof(T));
    for (int x = threadIdx.x; x < n * hs * lanes; x += kThreads) {
      const int d = x % lanes * 8, h = h0 + x / lanes % hs, i = x / lanes / hs;
      T* to = out + (t0 + i) * stride + static_cast<long>(h) * dim + d;
      if (held && p0 + i < len)
        get8<T, kBits, decltype(is_value)::value>(pool + (tile + static_cast<long>(h) * tpp) * size, dp, (p0 + i) & 31, d, to);
      else
        store8(to, bf16x8{});
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
  const int hkv = a.cache.n_kv_heads;
  int heads = 1;
  while (heads < hkv && tg.tiles * ((hkv + heads - 1) / heads) > kFill) heads *= 2;
  heads = heads < hkv ? heads : hkv;
  const int groups = (hkv + heads - 1) / heads;
  const dim3 grid(static_cast<unsigned>(tg.tiles), groups * (a.k && a.v ? 2 : 1));
  read_kernel<T, kK, kV><<<grid, kThreads, 0, s>>>(a, tg.each, heads, groups);
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
