// Attention of the step's new tokens over the paged cache.
//
// Per kv head, rows are (token, query head of the group) pairs, 32 to a wave.
// A wave forms the transposed scores of 32 keys x 32 rows, S^T = K Q^T, on the
// matrix cores: in the 32x32 result a lane holds 16 keys of ONE row (row
// lane%32; key 8j + 4(lane/32) + t in register 4j + t), so the softmax
// statistics of a row are a loop over registers and one exchange between the
// two halves of the wave, and the exponentials are already the B operand of
// O^T += V^T P^T: the cache stores the values' tokens in exactly the order of
// those registers (value_chunk), so probabilities never cross lanes and never
// touch LDS.  Softmax is online in base 2 (running maximum m and sum l); O and l
// are rescaled only when a row's maximum grew by more than 2^kLazy since the last
// time, which keeps every term below 2^kLazy and leaves the result unchanged.
#pragma once

#include <type_traits>

#include "cache.h"

namespace dmoe {
namespace attn {

typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr float kLazy = 8.f;
constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;

__device__ __forceinline__ void store4(float* p, const f32x4& v) { *reinterpret_cast<f32x4*>(p) = v; }
__device__ __forceinline__ void store4(bf16_t* p, const f32x4& v) {
  typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
  *reinterpret_cast<bf16x4*>(p) = __builtin_convertvector(v, bf16x4);
}

// c: values of a 16-byte chunk; a matrix operand (1 KiB, one chunk per lane)
// covers 2c elements of the head dimension (keys) or 2c tokens (values).
template <typename T>
struct Types;
template <>
struct Types<bf16_t> {
  typedef bf16x8 Frag;
  static constexpr int c = 8;
  static __device__ __forceinline__ void mma(f32x16& acc, const Frag& a, const Frag& b) {
    acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, acc, 0, 0, 0);
  }
  // probabilities of one operand: registers 8s .. 8s+7, rounded to nearest even
  static __device__ __forceinline__ Frag probs(const f32x16& p, int s) {
    Frag f;
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = static_cast<__bf16>(p[8 * s + i]);
    return f;
  }
  // the largest exponent field of f's values, in its place in a float32
  static __device__ __forceinline__ uint32_t exponent(const Frag& f) {
    const uint4 u = __builtin_bit_cast(uint4, f);
    auto top = [](uint32_t w) { return max(w & 0x7f800000u, w << 16 & 0x7f800000u); };
    return max(max(top(u.x), top(u.y)), max(top(u.z), top(u.w)));
  }
};
template <>
struct Types<float> {
  typedef f32x4 Frag;
  static constexpr int c = 4;
  static __device__ __forceinline__ void mma(f32x16& acc, const Frag& a, const Frag& b) {
#pragma unroll
    for (int t = 0; t < 4; ++t) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(a[t], b[t], acc, 0, 0, 0);
  }
  static __device__ __forceinline__ Frag probs(const f32x16& p, int s) {
    return Frag{p[4 * s], p[4 * s + 1], p[4 * s + 2], p[4 * s + 3]};
  }
  static __device__ __forceinline__ uint32_t exponent(const Frag& f) {
    const uint4 u = __builtin_bit_cast(uint4, f);
    return max(max(u.x & 0x7f800000u, u.y & 0x7f800000u), max(u.z & 0x7f800000u, u.w & 0x7f800000u));
  }
};

__device__ __forceinline__ float other_half_max(float v) {
  const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(s[0]), __uint_as_float(s[1]));
}
__device__ __forceinline__ float other_half_sum(float v) {
  const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(s[0]) + __uint_as_float(s[1]);
}
__device__ __forceinline__ float exp2_hw(float x) { return __builtin_amdgcn_exp2f(x); }

// Key index within a tile of register i in half h of the wave.
__device__ __forceinline__ constexpr int tile_key(int i, int h) { return 8 * (i / 4) + 4 * h + i % 4; }

template <typename T>
constexpr int waves_per_simd(int dp) {
  return two_per_cu(sizeof(T) == 4 ? DMOE_F32 : DMOE_BF16, dp) ? 2 : 1;
}

// Queries, keys, values and sums of a wave of the rows kernel pass its 512
// registers: the queries stay in LDS, and keys and values take turns in
// one set of registers.  fp32, 256 elements, 64 single tokens of 4096, 16 query
// and 4 kv heads: 923 us with all in registers, and much of it in scratch; 802 with
// the turns alone; 532 with both (2.1 GB of keys and values, 4.0 TB/s).
template <typename T>
constexpr bool rows_tight(int dp) {
  return dp * sizeof(T) > 768;
}

// A wave's 32 rows against tiles of 32 keys.
template <typename T, int DP, bool kQLds = false>
struct WaveRows {
  typedef Types<T> Ty;
  typedef typename Ty::Frag Frag;
  static constexpr int c = Ty::c;
  static constexpr int kK = DP / (2 * c);  // operands of a tile's keys
  static constexpr int kB = DP / 32;       // 32-wide blocks of the output
  static constexpr int kS = 16 / c;        // operands of a tile's values per block
  Frag q[kK];
  const Frag* ql;  // kQLds: the queries, read from here
  f32x16 o[kB];
  float m, l;  // l: of this half's keys
  int end;     // keys the row sees
  int lo, hi;  // the least and most of the wave's rows (uniform)

  __device__ __forceinline__ void clear() {
    m = -INFINITY;
    l = 0.f;
#pragma unroll
    for (int b = 0; b < kB; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[b][i] = 0.f;
  }

  // The sums' place between two products, where a wave has accumulation
  // registers beside its general ones: without it the compiler keeps them in general ones
  // because a raised maximum scales them there, copies all of them each stage
  // and has no room for the queries (two chunks of 2048 tokens over 4096, 16 query and 4 kv
  // heads: bf16 of 256 857 -> 423 us, of 192 401 -> 339; fp32 of 256 5376 -> 2663).
  __device__ __forceinline__ void pin() {
    if constexpr (waves_per_simd<T>(DP) == 1) {
#pragma unroll
      for (int b = 0; b < kB; ++b) asm volatile("" : "+a"(o[b]));
    }
  }

  __device__ __forceinline__ f32x16 scores(const Frag (&k)[kK]) const {
    f32x16 s;
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll
    for (int j = 0; j < kK; ++j) Ty::mma(s, k[j], kQLds ? ql[64 * j] : q[j]);
    return s;
  }

  // Scores (times scale log2 e) of consecutive tiles to probabilities relative
  // to the running maximum, which they raise first if they have to.  masked:
  // keys from `end - key0` on are not seen.
  template <int NT>
  __device__ __forceinline__ void softmax(f32x16 (&s)[NT], float scale2, int key0, bool masked, int half) {
    if (masked) {
      const int seen = end - key0;
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < 16; ++i) s[n][i] = n * kTileTokens + tile_key(i, half) < seen ? s[n][i] : -INFINITY;
    }
    float t = s[0][0];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int i = 0; i < 16; ++i) t = fmaxf(t, s[n][i]);
    t = other_half_max(t) * scale2;
    pin();
    if (__any(t > m + kLazy)) {
      const float nm = fmaxf(m, t);
      const float a = nm == m ? 1.f : exp2_hw(m - nm);
      m = nm;
      scale(a);
    }
    pin();
    const float off = m == -INFINITY ? 0.f : m;
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        s[n][i] = exp2_hw(__builtin_fmaf(s[n][i], scale2, -off));
        l += s[n][i];
      }
  }

  __device__ __forceinline__ void add(const f32x16& p, const Frag (&v)[kB][kS]) {
#pragma unroll
    for (int s = 0; s < kS; ++s) {
      const Frag f = Ty::probs(p, s);
#pragma unroll
      for (int b = 0; b < kB; ++b) Ty::mma(o[b], v[b][s], f);
    }
  }

  // For a tile in which some row does not see every key: values that no row
  // of the wave sees are not the sequence's, or a later token's, and become 0,
  // whatever they are.  True if the rest is finite: a value that some rows see
  // and others do not must not reach the others through 0 * value, so a tile
  // with one that is not is left to add_by_key.
  __device__ __forceinline__ bool cut(Frag (&v)[kB][kS], int key0, int half) const {
    const int seen = hi - key0;
    uint32_t top = 0;
#pragma unroll
    for (int s = 0; s < kS; ++s) {
      // all ones in the words (halves of words) of tokens that are seen
      uint32_t m[4];
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        constexpr int per = c / 4;
        auto on = [&](int e) { return 2 * c * s + 8 * (e / 4) + 4 * half + e % 4 < seen; };
        if constexpr (per == 1)
          m[x] = on(x) ? ~0u : 0u;
        else
          m[x] = (on(2 * x) ? 0xffffu : 0u) | (on(2 * x + 1) ? 0xffff0000u : 0u);
      }
#pragma unroll
      for (int b = 0; b < kB; ++b) {
        const uint4 u = __builtin_bit_cast(uint4, v[b][s]);
        v[b][s] = __builtin_bit_cast(Frag, make_uint4(u.x & m[0], u.y & m[1], u.z & m[2], u.w & m[3]));
        top = max(top, Ty::exponent(v[b][s]));
      }
    }
    return __all(top != 0x7f800000u);
  }
  // f with all elements but one set to 0 (slot -1: all).
  static __device__ __forceinline__ Frag only(const Frag& f, int slot) {
    constexpr int kPer = c / 4;  // elements of a 32-bit word
    const uint4 u = __builtin_bit_cast(uint4, f);
    const uint32_t bits = kPer == 1 ? ~0u : slot & 1 ? 0xffff0000u : 0x0000ffffu;
    const int word = slot < 0 ? -1 : slot / kPer;
    return __builtin_bit_cast(Frag, make_uint4(u.x & (word == 0 ? bits : 0), u.y & (word == 1 ? bits : 0), u.z & (word == 2 ? bits : 0),
                                               u.w & (word == 3 ? bits : 0)));
  }
  // Such tiles among kt, kt + step, ..., once the running maximum is the last
  // one: a key's products are added to the rows that see it.
  template <typename Map>
  __device__ __forceinline__ void add_by_key(const Map& map, int kt, int kt1, int step, float scale2, int half) {
    const int lane = threadIdx.x & 63;
#pragma unroll 1
    for (; kt < kt1; kt += step) {
      const int page = map.page(kt, kt1), key0 = kt * kTileTokens;
      if (!map.holds(page) || key0 >= hi) continue;
      const long at = map.at(kt, page);
      Frag v[kB][kS];
      load(v, map.v + at, lane);
      if (cut(v, key0, half)) continue;
      f32x16 s;
      {
        Frag k[kK];
        load(k, map.k + at, lane);
        s = scores(k);
      }
      const float off = m == -INFINITY ? 0.f : m;
#pragma unroll
      for (int i = 0; i < 16; ++i) s[i] = tile_key(i, half) < end - key0 ? exp2_hw(__builtin_fmaf(s[i], scale2, -off)) : 0.f;
      add_keys(s, v, key0, half);
    }
  }
  static __device__ __forceinline__ void load(Frag (&k)[kK], const T* p, int lane) {
#pragma unroll
    for (int j = 0; j < kK; ++j) k[j] = *reinterpret_cast<const Frag*>(p + j * 64 * c + lane * c);
  }
  static __device__ __forceinline__ void load(Frag (&v)[kB][kS], const T* p, int lane) {
#pragma unroll
    for (int b = 0; b < kB; ++b)
#pragma unroll
      for (int s = 0; s < kS; ++s) v[b][s] = *reinterpret_cast<const Frag*>(p + (b * kS + s) * 64 * c + lane * c);
  }
  __device__ __forceinline__ void add_keys(const f32x16& p, const Frag (&v)[kB][kS], int key0, int half) {
#pragma unroll
    for (int s = 0; s < kS; ++s) {
      const Frag f = Ty::probs(p, s);
#pragma unroll 1
      for (int r = 0; r < 2 * c; ++r) {
        const bool mine = (r >> 2 & 1) == half;
        const int slot = mine ? (r >> 3) * 4 + (r & 3) : -1;
        const bool sees = key0 + 2 * c * s + r < end;
        const Frag one = only(f, slot);
#pragma unroll
        for (int b = 0; b < kB; ++b) {
          const Frag x = only(v[b][s], slot);
          f32x16 t;
#pragma unroll
          for (int i = 0; i < 16; ++i) t[i] = 0.f;
          Ty::mma(t, x, one);
#pragma unroll
          for (int i = 0; i < 16; ++i) o[b][i] += sees ? t[i] : 0.f;
          __builtin_amdgcn_sched_barrier(0);  // one block's products at a time: registers are short here
        }
      }
    }
  }

  // This wave's rows joined with another's over other keys; fac scales this
  // one's sums.
  __device__ __forceinline__ void scale(float fac) {
    l *= fac;
#pragma unroll
    for (int b = 0; b < kB; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[b][i] *= fac;
  }
};

// Where a sequence's tiles of one kv head lie.
template <typename T, int DP>
struct TileMap {
  const T *k, *v;
  // nothing of a launch writes the table: scalar loads, as the constant address space has them
  const __attribute__((address_space(4))) int32_t* table;
  long page_len, layer0;
  int hkv, n_pages, shift;  // tiles of a page: 1 << shift, or -shift of them
  __device__ __forceinline__ TileMap(const AttnArgs& a, int slot, int hk) : hkv(a.cache.n_kv_heads), n_pages(a.cache.n_pages) {
    table = (const __attribute__((address_space(4))) int32_t*)(a.cache.table + static_cast<long>(slot) * a.cache.max_pages);
    const int tpp = a.cache.page_tokens / kTileTokens;
    shift = (tpp & (tpp - 1)) == 0 ? 31 - __builtin_clz(tpp) : -tpp;
    page_len = static_cast<long>(a.cache.page_tokens) * DP;
    layer0 = static_cast<long>(a.layer) * n_pages;
    k = static_cast<const T*>(a.cache.k) + hk * page_len;
    v = static_cast<const T*>(a.cache.v) + hk * page_len;
  }
  // page of a tile before `end`, else -1
  __device__ __forceinline__ int page(int kt, int end) const { return kt < end ? table[shift >= 0 ? kt >> shift : kt / -shift] : -1; }
  __device__ __forceinline__ bool holds(int page) const { return static_cast<unsigned>(page) < static_cast<unsigned>(n_pages); }
  // elements from k and v to a tile on a page that is held
  __device__ __forceinline__ long at(int kt, int page) const {
    const int in = shift >= 0 ? kt & ((1 << shift) - 1) : kt % -shift;
    return (layer0 + page) * hkv * page_len + in * (kTileTokens * DP);
  }
};

// The plan's item and whether there is one, in one round trip to memory (the
// array is as long as the grid).
__device__ __forceinline__ bool load_item(const AttnArgs& a, int i, AttnItem& it) {
  typedef int i32x16 __attribute__((ext_vector_type(16)));
  const auto* p = (const __attribute__((address_space(4))) int32_t*)a.plan;
  const int n = p[0];
  const i32x16 w = *(const __attribute__((address_space(4))) i32x16*)(p + sizeof(AttnPlanHead) / 4 + static_cast<long>(i) * 16);
  it = AttnItem{w[0], w[1], w[2], w[3], w[4], w[5], w[6], w[7], w[8], {w[9], w[10], w[11], w[12], w[13], w[14]}, 0};
  return i < n;
}

// The item's rows of this wave: row index, head and what they see; queries loaded.
template <typename T, int DP>
struct RowPlace {
  int row, tok, qh;
  bool live, any;
  template <typename Rows>
  __device__ __forceinline__ RowPlace(Rows& w, const AttnArgs& a, const AttnItem& it, int g, int hk, int row_lo, int lane) {
    constexpr int c = Types<T>::c;
    typedef typename Types<T>::Frag Frag;
    const int row_hi = min(row_lo + 32, it.rows) - 1;
    const int pos0 = it.len - it.n;
    row = row_lo + (lane & 31);
    live = row < it.rows;
    any = row_hi >= row_lo;
    tok = live ? row / g : 0;
    qh = hk * g + (live ? row - tok * g : 0);
    w.end = live ? visible_end(pos0 + tok, it.len, a.mask_block) : 0;
    // the ends grow with the rows; rows past the last are computed and dropped
    w.lo = any ? visible_end(pos0 + row_lo / g, it.len, a.mask_block) : 0;
    w.hi = any ? visible_end(pos0 + row_hi / g, it.len, a.mask_block) : 0;
    const T* qp = static_cast<const T*>(a.q) + (it.row0 + tok) * a.q_stride + static_cast<long>(qh) * a.cache.head_dim;
#pragma unroll
    for (int j = 0; j < Rows::kK; ++j) {
      const int d = (2 * j + (lane >> 5)) * c;
      Frag f{};
      if (live && d < a.cache.head_dim) f = *reinterpret_cast<const Frag*>(qp + d);
      w.q[j] = f;
    }
  }
  // The wave's sums: divided into out, or as they are into the workspace.
  template <typename Rows>
  __device__ __forceinline__ void store(const Rows& w, const AttnArgs& a, const AttnShape& sh, const AttnItem& it, int hk,
                                        int half, int part_rows) const {
    constexpr int kB = Rows::kB;
    if (!live) return;
    if (it.part >= 0) {
      const long at = (static_cast<long>(it.part) * a.cache.n_kv_heads + hk) * sh.tile_rows + (row - it.first);
      float* po = static_cast<float*>(a.workspace) + (at - (row - it.first)) * DP + partial_at(DP, row - it.first, 4 * half);
#pragma unroll
      for (int b = 0; b < kB; ++b)
#pragma unroll
        for (int i = 0; i < 16; i += 4)
          store4(po + partial_at(DP, 0, 32 * b + tile_key(i, 0)), f32x4{w.o[b][i], w.o[b][i + 1], w.o[b][i + 2], w.o[b][i + 3]});
      if (half == 0)
        *reinterpret_cast<float2*>(static_cast<float*>(a.workspace) + static_cast<long>(part_rows) * DP + at * 2) = make_float2(w.m, w.l);
      return;
    }
    const bool some = w.l > 0.f || w.l != w.l;
    const float inv = some ? 1.f / w.l : 0.f;
    T* op = static_cast<T*>(a.out) + (it.row0 + tok) * a.out_stride + static_cast<long>(qh) * a.cache.head_dim;
#pragma unroll
    for (int b = 0; b < kB; ++b)
#pragma unroll
      for (int i = 0; i < 16; i += 4) {
        const int d = 32 * b + tile_key(i, half);
        if (d < a.cache.head_dim)
          store4(op + d, f32x4{w.o[b][i] * inv, w.o[b][i + 1] * inv, w.o[b][i + 2] * inv, w.o[b][i + 3] * inv});
      }
    if (a.lse && half == 0)
      a.lse[static_cast<long>(it.row0 + tok) * a.n_heads + qh] = some ? (w.m + log2f(w.l)) * kLn2 : -INFINITY;
  }
};

// Few rows (one token a sequence, a small block): 32 kWR of one kv head per
// workgroup, 4 / kWR waves to 32 of them, each on every (4 / kWR)-th key tile,
// joined through LDS.  The cache goes straight into registers, past the caches
// where one wave alone reads a tile; the next tile's keys are issued when this
// one's are used up, its values likewise.
//
// Bound by the cache's bytes: bf16, 32 query and 8 kv heads of 128, one token
// over 131k: 537 MB in 85 us (6.3 TB/s); 64 of up to 16k: 1.08 GB in 181 us
// (6.0 TB/s).  The matrix instructions mostly multiply rows that are not there
// (4 of 32 here), which costs nothing: a CU's four could take 16 times the
// bytes it gets.  With loads through the caches the first took 96 us.  Short
// sequences are a chain of round trips: item and queries 1.6 us, keys and
// values 0.6, a tile's arithmetic 0.5 (fp32, 64 elements: 2.3), the join 1.1, the
// stores 0.5.
template <typename T, int DP, int kWR>
__global__ __launch_bounds__(256, waves_per_simd<T>(DP)) void attention_rows_kernel(AttnArgs a, AttnShape sh, int part_rows) {
  constexpr bool kTight = rows_tight<T>(DP);
  typedef WaveRows<T, DP, kTight> Rows;
  typedef typename Rows::Frag Frag;
  constexpr int c = Rows::c, kK = Rows::kK, kB = Rows::kB, kS = Rows::kS, kWK = 4 / kWR;
  extern __shared__ float lds[];
  const int hkv = a.cache.n_kv_heads;
  const int item_i = blockIdx.x / hkv, hk = blockIdx.x % hkv;
  AttnItem it;
  if (!load_item(a, item_i, it)) return;
  const int lane = threadIdx.x & 63, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wk = wave % kWK, wr = wave / kWK;
  Rows w;
  w.clear();
  const RowPlace<T, DP> rows(w, a, it, sh.group, hk, it.first + 32 * wr, lane);
  if constexpr (kTight) {
    Frag* ql = reinterpret_cast<Frag*>(lds) + wr * (kK * 64) + lane;
    if (wk == 0) {
#pragma unroll
      for (int j = 0; j < kK; ++j) ql[64 * j] = w.q[j];
    }
    w.ql = ql;
    __syncthreads();
  }
  const float scale2 = a.scale * kLog2e;
  const TileMap<T, DP> map(a, it.slot, hk);
  const int kt1 = min(it.kt1, (w.hi + kTileTokens - 1) / kTileTokens);
  Frag k[kK], v[kB][kS];
  auto load1 = [&](const T* p) {
    const Frag* f = reinterpret_cast<const Frag*>(p + lane * c);
    return kWR == 1 ? __builtin_nontemporal_load(f) : *f;
  };
  auto load_k = [&](const T* p) {
#pragma unroll
    for (int j = 0; j < kK; ++j) k[j] = load1(p + j * 64 * c);
  };
  auto load_v = [&](const T* p) {
#pragma unroll
    for (int b = 0; b < kB; ++b)
#pragma unroll
      for (int s = 0; s < kS; ++s) v[b][s] = load1(p + (b * kS + s) * 64 * c);
  };
  // page ids are known two of this wave's tiles ahead, its keys and values one
  int kt = it.kt0 + wk;
  int page = kt < kt1 ? (wk < 2 ? wk == 0 ? it.page[0] : it.page[1] : wk == 2 ? it.page[2] : it.page[3]) : -1;
  int page1 = map.page(kt + kWK, kt1);
  long at;
  auto first = [&] {
    at = map.holds(page) ? map.at(kt, page) : 0;
    if (map.holds(page)) {
      load_k(map.k + at);
      if (!kTight) load_v(map.v + at);
    }
  };
  first();
  if (const int now = map.page(kt, kt1); now != page) {  // moved since the plan was made
    page = now;
    first();
  }
  bool left = false;  // tiles for add_by_key
  auto turn = [&](auto masked) {
    w.pin();
    const int page2 = map.page(kt + 2 * kWK, kt1);
    const bool here = map.holds(page), more = map.holds(page1);
    const long at1 = more ? map.at(kt + kWK, page1) : 0;
    f32x16 s[1];
    if (here) s[0] = w.scores(k);
    if (kTight) {
      __builtin_amdgcn_sched_barrier(0);
      if (here) load_v(map.v + at);
    } else if (more) {
      load_k(map.k + at1);
    }
    if (here) {
      const int key0 = kt * kTileTokens;
      w.template softmax<1>(s, scale2, key0, masked, half);
      if (!masked || w.cut(v, key0, half))
        w.add(s[0], v);
      else
        left = true;
    }
    if (kTight) __builtin_amdgcn_sched_barrier(0);
    if (more) kTight ? load_k(map.k + at1) : load_v(map.v + at1);
    kt += kWK;
    at = at1;
    page = page1;
    page1 = page2;
  };
  // tiles that every row sees whole, then the others
  const int whole = min(kt1, w.lo / kTileTokens);
  while (kt < whole) turn(std::false_type());
  w.pin();
  const int first_masked = kt;
  while (kt < kt1) turn(std::true_type());
  w.pin();
  if (left) w.add_by_key(map, first_masked, kt1, kWK, scale2, half);
  w.l = other_half_sum(w.l);

  // join the waves two by two: the upper ones hand their sums to the lower
  // ones (fixed order)
  constexpr int kLen = (16 * kB + 2) * 64;
#pragma unroll
  for (int n = kWK / 2; n >= 1; n /= 2) {
    float* buf = lds + (kTight ? kWR * kK * 256 : 0) + (wr * (kWK / 2) + wk % n) * kLen;
    if (wk >= n && wk < 2 * n) {
      buf[lane] = w.m;
      buf[64 + lane] = w.l;
#pragma unroll
      for (int b = 0; b < kB; ++b)
#pragma unroll
        for (int i = 0; i < 16; i += 4)
          *reinterpret_cast<f32x4*>(buf + 128 + (4 * b + i / 4) * 256 + lane * 4) =
              f32x4{w.o[b][i], w.o[b][i + 1], w.o[b][i + 2], w.o[b][i + 3]};
    }
    __syncthreads();
    if (wk < n) {
      const float om = buf[lane], ol = buf[64 + lane];
      const float nm = fmaxf(w.m, om);
      const float fa = w.m == nm ? 1.f : exp2_hw(w.m - nm), fb = om == nm ? 1.f : exp2_hw(om - nm);
      w.scale(fa);
      w.m = nm;
      w.l += fb * ol;
#pragma unroll
      for (int b = 0; b < kB; ++b)
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
          const f32x4 x = *reinterpret_cast<const f32x4*>(buf + 128 + (4 * b + i / 4) * 256 + lane * 4);
#pragma unroll
          for (int t = 0; t < 4; ++t) w.o[b][i + t] += fb * x[t];
        }
    }
    __syncthreads();
  }
  if (wk == 0) rows.store(w, a, sh, it, hk, half, part_rows);
}

// 16 bytes per lane from global memory straight into LDS at dst + 16*lane.
template <typename T, typename Frag>
__device__ __forceinline__ void dma16(const T* src, Frag* dst) {
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)src,
                                   (__attribute__((address_space(3))) void*)dst, 16, 0, 0);
}

// Many rows: 128 of one kv head per workgroup, 32 to a wave, all four waves on
// the same keys.  Keys and values of kTS tiles go from memory straight into
// LDS, one stage ahead, in two buffers; one barrier a stage.
template <typename T, int DP>
struct BlockStage {
  static constexpr int kTileFrags = DP / (2 * Types<T>::c);           // operands of a tile's keys, or of its values
  static constexpr int kTS = stage_tiles(sizeof(T) == 4 ? DMOE_F32 : DMOE_BF16, DP);
  typename Types<T>::Frag f[kTS][2][kTileFrags][64];                  // [tile][keys, values][operand][lane]
};

//
// Bound by issue and power: bf16, 4096 tokens over 12k, 16 query and 4 kv heads of
// 128: 490 to 550 us, 880 to 980 TFLOP/s of 1430 that a library product of 8192^3
// reaches.  The matrix pipes are busy 51 % of the cycles and vector
// instructions fill most of the rest (about 75 a tile and wave, 16 of them
// exponentials at a quarter of the rate).  The clock falls under it: with values
// of 0 the same instructions take 450 us, with keys of 0 too 418.  Measured and not kept: the next
// tile's scores formed between the exponentials by scheduling groups (+5 %: the
// accumulators are copied more), operands read four ahead (+3 %), wave priorities
// around the matrix instructions (0 %).
//
// kWK = 2: eight waves, each four on one half of the item's keys, joined
// through LDS: half the partial results of two such workgroups, which matters
// where few row tiles are cut into many items (sixteen blocks of 32 tokens over up to
// 8k: kernel and join 22.3 + 7.1 -> 22.1 + 4.9 us; 64 MB of keys and values).
template <typename T, int DP, int kWK>
__global__ __launch_bounds__(256 * kWK, waves_per_simd<T>(DP)) void attention_block_kernel(AttnArgs a, AttnShape sh, int part_rows) {
  typedef WaveRows<T, DP> Rows;
  typedef typename Rows::Frag Frag;
  typedef BlockStage<T, DP> Stage;
  constexpr int c = Rows::c, kK = Rows::kK, kB = Rows::kB, kS = Rows::kS, kTS = Stage::kTS;
  __shared__ Stage s0s[kWK], s1s[kWK];  // apart, so that reads of one do not wait for loads into the other
  const int hkv = a.cache.n_kv_heads;
  const int item_i = blockIdx.x / hkv, hk = blockIdx.x % hkv;
  AttnItem it;
  if (!load_item(a, item_i, it)) return;
  const int lane = threadIdx.x & 63, half = lane >> 5;
  const int wk = kWK > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 8) : 0;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) & 3;
  Stage &s0 = s0s[wk], &s1 = s1s[wk];
  Rows w;
  w.clear();
  const RowPlace<T, DP> rows(w, a, it, sh.group, hk, it.first + 32 * wave, lane);
  const float scale2 = a.scale * kLog2e;
  const TileMap<T, DP> map(a, it.slot, hk);
  // this wave's keys; the first half has at least as many stages
  const int mid = kWK > 1 ? item_middle(it.kt0, it.kt1) : it.kt1;
  const int kt0 = wk ? mid : it.kt0, kt1 = wk ? it.kt1 : mid;
  const int turns = (mid - it.kt0 + kTS - 1) / kTS;
  struct Ids {
    int id[kTS];
  };
  auto pages = [&](int kt) {
    Ids p;
#pragma unroll
    for (int n = 0; n < kTS; ++n) p.id[n] = map.page(kt + n, kt1);
    return p;
  };
  // a wave's share of a stage: with two tiles the keys or the values of one,
  // with one tile half of its keys or values
  const T *mk = map.k, *mv = map.v;
  const T* share = wave & 1 ? mv : mk;
  auto load = [&](int kt, const Ids& pg, Stage& st) {
    const int n = kTS == 2 ? wave >> 1 : 0, kv = wave & 1;
    const int page = kTS == 2 && n ? pg.id[kTS - 1] : pg.id[0];
    if (!map.holds(page)) return;
    const T* p = share + map.at(kt + n, page) + lane * c;
    constexpr int kShare = kTS == 2 ? kK : kK / 2;
    const int j0 = kTS == 2 ? 0 : (wave >> 1) * kShare;
#pragma unroll
    for (int j = 0; j < kShare; ++j) dma16(p + (j0 + j) * 64 * c, &st.f[n][kv][j0 + j][0]);
  };
  // A stage that every row sees whole; its tiles may still lie on no page, or
  // behind the item's last.
  auto compute = [&](std::false_type, int kt, const Ids& pg, const Stage& st) {
    if (!rows.any) return;
    bool on[kTS];
    bool all = true, none = true;
#pragma unroll
    for (int n = 0; n < kTS; ++n) {
      on[n] = map.holds(pg.id[n]);
      all = all && on[n];
      none = none && !on[n];
    }
    if (none) return;
    f32x16 s[kTS];
#pragma unroll
    for (int n = 0; n < kTS; ++n) {
#pragma unroll
      for (int i = 0; i < 16; ++i) s[n][i] = 0.f;
#pragma unroll
      for (int j = 0; j < kK; ++j) Types<T>::mma(s[n], st.f[n][0][j][lane], w.q[j]);
    }
    if (!all) {
#pragma unroll
      for (int n = 0; n < kTS; ++n)
#pragma unroll
        for (int i = 0; i < 16; ++i) s[n][i] = on[n] ? s[n][i] : -INFINITY;
    }
    w.template softmax<kTS>(s, scale2, kt * kTileTokens, false, half);
#pragma unroll
    for (int n = 0; n < kTS; ++n) {
      if (!on[n]) continue;
#pragma unroll
      for (int x = 0; x < kS; ++x) {
        const Frag f = Types<T>::probs(s[n], x);
#pragma unroll
        for (int b = 0; b < kB; ++b) Types<T>::mma(w.o[b], st.f[n][1][b * kS + x][lane], f);
      }
    }
  };
  // Any stage, tile by tile (registers are short where values are cut).
  bool left = false;  // tiles for add_by_key
  auto compute_masked = [&](int kt, const Ids& pg, const Stage& st) {
#pragma unroll
    for (int n = 0; n < kTS; ++n) {
      const int key0 = (kt + n) * kTileTokens;
      if (!map.holds(pg.id[n]) || key0 >= w.hi) continue;
      f32x16 s[1];
#pragma unroll
      for (int i = 0; i < 16; ++i) s[0][i] = 0.f;
#pragma unroll
      for (int j = 0; j < kK; ++j) Types<T>::mma(s[0], st.f[n][0][j][lane], w.q[j]);
      w.template softmax<1>(s, scale2, key0, true, half);
      __builtin_amdgcn_sched_barrier(0);
      Frag v[kB][kS];
#pragma unroll
      for (int b = 0; b < kB; ++b)
#pragma unroll
        for (int x = 0; x < kS; ++x) v[b][x] = st.f[n][1][b * kS + x][lane];
      if (w.cut(v, key0, half))
        w.add(s[0], v);
      else
        left = true;
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  // page ids are known two stages ahead, keys and values one.  A stage's loads
  // are waited for by the wave that issued them, then by all: the barrier also
  // tells that the other buffer has been read.
  int kt = kt0;
  Ids pg, pg1;
#pragma unroll
  for (int n = 0; n < kTS; ++n) {
    pg.id[n] = wk ? it.page[4 + n] : kt + n < kt1 ? it.page[n] : -1;
  }
  load(kt, pg, s0);
  __builtin_amdgcn_sched_barrier(0);
  const Ids now = pages(kt);
  pg1 = pages(kt + kTS);
  bool moved = false;  // since the plan was made
#pragma unroll
  for (int n = 0; n < kTS; ++n) moved = moved || now.id[n] != pg.id[n];
  if (moved) {
    pg = now;
    __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0): the stage is loaded again
    load(kt, pg, s0);
  }
  __builtin_amdgcn_sched_barrier(0);
  auto turn = [&](auto masked, Stage& cur, Stage& fill) {
    w.pin();
    __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0)
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
    load(kt + kTS, pg1, fill);
    const Ids pg2 = pages(kt + 2 * kTS);
    __builtin_amdgcn_sched_barrier(0);
    if constexpr (masked)
      compute_masked(kt, pg, cur);
    else
      compute(masked, kt, pg, cur);
    __builtin_amdgcn_sched_barrier(0);
    kt += kTS;
    pg = pg1;
    pg1 = pg2;
  };
  // stages whose keys every row of the workgroup sees, then the others; every
  // wave takes all turns, for their barriers
  const int whole = visible_end(it.len - it.n + it.first / sh.group, it.len, a.mask_block) / kTileTokens;
  const int stages = whole >= kt1 ? max(kt1 - kt + kTS - 1, 0) / kTS : max(whole - kt, 0) / kTS;
  const int first_masked = kt + stages * kTS;
  int done = 0;
  for (; done + 2 <= stages; done += 2) {
    turn(std::false_type(), s0, s1);
    turn(std::false_type(), s1, s0);
  }
  if (done < stages) {
    turn(std::false_type(), s0, s1);
    ++done;
  }
  for (; done < turns; ++done) {
    if (done & 1)
      turn(std::true_type(), s1, s0);
    else
      turn(std::true_type(), s0, s1);
  }
  if (left) w.add_by_key(map, first_masked, kt1, 1, scale2, half);
  w.l = other_half_sum(w.l);
  if constexpr (kWK > 1) {
    // the second half's sums to the first's waves; the stages are done with
    __syncthreads();
    float* sums = reinterpret_cast<float*>(wave < 2 ? s0s : s1s) + (wave & 1) * (16 * kB * 64);
    static_assert(sizeof(s0s) >= 2 * 16 * kB * 64 * sizeof(float));
    __shared__ float2 stats[4][64];
    if (wk) {
      stats[wave][lane] = make_float2(w.m, w.l);
#pragma unroll
      for (int b = 0; b < kB; ++b)
#pragma unroll
        for (int i = 0; i < 16; i += 4)
          store4(sums + (4 * b + i / 4) * 256 + lane * 4, f32x4{w.o[b][i], w.o[b][i + 1], w.o[b][i + 2], w.o[b][i + 3]});
    }
    __syncthreads();
    if (wk) return;
    const float2 other = stats[wave][lane];
    const float nm = fmaxf(w.m, other.x);
    const float fa = w.m == nm ? 1.f : exp2_hw(w.m - nm), fb = other.x == nm ? 1.f : exp2_hw(other.x - nm);
    w.scale(fa);
    w.m = nm;
    w.l += fb * other.y;
#pragma unroll
    for (int b = 0; b < kB; ++b)
#pragma unroll
      for (int i = 0; i < 16; i += 4) {
        const f32x4 x = *reinterpret_cast<const f32x4*>(sums + (4 * b + i / 4) * 256 + lane * 4);
#pragma unroll
        for (int t = 0; t < 4; ++t) w.o[b][i + t] += fb * x[t];
      }
  }
  rows.store(w, a, sh, it, hk, half, part_rows);
}

// Partial results of a row tile joined, pieces in fixed order.  A workgroup
// takes 8 rows, which lie side by side in every KiB of the partial sums: a
// wave reads 128 bytes of each, lane = (16-byte piece of the KiB, row), and the
// waves share the pieces.  4.2 us for 17 pieces of 512 rows, 4.9 for 7 of 8192;
// with the sums stored row by row and a workgroup per row 14 and 15.  Eight waves
// were faster for one sequence's 127 pieces (8.3 against 11.4 us) and slower for
// many rows (9.4 against 4.8).
constexpr int kMergeWaves = 4, kMergeRows = 8;

template <typename T, int DP>
__global__ __launch_bounds__(64 * kMergeWaves) void attention_merge_kernel(AttnArgs a, AttnShape sh, int part_rows) {
  constexpr int kV = DP / 32;  // f32x4 of a lane: 8 lanes of a row cover 32 elements
  __shared__ f32x4 so[kMergeWaves - 1][kV][64];
  __shared__ float2 sml[kMergeWaves][kMergeRows];
  const int hkv = a.cache.n_kv_heads;
  const int groups = sh.tile_rows / kMergeRows;
  // the number of merges and the first one are loaded together: the grid is within their array
  const auto* plan = (const __attribute__((address_space(4))) int32_t*)a.plan;
  const int units = plan[1] * hkv * groups;
  const long merges = (sizeof(AttnPlanHead) + sh.max_items() * sizeof(AttnItem)) / sizeof(int);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = lane % kMergeRows, col = lane / kMergeRows;  // row; piece of 4 elements of every 32
  const float* po = static_cast<const float*>(a.workspace);
  const float2* ml = reinterpret_cast<const float2*>(po + static_cast<long>(part_rows) * DP);
  const long step = static_cast<long>(hkv) * sh.tile_rows;
  int u = blockIdx.x;
  do {
    typedef int i32x8 __attribute__((ext_vector_type(8)));
    const int row0 = u % groups * kMergeRows, hk = u / groups % hkv;
    const i32x8 mw = *(const __attribute__((address_space(4))) i32x8*)(plan + merges + u / groups / hkv * 8l);
    const AttnMerge mg{mw[0], mw[1], mw[2], mw[3], mw[4], {0, 0, 0}};
    if (u >= units) return;
    if (mg.first + row0 >= mg.rows) continue;
    const int row = mg.first + row0 + r;
    const bool live = row < mg.rows;
    const long tile = (static_cast<long>(mg.part) * hkv + hk) * sh.tile_rows;
    const float* pr = po + tile * DP + partial_at(DP, row0 + r, 4 * col);
    const float2* mr = ml + tile + row0 + r;
    // online over this wave's pieces: all their loads are in flight together
    float m = -INFINITY, l = 0.f;
    f32x4 o[kV];
#pragma unroll
    for (int j = 0; j < kV; ++j) o[j] = f32x4{0.f, 0.f, 0.f, 0.f};
    constexpr int kBatch = kV <= 4 ? 4 : 2;
    for (int i0 = wave; i0 < mg.pieces; i0 += kMergeWaves * kBatch) {
      float2 x[kBatch];
      f32x4 p[kBatch][kV];
      float nm = m;
#pragma unroll
      for (int y = 0; y < kBatch; ++y) {
        const int i = i0 + y * kMergeWaves;
        x[y] = make_float2(-INFINITY, 0.f);
        if (live && i < mg.pieces) {
          x[y] = mr[i * step];
#pragma unroll
          for (int j = 0; j < kV; ++j) p[y][j] = *reinterpret_cast<const f32x4*>(pr + i * step * DP + partial_at(DP, 0, 32 * j));
        } else {
#pragma unroll
          for (int j = 0; j < kV; ++j) p[y][j] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
      }
#pragma unroll
      for (int y = 0; y < kBatch; ++y) nm = fmaxf(nm, x[y].x);
      const float f0 = m == nm ? 1.f : exp2_hw(m - nm);
      m = nm;
      l *= f0;
#pragma unroll
      for (int j = 0; j < kV; ++j) o[j] *= f0;
#pragma unroll
      for (int y = 0; y < kBatch; ++y) {
        const float f = x[y].x == m ? 1.f : exp2_hw(x[y].x - m);
        l += f * x[y].y;
#pragma unroll
        for (int j = 0; j < kV; ++j) o[j] += f * p[y][j];
      }
    }
    __syncthreads();  // the previous unit's sums have been read
    if (col == 0) sml[wave][r] = make_float2(m, l);
    if (wave > 0) {
#pragma unroll
      for (int j = 0; j < kV; ++j) so[wave - 1][j][lane] = o[j];
    }
    __syncthreads();
    if (wave != 0 || !live) continue;
    float mm = -INFINITY;
#pragma unroll
    for (int i = 0; i < kMergeWaves; ++i) mm = fmaxf(mm, sml[i][r].x);
    l = 0.f;
#pragma unroll
    for (int i = 0; i < kMergeWaves; ++i) {
      const float2 x = sml[i][r];
      const float f = x.x == mm ? 1.f : exp2_hw(x.x - mm);
      l += f * x.y;
#pragma unroll
      for (int j = 0; j < kV; ++j) o[j] = i == 0 ? f * o[j] : o[j] + f * so[i > 0 ? i - 1 : 0][j][lane];
    }
    const bool some = l > 0.f || l != l;
    const float inv = some ? 1.f / l : 0.f;
    const int tok = row / sh.group, qh = hk * sh.group + row - tok * sh.group;
    T* op = static_cast<T*>(a.out) + (mg.row0 + tok) * a.out_stride + static_cast<long>(qh) * a.cache.head_dim + col * 4;
#pragma unroll
    for (int j = 0; j < kV; ++j)
      if (32 * j + col * 4 < a.cache.head_dim) store4(op + 32 * j, o[j] * inv);
    if (a.lse && col == 0)
      a.lse[static_cast<long>(mg.row0 + tok) * a.n_heads + qh] = some ? (mm + log2f(l)) * kLn2 : -INFINITY;
  } while ((u += gridDim.x) < units);
}

constexpr long kMergeGrid = 1024;

template <typename T, int DP>
hipError_t launch_dim(const AttnArgs& a, const AttnShape& sh, hipStream_t s) {
  const int hkv = a.cache.n_kv_heads;
  const unsigned items = static_cast<unsigned>(sh.max_items() * hkv);
  const int part_rows = static_cast<int>(sh.max_parts() * hkv * sh.tile_rows);
  if (sh.tile_rows <= 64) {
    const size_t lds = 2 * (16 * (DP / 32) + 2) * 64 * sizeof(float) + (rows_tight<T>(DP) ? sh.tile_rows * DP * sizeof(T) : 0);
    if (sh.tile_rows == 32)
      attention_rows_kernel<T, DP, 1><<<items, 256, lds, s>>>(a, sh, part_rows);
    else
      attention_rows_kernel<T, DP, 2><<<items, 256, lds, s>>>(a, sh, part_rows);
  } else {
    if constexpr (waves_per_simd<T>(DP) == 2) {
      if (sh.wide)
        attention_block_kernel<T, DP, 2><<<items, 512, 0, s>>>(a, sh, part_rows);
      else
        attention_block_kernel<T, DP, 1><<<items, 256, 0, s>>>(a, sh, part_rows);
    } else {
      attention_block_kernel<T, DP, 1><<<items, 256, 0, s>>>(a, sh, part_rows);
    }
  }
  // no sequence is long enough to be split: nothing to join
  if (static_cast<long>(a.cache.max_pages) * a.cache.page_tokens <= static_cast<long>(sh.min_tiles) * kTileTokens) return hipGetLastError();
  const long units = sh.split_items * hkv * (sh.tile_rows / kMergeRows);
  attention_merge_kernel<T, DP><<<static_cast<unsigned>(units < kMergeGrid ? units : kMergeGrid), 64 * kMergeWaves, 0, s>>>(a, sh, part_rows);
  return hipGetLastError();
}

template <typename T>
hipError_t launch_type(const AttnArgs& a, const AttnShape& sh, hipStream_t s) {
  switch (padded_dim(a.cache.head_dim)) {
    case 32: return launch_dim<T, 32>(a, sh, s);
    case 64: return launch_dim<T, 64>(a, sh, s);
    case 96: return launch_dim<T, 96>(a, sh, s);
    case 128: return launch_dim<T, 128>(a, sh, s);
    case 192: return launch_dim<T, 192>(a, sh, s);
    default: return launch_dim<T, 256>(a, sh, s);
  }
}

}  // namespace attn
}  // namespace dmoe
