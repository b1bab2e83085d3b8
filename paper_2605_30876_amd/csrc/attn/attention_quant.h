// Attention over a cache of few bits.
//
// The products are those of attention.h on the bf16 matrix cores: S^T = K Q^T with a
// row to a lane, online softmax in base 2, O^T += V^T P^T, on tiles of 32 or 16
// rows.  code * scale is exact in bf16, so codes become matrix operands by the
// conversion instructions alone, two values each, the scale applied by them.  A page holds
// keys and values alike, token by token: a lane's 16 bytes are consecutive elements of
// one token, which is a key operand as it is (the order of a reduction's elements is free,
// as long as queries are loaded in the same one); values are written to LDS
// in rows of tokens and read back turned (ds_read_b64_tr_b16: four tokens of one
// element a lane), in the order of the registers that hold probabilities.
//
// Not used: the matrix instructions that take codes and scales as they are.  They align a
// product's terms to the largest and keep 12 bits below it (measured: sums of 64 off by 2^-12
// of the largest term), where the bf16 ones keep float32's.
//
// fp32 rows: queries and probabilities are cut into three bf16 parts of eight bits, which hold
// them exactly, and multiplied one after another: three bf16 products take 96 cycles where
// the fp32 one takes 512.
#pragma once

#include "attention.h"
#include "quant.h"

namespace dmoe {
namespace attn {

using quant::decode;
using quant::scale_of;

typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// A plan's shape and what kernels divide by.
struct QuantShape : AttnShape {
  FastDiv by_group, by_page, by_mask;  // query heads of a kv head, tiles of a page, mask_block (where there is one)
};

// bf16 parts of a row's queries and probabilities.
template <typename T>
constexpr int kParts = sizeof(T) == 4 ? 3 : 1;

// Eight values as parts that add up to them: the first 8 bits, the next, the
// rest.  What is not finite is in the first part.
__device__ __forceinline__ void split(const float (&x)[8], bf16x8 (&f)[3]) {
  uint32_t w[3][4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint32_t a[2][3];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const uint32_t u = __float_as_uint(x[2 * i + e]), hi = u & 0xffff0000u;
      const bool finite = (u & 0x7f800000u) != 0x7f800000u;
      const float r = finite ? x[2 * i + e] - __uint_as_float(hi) : 0.f;
      const uint32_t mid = __float_as_uint(r) & 0xffff0000u;
      a[e][0] = hi | (!finite && (u & 0xffffu) ? 0x10000u : 0u);  // a NaN stays one
      a[e][1] = mid;
      a[e][2] = __float_as_uint(r - __uint_as_float(mid));
    }
#pragma unroll
    for (int p = 0; p < 3; ++p) w[p][i] = (a[0][p] >> 16) | (a[1][p] & 0xffff0000u);
  }
#pragma unroll
  for (int p = 0; p < 3; ++p) f[p] = __builtin_bit_cast(bf16x8, make_uint4(w[p][0], w[p][1], w[p][2], w[p][3]));
}

// Codes and scale bytes of a token that nobody sees become 0; false if what is left is perhaps not finite.
template <int kBits, int kN>
__device__ __forceinline__ bool cut_codes(u32x4 (&c)[kN], uint8_t (&s)[kN], int i, bool seen) {
  bool finite = s[i] <= quant::kHighest<kBits>;
#pragma unroll
  for (int x = 0; x < 4; ++x) {
    // 8 bits: 0x7f is NaN
    if constexpr (kBits == 8) finite = finite && (((c[i][x] & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u) == 0;
    c[i][x] = seen ? c[i][x] : 0;
  }
  s[i] = seen ? s[i] : 127;
  return finite || !seen;
}

// A token's codes as the kG lanes that share it load them: pieces of 16 bytes a lane, then of
// 8 and 4 where the rest is less.  Piece i of lane group g is kBytes(i) bytes from at(i) + g * kBytes(i) on.
template <int DP, int kBits, int kG>
struct LaneCodes {
  static constexpr int kRow = DP * kBits / 8;                        // bytes of a token
  static constexpr int kFull = kRow / (16 * kG), kRest = kRow % (16 * kG);
  static constexpr int kPieces = kFull + (kRest >= 8 * kG) + (kRest % (8 * kG) >= 4 * kG);
  static __host__ __device__ constexpr int bytes(int i) { return i < kFull ? 16 : i == kFull && kRest >= 8 * kG ? 8 : 4; }
  static __host__ __device__ constexpr int at(int i) {
    return i <= kFull ? i * 16 * kG : kFull * 16 * kG + 8 * kG;
  }
  static __host__ __device__ constexpr int operands(int i) { return bytes(i) / kBits; }  // of 8 elements
  static __host__ __device__ constexpr int first(int i) { return at(i) / (kG * kBits); }  // operands before piece i
  static constexpr int kOperands = kRow / (kG * kBits);
  // first element of operand o of piece i
  static __host__ __device__ constexpr int element(int i, int o, int g) { return (at(i) + g * bytes(i)) * 8 / kBits + 8 * o; }

  u32x4 c[kPieces];
  uint8_t s[kPieces];  // scale bytes
  template <bool kStream>
  __device__ __forceinline__ void load(const uint8_t* tile, int r, int g) {
    auto get = [](const auto* p) { return kStream ? __builtin_nontemporal_load(p) : *p; };
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      const int x = at(i) + g * bytes(i);
      const uint8_t* p = tile + (x / 16 * kTileTokens + r) * 16 + x % 16;
      if (bytes(i) == 16) {
        c[i] = get(reinterpret_cast<const u32x4*>(p));
      } else if (bytes(i) == 8) {
        const u32x2 w = get(reinterpret_cast<const u32x2*>(p));
        c[i] = u32x4{w[0], w[1], 0, 0};
      } else {
        c[i] = u32x4{get(reinterpret_cast<const uint32_t*>(p)), 0, 0, 0};
      }
      s[i] = tile[scale_at<kBits>(DP, r) + x * 8 / kBits / kGroup];
    }
  }
  __device__ __forceinline__ bf16x8 operand(int i, int o, float scale) const {
    const uint32_t w[2] = {c[i][o * kBits / 4], c[i][kBits == 8 ? 2 * o + 1 : o]};
    return decode<kBits>(w, scale);
  }
  __device__ __forceinline__ bool cut(bool seen) {
    bool finite = true;
#pragma unroll
    for (int i = 0; i < kPieces; ++i) finite = cut_codes<kBits>(c, s, i, seen) && finite;
    return finite;
  }
};

// Values of a tile in LDS: 32 rows of tokens, kRow bytes apart.  Rows of four tokens lie in
// different banks (kRow is 64 bytes more than a multiple of 256, or 64 less), and the 16-byte pieces of every 64
// bytes change places with the token's second pair of bits, so that writes of
// one piece by 32 tokens use all banks too.
template <int DP>
struct TurnedValues {
  static constexpr int kRow = DP * 2 + (DP % 64 == 0 ? 64 : 0);
  static constexpr int kBytes = kTileTokens * kRow;
  static __device__ __forceinline__ int piece(int r, int p) { return r * kRow + (p ^ (r >> 2 & 3)) * 16; }
  static __device__ __forceinline__ void write(char* lds, int r, int p, const bf16x8& x) { *reinterpret_cast<bf16x8*>(lds + piece(r, p)) = x; }
};

// Reads of values turned, for results of kR rows: operand s of block b, element 4j + t of lane (element d = lane % kR of
// the block, group g = lane / kR), is token 4G (2s + j) + 4g + t, G = 64 / kR.  Within 16 lanes, lane i
// points at token i / 4 of four, elements 4 (i % 4) on, and receives element i of the four tokens.
template <int DP, int kR>
struct TurnedRead {
  static constexpr int kG = 64 / kR, kRow = TurnedValues<DP>::kRow;
  int at[2];
  __device__ __forceinline__ TurnedRead(int lane) {
    const int g = lane / kR, i = lane & 15, p = (kR == 32 ? (lane >> 4 & 1) * 2 : 0) + (i & 3) / 2;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int t = 4 * kG * j + 4 * g;  // the first of the four tokens
      at[j] = (t + i / 4) * kRow + (p ^ (t >> 2 & 3)) * 16 + (i & 1) * 8;
    }
  }
  __device__ __forceinline__ bf16x8 read(const char* lds, int b, int s) const {
    bf16x4 x[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      // 16 elements on are two pieces on: with pieces that change places, another bit of the place
      const int a = kR == 16 && (b & 1) ? at[j] ^ 32 : at[j];
      x[j] = __builtin_amdgcn_ds_read_tr16_b64_v4bf16(
          (__attribute__((address_space(3))) bf16x4*)(lds + a + s * (8 * kG * kRow) + b * kR / 32 * 64));
    }
    return __builtin_shufflevector(x[0], x[1], 0, 1, 2, 3, 4, 5, 6, 7);
  }
};

// What is written to LDS before is read after, and the other way round: a wave's LDS
// instructions act in their order.
__device__ __forceinline__ void lds_order() { asm volatile("" ::: "memory"); }

template <int kG>
__device__ __forceinline__ float groups_max(float v) {
  if constexpr (kG == 4) {
    const auto s = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = fmaxf(__uint_as_float(s[0]), __uint_as_float(s[1]));
  }
  return other_half_max(v);
}
template <int kG>
__device__ __forceinline__ float groups_sum(float v) {
  if constexpr (kG == 4) {
    const auto s = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(s[0]) + __uint_as_float(s[1]);
  }
  return other_half_sum(v);
}

// A wave's kR rows (lane % kR) against tiles of 32 keys.  Group g = lane / kR of the wave holds keys 4G (i / 4) + 4g +
// i % 4 in register i of a tile's scores, G = 64 / kR, and elements kR b + 4G (i / 4) + 4g + i % 4 in register i of block b of
// the sums.
template <typename T, int DP, int kR, bool kPin>
struct QuantRows {
  static constexpr int kG = 64 / kR, kP = kParts<T>;
  static constexpr int kK = DP / (8 * kG);  // operands of a token's keys: 8 elements of every group
  static constexpr int kS = 4 / kG;         // operands of a tile's values
  static constexpr int kB = DP / kR;        // blocks of the output
  static constexpr int kN = 32 / kG;        // scores of a tile in a lane
  static constexpr int kO = kR * kR / 64;   // registers of a block
  typedef float Sums __attribute__((ext_vector_type(kO)));
  bf16x8 q[kP][kK];
  Sums o[kB];
  float m, l;  // l: of this group's keys
  int end;     // keys the row sees
  int lo, hi;  // the least and most of the wave's rows (uniform)

  static __device__ __forceinline__ constexpr int key(int i, int g) { return 4 * kG * (i / 4) + 4 * g + i % 4; }
  static __device__ __forceinline__ constexpr int element(int b, int i, int g) { return kR * b + key(i, g); }

  // element(j): the first element of operand j
  template <typename Place, typename F>
  __device__ __forceinline__ void load(const Place& rows, const AttnArgs& a, const AttnItem& it, F element) {
    const T* qp = rows.query(a, it);
#pragma unroll
    for (int j = 0; j < kK; ++j) {
      const int d = element(j);
      const bool on = rows.live && d < a.cache.head_dim;
      if constexpr (kP == 1) {
        bf16x8 f{};
        if (on) f = *reinterpret_cast<const bf16x8*>(qp + d);
        q[0][j] = f;
      } else {
        float x[8] = {};
        if (on) {
          const f32x4 u = *reinterpret_cast<const f32x4*>(qp + d), v = *reinterpret_cast<const f32x4*>(qp + d + 4);
#pragma unroll
          for (int e = 0; e < 4; ++e) x[e] = u[e], x[4 + e] = v[e];
        }
        bf16x8 f[3];
        split(x, f);
#pragma unroll
        for (int p = 0; p < 3; ++p) q[p][j] = f[p];
      }
    }
  }
  __device__ __forceinline__ void clear() {
    m = -INFINITY;
    l = 0.f;
#pragma unroll
    for (int b = 0; b < kB; ++b)
#pragma unroll
      for (int i = 0; i < kO; ++i) o[b][i] = 0.f;
  }
  // WaveRows::pin
  __device__ __forceinline__ void pin() {
    if constexpr (kPin) {
#pragma unroll
      for (int b = 0; b < kB; ++b) asm volatile("" : "+a"(o[b]));
    }
  }
  static __device__ __forceinline__ void mma(Sums& acc, const bf16x8& a, const bf16x8& b) {
    if constexpr (kR == 32)
      acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, acc, 0, 0, 0);
    else
      acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, acc, 0, 0, 0);
  }
  // operand j of keys kR x .. kR x + kR - 1 of a tile
  __device__ __forceinline__ void score(float (&s)[kN], int x, const bf16x8& k, int j) const {
    Sums acc;
#pragma unroll
    for (int i = 0; i < kO; ++i) acc[i] = s[kO * x + i];
    // smallest parts first
#pragma unroll
    for (int p = kP - 1; p >= 0; --p) mma(acc, k, q[p][j]);
#pragma unroll
    for (int i = 0; i < kO; ++i) s[kO * x + i] = acc[i];
  }
  // WaveRows::softmax; the groups' maxima meet only where one of them has to be raised.  masked: keys of tile n from
  // seen[n] on are not seen.
  template <int NT>
  __device__ __forceinline__ void softmax(float (&s)[NT][kN], float scale2, bool masked, const int (&seen)[NT], int g) {
    if (masked) {
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < kN; ++i) s[n][i] = key(i, g) < seen[n] ? s[n][i] : -INFINITY;
    }
    float t = s[0][0];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int i = 0; i < kN; ++i) t = fmaxf(t, s[n][i]);
    t *= scale2;
    pin();
    if (__any(t > m + kLazy)) {
      const float nm = fmaxf(m, groups_max<kG>(t));
      const float a = nm == m ? 1.f : exp2_hw(m - nm);
      m = nm;
      scale(a);
    }
    pin();
    const float off = m == -INFINITY ? 0.f : m;
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int i = 0; i < kN; ++i) {
        s[n][i] = exp2_hw(__builtin_fmaf(s[n][i], scale2, -off));
        l += s[n][i];
      }
  }
  __device__ __forceinline__ void scale(float fac) {
    l *= fac;
#pragma unroll
    for (int b = 0; b < kB; ++b)
#pragma unroll
      for (int i = 0; i < kO; ++i) o[b][i] *= fac;
  }
  // probabilities of operand s of a tile's values
  static __device__ __forceinline__ void probs(const float (&p)[kN], int s, bf16x8 (&f)[kP]) {
    if constexpr (kP == 1) {
#pragma unroll
      for (int i = 0; i < 8; ++i) f[0][i] = static_cast<__bf16>(p[8 * s + i]);
    } else {
      float x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = p[8 * s + i];
      split(x, f);
    }
  }
  template <typename F>
  __device__ __forceinline__ void add(const float (&p)[kN], F value) {
#pragma unroll
    for (int s = 0; s < kS; ++s) {
      bf16x8 f[kP];
      probs(p, s, f);
#pragma unroll
      for (int b = 0; b < kB; ++b) {
        const bf16x8 v = value(b, s);
#pragma unroll
        for (int x = kP - 1; x >= 0; --x) mma(o[b], v, f[x]);
      }
    }
  }
  // WaveRows::add_keys: a key's products are added to the rows that see it
  __device__ __forceinline__ void add_keys(const float (&p)[kN], const bf16x8 (&v)[kB][kS], int key0, int g) {
#pragma unroll
    for (int s = 0; s < kS; ++s) {
      bf16x8 f[kP];
      probs(p, s, f);
#pragma unroll 1
      for (int r = 0; r < 8 * kG; ++r) {
        const int slot = r / 4 % kG == g ? r / (4 * kG) * 4 + r % 4 : -1;
        const bool sees = key0 + 8 * kG * s + r < end;
#pragma unroll
        for (int b = 0; b < kB; ++b) {
          const bf16x8 x = WaveRows<bf16_t, 32>::only(v[b][s], slot);
          Sums t;
#pragma unroll
          for (int i = 0; i < kO; ++i) t[i] = 0.f;
#pragma unroll
          for (int y = kP - 1; y >= 0; --y) mma(t, x, WaveRows<bf16_t, 32>::only(f[y], slot));
#pragma unroll
          for (int i = 0; i < kO; ++i) o[b][i] += sees ? t[i] : 0.f;
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    }
  }
};

// The item's rows of a wave, kR of them: as RowPlace.
template <typename T, int DP, int kR>
struct QuantPlace {
  int row, tok, qh;
  bool live, any;
  template <typename Rows>
  __device__ __forceinline__ QuantPlace(Rows& w, const AttnArgs& a, const QuantShape& sh, const AttnItem& it, int hk, int row_lo, int lane) {
    row = row_lo + lane % kR;
    live = row < it.rows;
    any = row_lo < it.rows;
    tok = live ? sh.by_group.of(row) : 0;
    qh = hk * sh.group + (live ? row - tok * sh.group : 0);
    w.end = live ? seen_end(a, sh, it, tok) : 0;
    w.lo = any ? seen_end(a, sh, it, sh.by_group.of(row_lo)) : 0;
    w.hi = any ? seen_end(a, sh, it, sh.by_group.of(min(row_lo + kR, it.rows) - 1)) : 0;
  }
  // visible_end of the item's token
  static __device__ __forceinline__ int seen_end(const AttnArgs& a, const QuantShape& sh, const AttnItem& it, int tok) {
    const int p = it.len - it.n + tok;
    if (p < 0) return 0;
    if (a.mask_block <= 0) return it.len;
    const long e = (static_cast<long>(sh.by_mask.of(p)) + 1) * a.mask_block;
    return e < it.len ? static_cast<int>(e) : it.len;
  }
  __device__ __forceinline__ const T* query(const AttnArgs& a, const AttnItem& it) const {
    return static_cast<const T*>(a.q) + (it.row0 + tok) * a.q_stride + static_cast<long>(qh) * a.cache.head_dim;
  }
  // The row's sums, x(i) elements d(i) .. d(i) + 3 of them for i < kN: divided into out, or as they are into the workspace;
  // with `whole`, what belongs to the row once.
  template <int kN, typename X, typename D>
  __device__ __forceinline__ void store(X x, D d, float m, float l, bool whole, const AttnArgs& a, const QuantShape& sh, const AttnItem& it,
                                        int hk, int part_rows) const {
    if (!live) return;
    if (it.part >= 0) {
      const long tile = (static_cast<long>(it.part) * a.cache.n_kv_heads + hk) * sh.tile_rows;
      const int r = row - it.first;
      float* po = static_cast<float*>(a.workspace) + tile * DP;
#pragma unroll
      for (int i = 0; i < kN; ++i) store4(po + partial_at(DP, r, d(i)), x(i));
      if (whole) reinterpret_cast<float2*>(static_cast<float*>(a.workspace) + static_cast<long>(part_rows) * DP)[tile + r] = make_float2(m, l);
      return;
    }
    const bool some = l > 0.f || l != l;
    const float inv = some ? 1.f / l : 0.f;
    T* op = static_cast<T*>(a.out) + (it.row0 + tok) * a.out_stride + static_cast<long>(qh) * a.cache.head_dim;
#pragma unroll
    for (int i = 0; i < kN; ++i)
      if (d(i) < a.cache.head_dim) store4(op + d(i), divided(x(i), some, inv));
    if (whole && a.lse) a.lse[static_cast<long>(it.row0 + tok) * a.n_heads + qh] = some ? (m + log2f(l)) * kLn2 : -INFINITY;
  }
};

// Where a sequence's tiles of one kv head lie: as TileMap, in bytes.
template <int DP, int kKB, int kVB>
struct QuantMap {
  static constexpr int kKTile = quant_tile(kKB, DP), kVTile = quant_tile(kVB, DP);
  const uint8_t *k, *v;
  const __attribute__((address_space(4))) int32_t* table;
  long layer0;
  int n_pages, tpp, per_page;  // tiles of a page of one kv head, of all
  FastDiv by_page;
  __device__ __forceinline__ QuantMap(const AttnArgs& a, const QuantShape& sh, int slot, int hk)
      : n_pages(a.cache.n_pages), tpp(a.cache.page_tokens / kTileTokens), by_page(sh.by_page) {
    table = (const __attribute__((address_space(4))) int32_t*)(a.cache.table + static_cast<long>(slot) * a.cache.max_pages);
    per_page = tpp * a.cache.n_kv_heads;
    layer0 = static_cast<long>(a.layer) * n_pages;
    k = static_cast<const uint8_t*>(a.cache.k) + static_cast<long>(hk * tpp) * kKTile;
    v = static_cast<const uint8_t*>(a.cache.v) + static_cast<long>(hk * tpp) * kVTile;
  }
  __device__ __forceinline__ int page(int kt, int end) const { return kt < end ? table[by_page.of(kt)] : -1; }
  __device__ __forceinline__ bool holds(int page) const { return static_cast<unsigned>(page) < static_cast<unsigned>(n_pages); }
  // tiles from k and v to a tile on a page; of no page: some tile of the pool
  __device__ __forceinline__ long at(int kt, int page) const {
    return (layer0 + (holds(page) ? page : 0)) * per_page + (kt - by_page.of(kt) * tpp);
  }
  __device__ __forceinline__ const uint8_t* key(long tile) const { return k + tile * kKTile; }
  __device__ __forceinline__ const uint8_t* value(long tile) const { return v + tile * kVTile; }
};

// A tile's codes in a wave's registers: keys by kR tokens, values by 32.
template <int DP, int kKB, int kVB, int kR>
struct WaveTile {
  typedef LaneCodes<DP, kKB, 64 / kR> Keys;
  typedef LaneCodes<DP, kVB, 2> Values;
  Keys k[32 / kR];
  Values v;
  template <bool kStream>
  __device__ __forceinline__ void load_keys(const uint8_t* tile, int lane) {
#pragma unroll
    for (int x = 0; x < 32 / kR; ++x) k[x].template load<kStream>(tile, kR * x + lane % kR, lane / kR);
  }
  template <bool kStream>
  __device__ __forceinline__ void load_values(const uint8_t* tile, int lane) {
    v.template load<kStream>(tile, lane % 32, lane / 32);
  }
  template <typename Rows>
  __device__ __forceinline__ void scores(const Rows& w, float (&s)[Rows::kN]) const {
#pragma unroll
    for (int i = 0; i < Rows::kN; ++i) s[i] = 0.f;
#pragma unroll
    for (int i = 0; i < Keys::kPieces; ++i)
#pragma unroll
      for (int x = 0; x < 32 / kR; ++x) {
        const float scale = scale_of(k[x].s[i]);
#pragma unroll
        for (int o = 0; o < Keys::operands(i); ++o) w.score(s, x, k[x].operand(i, o, scale), Keys::first(i) + o);
      }
  }
  // the values to this wave's place in LDS
  __device__ __forceinline__ void open_values(char* lds, int lane) const {
    lds_order();
#pragma unroll
    for (int i = 0; i < Values::kPieces; ++i) {
      const float scale = scale_of(v.s[i]);
      const int p = Values::element(i, 0, lane / 32) / 8;
#pragma unroll
      for (int o = 0; o < Values::operands(i); ++o) TurnedValues<DP>::write(lds, lane % 32, p + o, v.operand(i, o, scale));
    }
    lds_order();
  }
};

// Tiles left out because they hold, before token hi, a value that is perhaps not finite, once the running maximum is the
// last one (WaveRows::add_by_key).  masked(kt): the tile was looked at for that; scores(s, keys): a tile's scores.
template <int DP, int kKB, int kVB, int kR, typename Rows, typename Map, typename Masked, typename Scores>
__device__ __forceinline__ void add_by_key(Rows& w, const Map& map, int kt, int kt1, int step, int hi, float scale2, int lane, char* lds,
                                           Masked masked, Scores scores) {
  const int g = lane / kR;
#pragma unroll 1
  for (; kt < kt1; kt += step) {
    const int page = map.page(kt, kt1), key0 = kt * kTileTokens;
    if (!map.holds(page) || key0 >= w.hi || !masked(kt)) continue;
    const long at = map.at(kt, page);
    bf16x8 v[Rows::kB][Rows::kS];
    {
      WaveTile<DP, kKB, kVB, kR> t;
      t.template load_values<false>(map.value(at), lane);
      if (__all(t.v.cut(lane % 32 < hi - key0))) continue;
      t.open_values(lds, lane);
      const TurnedRead<DP, kR> turned(lane);
#pragma unroll
      for (int b = 0; b < Rows::kB; ++b)
#pragma unroll
        for (int s = 0; s < Rows::kS; ++s) v[b][s] = turned.read(lds, b, s);
    }
    float s[Rows::kN];
    scores(s, map.key(at));
    const float off = w.m == -INFINITY ? 0.f : w.m;
#pragma unroll
    for (int i = 0; i < Rows::kN; ++i) s[i] = Rows::key(i, g) < w.end - key0 ? exp2_hw(__builtin_fmaf(s[i], scale2, -off)) : 0.f;
    w.add_keys(s, v, key0, g);
  }
}

// The sums of kW waves over different keys joined and stored: every wave lays its own in LDS, then takes an equal share of all.
// (A tree of pairs had eight waves wait for 3.5 us; code that runs once costs its way into the instruction cache.)
template <int kW, typename Rows, typename Place>
__device__ __forceinline__ void join_store(const Rows& w, float* lds, int wave, int lane, const Place& rows, const AttnArgs& a, const QuantShape& sh,
                                           const AttnItem& it, int hk, int part_rows) {
  constexpr int kUnits = Rows::kO * Rows::kB / 4, kLen = (4 * kUnits + 2) * 64, kMine = (kUnits + kW - 1) / kW;
  static_assert(Rows::kO == 4 || Rows::kO == 16);
  float* mine = lds + wave * kLen;
  mine[lane] = w.m;
  mine[64 + lane] = w.l;
#pragma unroll
  for (int u = 0; u < kUnits; ++u) {
    const int b = u / (Rows::kO / 4), i = u % (Rows::kO / 4) * 4;
    store4(mine + 128 + u * 256 + lane * 4, f32x4{w.o[b][i], w.o[b][i + 1], w.o[b][i + 2], w.o[b][i + 3]});
  }
  __syncthreads();
  if (kUnits % kW && wave * kMine >= kUnits) return;
  float f[kW], m = -INFINITY, l = 0.f;
#pragma unroll
  for (int x = 0; x < kW; ++x) {
    f[x] = lds[x * kLen + lane];
    m = fmaxf(m, f[x]);
  }
#pragma unroll
  for (int x = 0; x < kW; ++x) {
    f[x] = f[x] == m ? 1.f : exp2_hw(f[x] - m);
    l += f[x] * lds[x * kLen + 64 + lane];
  }
  const int g = lane / (64 / Rows::kG);
  f32x4 o[kMine];
#pragma unroll
  for (int y = 0; y < kMine; ++y) {
    o[y] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int x = 0; x < kW; ++x) o[y] += f[x] * *reinterpret_cast<const f32x4*>(lds + x * kLen + 128 + (wave * kMine + y) * 256 + lane * 4);
  }
  rows.template store<kMine>([&](int y) { return o[y]; },
                             [&](int y) {
                               const int u = wave * kMine + y;
                               return Rows::element(u / (Rows::kO / 4), u % (Rows::kO / 4) * 4, g);
                             },
                             m, l, wave == 0 && g == 0, a, sh, it, hk, part_rows);
}

template <typename T, int DP, int kKB, int kVB, int kR>
constexpr int rows_waves = quant_rows_waves(kParts<T>, DP, kKB + kVB, kR);

// Few rows: kR of one kv head per workgroup, its kW waves each on every kW-th key tile, joined through LDS.  Codes go
// straight into registers, past the caches, the next tile's while one is used.  Bound by those loads: 64 single tokens
// over 363,063 (32 and 8 heads of 128 in 4 bits, page 64; 396 MB) 85 us, 4.7 TB/s, of which 70 are left with
// loads alone; one over 131,000 (143 MB) 35 us with plan and merge.  Loads further ahead, or a third wave of a SIMD: as
// fast; through the caches 98.  Eight waves take 94 us for the 64, and win where there are few (attn_shape).  A block of 32 tokens over 4096, four kv heads of 32 rows by 4: a
// chain of one load after another, 10 us where 7 TB/s would take 1.
template <typename T, int DP, int kKB, int kVB, int kR, int kW>
__global__ __launch_bounds__(64 * kW, (rows_waves<T, DP, kKB, kVB, kR>)) void quant_rows_kernel(AttnArgs a, QuantShape sh, int part_rows) {
  constexpr bool kPin = rows_waves<T, DP, kKB, kVB, kR> == 1;
  typedef QuantRows<T, DP, kR, kPin> Rows;
  typedef WaveTile<DP, kKB, kVB, kR> Tile;
  typedef typename Tile::Keys Keys;
  extern __shared__ float lds[];
  const int hkv = a.cache.n_kv_heads;
  const int item_i = blockIdx.x / hkv, hk = blockIdx.x % hkv;
  AttnItem it;
  if (!load_item(a, item_i, it)) return;
  const int lane = threadIdx.x & 63, g = lane / kR;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  char* mine = reinterpret_cast<char*>(lds) + wave * TurnedValues<DP>::kBytes;
  const TurnedRead<DP, kR> turned(lane);
  Rows w;
  w.clear();
  const QuantPlace<T, DP, kR> rows(w, a, sh, it, hk, it.first, lane);
  const float scale2 = a.scale * kLog2e;
  const QuantMap<DP, kKB, kVB> map(a, sh, it.slot, hk);
  const int kt1 = min(it.kt1, (w.hi + kTileTokens - 1) / kTileTokens);
  // page ids are known two of this wave's tiles ahead, codes one; of no page, and behind the last tile, some tile of the pool's
  int kt = it.kt0 + wave;
  int page = -1;
  if (wave >= 4)
    page = map.page(kt, kt1);
  else if (kt < kt1)
    page = wave < 2 ? wave == 0 ? it.page[0] : it.page[1] : wave == 2 ? it.page[2] : it.page[3];
  Tile t;
  auto fetch = [&](int at_kt, int pg) {
    const long at = map.at(at_kt, pg);
    t.template load_keys<true>(map.key(at), lane);
    t.template load_values<true>(map.value(at), lane);
  };
  fetch(kt, page);
  const int now = map.page(kt, kt1);
  int page1 = map.page(kt + kW, kt1);
  w.load(rows, a, it, [&](int j) {
    int d = 0;
#pragma unroll
    for (int i = 0; i < Keys::kPieces; ++i)
      if (j >= Keys::first(i)) d = Keys::element(i, j - Keys::first(i), g);
    return d;
  });
  if (now != page) {  // moved since the plan was made
    page = now;
    fetch(kt, page);
  }
  // tiles that every row sees whole come first
  const int whole = min(kt1, w.lo / kTileTokens);
  int left = kt1;  // the first tile for add_by_key
  while (kt < kt1) {
    w.pin();
    const int page2 = map.page(kt + 2 * kW, kt1), key0 = kt * kTileTokens;
    const bool masked = kt >= whole;
    bool finite = true;
    if (masked) finite = __all(t.v.cut(lane % 32 < w.hi - key0));
    float s[1][Rows::kN];
    t.scores(w, s[0]);
    t.open_values(mine, lane);
    fetch(kt + kW, page1);
    if (map.holds(page)) {
      const int seen[1] = {w.end - key0};
      w.template softmax<1>(s, scale2, masked, seen, g);
      // a value that is not finite must not reach the rows that do not see it
      if (finite)
        w.add(s[0], [&](int b, int x) { return turned.read(mine, b, x); });
      else
        left = min(left, kt);
    }
    kt += kW;
    page = page1;
    page1 = page2;
  }
  w.pin();
  if (left < kt1)
    add_by_key<DP, kKB, kVB, kR>(w, map, left, kt1, kW, w.hi, scale2, lane, mine, [](int) { return true; }, [&](float (&s)[Rows::kN], const uint8_t* p) {
      Tile other;
      other.template load_keys<false>(p, lane);
      other.scores(w, s);
    });
  w.l = groups_sum<Rows::kG>(w.l);
  __syncthreads();  // the values' places are taken by the sums
  join_store<kW>(w, lds, wave, lane, rows, a, sh, it, hk, part_rows);
}

// Keys and values of kTS tiles in LDS: keys as operands, element 16j + 8 half + e of
// token r at [j][32 half + r][e], values in rows.
template <int DP>
struct QuantStage {
  static constexpr int kTS = stage_tiles(DMOE_BF16, DP), kK = DP / 16;
  bf16x8 k[kTS][kK][64];
  char v[kTS][TurnedValues<DP>::kBytes];
  int bad[4];  // the tile whose values are perhaps not all finite, where rows see some of them and not others
  char more[kTS == 1 ? TurnedValues<DP>::kBytes - DP * 64 : 64];  // the two stages hold a tile's values of four waves
};

// A thread's share of a stage's keys (or values): chunk u of [tile][chunk][token], u = thread, thread + 256, ...
template <int DP, int kBits, int kTS>
struct StageCodes {
  static constexpr int kChunks = DP * kBits / 128, kUnits = kTS * kChunks * kTileTokens, kMine = (kUnits + 255) / 256;
  u32x4 c[kMine] = {};
  uint8_t s[kMine] = {};
  static __device__ __forceinline__ bool has(int i) { return kUnits % 256 == 0 || static_cast<int>(threadIdx.x) + 256 * i < kUnits; }
  static __device__ __forceinline__ int tile(int i) { return (threadIdx.x + 256 * i) / (kChunks * kTileTokens); }
  static __device__ __forceinline__ int chunk(int i) { return (threadIdx.x + 256 * i) / kTileTokens % kChunks; }
  // base[n]: where tile n lies
  __device__ __forceinline__ void load(const uint8_t* const (&base)[kTS]) {
    const int r = threadIdx.x % kTileTokens;
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
      const uint8_t* p = base[0];
#pragma unroll
      for (int n = 1; n < kTS; ++n) p = tile(i) == n ? base[n] : p;
      if (!has(i)) continue;
      c[i] = *reinterpret_cast<const u32x4*>(p + (chunk(i) * kTileTokens + r) * 16);
      s[i] = p[scale_at<kBits>(DP, r) + chunk(i) * 128 / (kBits * kGroup)];
    }
  }
  // seen[n]: tokens of tile n that are seen by some row; bad(n): it holds a value that is perhaps not finite
  template <typename F>
  __device__ __forceinline__ void cut(const int (&seen)[kTS], F bad) {
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
      int upto = seen[0];
#pragma unroll
      for (int n = 1; n < kTS; ++n) upto = tile(i) == n ? seen[n] : upto;
      if (!cut_codes<kBits>(c, s, i, static_cast<int>(threadIdx.x) % kTileTokens < upto) && has(i)) bad(tile(i));
    }
  }
  template <typename F>
  __device__ __forceinline__ void open(F put) const {
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
      if (!has(i)) continue;
      const float scale = scale_of(s[i]);
#pragma unroll
      for (int o = 0; o < 16 / kBits; ++o) {
        const uint32_t w[2] = {c[i][o * kBits / 4], c[i][kBits == 8 ? 2 * o + 1 : o]};
        put(tile(i), chunk(i) * (16 / kBits) + o, decode<kBits>(w, scale));
      }
    }
  }
};

template <typename T>
constexpr int quant_waves(int dp) {
  return quant_two_per_cu(sizeof(T) == 4 ? DMOE_F32 : DMOE_BF16, dp) ? 2 : 1;
}

// Many rows: 128 of one kv head per workgroup, 32 to a wave, all four waves on the same keys.  Codes of kTS tiles
// are loaded two stages ahead, opened into LDS one stage ahead, each by one of the
// threads; one barrier a stage.  Bound by matrix products and the exponentials between them: 4096 rows of 16 heads of 128
// over 16384 keys in 4 bits, 525 us, 920 TFLOP/s (a library product 1210; a cache of bf16 490 us); the first calls after a
// pause take 570 to 650, until the clock has risen.  fp32 rows of 256 elements have no room for the queries' parts and spill 460
// to 524 bytes a lane; so does the form of 32 rows (440 to 484), which took 303 us for 1024 tokens of 8 and 4 heads over 4096 where
// this one took 258.
template <typename T, int DP, int kKB, int kVB>
__global__ __launch_bounds__(256, quant_waves<T>(DP)) void quant_block_kernel(AttnArgs a, QuantShape sh, int part_rows) {
  typedef QuantStage<DP> Stage;
  typedef QuantRows<T, DP, 32, quant_waves<T>(DP) == 1> Rows;
  constexpr int kK = Stage::kK, kTS = Stage::kTS;
  __shared__ Stage s0, s1;
  const int hkv = a.cache.n_kv_heads;
  const int item_i = blockIdx.x / hkv, hk = blockIdx.x % hkv;
  AttnItem it;
  if (!load_item(a, item_i, it)) return;
  const int lane = threadIdx.x & 63, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const TurnedRead<DP, 32> turned(lane);
  Rows w;
  w.clear();
  const QuantPlace<T, DP, 32> rows(w, a, sh, it, hk, it.first + 32 * wave, lane);
  w.load(rows, a, it, [&](int j) { return 16 * j + 8 * half; });
  const float scale2 = a.scale * kLog2e;
  const QuantMap<DP, kKB, kVB> map(a, sh, it.slot, hk);
  const int kt0 = it.kt0, kt1 = it.kt1, turns = (kt1 - kt0 + kTS - 1) / kTS;
  struct Ids {
    int id[kTS];
  };
  auto pages = [&](int kt) {
    Ids p;
#pragma unroll
    for (int n = 0; n < kTS; ++n) p.id[n] = map.page(kt + n, kt1);
    return p;
  };
  StageCodes<DP, kKB, kTS> kc;
  StageCodes<DP, kVB, kTS> vc;
  auto load = [&](int kt, const Ids& pg) {
    const uint8_t *kb[kTS], *vb[kTS];
#pragma unroll
    for (int n = 0; n < kTS; ++n) {
      const long at = map.at(kt + n, pg.id[n]);
      kb[n] = map.key(at);
      vb[n] = map.value(at);
    }
    kc.load(kb);
    vc.load(vb);
  };
  // stages whose keys every row of the workgroup sees, all of them on pages, come first in a sequence that has them
  auto end_of = [&](int row) { return rows.seen_end(a, sh, it, sh.by_group.of(row)); };
  const int whole = end_of(it.first) / kTileTokens, hi = end_of(min(it.first + 128, it.rows) - 1);
  auto plain = [&](int kt, const Ids& pg) {
    bool all = kt + kTS <= whole;
#pragma unroll
    for (int n = 0; n < kTS; ++n) all = all && map.holds(pg.id[n]);
    return all;
  };
  auto open = [&](int kt, const Ids& pg, Stage& st) {
    const int r = threadIdx.x % kTileTokens;
    if (!plain(kt, pg)) {
      int seen[kTS];
#pragma unroll
      for (int n = 0; n < kTS; ++n) seen[n] = map.holds(pg.id[n]) ? hi - (kt + n) * kTileTokens : 0;
      kc.cut(seen, [](int) {});
      vc.cut(seen, [&](int n) { st.bad[n] = kt + n; });
    }
    kc.open([&](int n, int p, const bf16x8& x) { st.k[n][p / 2][32 * (p & 1) + r] = x; });
    vc.open([&](int n, int p, const bf16x8& x) { TurnedValues<DP>::write(st.v[n], r, p, x); });
  };
  int left = it.kt1;  // the first tile for add_by_key
  auto compute = [&](int kt, const Ids& pg, const Stage& st) {
    if (!rows.any) return;
    float s[kTS][Rows::kN];
#pragma unroll
    for (int n = 0; n < kTS; ++n) {
#pragma unroll
      for (int i = 0; i < Rows::kN; ++i) s[n][i] = 0.f;
#pragma unroll
      for (int j = 0; j < kK; ++j) w.score(s[n], 0, st.k[n][j][lane], j);
    }
    const bool masked = !plain(kt, pg);
    int seen[kTS];
#pragma unroll
    for (int n = 0; n < kTS; ++n) seen[n] = map.holds(pg.id[n]) ? w.end - (kt + n) * kTileTokens : 0;
    w.template softmax<kTS>(s, scale2, masked, seen, half);
#pragma unroll
    for (int n = 0; n < kTS; ++n) {
      // a value that is not finite must not reach the rows that do not see it
      if (masked && __builtin_amdgcn_readfirstlane(st.bad[n]) == kt + n)
        left = min(left, kt + n);
      else
        w.add(s[n], [&](int b, int x) { return turned.read(st.v[n], b, x); });
    }
  };
  int kt = kt0;
  Ids pg = pages(kt), pg1 = pages(kt + kTS);
  if (threadIdx.x < 2 * kTS) (threadIdx.x < kTS ? s0 : s1).bad[threadIdx.x % kTS] = -1;
  load(kt, pg);
  __syncthreads();
  open(kt, pg, s0);
  load(kt + kTS, pg1);
  // every wave takes all turns, for their barriers
  auto turn = [&](Stage& cur, Stage& fill) {
    w.pin();
    // a stage's writes are done, by all; the other buffer has been read
    lds_order();
    __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
    lds_order();
    const Ids pg2 = pages(kt + 2 * kTS);
    open(kt + kTS, pg1, fill);
    load(kt + 2 * kTS, pg2);
    __builtin_amdgcn_sched_barrier(0);
    compute(kt, pg, cur);
    kt += kTS;
    pg = pg1;
    pg1 = pg2;
  };
  int done = 0;
  for (; done + 2 <= turns; done += 2) {
    turn(s0, s1);
    turn(s1, s0);
  }
  if (done < turns) turn(s0, s1);
  __syncthreads();  // the stages are done with
  if (left < kt1) {
    static_assert(sizeof(Stage) >= 2 * TurnedValues<DP>::kBytes);
    char* room = reinterpret_cast<char*>(wave < 2 ? &s0 : &s1) + (wave & 1) * TurnedValues<DP>::kBytes;
    // the workgroup's flags, not the wave's: a tile may be left out for what only other waves' rows see
    auto masked = [&](int kt) {
      const int first = kt0 + (kt - kt0) / kTS * kTS;
      return !plain(first, pages(first));
    };
    add_by_key<DP, kKB, kVB, 32>(w, map, left, kt1, 1, hi, scale2, lane, room, masked, [&](float (&s)[Rows::kN], const uint8_t* p) {
      // operands in the queries' order, straight from memory: the lane's token, elements 16j + 8 half on
      const int r = lane & 31;
#pragma unroll
      for (int i = 0; i < Rows::kN; ++i) s[i] = 0.f;
#pragma unroll
      for (int j = 0; j < kK; ++j) {
        const int d = 16 * j + 8 * half;
        const uint32_t* c = reinterpret_cast<const uint32_t*>(p + code_at<kKB>(r, d));
        const uint32_t x[2] = {c[0], kKB == 8 ? c[1] : 0u};
        w.score(s, 0, decode<kKB>(x, scale_of(p[scale_at<kKB>(DP, r) + d / kGroup])), j);
      }
    });
  }
  w.l = other_half_sum(w.l);
  rows.template store<4 * Rows::kB>([&](int y) { return f32x4{w.o[y / 4][y % 4 * 4], w.o[y / 4][y % 4 * 4 + 1], w.o[y / 4][y % 4 * 4 + 2], w.o[y / 4][y % 4 * 4 + 3]}; },
                                    [&](int y) { return Rows::element(y / 4, y % 4 * 4, half); }, w.m, w.l, half == 0, a, sh, it, hk, part_rows);
}

template <typename T, int DP, int kKB, int kVB, int kR, int kW>
void launch_quant_rows(const AttnArgs& a, const QuantShape& sh, unsigned items, int part_rows, hipStream_t s) {
  constexpr size_t join = kW * (kR * DP / 64 + 2) * 64 * sizeof(float), values = kW * TurnedValues<DP>::kBytes;
  quant_rows_kernel<T, DP, kKB, kVB, kR, kW><<<items, 64 * kW, join > values ? join : values, s>>>(a, sh, part_rows);
}

template <typename T, int DP, int kKB, int kVB>
hipError_t launch_quant_dim(const AttnArgs& a, const QuantShape& sh, hipStream_t s) {
  const int hkv = a.cache.n_kv_heads;
  const unsigned items = static_cast<unsigned>(sh.max_items() * hkv);
  const int part_rows = static_cast<int>(sh.max_parts() * hkv * sh.tile_rows);
  const long most = static_cast<long>(a.batch.max_new < a.batch.T ? a.batch.max_new : a.batch.T) * sh.group;
  if (sh.tile_rows == 128)
    quant_block_kernel<T, DP, kKB, kVB><<<items, 256, 0, s>>>(a, sh, part_rows);
  else if (most <= 16 && sh.wide)
    launch_quant_rows<T, DP, kKB, kVB, 16, rows_waves<T, DP, kKB, kVB, 16> == 2 ? 8 : 4>(a, sh, items, part_rows, s);
  else if (most <= 16)
    launch_quant_rows<T, DP, kKB, kVB, 16, 4>(a, sh, items, part_rows, s);
  else
    launch_quant_rows<T, DP, kKB, kVB, 32, rows_waves<T, DP, kKB, kVB, 32> == 2 ? 8 : 4>(a, sh, items, part_rows, s);
  return launch_merge<T, DP>(a, sh, part_rows, s);
}

}  // namespace attn

template <typename T, int kKB, int kVB>
hipError_t launch_attention_quant(const AttnArgs& a, const AttnShape& shape, hipStream_t s) {
  const attn::QuantShape sh{shape, fast_div(shape.group), fast_div(a.cache.page_tokens / kTileTokens),
                            fast_div(a.mask_block > 0 ? a.mask_block : 1)};
  switch (padded_dim(a.cache.head_dim)) {
    case 32: return attn::launch_quant_dim<T, 32, kKB, kVB>(a, sh, s);
    case 64: return attn::launch_quant_dim<T, 64, kKB, kVB>(a, sh, s);
    case 96: return attn::launch_quant_dim<T, 96, kKB, kVB>(a, sh, s);
    case 128: return attn::launch_quant_dim<T, 128, kKB, kVB>(a, sh, s);
    case 192: return attn::launch_quant_dim<T, 192, kKB, kVB>(a, sh, s);
    default: return attn::launch_quant_dim<T, 256, kKB, kVB>(a, sh, s);
  }
}

}  // namespace dmoe
