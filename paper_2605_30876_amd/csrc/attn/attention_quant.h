// Attention over a cache of few bits.
//
// The products are those of attention.h on the bf16 matrix cores: S^T = K Q^T with a
// row to a lane, online softmax in base 2, O^T += V^T P^T.  code * scale is exact in bf16, so
// codes become matrix operands by the conversion instructions alone, two
// values each, the scale applied by them.  A page holds keys and values alike, token by token:
// a lane's 16 bytes are consecutive elements of one token, which is a key operand as it is
// (the order of a reduction's elements is free, as long as queries are loaded in the same one);
// values are written to LDS in rows of tokens and read back turned (ds_read_b64_tr_b16:
// four tokens of one element a lane), in the order of the registers that hold probabilities.
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
      const float r = (u & 0x7f800000u) == 0x7f800000u ? 0.f : x[2 * i + e] - __uint_as_float(hi);
      const uint32_t mid = __float_as_uint(r) & 0xffff0000u;
      a[e][0] = hi | ((u & 0x7f800000u) == 0x7f800000u && (u & 0xffffu) ? 0x10000u : 0u);
      a[e][1] = mid;
      a[e][2] = __float_as_uint(r - __uint_as_float(mid));
    }
#pragma unroll
    for (int p = 0; p < 3; ++p) w[p][i] = (a[0][p] >> 16) | (a[1][p] & 0xffff0000u);
  }
#pragma unroll
  for (int p = 0; p < 3; ++p) f[p] = __builtin_bit_cast(bf16x8, make_uint4(w[p][0], w[p][1], w[p][2], w[p][3]));
}

// A token's scale bytes.
template <int DP>
struct Scales {
  uint32_t w[DP > 128 ? 2 : 1];
  __device__ __forceinline__ void load(const uint8_t* p) {
    if constexpr (scale_row(DP) == 1)
      w[0] = *p;
    else if constexpr (scale_row(DP) == 2)
      w[0] = *reinterpret_cast<const uint16_t*>(p);
    else if constexpr (scale_row(DP) == 4)
      w[0] = *reinterpret_cast<const uint32_t*>(p);
    else {
      const uint2 x = *reinterpret_cast<const uint2*>(p);
      w[0] = x.x;
      w[1] = x.y;
    }
  }
  // of group g, or of group g + 1 in the second half of the wave
  __device__ __forceinline__ float of(int g) const { return scale_of(w[g / 4] >> (8 * (g % 4)) & 255u); }
  __device__ __forceinline__ float of_two(int g, int half) const { return scale_of(w[g / 4] >> (8 * (g % 4) + 8 * half) & 255u); }
};

// A tile's keys (or values) as a wave loads them: load j of a lane (token lane % 32, half
// lane / 32) is the token's chunk 2j + half.
template <int DP, int kBits>
struct TileCodes {
  static constexpr int kChunks = DP * kBits / 128;      // of a token
  static constexpr int kLoads = (kChunks + 1) / 2;      // the last of an odd number: only the first half has one
  static constexpr int kPer = 16 / kBits;               // operands of a load: 8 elements each
  u32x4 c[kLoads];
  Scales<DP> s;
  template <bool kStream>
  __device__ __forceinline__ void load(const uint8_t* tile, int lane) {
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
      if (2 * j + 1 < kChunks || lane < 32) {
        const u32x4* p = reinterpret_cast<const u32x4*>(tile + (j * 64 + lane) * 16);
        c[j] = kStream ? __builtin_nontemporal_load(p) : *p;
      } else {
        c[j] = u32x4{0, 0, 0, 0};
      }
    }
    s.load(tile + scale_at<kBits>(DP, lane & 31));
  }
  __device__ __forceinline__ float scale(int j, int half) const {
    if constexpr (kBits == 8) return s.of(j);
    // an odd number of groups: there is nothing in the second half, and codes of 0 at any finite scale
    if (2 * j + 1 >= kChunks) return half ? 1.f : s.of(2 * j);
    return s.of_two(2 * j, half);
  }
  // operand o of load j
  __device__ __forceinline__ bf16x8 operand(int j, int o, float scale) const {
    const uint32_t w[2] = {c[j][o * kBits / 4], c[j][kBits == 8 ? 2 * o + 1 : o]};
    return decode<kBits>(w, scale);
  }
  // first element of a lane's operand o of load j
  static __device__ __forceinline__ int element(int j, int o, int half) { return (128 / kBits) * (2 * j + half) + 8 * o; }
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
  // Where a lane's pieces of 4 tokens x 16 elements start: within a group of 16 lanes, lane i points at
  // token i / 4, elements 4 (i % 4) on, and receives element i of the four tokens.
  int at[2];
  __device__ __forceinline__ TurnedValues(int lane) {
    const int half = lane >> 5, i = lane & 15, p = (lane >> 4 & 1) * 2 + (i & 3) / 2;
#pragma unroll
    for (int j = 0; j < 2; ++j) at[j] = (8 * j + 4 * half + i / 4) * kRow + (p ^ ((2 * j + half) & 3)) * 16 + (i & 1) * 8;
  }
  // tokens 16s + 8j + 4 half + t (element 4j + t) of element 32b + lane % 32
  __device__ __forceinline__ bf16x8 read(const char* lds, int b, int s) const {
    bf16x4 x[2];
#pragma unroll
    for (int j = 0; j < 2; ++j)
      x[j] = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((__attribute__((address_space(3))) bf16x4*)(lds + at[j] + s * (16 * kRow) + b * 64));
    return __builtin_shufflevector(x[0], x[1], 0, 1, 2, 3, 4, 5, 6, 7);
  }
};

// What is written to LDS before is read after, and the other way round: a wave's LDS
// instructions act in their order.
__device__ __forceinline__ void lds_order() { asm volatile("" ::: "memory"); }

// A wave's 32 rows: WaveRows' sums and softmax, with queries in kK operands of parts.
template <typename T, int DP, int kK>
struct QuantRows : WaveRows<bf16_t, DP> {
  typedef WaveRows<bf16_t, DP> Base;
  typedef Types<bf16_t> Ty;
  static constexpr int kB = Base::kB, kS = Base::kS, kP = kParts<T>;
  bf16x8 q[kP][kK];

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
  __device__ __forceinline__ void score(f32x16& s, const bf16x8& k, int j) const {
    // smallest parts first
#pragma unroll
    for (int p = kP - 1; p >= 0; --p) Ty::mma(s, k, q[p][j]);
  }
  // probabilities of operand s of a tile's values
  static __device__ __forceinline__ void probs(const f32x16& p, int s, bf16x8 (&f)[kP]) {
    if constexpr (kP == 1) {
      f[0] = Ty::probs(p, s);
    } else {
      float x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = p[8 * s + i];
      split(x, f);
    }
  }
  template <typename F>
  __device__ __forceinline__ void add(const f32x16& p, F value) {
#pragma unroll
    for (int s = 0; s < kS; ++s) {
      bf16x8 f[kP];
      probs(p, s, f);
#pragma unroll
      for (int b = 0; b < kB; ++b) {
        const bf16x8 v = value(b, s);
#pragma unroll
        for (int x = kP - 1; x >= 0; --x) Ty::mma(this->o[b], v, f[x]);
      }
    }
  }
  // Base::add_keys with parts
  __device__ __forceinline__ void add_keys(const f32x16& p, const bf16x8 (&v)[kB][kS], int key0, int half) {
#pragma unroll
    for (int s = 0; s < kS; ++s) {
      bf16x8 f[kP];
      probs(p, s, f);
#pragma unroll 1
      for (int r = 0; r < 16; ++r) {
        const bool mine = (r >> 2 & 1) == half;
        const int slot = mine ? (r >> 3) * 4 + (r & 3) : -1;
        const bool sees = key0 + 16 * s + r < this->end;
#pragma unroll
        for (int b = 0; b < kB; ++b) {
          const bf16x8 x = Base::only(v[b][s], slot);
          f32x16 t;
#pragma unroll
          for (int i = 0; i < 16; ++i) t[i] = 0.f;
#pragma unroll
          for (int y = kP - 1; y >= 0; --y) Ty::mma(t, x, Base::only(f[y], slot));
#pragma unroll
          for (int i = 0; i < 16; ++i) this->o[b][i] += sees ? t[i] : 0.f;
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    }
  }
};

// Where a sequence's tiles of one kv head lie: as TileMap, in bytes.
template <int DP, int kKB, int kVB>
struct QuantMap {
  static constexpr int kKTile = quant_tile(kKB, DP), kVTile = quant_tile(kVB, DP);
  const uint8_t *k, *v;
  const __attribute__((address_space(4))) int32_t* table;
  long layer0;
  int n_pages, shift, per_page;  // per_page: tiles of all kv heads
  __device__ __forceinline__ QuantMap(const AttnArgs& a, int slot, int hk) : n_pages(a.cache.n_pages) {
    table = (const __attribute__((address_space(4))) int32_t*)(a.cache.table + static_cast<long>(slot) * a.cache.max_pages);
    const int tpp = a.cache.page_tokens / kTileTokens;
    shift = (tpp & (tpp - 1)) == 0 ? 31 - __builtin_clz(tpp) : -tpp;
    per_page = tpp * a.cache.n_kv_heads;
    layer0 = static_cast<long>(a.layer) * n_pages;
    k = static_cast<const uint8_t*>(a.cache.k) + static_cast<long>(hk * tpp) * kKTile;
    v = static_cast<const uint8_t*>(a.cache.v) + static_cast<long>(hk * tpp) * kVTile;
  }
  __device__ __forceinline__ int page(int kt, int end) const { return kt < end ? table[shift >= 0 ? kt >> shift : kt / -shift] : -1; }
  __device__ __forceinline__ bool holds(int page) const { return static_cast<unsigned>(page) < static_cast<unsigned>(n_pages); }
  // tiles from k and v to a tile on a page that is held
  __device__ __forceinline__ long at(int kt, int page) const {
    return (layer0 + page) * per_page + (shift >= 0 ? kt & ((1 << shift) - 1) : kt % -shift);
  }
  __device__ __forceinline__ const uint8_t* key(long tile) const { return k + tile * kKTile; }
  __device__ __forceinline__ const uint8_t* value(long tile) const { return v + tile * kVTile; }
};

// A tile's values, loaded by this wave, through its LDS.
template <int DP, int kVB>
__device__ __forceinline__ void turn_values(const TileCodes<DP, kVB>& c, char* lds, int lane) {
  typedef TileCodes<DP, kVB> Codes;
  const int half = lane >> 5, r = lane & 31;
  lds_order();
#pragma unroll
  for (int j = 0; j < Codes::kLoads; ++j) {
    const float scale = c.scale(j, half);
    if (2 * j + 1 < Codes::kChunks || lane < 32) {
#pragma unroll
      for (int o = 0; o < Codes::kPer; ++o)
        TurnedValues<DP>::write(lds, r, (2 * j + half) * Codes::kPer + o, c.operand(j, o, scale));
    }
  }
  lds_order();
}

// Tiles of a masked stretch that hold values that are not finite, once the running maximum is the last one (WaveRows::add_by_key).
template <typename Rows, typename Map, int DP, int kKB, int kVB, typename Element>
__device__ __forceinline__ void add_by_key(Rows& w, const Map& map, int kt, int kt1, int step, float scale2, int lane, char* lds, Element query_operand) {
  const int half = lane >> 5;
#pragma unroll 1
  for (; kt < kt1; kt += step) {
    const int page = map.page(kt, kt1), key0 = kt * kTileTokens;
    if (!map.holds(page) || key0 >= w.hi) continue;
    const long at = map.at(kt, page);
    bf16x8 v[Rows::kB][Rows::kS];
    {
      TileCodes<DP, kVB> vc;
      vc.template load<false>(map.value(at), lane);
      turn_values<DP, kVB>(vc, lds, lane);
      const TurnedValues<DP> turned(lane);
#pragma unroll
      for (int b = 0; b < Rows::kB; ++b)
#pragma unroll
        for (int s = 0; s < Rows::kS; ++s) v[b][s] = turned.read(lds, b, s);
    }
    if (w.cut(v, key0, half)) continue;
    f32x16 s;
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = 0.f;
    query_operand(s, map.key(at));
    const float off = w.m == -INFINITY ? 0.f : w.m;
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = tile_key(i, half) < w.end - key0 ? exp2_hw(__builtin_fmaf(s[i], scale2, -off)) : 0.f;
    w.add_keys(s, v, key0, half);
  }
}

template <typename T>
constexpr int quant_waves(int dp) {
  return quant_two_per_cu(sizeof(T) == 4 ? DMOE_F32 : DMOE_BF16, dp) ? 2 : 1;
}

// Few rows: attention_rows_kernel's split of the work (32 kWR rows of one kv head per workgroup, 4 / kWR waves to 32 of
// them, each on every (4 / kWR)-th key tile), the codes of the next tile on their way while one is used.
template <typename T, int DP, int kKB, int kVB, int kWR>
__global__ __launch_bounds__(256, quant_waves<T>(DP)) void quant_rows_kernel(AttnArgs a, AttnShape sh, int part_rows) {
  typedef TileCodes<DP, kKB> KCodes;
  typedef TileCodes<DP, kVB> VCodes;
  typedef QuantRows<T, DP, KCodes::kLoads * KCodes::kPer> Rows;
  constexpr int kB = Rows::kB, kS = Rows::kS, kWK = 4 / kWR;
  constexpr bool kStream = kWR == 1;
  extern __shared__ float lds[];
  const int hkv = a.cache.n_kv_heads;
  const int item_i = blockIdx.x / hkv, hk = blockIdx.x % hkv;
  AttnItem it;
  if (!load_item(a, item_i, it)) return;
  const int lane = threadIdx.x & 63, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wk = wave % kWK, wr = wave / kWK;
  char* mine = reinterpret_cast<char*>(lds) + wave * TurnedValues<DP>::kBytes;
  const TurnedValues<DP> turned(lane);
  Rows w;
  w.clear();
  const RowPlace<T, DP> rows(w, a, it, sh.group, hk, it.first + 32 * wr, lane);
  w.load(rows, a, it, [&](int j) { return KCodes::element(j / KCodes::kPer, j % KCodes::kPer, half); });
  const float scale2 = a.scale * kLog2e;
  const QuantMap<DP, kKB, kVB> map(a, it.slot, hk);
  const int kt1 = min(it.kt1, (w.hi + kTileTokens - 1) / kTileTokens);
  KCodes kc;
  VCodes vc;
  auto scores = [&](f32x16& s, const KCodes& c) {
#pragma unroll
    for (int j = 0; j < KCodes::kLoads; ++j) {
      const float scale = c.scale(j, half);
#pragma unroll
      for (int o = 0; o < KCodes::kPer; ++o) w.score(s, c.operand(j, o, scale), j * KCodes::kPer + o);
    }
  };
  // page ids are known two of this wave's tiles ahead, its keys and values one
  int kt = it.kt0 + wk;
  int page = kt < kt1 ? (wk < 2 ? wk == 0 ? it.page[0] : it.page[1] : wk == 2 ? it.page[2] : it.page[3]) : -1;
  int page1 = map.page(kt + kWK, kt1);
  auto first = [&] {
    if (!map.holds(page)) return;
    const long at = map.at(kt, page);
    kc.template load<kStream>(map.key(at), lane);
    vc.template load<kStream>(map.value(at), lane);
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
    if (here) {
#pragma unroll
      for (int i = 0; i < 16; ++i) s[0][i] = 0.f;
      scores(s[0], kc);
    }
    if (more) kc.template load<kStream>(map.key(at1), lane);
    if (here) turn_values<DP, kVB>(vc, mine, lane);
    if (more) vc.template load<kStream>(map.value(at1), lane);
    if (here) {
      const int key0 = kt * kTileTokens;
      w.template softmax<1>(s, scale2, key0, masked, half);
      if constexpr (!masked) {
        w.add(s[0], [&](int b, int x) { return turned.read(mine, b, x); });
      } else {
        bf16x8 v[kB][kS];
#pragma unroll
        for (int b = 0; b < kB; ++b)
#pragma unroll
          for (int x = 0; x < kS; ++x) v[b][x] = turned.read(mine, b, x);
        if (w.cut(v, key0, half))
          w.add(s[0], [&](int b, int x) { return v[b][x]; });
        else
          left = true;
      }
    }
    kt += kWK;
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
  if (left)
    add_by_key<Rows, QuantMap<DP, kKB, kVB>, DP, kKB, kVB>(w, map, first_masked, kt1, kWK, scale2, lane, mine, [&](f32x16& s, const uint8_t* p) {
      KCodes c;
      c.template load<false>(p, lane);
      scores(s, c);
    });
  w.l = other_half_sum(w.l);
  if constexpr (kWK > 1) __syncthreads();  // the values' places are taken by the sums
  join_waves<kWK, kB>(w, lds, wr * (kWK / 2), wk, lane);
  if (wk == 0) rows.store(w, a, sh, it, hk, half, part_rows);
}

// Keys and values of kTS tiles in LDS: keys as operands, element 16j + 8 half + e of
// token r at [j][32 half + r][e], values in rows.
template <int DP>
struct QuantStage {
  static constexpr int kTS = stage_tiles(DMOE_BF16, DP), kK = DP / 16;
  bf16x8 k[kTS][kK][64];
  char v[kTS][TurnedValues<DP>::kBytes];
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
  // base[n]: where tile n lies, or nullptr
  __device__ __forceinline__ void load(const uint8_t* const (&base)[kTS]) {
    const int r = threadIdx.x % kTileTokens;
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
      const uint8_t* p = base[0];
#pragma unroll
      for (int n = 1; n < kTS; ++n) p = tile(i) == n ? base[n] : p;
      if (!has(i) || !p) continue;
      c[i] = *reinterpret_cast<const u32x4*>(p + (chunk(i) * kTileTokens + r) * 16);
      s[i] = p[scale_at<kBits>(DP, r) + chunk(i) * 128 / (kBits * kGroup)];
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

// Many rows: 128 of one kv head per workgroup, 32 to a wave, all four waves on the same keys.  Codes of kTS tiles
// are loaded two stages ahead, opened into LDS one stage ahead, each by one of the
// threads; one barrier a stage.
template <typename T, int DP, int kKB, int kVB>
__global__ __launch_bounds__(256, quant_waves<T>(DP)) void quant_block_kernel(AttnArgs a, AttnShape sh, int part_rows) {
  typedef QuantStage<DP> Stage;
  typedef QuantRows<T, DP, Stage::kK> Rows;
  constexpr int kB = Rows::kB, kS = Rows::kS, kK = Stage::kK, kTS = Stage::kTS;
  __shared__ Stage s0, s1;
  const int hkv = a.cache.n_kv_heads;
  const int item_i = blockIdx.x / hkv, hk = blockIdx.x % hkv;
  AttnItem it;
  if (!load_item(a, item_i, it)) return;
  const int lane = threadIdx.x & 63, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const TurnedValues<DP> turned(lane);
  Rows w;
  w.clear();
  const RowPlace<T, DP> rows(w, a, it, sh.group, hk, it.first + 32 * wave, lane);
  w.load(rows, a, it, [&](int j) { return 16 * j + 8 * half; });
  const float scale2 = a.scale * kLog2e;
  const QuantMap<DP, kKB, kVB> map(a, it.slot, hk);
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
      const bool on = map.holds(pg.id[n]);
      const long at = on ? map.at(kt + n, pg.id[n]) : 0;
      kb[n] = on ? map.key(at) : nullptr;
      vb[n] = on ? map.value(at) : nullptr;
    }
    kc.load(kb);
    vc.load(vb);
  };
  // what lies on no page leaves something in LDS that is not used
  auto open = [&](Stage& st) {
    const int r = threadIdx.x % kTileTokens;
    kc.open([&](int n, int p, const bf16x8& x) { st.k[n][p / 2][32 * (p & 1) + r] = x; });
    vc.open([&](int n, int p, const bf16x8& x) { TurnedValues<DP>::write(st.v[n], r, p, x); });
  };
  auto score = [&](f32x16& s, const Stage& st, int n) {
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll
    for (int j = 0; j < kK; ++j) w.score(s, st.k[n][j][lane], j);
  };
  // A stage that every row sees whole; its tiles may still lie on no page, or behind the item's last.
  auto compute = [&](const Ids& pg, const Stage& st) {
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
    for (int n = 0; n < kTS; ++n) score(s[n], st, n);
    if (!all) {
#pragma unroll
      for (int n = 0; n < kTS; ++n)
#pragma unroll
        for (int i = 0; i < 16; ++i) s[n][i] = on[n] ? s[n][i] : -INFINITY;
    }
    w.template softmax<kTS>(s, scale2, 0, false, half);
#pragma unroll
    for (int n = 0; n < kTS; ++n) {
      if (!on[n]) continue;
      w.add(s[n], [&](int b, int x) { return turned.read(st.v[n], b, x); });
    }
  };
  // Any stage, tile by tile.
  bool left = false;  // tiles for add_by_key
  auto compute_masked = [&](int kt, const Ids& pg, const Stage& st) {
#pragma unroll
    for (int n = 0; n < kTS; ++n) {
      const int key0 = (kt + n) * kTileTokens;
      if (!map.holds(pg.id[n]) || key0 >= w.hi) continue;
      f32x16 s[1];
      score(s[0], st, n);
      w.template softmax<1>(s, scale2, key0, true, half);
      __builtin_amdgcn_sched_barrier(0);
      bf16x8 v[kB][kS];
#pragma unroll
      for (int b = 0; b < kB; ++b)
#pragma unroll
        for (int x = 0; x < kS; ++x) v[b][x] = turned.read(st.v[n], b, x);
      if (w.cut(v, key0, half))
        w.add(s[0], [&](int b, int x) { return v[b][x]; });
      else
        left = true;
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  int kt = kt0;
  Ids pg = pages(kt), pg1 = pages(kt + kTS);
  load(kt, pg);
  open(s0);
  load(kt + kTS, pg1);
  auto turn = [&](auto masked, Stage& cur, Stage& fill) {
    w.pin();
    // a stage's writes are done, by all; the other buffer has been read
    lds_order();
    __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
    lds_order();
    const Ids pg2 = pages(kt + 2 * kTS);
    open(fill);
    load(kt + 2 * kTS, pg2);
    if constexpr (masked)
      compute_masked(kt, pg, cur);
    else
      compute(pg, cur);
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
  __syncthreads();  // the stages are done with
  if (left) {
    static_assert(sizeof(Stage) >= 2 * TurnedValues<DP>::kBytes);
    char* room = reinterpret_cast<char*>(wave < 2 ? &s0 : &s1) + (wave & 1) * TurnedValues<DP>::kBytes;
    add_by_key<Rows, QuantMap<DP, kKB, kVB>, DP, kKB, kVB>(w, map, first_masked, kt1, 1, scale2, lane, room, [&](f32x16& s, const uint8_t* p) {
      // operands in the queries' order, straight from memory: lane's token, elements 16j + 8 half on
      const int r = lane & 31;
#pragma unroll 1
      for (int j = 0; j < kK; ++j) {
        const int d = 16 * j + 8 * half;
        uint32_t x[2];
        const uint8_t* c = p + code_at<kKB>(r, d);
        x[0] = *reinterpret_cast<const uint32_t*>(c);
        x[1] = kKB == 8 ? *reinterpret_cast<const uint32_t*>(c + 4) : 0;
        const bf16x8 k = decode<kKB>(x, scale_of(p[scale_at<kKB>(DP, r) + d / kGroup]));
#pragma unroll
        for (int y = 0; y < kK; ++y)
          if (y == j) w.score(s, k, y);
      }
    });
  }
  w.l = other_half_sum(w.l);
  rows.store(w, a, sh, it, hk, half, part_rows);
}

template <typename T, int DP, int kKB, int kVB>
hipError_t launch_quant_dim(const AttnArgs& a, const AttnShape& sh, hipStream_t s) {
  const int hkv = a.cache.n_kv_heads;
  const unsigned items = static_cast<unsigned>(sh.max_items() * hkv);
  const int part_rows = static_cast<int>(sh.max_parts() * hkv * sh.tile_rows);
  if (sh.tile_rows <= 64) {
    const size_t join = 2 * (16 * (DP / 32) + 2) * 64 * sizeof(float), values = 4 * TurnedValues<DP>::kBytes;
    const size_t lds = join > values ? join : values;
    if (sh.tile_rows == 32)
      quant_rows_kernel<T, DP, kKB, kVB, 1><<<items, 256, lds, s>>>(a, sh, part_rows);
    else
      quant_rows_kernel<T, DP, kKB, kVB, 2><<<items, 256, lds, s>>>(a, sh, part_rows);
  } else {
    quant_block_kernel<T, DP, kKB, kVB><<<items, 256, 0, s>>>(a, sh, part_rows);
  }
  return launch_merge<T, DP>(a, sh, part_rows, s);
}

}  // namespace attn

template <typename T, int kKB, int kVB>
hipError_t launch_attention_quant(const AttnArgs& a, const AttnShape& sh, hipStream_t s) {
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
