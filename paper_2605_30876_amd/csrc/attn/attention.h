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
  static __device__ __forceinline__ float rounded(float p) { return static_cast<float>(static_cast<__bf16>(p)); }
  static __device__ __forceinline__ bool finite(const Frag& f) {
    const uint4 u = __builtin_bit_cast(uint4, f);
    auto bad = [](uint32_t w) { return (w & 0x7f80u) == 0x7f80u || (w & 0x7f800000u) == 0x7f800000u; };
    return !(bad(u.x) || bad(u.y) || bad(u.z) || bad(u.w));
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
  static __device__ __forceinline__ float rounded(float p) { return p; }
  static __device__ __forceinline__ bool finite(const Frag& f) {
    bool ok = true;
#pragma unroll
    for (int i = 0; i < 4; ++i) ok = ok && (__float_as_uint(f[i]) & 0x7f800000u) != 0x7f800000u;
    return ok;
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

// A wave's 32 rows against tiles of 32 keys.
template <typename T, int DP>
struct WaveRows {
  typedef Types<T> Ty;
  typedef typename Ty::Frag Frag;
  static constexpr int c = Ty::c;
  static constexpr int kK = DP / (2 * c);  // operands of a tile's keys
  static constexpr int kB = DP / 32;       // 32-wide blocks of the output
  static constexpr int kS = 16 / c;        // operands of a tile's values per block
  Frag q[kK];
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

  __device__ __forceinline__ f32x16 scores(const Frag (&k)[kK]) const {
    f32x16 s;
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll
    for (int j = 0; j < kK; ++j) Ty::mma(s, k[j], q[j]);
    return s;
  }

  // Scores (times scale log2 e) to probabilities relative to the running
  // maximum, which they raise first if they have to.  masked: keys from
  // `end - key0` on are not seen.
  __device__ __forceinline__ void softmax(f32x16& s, float scale2, int key0, bool masked, int half) {
    if (masked) {
      const int seen = end - key0;
#pragma unroll
      for (int i = 0; i < 16; ++i) s[i] = tile_key(i, half) < seen ? s[i] : -INFINITY;
    }
    float t = s[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) t = fmaxf(t, s[i]);
    t = other_half_max(t) * scale2;
    if (__any(t > m + kLazy)) {
      const float nm = fmaxf(m, t);
      const float a = nm == m ? 1.f : exp2_hw(m - nm);
      m = nm;
      l *= a;
#pragma unroll
      for (int b = 0; b < kB; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[b][i] *= a;
    }
    const float off = m == -INFINITY ? 0.f : m;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      s[i] = exp2_hw(__builtin_fmaf(s[i], scale2, -off));
      l += s[i];
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

  // A tile in which some row does not see every key.  Values that no row of
  // the wave sees are not the sequence's, or a later token's: they become 0,
  // whatever they are.  A value that some rows see and others do not must not
  // reach the others through 0 * value: where one is not finite (v0: the
  // tile's values in memory), the tile is added key by key.
  __device__ __forceinline__ void add_masked(const f32x16& p, Frag (&v)[kB][kS], int key0, int half, const T* v0) {
    const int seen = hi - key0;
    bool fine = true;
#pragma unroll
    for (int s = 0; s < kS; ++s)
#pragma unroll
      for (int b = 0; b < kB; ++b) {
#pragma unroll
        for (int e = 0; e < c; ++e)
          if (2 * c * s + 8 * (e / 4) + 4 * half + e % 4 >= seen) v[b][s][e] = 0;
        fine = fine && Ty::finite(v[b][s]);
      }
    if (__all(fine)) {
      add(p, v);
      return;
    }
    const int lane = threadIdx.x & 63;
    for (int key = 0; key < kTileTokens; ++key) {
      if (key >= seen) break;
      const int reg = 4 * (key >> 3) + (key & 3), kh = (key >> 2) & 1;
      float w = 0.f;
#pragma unroll
      for (int i = 0; i < 16; ++i) w = i == reg ? p[i] : w;
      w = Ty::rounded(__shfl(w, (lane & 31) + 32 * kh));
      if (key0 + key >= end) continue;
      const int r = key % (2 * c);
#pragma unroll
      for (int b = 0; b < kB; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i)
          o[b][i] += w * load_as_f32<T>(v0 + value_chunk<c>(32 * b + tile_key(i, half), key / (2 * c), r % 8 / 4) +
                                        r / 8 * 4 + r % 4);
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

// One item of one kv head per workgroup: kWR waves along the rows (tiles of
// 32*kWR), kWK along the keys (every kWK-th tile), joined through LDS.
template <typename T, int DP, int kWR, int kWK>
__global__ __launch_bounds__(64 * kWR * kWK) void attention_kernel(AttnArgs a, AttnShape sh, int part_rows) {
  typedef WaveRows<T, DP> Rows;
  typedef typename Rows::Frag Frag;
  constexpr int c = Rows::c, kK = Rows::kK, kB = Rows::kB, kS = Rows::kS;
  extern __shared__ float lds[];
  const int hkv = a.cache.n_kv_heads;
  const AttnPlanHead* head = reinterpret_cast<const AttnPlanHead*>(a.plan);
  const int item_i = blockIdx.x / hkv, hk = blockIdx.x % hkv;
  if (item_i >= head->n_items) return;
  const AttnItem it = plan_items(a.plan)[item_i];
  const int lane = threadIdx.x & 63, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wr = wave / kWK, wk = wave % kWK;
  const int g = sh.group;

  Rows w;
  w.clear();
  const int row_lo = it.first + 32 * wr;
  const int row_hi = min(row_lo + 32, it.rows) - 1;
  const int row = row_lo + (lane & 31);
  const bool live = row < it.rows;
  const int pos0 = it.len - it.n;
  const int tok = live ? row / g : 0;
  const int qh = hk * g + (live ? row - tok * g : 0);
  w.end = live ? visible_end(pos0 + tok, it.len, a.mask_block) : 0;
  if (row_hi >= row_lo) {
    // the ends grow with the rows; rows past the last are computed and dropped
    w.lo = visible_end(pos0 + row_lo / g, it.len, a.mask_block);
    w.hi = visible_end(pos0 + row_hi / g, it.len, a.mask_block);
    const T* qp = static_cast<const T*>(a.q) + (it.row0 + tok) * a.q_stride + static_cast<long>(qh) * a.cache.head_dim;
#pragma unroll
    for (int j = 0; j < kK; ++j) {
      const int d = (2 * j + half) * c;
      Frag f{};
      if (live && d < a.cache.head_dim) f = *reinterpret_cast<const Frag*>(qp + d);
      w.q[j] = f;
    }
    const float scale2 = a.scale * kLog2e;
    const int tpp = a.cache.page_tokens / kTileTokens;
    const long page_len = static_cast<long>(a.cache.page_tokens) * DP;
    const int32_t* table = a.cache.table + static_cast<long>(it.slot) * a.cache.max_pages;
    const T* kbase = static_cast<const T*>(a.cache.k) + hk * page_len;
    const T* vbase = static_cast<const T*>(a.cache.v) + hk * page_len;
    const int kt1 = min(it.kt1, (w.hi + kTileTokens - 1) / kTileTokens);
    for (int kt = it.kt0 + wk; kt < kt1; kt += kWK) {
      const int page = __builtin_amdgcn_readfirstlane(table[kt / tpp]);
      if (page < 0 || page >= a.cache.n_pages) continue;
      const long at = (static_cast<long>(a.layer) * a.cache.n_pages + page) * hkv * page_len + (kt % tpp) * (kTileTokens * DP);
      const T* kp = kbase + at;
      const T* vp = vbase + at;
      Frag k[kK], v[kB][kS];
#pragma unroll
      for (int j = 0; j < kK; ++j) k[j] = *reinterpret_cast<const Frag*>(kp + j * 64 * c + lane * c);
#pragma unroll
      for (int b = 0; b < kB; ++b)
#pragma unroll
        for (int s = 0; s < kS; ++s) v[b][s] = *reinterpret_cast<const Frag*>(vp + (b * kS + s) * 64 * c + lane * c);
      f32x16 s = w.scores(k);
      const int key0 = kt * kTileTokens;
      const bool masked = key0 + kTileTokens > w.lo;
      w.softmax(s, scale2, key0, masked, half);
      if (masked)
        w.add_masked(s, v, key0, half, vp);
      else
        w.add(s, v);
    }
  }
  w.l = other_half_sum(w.l);

  if constexpr (kWK > 1) {
    // join the waves of a row tile two by two: the upper ones hand their sums
    // to the lower ones (fixed order)
    constexpr int kLen = (16 * kB + 2) * 64;
#pragma unroll
    for (int n = kWK / 2; n >= 1; n /= 2) {
      float* buf = lds + (wr * (kWK / 2) + wk % n) * kLen;
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
  }
  if (wk != 0 || !live) return;

  if (it.part >= 0) {
    const long slot = static_cast<long>(it.part) * hkv + hk;
    float* po = static_cast<float*>(a.workspace) + (slot * sh.tile_rows + (row - it.first)) * DP;
#pragma unroll
    for (int b = 0; b < kB; ++b)
#pragma unroll
      for (int i = 0; i < 16; i += 4)
        *reinterpret_cast<f32x4*>(po + 32 * b + tile_key(i, half)) = f32x4{w.o[b][i], w.o[b][i + 1], w.o[b][i + 2], w.o[b][i + 3]};
    if (half == 0) {
      float* ml = static_cast<float*>(a.workspace) + static_cast<long>(part_rows) * DP + (slot * sh.tile_rows + (row - it.first)) * 2;
      ml[0] = w.m;
      ml[1] = w.l;
    }
    return;
  }
  const float inv = w.l > 0.f || w.l != w.l ? 1.f / w.l : 0.f;
  T* op = static_cast<T*>(a.out) + (it.row0 + tok) * a.out_stride + static_cast<long>(qh) * a.cache.head_dim;
#pragma unroll
  for (int b = 0; b < kB; ++b)
#pragma unroll
    for (int i = 0; i < 16; i += 4) {
      const int d = 32 * b + tile_key(i, half);
      if (d < a.cache.head_dim)
#pragma unroll
        for (int t = 0; t < 4; ++t) store_from_f32<T>(op + d + t, w.o[b][i + t] * inv);
    }
  if (a.lse && half == 0)
    a.lse[static_cast<long>(it.row0 + tok) * a.n_heads + qh] = w.l > 0.f || w.l != w.l ? (w.m + log2f(w.l)) * kLn2 : -INFINITY;
}

// Partial results of a row tile joined: a wave per row, its lanes along the
// head dimension, pieces in order.
template <typename T, int DP>
__global__ __launch_bounds__(256) void attention_merge_kernel(AttnArgs a, AttnShape sh, int part_rows) {
  const int hkv = a.cache.n_kv_heads;
  const AttnPlanHead* head = reinterpret_cast<const AttnPlanHead*>(a.plan);
  const int mi = blockIdx.x / hkv, hk = blockIdx.x % hkv;
  if (mi >= head->n_merges) return;
  const AttnMerge* merges = reinterpret_cast<const AttnMerge*>(plan_items(a.plan) + sh.max_items());
  const AttnMerge mg = merges[mi];
  const int lane = threadIdx.x & 63;
  const int r = blockIdx.y * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int row = mg.first + r;
  if (r >= sh.tile_rows || row >= mg.rows) return;
  const float* po = static_cast<const float*>(a.workspace);
  const float* ml = po + static_cast<long>(part_rows) * DP;
  const long step = static_cast<long>(hkv) * sh.tile_rows;
  const long at = (static_cast<long>(mg.part) * hkv + hk) * sh.tile_rows + r;
  float m = -INFINITY;
  for (int i = lane; i < mg.pieces; i += 64) m = fmaxf(m, ml[(at + i * step) * 2]);
#pragma unroll
  for (int x = 32; x >= 1; x /= 2) m = fmaxf(m, __shfl_xor(m, x));
  constexpr int kV = (DP + 63) / 64;
  float o[kV] = {}, l = 0.f;
  const float off = m == -INFINITY ? 0.f : m;
  for (int i = 0; i < mg.pieces; ++i) {
    const float pm = ml[(at + i * step) * 2];
    const float f = pm == m ? 1.f : exp2_hw(pm - off);
    l += f * ml[(at + i * step) * 2 + 1];
#pragma unroll
    for (int j = 0; j < kV; ++j)
      if (lane + 64 * j < DP) o[j] += f * po[(at + i * step) * DP + lane + 64 * j];
  }
  const bool any = l > 0.f || l != l;
  const float inv = any ? 1.f / l : 0.f;
  const int tok = row / sh.group, qh = hk * sh.group + row - tok * sh.group;
  T* op = static_cast<T*>(a.out) + (mg.row0 + tok) * a.out_stride + static_cast<long>(qh) * a.cache.head_dim;
#pragma unroll
  for (int j = 0; j < kV; ++j)
    if (lane + 64 * j < a.cache.head_dim) store_from_f32<T>(op + lane + 64 * j, o[j] * inv);
  if (a.lse && lane == 0)
    a.lse[static_cast<long>(mg.row0 + tok) * a.n_heads + qh] = any ? (m + log2f(l)) * kLn2 : -INFINITY;
}

template <typename T, int DP>
hipError_t launch_dim(const AttnArgs& a, const AttnShape& sh, hipStream_t s) {
  const int hkv = a.cache.n_kv_heads;
  const unsigned items = static_cast<unsigned>(sh.max_items() * hkv);
  const int part_rows = static_cast<int>(sh.max_parts() * hkv * sh.tile_rows);
  if (sh.tile_rows == 32) {
    constexpr size_t lds = 2 * (16 * (DP / 32) + 2) * 64 * sizeof(float);
    attention_kernel<T, DP, 1, 4><<<items, 256, lds, s>>>(a, sh, part_rows);
  } else {
    attention_kernel<T, DP, 4, 1><<<items, 256, 0, s>>>(a, sh, part_rows);
  }
  attention_merge_kernel<T, DP><<<dim3(static_cast<unsigned>(sh.split_items * hkv), sh.tile_rows / 4), 256, 0, s>>>(a, sh, part_rows);
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
