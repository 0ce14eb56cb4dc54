// Attention of sequences that share a prefix (or of caches of bounded size), and the
// weight that queries give to each key.
#include <type_traits>

#include "common.h"
#include "merge.h"
#include "tiles.h"

namespace louiskv {
namespace {

constexpr int64_t kMaxQueries = 1 << 25;   // of a call, times heads

// The rows of a prefix, or of the slices' own caches.
struct Side {
  const void* k;
  const void* v;
  const int32_t* n;
  int rows;
  int row_groups, splits;   // blocks that a slice's queries, and parts that its keys, are cut into
};

struct AttnArgs {
  const void* q;
  int group_size, n_q, n_seqs;
  float scale;
  int64_t n_prefix_slices;
  Side prefix, own;
  int64_t prefix_blocks;
  int n_parts;              // of a query: the prefix's, then its own rows'
  int stream;               // rows that one block reads bypass the caches
  float* part;
  float* logits;            // [slices][group_size * n_q][logit_stride], base 2, or NULL
  int logit_stride;
  float* weights;
  void* out;
  int out_bf16;
  float* lse_out;
};

__device__ __forceinline__ int length_of(const int32_t* n, int64_t s, int rows) {
  return n ? max(0, min(n[s], rows)) : rows;
}

// Channel c of row r of a [..][128] buffer.
template <class T>
__device__ __forceinline__ float at(const void* p, int64_t r, int c) {
  return load_as_f32(static_cast<const T*>(p), r * kHeadDim + c);
}

constexpr int kTile = 32;            // keys of a product
constexpr int kBlockWaves = 4;
constexpr int kStage = 64;           // keys of a stage that the block's waves share
constexpr float kGrow = 8.0f;        // base-2 logits may pass the base by this much before the sums are rescaled
template <class T> constexpr int kRowBytes = kHeadDim * sizeof(T);
constexpr int kNearLogits = 3584;    // logits that LDS holds: two blocks of 80 KB a CU
// keys and values of a tile for each wave, or of two stages
template <class T> constexpr int kRingBytes = kBlockWaves * kTile * 2 * kRowBytes<T>;

// A block's place: the queries and keys that it attends.
struct Place {
  int64_t s;         // slice, or prefix slice
  int rgrp, split;
  int n_rows;        // queries of the (prefix) slice
  int64_t kv_row;    // first row of the slice in k and v
  int n;             // rows held
};

__device__ __forceinline__ Place place_of(const AttnArgs& a, const Side& x, bool own, int64_t id) {
  if (!own && a.prefix_blocks >= 64) {
    // blocks that read the same keys go to one XCD (blocks are dealt to the eight in turn)
    const int64_t per = a.prefix_blocks >> 3, rest = a.prefix_blocks & 7, xcd = id & 7;
    id = xcd * per + min<int64_t>(xcd, rest) + (id >> 3);
  }
  Place p;
  p.rgrp = (int)(id % x.row_groups);
  id /= x.row_groups;
  p.split = (int)(id % x.splits);
  p.s = id / x.splits;
  p.n_rows = a.group_size * a.n_q * (own ? 1 : a.n_seqs);
  p.kv_row = p.s * x.rows;
  p.n = length_of(x.n, p.s, x.rows);
  return p;
}

// Query r of a place as its row in q and out.
__device__ __forceinline__ int64_t query_row(const AttnArgs& a, const Place& p, bool own, int r) {
  const int per = a.group_size * a.n_q;
  if (own) return p.s * per + r;
  const int seq = r / per;
  return ((int64_t)seq * a.n_prefix_slices + p.s) * per + (r - seq * per);
}

// Keys that query r of a place sees.
__device__ __forceinline__ int limit_of(const AttnArgs& a, const Place& p, bool own, int r) {
  return own ? max(0, p.n - a.n_q + r % a.n_q + 1) : p.n;
}

// The fewest and most keys that queries r0..r1 see.
__device__ __forceinline__ void limits_of(const AttnArgs& a, const Place& p, bool own, int r0, int r1, int& least, int& most) {
  const bool wraps = own && r0 / a.n_q != r1 / a.n_q;
  least = wraps ? max(0, p.n - a.n_q + 1) : limit_of(a, p, own, r0);
  most = wraps ? p.n : limit_of(a, p, own, r1);
}

typedef const __attribute__((address_space(3))) bf16x8* lds_bf16x8;
typedef const __attribute__((address_space(3))) f32x4* lds_f32x4;
typedef const __attribute__((address_space(3))) float* lds_f32;
typedef __attribute__((address_space(3))) s16x4* lds_s16x4;

// A wave's 32 queries, a lane (of two) a query n = lane % 32: S^T = K Q^T of 32 keys leaves
// the lane 16 scores, of keys (i & 3) + 8 (i >> 2) + 4 h with h = lane / 32, and their
// exponentials are, unmoved, the B operand of O^T += V^T P^T.
template <class T>
struct Wave {
  static constexpr bool kBf16 = sizeof(T) == 2;
  typedef typename std::conditional<kBf16, bf16x8, f32x4>::type QPiece;
  typedef typename std::conditional<kBf16, bf16x8[8], int>::type Keys;       // float32: read where they are used
  typedef typename std::conditional<kBf16, s16x8[2][4], int>::type Values;
  typedef typename std::conditional<kBf16, bf16x8[2], f32x16>::type Weights;
  static constexpr int kQ = kBf16 ? 8 : 16;

  int lane, h, n;
  QPiece q[kQ];              // 16-byte pieces 2 c + h (bfloat16) or 16 h + c (float32)
  float mult;                // |scale| log2(e); the queries' signs are flipped where the scale is negative
  int limit;                 // keys that the lane's query sees
  f32x16 o[4];
  float base = 0.f, grow_at = -__builtin_inff(), sum = 0.f;
  uint32_t k_at[8], v_at[4][2];   // LDS addresses of the lane's reads in a tile at address 0

  __device__ __forceinline__ void init(const AttnArgs& a, int64_t row, int lim) {
    lane = threadIdx.x & 63;
    h = lane >> 5;
    n = lane & 31;
    limit = lim;
    const float qs = a.scale * kLog2E;
    const uint32_t flip = qs < 0.f ? (kBf16 ? 0x80008000u : 0x80000000u) : 0u;
    mult = fabsf(qs);
    const uint4* src = reinterpret_cast<const uint4*>(static_cast<const T*>(a.q) + row * kHeadDim);
#pragma unroll
    for (int c = 0; c < kQ; ++c) {
      uint4 v = src[kBf16 ? 2 * c + h : 16 * h + c];
      v.x ^= flip; v.y ^= flip; v.z ^= flip; v.w ^= flip;
      q[c] = __builtin_bit_cast(QPiece, v);
    }
#pragma unroll
    for (int dt = 0; dt < 4; ++dt)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[dt][i] = 0.f;
  }

  // bfloat16: pieces 2 c + h of key n, and of the values rows 4 h + 0..3 and, in the
  // second, those + 8 (the same swizzle but for bit 1) of channels 32 dt + 0..31.
  // float32: pieces 16 h + c of key n, and channel n % 4 of piece n / 4 (+ 8 dt) of rows
  // 4 h + i.
  __device__ __forceinline__ void addresses(uint32_t k0, uint32_t v0) {
    constexpr int kRow = kRowBytes<T>;
    if constexpr (kBf16) {
      const uint32_t kp = (h ^ swizzle<T>(n & 15)) << 4, kr = k0 + n * kRow;
      const int j4 = (lane & 15) >> 2, xp = (((lane >> 4) & 1) << 1) | ((lane & 3) >> 1);
      const uint32_t v1 = v0 + (4 * h + j4) * kRow + ((lane & 1) << 3), vp = ((j4 << 2) | (xp ^ h)) << 4;
#pragma unroll
      for (int c = 0; c < 8; ++c) k_at[c] = kr + (kp ^ (c << 5));
#pragma unroll
      for (int dt = 0; dt < 4; ++dt) {
        v_at[dt][0] = v1 + (vp ^ (dt << 6));
        v_at[dt][1] = v1 + 8 * kRow + (vp ^ (dt << 6) ^ 32);
      }
    } else {
#pragma unroll
      for (int c = 0; c < 8; ++c) k_at[c] = k0 + n * kRow + h * 256 + ((c ^ swizzle<T>(n & 15)) << 4);   // and ^ 128 for c + 8
      // row (i & 3) + 8 (i >> 2) + 4 h: its swizzle is (i & 3) | (i >> 2 & 1) << 2 | h << 3
#pragma unroll
      for (int dt = 0; dt < 4; ++dt)
        v_at[dt][0] = v0 + 4 * h * kRow + (((8 * dt + (n >> 2)) ^ (h << 3)) << 4) + ((n & 3) << 2);
    }
  }

  __device__ __forceinline__ void load_keys(uint32_t off, Keys& kf) {
    if constexpr (kBf16) {
#pragma unroll
      for (int c = 0; c < 8; ++c) kf[c] = *(lds_bf16x8)(uintptr_t)(k_at[c] + off);
    }
  }
  __device__ __forceinline__ void load_values(uint32_t off, Values& vf) {
    if constexpr (kBf16) {
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int dt = 0; dt < 4; ++dt) {
          const uint32_t x = off + 16 * k * kRowBytes<T>;
          const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(uintptr_t)(v_at[dt][0] + x));
          const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(uintptr_t)(v_at[dt][1] + x));
          vf[k][dt] = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        }
    }
  }
  __device__ __forceinline__ f32x16 scores(uint32_t off, const Keys& kf) {
    f32x16 sc;
#pragma unroll
    for (int i = 0; i < 16; ++i) sc[i] = 0.f;
    if constexpr (kBf16) {
#pragma unroll
      for (int c = 0; c < 8; ++c) sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[c], q[c], sc, 0, 0, 0);
    } else {
#pragma unroll
      for (int c = 0; c < 16; ++c) {
        const f32x4 k = *(lds_f32x4)(uintptr_t)((k_at[c & 7] ^ (c >> 3 << 7)) + off);
#pragma unroll
        for (int e = 0; e < 4; ++e) sc = __builtin_amdgcn_mfma_f32_32x32x2f32(k[e], q[c][e], sc, 0, 0, 0);
      }
    }
    return sc;
  }
  // Raises the base where a lane's scores pass it.
  __device__ __forceinline__ void rebase(float top) {
    if (!__builtin_amdgcn_ballot_w64(top > grow_at)) return;
    top = fmaxf(top, __shfl_xor(top, 32, kWave));
    const bool grows = top > grow_at;
    // before the first finite score the sums are 0 (or NaN): any factor does
    const float f = grows && grow_at != -__builtin_inff() ? __builtin_amdgcn_exp2f(base - top) : 1.f;
    base = grows ? top : base;
    grow_at = grows ? top + kGrow : grow_at;
    sum *= f;
#pragma unroll
    for (int dt = 0; dt < 4; ++dt) o[dt] *= f;
  }
  // Scores of keys p0.. become base-2 logits (masked: -inf where the query does not see the
  // key), and their weights pb.  bfloat16: rest is what the rounding leaves over, and
  // pb that too where `low` is set.
  __device__ __forceinline__ void soften(f32x16& sc, int p0, bool masked, bool low, Weights& pb, Weights& rest) {
    float m = mult;
    if (masked) {
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int key = p0 + (i & 3) + 8 * (i >> 2) + 4 * h;
        sc[i] = key < limit ? sc[i] * mult : -__builtin_inff();
      }
      m = 1.f;
    }
    float top = sc[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) top = fmaxf(top, sc[i]);
    rebase(top * m);
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const float p = __builtin_amdgcn_exp2f(fmaf(sc[i], m, -base));
      sum += p;
      if constexpr (kBf16) {
        const __bf16 b = (__bf16)p, r = (__bf16)(p - (float)b);
        pb[i >> 3][i & 7] = low ? r : b;
        rest[i >> 3][i & 7] = r;
      } else {
        pb[i] = p;
      }
    }
    if (!masked) {
#pragma unroll
      for (int i = 0; i < 16; ++i) sc[i] *= mult;      // dead where nobody stores the logits
    }
  }
  __device__ __forceinline__ void add_values(uint32_t off, const Values& vf, const Weights& pb) {
    if constexpr (kBf16) {
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int dt = 0; dt < 4; ++dt)
          o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, vf[k][dt]), pb[k], o[dt], 0, 0, 0);
    } else {
#pragma unroll
      for (int i = 0; i < 16; ++i)
#pragma unroll
        for (int dt = 0; dt < 4; ++dt) {
          const uint32_t x = v_at[dt][0] + ((i & 3) + 8 * (i >> 2)) * kRowBytes<T>;
          const float v = *(lds_f32)(uintptr_t)((x ^ (((i & 3) | ((i >> 2) & 1) << 2) << 4)) + off);
          o[dt] = __builtin_amdgcn_mfma_f32_32x32x2f32(v, pb[i], o[dt], 0, 0, 0);
        }
    }
  }
  // Whether the values, not the scores, make the lane's sums infinite or NaN.
  __device__ __forceinline__ bool met_not_finite() const {
    float zero = 0.f;
#pragma unroll
    for (int dt = 0; dt < 4; ++dt)
#pragma unroll
      for (int i = 0; i < 16; ++i) zero = fmaf(o[dt][i], 0.f, zero);
    return zero != 0.f && __builtin_isfinite(sum);
  }
  __device__ __forceinline__ void restart() {
    base = sum = 0.f;
    grow_at = -__builtin_inff();
#pragma unroll
    for (int dt = 0; dt < 4; ++dt)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[dt][i] = 0.f;
  }
  // A value that is not finite, of row `key`, to the queries that see it.
  __device__ __forceinline__ void add_not_finite(const void* v, int64_t row, int key, bool skip) {
#pragma unroll
    for (int dt = 0; dt < 4; ++dt)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float f = at<T>(v, row, 32 * dt + (i & 3) + 8 * (i >> 2) + 4 * h);
        o[dt][i] += key < limit && !skip && !__builtin_isfinite(f) ? f : 0.f;
      }
  }
};

// Rows first..first + kN - 1 of a slice (row0 its first, n rows held; rows from n on repeat
// the last) to LDS, permuted as `swizzle` says.
template <class T, int kN>
__device__ __forceinline__ void copy_rows(const void* p, int64_t row0, int first, int n, uint32_t lds, bool stream) {
  constexpr int kRow = kRowBytes<T>, kPieces = kRow / 16, kRows = 1024 / kRow;   // rows of one copy of 64 x 16 bytes
  const int lane = threadIdx.x & 63, from = min(first, n - 1);
  const char* base = static_cast<const char*>(p) + (row0 + from) * kRow;
  auto copies = [&](auto&& copy) {
#pragma unroll
    for (int c = 0; c < kN / kRows; ++c) {
      const int r = c * kRows + lane / kPieces;
      copy(base, min(r, n - 1 - from) * kRow + (((lane % kPieces) ^ swizzle<T>(r)) << 4), lds + c * 1024);
    }
  };
  if (stream) copies([](const void* b, uint32_t off, uint32_t to) { stream_to_lds(b, off, to); });
  else copies([](const void* b, uint32_t off, uint32_t to) { copy_to_lds(b, off, to); });
}

// Makes values that are not finite 0 in kBytes of LDS that this wave's lanes share;
// whether there were any.
template <class T, int kBytes>
__device__ __forceinline__ bool clear_not_finite(char* p) {
  bool any = false;
#pragma unroll
  for (int i = 0; i < kBytes / 1024; ++i) {
    uint4* v = reinterpret_cast<uint4*>(p + i * 1024) + (threadIdx.x & 63);
    uint4 u = *v;
    uint32_t* e = &u.x;
    bool bad = false;
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const bool b0 = sizeof(T) == 2 && (e[c] & 0x7f80u) == 0x7f80u, b1 = (e[c] & 0x7f800000u) == 0x7f800000u;
      e[c] &= (b0 ? 0xffff0000u : ~0u) & (b1 ? (sizeof(T) == 2 ? 0x0000ffffu : 0u) : ~0u);
      bad |= b0 | b1;
    }
    if (bad) *v = u;
    any |= bad;
  }
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  return any;
}

// 16 channels of a query's sums, 32 dt + (i & 3) + 8 (i >> 2) + 4 h, as results or as a part.
__device__ __forceinline__ void store_sums(const AttnArgs& a, int64_t row, int part, int dt, int h, const f32x16& o,
                                           float m, float l) {
  if (a.n_parts > 1) {
    float* p = a.part + (row * a.n_parts + part) * kPartFloats;
    if (dt == 0 && h == 0) *reinterpret_cast<float2*>(p) = make_float2(m, l);
#pragma unroll
    for (int i = 0; i < 16; i += 2)
      *reinterpret_cast<float2*>(p + 2 + 32 * dt + (i & 3) + 8 * (i >> 2) + 4 * h) = make_float2(o[i], o[i + 1]);
    return;
  }
  const float inv = inv_sum(l);
  if (a.lse_out && dt == 0 && h == 0) a.lse_out[row] = lse_of(m, l);
#pragma unroll
  for (int i = 0; i < 16; i += 4) {
    const size_t x = row * kHeadDim + 32 * dt + 2 * i + 4 * h;
    const float y0 = o[i] * inv, y1 = o[i + 1] * inv, y2 = o[i + 2] * inv, y3 = o[i + 3] * inv;
    if (a.out_bf16) {
      *reinterpret_cast<uint2*>(static_cast<uint16_t*>(a.out) + x) =
          make_uint2(f32_to_bf16(y0) | (uint32_t)f32_to_bf16(y1) << 16, f32_to_bf16(y2) | (uint32_t)f32_to_bf16(y3) << 16);
    } else {
      *reinterpret_cast<float4*>(static_cast<float*>(a.out) + x) = make_float4(y0, y1, y2, y3);
    }
  }
}

// Adds to the weights of rows i .. i + 3 of n what n_queries give them: 2^(logit - lse), lse
// infinite where a query sees nothing.
__device__ __forceinline__ void add_weights(const float* logits, int stride, int n_queries, const float* lse, int n, int i,
                                            float* weights) {
  float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
  for (int q = 0; q < n_queries; ++q) {
    const float4 v = *reinterpret_cast<const float4*>(logits + (int64_t)q * stride + i);
    const float e = lse[q];
    y.x += __builtin_amdgcn_exp2f(v.x - e);
    y.y += __builtin_amdgcn_exp2f(v.y - e);
    y.z += __builtin_amdgcn_exp2f(v.z - e);
    y.w += __builtin_amdgcn_exp2f(v.w - e);
  }
  weights[i] += y.x;
  if (i + 1 < n) weights[i + 1] += y.y;
  if (i + 2 < n) weights[i + 2] += y.z;
  if (i + 3 < n) weights[i + 3] += y.w;
}

// Up to 32 queries: every wave takes every fourth 32 keys, through its own place in LDS, so
// that no wave waits for another.  bfloat16: what the rounding of a weight leaves over meets the
// values too, in products of its own, or with up to 16 queries, which lanes n and n + 16 both
// hold then, as the second's weights, in columns that would be idle.  Such a rest is 0 or negative
// as often as not, and an infinite value that it met NaN: a wave whose sums the values leave not
// finite takes its tiles once more, with such values set to 0 and added apart.
//
// Memory bounds it: without any arithmetic the same copies took as long (a prefix of 32768 rows
// of 8 slices, 38.3 us for 40.5 then).  Four sequences over that prefix: 28.0 us and 4.1 for the
// joining launch; from the first to the last copy of a block 6.6 TB/s, where plain streaming
// reads reach 6.8 to 7.0, the rest is some 1.5 us before the first copy and 2 after the last.
// Caches of 1024 slices (930 MB, weights added): 163 us, without weights 140.  float32: the
// products, two channels or keys at a time, take 3.4 us a tile, more than its bytes.
template <class T>
__device__ __forceinline__ void attend_few(const AttnArgs& a, bool own, int64_t id, char* s_ring, float* s_m, float* s_l, float* s_logits) {
  constexpr int kTileBytes = kTile * kRowBytes<T>;
  const Side& x = own ? a.own : a.prefix;
  const Place p = place_of(a, x, own, id);
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r0 = p.rgrp * 32, n_rows = min(32, p.n_rows - r0);
  const bool twice = Wave<T>::kBf16 && n_rows <= 16, low = twice && (lane & 16);
  const int r = r0 + min(lane & (twice ? 15 : 31), n_rows - 1);
  int least, most;
  limits_of(a, p, own, r0, r0 + n_rows - 1, least, most);
  const int tiles = (most + kTile - 1) / kTile;
  const int t0 = (int)((int64_t)tiles * p.split / x.splits), t1 = (int)((int64_t)tiles * (p.split + 1) / x.splits);
  const uint32_t slot = __builtin_amdgcn_readfirstlane(lds_addr(s_ring) + w * 2 * kTileBytes);
  auto copy_k = [&](int tile) { copy_rows<T, kTile>(x.k, p.kv_row, tile * kTile, p.n, slot, a.stream && x.row_groups == 1); };
  auto copy_v = [&](int tile) {
    copy_rows<T, kTile>(x.v, p.kv_row, tile * kTile, p.n, slot + kTileBytes, a.stream && x.row_groups == 1);
  };
  Wave<T> f;
  f.init(a, query_row(a, p, own, r), limit_of(a, p, own, r));
  f.addresses(slot, slot + kTileBytes);
  // A block that sees all of a slice keeps the logits of its first rows in LDS: 1024 slices of 1781
  // rows took 141 us without logits, 175 with all of them through memory.
  const int near = a.n_parts == 1 ? kNearLogits / n_rows / kTile * kTile : 0;
  // bfloat16: a tile's operands all fit the registers, so that the next one is under way during
  // its arithmetic.  float32: the next keys follow the scores, the next values the sums.
  constexpr bool kBf16 = Wave<T>::kBf16;
  constexpr int kCopies = kTileBytes / 1024;
  static_assert(kBf16 || kCopies == 16, "the waits below count copies");
  if (t0 + w < t1) {
    copy_k(t0 + w);
    copy_v(t0 + w);
  }
#pragma unroll
  for (int c = 0; c < Wave<T>::kQ; ++c) asm volatile("" : "+v"(f.q[c]));   // waits for the queries here, not in the loop
  bool bad = false, careful = false;
again:
  for (int tile = t0 + w; tile < t1; tile += kBlockWaves) {
    const int p0 = tile * kTile;
    const bool masked = p0 + kTile > least, more = tile + kBlockWaves < t1;
    // values that a query may not see must not reach it: 0 * inf is NaN
    auto clear = [&]() {
      if (masked || careful) bad |= __builtin_amdgcn_ballot_w64(clear_not_finite<T, kTileBytes>(s_ring + (w * 2 + 1) * kTileBytes)) != 0;
    };
    typename Wave<T>::Keys kf;
    typename Wave<T>::Values vf;
    typename Wave<T>::Weights pb, rest;
    if constexpr (kBf16) {
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      clear();
      f.load_keys(0, kf);
      f.load_values(0, vf);
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      if (more) {
        copy_k(tile + kBlockWaves);
        copy_v(tile + kBlockWaves);
      }
    } else {
      asm volatile("s_waitcnt vmcnt(16)" ::: "memory");        // all but the values
    }
    f32x16 sc = f.scores(0, kf);
    if constexpr (!kBf16) {
#pragma unroll
      for (int i = 0; i < 16; ++i) asm volatile("" : "+v"(sc[i]));    // the keys have been read
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      if (more) copy_k(tile + kBlockWaves);
    }
    f.soften(sc, p0, masked, low, pb, rest);
    if constexpr (!kBf16) {
      if (more) asm volatile("s_waitcnt vmcnt(16)" ::: "memory");     // all but the next keys
      else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      clear();
    }
    if (own && a.logits && f.n < n_rows) {
      float* to = p0 < near ? s_logits + f.n * near + p0 : a.logits + (p.s * p.n_rows + r) * a.logit_stride + p0;
      to += 4 * f.h;
#pragma unroll
      for (int i = 0; i < 16; i += 4)
        *reinterpret_cast<float4*>(to + 2 * i) = make_float4(sc[i], sc[i + 1], sc[i + 2], sc[i + 3]);
    }
    f.add_values(0, vf, pb);
    if constexpr (kBf16) {
      if (!twice) f.add_values(0, vf, rest);
    }
    if constexpr (!kBf16) {
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      if (more) copy_v(tile + kBlockWaves);
    }
  }
  if (kBf16 && !careful && __builtin_amdgcn_ballot_w64(f.met_not_finite())) {
    careful = true;
    f.restart();
    copy_k(t0 + w);
    copy_v(t0 + w);
    goto again;
  }
  if (bad) {                                    // rare
#pragma unroll 1
    for (int tile = t0 + w; tile < t1; tile += kBlockWaves) {
      if (!careful && tile * kTile + kTile <= least) continue;
#pragma unroll 1
      for (int key = tile * kTile; key < min(tile * kTile + kTile, most); ++key)
        f.add_not_finite(x.v, p.kv_row + key, key, low);
    }
  }
  // the waves' sums, in their places in LDS; wave w joins channels 32 w..
  const float m = f.grow_at == -__builtin_inff() ? -__builtin_inff() : f.base;
  const float total = f.sum + __shfl_xor(f.sum, 32, kWave);
  // (a lane's 64 sums in 16-byte pieces, permuted so that sixteen lanes meet in no bank)
  f32x4* mine = reinterpret_cast<f32x4*>(s_ring + w * 2 * kTileBytes) + lane * 16;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const f32x16& y = f.o[i >> 2];
    const int e = (i & 3) * 4;
    mine[i ^ (lane & 15)] = f32x4{y[e], y[e + 1], y[e + 2], y[e + 3]};
  }
  if (f.h == 0) {
    s_m[w * 32 + f.n] = m;
    s_l[w * 32 + f.n] = total;
  }
  __syncthreads();
  float mm = s_m[f.n];
#pragma unroll
  for (int i = 1; i < kBlockWaves; ++i) mm = fmaxf(mm, s_m[i * 32 + f.n]);
  float l = 0.f;
  f32x16 o;
#pragma unroll
  for (int i = 0; i < 16; ++i) o[i] = 0.f;
#pragma unroll 1
  for (int v = 0; v < kBlockWaves; ++v) {
    const float e = __builtin_amdgcn_exp2f(s_m[v * 32 + f.n] - max_base(mm));
    l += s_l[v * 32 + f.n] * e;
    const f32x4* from = reinterpret_cast<const f32x4*>(s_ring + v * 2 * kTileBytes);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f32x4 y = from[lane * 16 + ((4 * w + i) ^ (lane & 15))];
      if (twice) y += from[(lane ^ 16) * 16 + ((4 * w + i) ^ (lane & 15))];
#pragma unroll
      for (int c = 0; c < 4; ++c) o[4 * i + c] += y[c] * e;
    }
  }
  if (f.n < n_rows)
    store_sums(a, query_row(a, p, own, r), (own && a.prefix_blocks ? a.prefix.splits : 0) + p.split, w, f.h, o, mm, l);
  if (!own || !a.logits || a.n_parts > 1) return;
  // the block has seen all there is: its rows' weights from the logits that its waves left
  // (behind the maxima, which other waves may still be reading)
  float* s_lse = s_m + kBlockWaves * 32;
  if (w == 0 && f.h == 0) s_lse[f.n] = l == 0.f ? __builtin_inff() : max_base(mm) + log2f(l);
  __syncthreads();
  const float* far = a.logits + p.s * p.n_rows * a.logit_stride;
  for (int i = threadIdx.x * 4; i < p.n; i += kBlockWaves * 64 * 4)
    add_weights(i < near ? s_logits : far, i < near ? near : a.logit_stride, p.n_rows, s_lse, p.n, i, a.weights + p.s * x.rows);
}

// Up to 32 WR queries, 32 a wave; the waves share stages of 64 keys (two places in LDS, one
// in flight), WR = 2 in halves.
//
// Eight chunks of 77 tokens over 20011 rows (2464 queries a slice): 228 to 237 us, 0.86
// PFLOP/s of the 1.35 to 1.37 of a large product.  A tile of a wave has 16 products (512 cycles),
// 16 exponentials (256) and 80 other vector operations; two waves of a SIMD overlap them in
// part (matrix cores busy 50%, no LDS bank conflicts), at clocks of 1.9 to 2.1 GHz under this
// load.  The next tile's keys read before the exponentials: 247 us for 258 on one part, both
// scores first 244; a raised wave priority around the products 234 for 232.
// The weights are rounded to bfloat16 (2^-8 of each), as the products of what that leaves over
// would take 304 us for 227, and 64 sequences over 32768 rows 83.5 for 72.5, all these on one part:
// outputs are 2.1e-3 of their size off instead of 1.7e-3, a bfloat16 result's own rounding.
template <class T, int WR, bool own>
__device__ __forceinline__ void attend_many(const AttnArgs& a, int64_t id, char* s_ring, int* s_bad) {
  constexpr int kRow = kRowBytes<T>, kHalf = kStage * kRow, WK = kBlockWaves / WR;
  const Side& x = own ? a.own : a.prefix;
  const Place p = place_of(a, x, own, id);
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wr = w % WR, wk = w / WR;
  const int b0 = p.rgrp * WR * 32, b1 = min(b0 + WR * 32, p.n_rows) - 1;     // the block's queries
  const int r0 = min(b0 + wr * 32, p.n_rows - 1), r1 = min(r0 + 31, p.n_rows - 1);
  const int r = min(b0 + wr * 32 + (lane & 31), p.n_rows - 1);
  int least, most, w_least, w_most;
  limits_of(a, p, own, b0, b1, least, most);
  limits_of(a, p, own, r0, r1, w_least, w_most);
  const int stages = (most + kStage - 1) / kStage;
  const int st0 = (int)((int64_t)stages * p.split / x.splits), st1 = (int)((int64_t)stages * (p.split + 1) / x.splits);
  const uint32_t ring = __builtin_amdgcn_readfirstlane(lds_addr(s_ring));
  // a wave's share: 16 rows
  auto copy = [&](int st, int place) {
    const uint32_t to = ring + place * 2 * kHalf + w * 16 * kRow;
    copy_rows<T, 16>(x.k, p.kv_row, st * kStage + w * 16, p.n, to, a.stream && x.row_groups == 1);
    copy_rows<T, 16>(x.v, p.kv_row, st * kStage + w * 16, p.n, to + kHalf, a.stream && x.row_groups == 1);
  };
  Wave<T> f;
  f.init(a, query_row(a, p, own, r), limit_of(a, p, own, r));
  f.addresses(ring, ring + kHalf);
  if (threadIdx.x == 0) *s_bad = 0;
  __syncthreads();
  if (st0 < st1) copy(st0, 0);
#pragma unroll
  for (int c = 0; c < Wave<T>::kQ; ++c) asm volatile("" : "+v"(f.q[c]));   // waits for the queries here, not in the loop
  // Stage st, which lies at place `place` of the ring (a constant where it is inlined).
  auto stage = [&](int st, int place) {
    const int p0 = st * kStage;
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    if (p0 + kStage > least) {                  // block-uniform
      if (clear_not_finite<T, 16 * kRow>(s_ring + place * 2 * kHalf + kHalf + w * 16 * kRow)) *s_bad = 1;
    }
    sync_stage();                               // the stage is in LDS; the other place is free
    if (st + 1 < st1) copy(st + 1, place ^ 1);
    typename Wave<T>::Keys kf;
    typename Wave<T>::Values vf;
    typename Wave<T>::Weights pb, rest;
    auto half = [&](int x, bool more) {
      const int k0 = p0 + x * kTile;
      const uint32_t off = place * 2 * kHalf + x * kTile * kRow;
      f32x16 sc = f.scores(off, kf);
      f.load_values(off, vf);
      if (more) f.load_keys(off + kTile * kRow, kf);   // the next tile's, before the exponentials
      __builtin_amdgcn_sched_barrier(0);
      f.soften(sc, k0, k0 + kTile > w_least, false, pb, rest);
      f.add_values(off, vf, pb);
    };
    if constexpr (WK == 1) {
      if (p0 >= w_most) return;
      f.load_keys(place * 2 * kHalf, kf);
      half(0, true);
      if (p0 + kTile < w_most) half(1, false);
    } else {
      if (p0 + wk * kTile >= w_most) return;
      f.load_keys(place * 2 * kHalf + wk * kTile * kRow, kf);
      half(wk, false);
    }
  };
  for (int st = st0; st < st1; st += 2) {
    stage(st, 0);
    if (st + 1 < st1) stage(st + 1, 1);
  }
  sync_stage();
  if (*s_bad) {                                 // block-uniform, rare
#pragma unroll 1
    for (int st = st0; st < st1; ++st) {
      if (st * kStage + kStage <= least) continue;
#pragma unroll 1
      for (int key = st * kStage; key < min(st * kStage + kStage, w_most); ++key)
        if (WK == 1 || (key / kTile) % 2 == wk) f.add_not_finite(x.v, p.kv_row + key, key, false);
    }
  }
  float m = f.grow_at == -__builtin_inff() ? -__builtin_inff() : f.base;
  float total = f.sum + __shfl_xor(f.sum, 32, kWave);
  if constexpr (WK == 2) {
    // wk = 1 leaves its sums in LDS, wk = 0 adds them
    float* mine = reinterpret_cast<float*>(s_ring) + wr * 66 * 64 + lane;
    __syncthreads();                            // every wave has read s_bad and its last stage
    if (wk == 1) {
#pragma unroll
      for (int i = 0; i < 64; ++i) mine[i * 64] = f.o[i >> 4][i & 15];
      mine[64 * 64] = m;
      mine[65 * 64] = total;
    }
    __syncthreads();
    if (wk == 1) return;
    const float m1 = mine[64 * 64], mm = fmaxf(m, m1);
    const float f0 = __builtin_amdgcn_exp2f(m - max_base(mm)), f1 = __builtin_amdgcn_exp2f(m1 - max_base(mm));
    m = mm;
    total = total * f0 + mine[65 * 64] * f1;
#pragma unroll
    for (int i = 0; i < 64; ++i) f.o[i >> 4][i & 15] = f.o[i >> 4][i & 15] * f0 + mine[i * 64] * f1;
  }
  if (b0 + wr * 32 + f.n > b1) return;
  const int64_t row = query_row(a, p, own, r);
  const int part = (own && a.prefix_blocks ? a.prefix.splits : 0) + p.split;
#pragma unroll
  for (int dt = 0; dt < 4; ++dt) store_sums(a, row, part, dt, f.h, f.o[dt], m, total);
}

// Blocks of the prefix (WP waves of queries), then of the own rows (WO).
template <class T, int WP, int WO>
__global__ __launch_bounds__(kBlockWaves * 64, sizeof(T) == 2 ? 2 : 1)
void attn_kernel(const AttnArgs a) {
  __shared__ __align__(256) char s_ring[kRingBytes<T>];
  __shared__ float s_m[(kBlockWaves + 1) * 32], s_l[kBlockWaves * 32];
  __shared__ __align__(16) float s_logits[WO == 1 ? kNearLogits : 4];
  __shared__ int s_bad;
  const bool own = blockIdx.x >= a.prefix_blocks;
  const int64_t id = own ? blockIdx.x - a.prefix_blocks : blockIdx.x;
  if constexpr (WP == 1) {
    // one code for both: such blocks run a few iterations, and what they run has to be fetched first
    attend_few<T>(a, own, id, s_ring, s_m, s_l, s_logits);
  } else if (!own) {
    attend_many<T, WP, false>(a, id, s_ring, &s_bad);
  } else if constexpr (WO == 1) {
    attend_few<T>(a, true, id, s_ring, s_m, s_l, s_logits);
  } else {
    attend_many<T, WO, true>(a, id, s_ring, &s_bad);
  }
}

// How a call is cut into blocks.
struct Cut {
  int waves_p, waves_o;            // of queries of a block: 1, 2 or 4
  int groups_p, groups_o;          // blocks that a slice's queries are cut into
  int splits_p, splits_o;          // parts that its keys are cut into
  int64_t blocks_p, blocks_o;
  int n_parts() const { return splits_p + splits_o; }
};

// Parts that the keys of `units` slices' query blocks are cut into, for `slots` blocks at a time:
// the fewest of those that make the rounds of blocks times their tiles least.  A block's start
// and end count as tiles, more where it leaves more partials; waves that take turns (w = 1)
// take four tiles at once.
int splits_of(int64_t units, int64_t tiles, int w, int64_t slots) {
  if (units < 1 || tiles < 1) return 0;
  const int64_t ends = 4 * w + 2;
  auto length = [&](int64_t s) {
    const int64_t t = (tiles + s - 1) / s;
    return (w == 1 ? (t + 3) / 4 * 4 : t) + ends;
  };
  const int64_t most = std::max<int64_t>(1, tiles / (4 * w));
  int64_t best = 1, cost = (units + slots - 1) / slots * length(1);
  for (int64_t rounds = (units + slots - 1) / slots, i = 0; i < 8; ++i, ++rounds) {
    int64_t s = std::min(most, rounds * slots / units);
    if (s < 1) continue;
    const int64_t len = length(s);
    const int64_t per = w == 1 ? len - ends : (tiles + s - 1) / s;    // the fewest parts of that length
    s = std::max<int64_t>(1, std::min(s, (tiles + per - 1) / per));
    if (rounds * len < cost) cost = rounds * len, best = s;
  }
  return (int)best;
}

// float32 leaves no registers for stages that waves share: always 32 queries a block.
Cut cut_of(int64_t n_slices, int64_t n_prefix_slices, int group_size, int n_q, int64_t prefix_rows, int64_t own_rows,
           int dtype) {
  Cut c{};
  const bool bf16 = dtype == LOUISKV_BF16;
  const int64_t resident = bf16 ? 512 : 256;      // blocks that the chip holds, two or one a CU
  const int64_t mine = (int64_t)group_size * n_q, all = prefix_rows ? mine * (n_slices / n_prefix_slices) : 0;
  auto waves = [&](int64_t rows) { return !bf16 || rows <= 32 ? 1 : rows <= 64 ? 2 : 4; };
  auto groups = [](int64_t rows, int w) { return (int)((rows + 32 * w - 1) / (32 * w)); };
  c.waves_o = waves(mine);
  c.waves_p = std::max(waves(all), c.waves_o);
  c.groups_o = groups(mine, c.waves_o);
  c.groups_p = groups(all, c.waves_p);
  const int64_t tiles_p = (prefix_rows + kTile - 1) / kTile, tiles_o = (own_rows + kTile - 1) / kTile;
  const int64_t unit_p = prefix_rows ? n_prefix_slices * c.groups_p : 0, unit_o = own_rows ? n_slices * c.groups_o : 0;
  // the two run side by side, each in its share of the chip; a few blocks of own rows get a place
  // each, so that none waits for a prefix block to end
  const double work_p = (double)unit_p * tiles_p, work_o = (double)unit_o * tiles_o;
  int64_t slots = !unit_o ? resident : (int64_t)(resident * (work_p / (work_p + work_o)) + 0.5);
  if (unit_o <= resident / 8) slots = std::min(slots, resident - unit_o);
  slots = std::max<int64_t>(1, std::min(slots, resident - (unit_o > 0)));
  c.splits_p = splits_of(unit_p, tiles_p, c.waves_p, slots);
  c.splits_o = splits_of(unit_o, tiles_o, c.waves_o, unit_p ? resident - slots : resident);
  c.blocks_p = unit_p * c.splits_p;
  c.blocks_o = unit_o * c.splits_o;
  return c;
}

// Rows of calls that read more than the L2s hold bypass the caches where one block reads
// them: caches of 930 MB took 178 us (201 through the caches) when all logits went through memory,
// a prefix of 134 MB 34.6 us (38.4) before its waves joined in 16-byte pieces; 8 MB stay (12.0 us;
// 13.5 past the caches).
template <class T>
void launch_attn(const AttnArgs& a, const Cut& c, hipStream_t hs) {
  const unsigned grid = (unsigned)(c.blocks_p + c.blocks_o);
  constexpr int kThreads = kBlockWaves * 64;
  if constexpr (sizeof(T) == 4) {
    attn_kernel<T, 1, 1><<<grid, kThreads, 0, hs>>>(a);
  } else {
    switch (c.waves_p * 8 + c.waves_o) {
      case 8 + 1: attn_kernel<T, 1, 1><<<grid, kThreads, 0, hs>>>(a); break;
      case 16 + 1: attn_kernel<T, 2, 1><<<grid, kThreads, 0, hs>>>(a); break;
      case 16 + 2: attn_kernel<T, 2, 2><<<grid, kThreads, 0, hs>>>(a); break;
      case 32 + 1: attn_kernel<T, 4, 1><<<grid, kThreads, 0, hs>>>(a); break;
      case 32 + 2: attn_kernel<T, 4, 2><<<grid, kThreads, 0, hs>>>(a); break;
      default: attn_kernel<T, 4, 4><<<grid, kThreads, 0, hs>>>(a); break;
    }
  }
}

struct WeightArgs {
  const void* q;
  int group_size, n_q;
  float scale;       // times log2(e), rounded
  double per_lse;    // what turns an lse into base 2 by that same rounded factor
  const void* keys;
  int key_rows;
  const int32_t* n_keys;
  const float* lse;
  float* weights;
  int64_t n_slices;
  int splits;        // parts of the queries
  float* part;       // [splits][slices][key_rows] sums
};

// 32-key tiles of a wave as the operand K^T, and what 32 queries at a time add to their sums:
// Q K^T leaves a lane 16 queries of one key, which it adds up.
template <class T, int KT>
struct KeyTiles {
  static constexpr bool kBf16 = sizeof(T) == 2;
  static constexpr int kPieces = kBf16 ? 8 : 16;       // 16-byte pieces 2 c + h (bfloat16) or 16 h + c (float32) of key n
  typedef typename std::conditional<kBf16, bf16x8, f32x4>::type Piece;
  Piece k[KT][kPieces];
  float sum[KT];
  int first;                                           // the first key

  // Keys first.. of a slice of n (rows from n on repeat the last).
  __device__ __forceinline__ void load(const void* keys, int64_t row0, int first_, int n) {
    const int lane = threadIdx.x & 63, h = lane >> 5;
    first = first_;
#pragma unroll
    for (int x = 0; x < KT; ++x) {
      const int key = min(first + x * kTile + (lane & 31), n - 1);
      const Piece* from = reinterpret_cast<const Piece*>(static_cast<const T*>(keys) + (row0 + key) * kHeadDim);
#pragma unroll
      for (int c = 0; c < kPieces; ++c) k[x][c] = from[kBf16 ? 2 * c + h : 16 * h + c];
      sum[x] = 0.f;
    }
  }
  // Waits for the keys here, not where they are used.
  __device__ __forceinline__ void arrive() {
#pragma unroll
    for (int x = 0; x < KT; ++x)
#pragma unroll
      for (int c = 0; c < kPieces; ++c) asm volatile("" : "+v"(k[x][c]));
  }
  // LDS addresses of the lane's reads of a 32-query tile at `to`.
  static __device__ __forceinline__ void addresses(uint32_t to, uint32_t (&q_at)[8]) {
    const int lane = threadIdx.x & 63, h = lane >> 5, r = lane & 31;
#pragma unroll
    for (int c = 0; c < 8; ++c)
      q_at[c] = to + r * kRowBytes<T> + (kBf16 ? ((h ^ swizzle<T>(r & 15)) << 4) ^ (c << 5)
                                               : h * 256 + ((c ^ swizzle<T>(r & 15)) << 4));
  }
  // The tile of queries `off` bytes on: their -lse in base 2, and the keys that each sees, of
  // which the keys below `least` all do if none is `dead`.
  __device__ __forceinline__ void weigh(const uint32_t (&q_at)[8], uint32_t off, const float* lse, const int* limits, int least,
                                        bool dead, float scale) {
    const int lane = threadIdx.x & 63, h = lane >> 5;
    Piece q[kBf16 ? 8 : 1];
    if constexpr (kBf16) {
#pragma unroll
      for (int c = 0; c < 8; ++c) q[c] = *(lds_bf16x8)(uintptr_t)(q_at[c] + off);
    }
    f32x4 nl[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) nl[i] = *reinterpret_cast<const f32x4*>(lse + 8 * i + 4 * h);
#pragma unroll
    for (int x = 0; x < KT; ++x) {
      f32x16 sc;
#pragma unroll
      for (int i = 0; i < 16; ++i) sc[i] = 0.f;
      if constexpr (kBf16) {
#pragma unroll
        for (int c = 0; c < 8; ++c) sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(q[c], k[x][c], sc, 0, 0, 0);
      } else {
#pragma unroll
        for (int c = 0; c < 16; ++c) {
          const f32x4 y = *(lds_f32x4)(uintptr_t)((q_at[c & 7] ^ (c >> 3 << 7)) + off);
#pragma unroll
          for (int e = 0; e < 4; ++e) sc = __builtin_amdgcn_mfma_f32_32x32x2f32(y[e], k[x][c][e], sc, 0, 0, 0);
        }
      }
      const int key = first + x * kTile + (lane & 31);
      float part = 0.f;
      if (dead || first + x * kTile + kTile > least) {
#pragma unroll
        for (int i = 0; i < 16; ++i)
          part += key < limits[(i & 3) + 8 * (i >> 2) + 4 * h]
                      ? __builtin_amdgcn_exp2f(fmaf(sc[i], scale, nl[i >> 2][i & 3])) : 0.f;
      } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) part += __builtin_amdgcn_exp2f(fmaf(sc[i], scale, nl[i >> 2][i & 3]));
      }
      sum[x] += part;
    }
  }
  // f(key, sum) for the keys of the lanes below 32 that there are
  template <class F>
  __device__ __forceinline__ void each_sum(int n, F&& f) const {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int x = 0; x < KT; ++x) {
      const float y = sum[x] + __shfl_xor(sum[x], 32, kWave);
      const int key = first + x * kTile + (lane & 31);
      if (lane < 32 && key < n) f(key, y);
    }
  }
};

// Query f of those of a slice that count, the last token first, a token's heads together:
// x / g = x * magic >> 16 for x below 1024.
struct QueryOrder {
  int g, n_q, magic;
  __device__ __forceinline__ QueryOrder(int g_, int n_q_) : g(g_), n_q(n_q_), magic(65536 / g_ + 1) {}
  // query base + r (base uniform, r below 512) as its head and token
  __device__ __forceinline__ void at(int base, int r, int& head, int& token) const {
    const int t = base / g, x = r + base - t * g, dt = x * magic >> 16;
    head = x - dt * g;
    token = n_q - 1 - t - dt;
  }
};

// Sums of softmax weights by key.  Block: keys, which stay in registers as the operand K^T
// (KT 32-key tiles a wave), and a part of the queries that see them, 64 at a time through LDS
// (two places, one in flight), the last tokens first, a token's heads together: blocks
// of a slice begin with the same queries and meet them in the L2.  Q K^T leaves a lane 16
// queries of one key, which it adds up.
//
// A tile has 8 products (256 cycles), and a multiply-add, an exponential and an add of 16 scores
// (384), which bound it: a 32K prompt of 8 slices 4.6 to 4.7 ms, 0.95 PFLOP/s, some 520 cycles a
// tile at the 1.93 GHz that the clock falls to; without the exponentials 4.1, with an eighth
// of the products 2.9.  Three waves a SIMD 4.7 ms for two's 4.9; products of two tiles in turn
// 4.9, a raised wave priority around them 4.8.
constexpr int kQueries = 64;                            // of a stage
constexpr int block_keys(int key_tiles) { return kBlockWaves * key_tiles * kTile; }

template <class T, int KT>
__global__ __launch_bounds__(kBlockWaves * 64, sizeof(T) == 2 ? KT == 2 ? 3 : 4 : 2)
void weights_kernel(const WeightArgs a) {
  constexpr bool kBf16 = sizeof(T) == 2;
  constexpr int kRow = kRowBytes<T>, kPlace = kQueries * kRow;
  __shared__ __align__(256) char s_ring[2][kPlace];
  __shared__ float s_lse[2][kQueries];                  // -lse in base 2
  __shared__ int s_limit[2][kQueries], s_dead[2];       // keys that a query sees; a stage with a query that adds nothing
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5, n32 = lane & 31;
  int64_t id = blockIdx.x;
  const int64_t s = id % a.n_slices;                    // slices are dealt to the XCDs
  id /= a.n_slices;
  const int split = (int)(id % a.splits), kb = (int)(id / a.splits) * block_keys(KT);
  const int n = length_of(a.n_keys, s, a.key_rows), g = a.group_size;
  if (kb >= n) return;
  const int first = max(0, kb - (n - a.n_q));           // the first token that sees one of the keys
  const int total = (a.n_q - first) * g, stages = (total + kQueries - 1) / kQueries;
  const int st0 = (int)((int64_t)stages * split / a.splits), st1 = (int)((int64_t)stages * (split + 1) / a.splits);
  const QueryOrder order(g, a.n_q);
  const int wk0 = kb + w * KT * kTile;                  // the wave's first key
  KeyTiles<T, KT> keys;
  keys.load(a.keys, s * a.key_rows, wk0, n);
  auto query = [&](int st, int r, int& head, int& token) {   // past the last one, that
    order.at(st * kQueries, min(r, total - 1 - st * kQueries), head, token);
  };
  float lse_next = 0.f;
  int limit_next = 0;
  const uint32_t ring = __builtin_amdgcn_readfirstlane(lds_addr(s_ring));
  const char* qs = static_cast<const char*>(a.q) + s * g * a.n_q * (int64_t)kRow;
  auto copy = [&](int st, int place) {
    constexpr int kPieces = kRow / 16, kRows = 1024 / kRow;
#pragma unroll
    for (int c = 0; c < 16 / kRows; ++c) {
      const int r = w * 16 + c * kRows + lane / kPieces;
      int head, token;
      query(st, r, head, token);
      const char* from = qs + ((int64_t)head * a.n_q + token) * kRow + (((lane % kPieces) ^ swizzle<T>(r & 15)) << 4);
      const uint32_t to = ring + place * kPlace + (w * 16 + c * kRows) * kRow;
      asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(from), "s"(to) : "memory", "m0");
    }
    if (w == 0) {
      int head, token;
      query(st, lane, head, token);
      lse_next = a.lse[(s * g + head) * a.n_q + token];
      limit_next = st * kQueries + lane < total ? n - a.n_q + token + 1 : 0;
    }
  };
  uint32_t q_at[8];
  keys.addresses(ring, q_at);
  if (st0 < st1) copy(st0, 0);
  keys.arrive();
  auto stage = [&](int st, int place) {
    asm volatile("s_waitcnt vmcnt(0)" : "+v"(lse_next), "+v"(limit_next)::"memory");
    if (w == 0) {
      const bool none = lse_next == -__builtin_inff() || limit_next <= 0;
      s_lse[place][lane] = none ? -__builtin_inff() : (float)(-lse_next * a.per_lse);
      s_limit[place][lane] = none ? 0 : limit_next;
      const bool any = __builtin_amdgcn_ballot_w64(none) != 0;
      if (lane == 0) s_dead[place] = any;
    }
    sync_stage();
    if (st + 1 < st1) copy(st + 1, place ^ 1);
    const bool dead = __builtin_amdgcn_readfirstlane(s_dead[place]) != 0;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      // the tokens of the tile's last and first query bound what is seen
      const int f0 = st * kQueries + half * 32, f1 = min(f0 + 31, total - 1);
      if (f0 >= total) break;
      const int most = n - f0 / g, least = n - f1 / g;
      if (wk0 >= most) continue;
      keys.weigh(q_at, place * kPlace + half * 32 * kRow, &s_lse[place][half * 32], &s_limit[place][half * 32], least, dead,
                 a.scale);
    }
  };
  for (int st = st0; st < st1; st += 2) {
    stage(st, 0);
    if (st + 1 < st1) stage(st + 1, 1);
  }
  keys.each_sum(n, [&](int key, float y) {
    if (a.splits > 1) a.part[((int64_t)split * a.n_slices + s) * a.key_rows + key] = y;
    else a.weights[s * a.key_rows + key] += y;
  });
}

// The same for up to kFewQueries queries, which stay in LDS while the keys pass: wave w of a
// block takes every eighth tile of the block's keys.  Four waves a SIMD wait for keys in turn
// (64 queries, 32768 keys of 8 slices: 24.0 us; two waves with the next keys on their way
// 26.8, with two tiles at a time 28.7).
constexpr int kFewWaves = 8;
template <class T> constexpr int kFewQueries = 65536 / kRowBytes<T>;
template <class T>
__global__ __launch_bounds__(kFewWaves * 64, 4)
void weights_few_kernel(const WeightArgs a) {
  constexpr int kRow = kRowBytes<T>, kFew = kFewQueries<T>, kPieces = kRow / 16, kRows = 1024 / kRow;
  __shared__ __align__(256) char s_q[kFew * kRow];
  __shared__ float s_lse[kFew];                         // -lse in base 2
  __shared__ int s_limit[kFew], s_dead;
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int64_t s = blockIdx.x % a.n_slices;
  const int split = (int)(blockIdx.x / a.n_slices);     // of the keys
  const int n = length_of(a.n_keys, s, a.key_rows), g = a.group_size, total = g * a.n_q;
  const int groups = (n + kTile - 1) / kTile;
  const int g1 = (int)((int64_t)groups * (split + 1) / a.splits);
  int at = (int)((int64_t)groups * split / a.splits) + w;
  if (at - w >= g1) return;                             // block-uniform
  const QueryOrder order(g, a.n_q);
  KeyTiles<T, 1> keys;
  keys.load(a.keys, s * a.key_rows, min(at, g1 - 1) * kTile, n);
  const int tiles = (total + 31) / 32;
  const uint32_t base = __builtin_amdgcn_readfirstlane(lds_addr(s_q));
  const char* qs = static_cast<const char*>(a.q) + s * total * (int64_t)kRow;
  for (int c = w; c < tiles * 32 / kRows; c += kFewWaves) {
    const int r = c * kRows + lane / kPieces;
    int head, token;
    order.at(0, min(r, total - 1), head, token);
    const char* from = qs + ((int64_t)head * a.n_q + token) * kRow + (((lane % kPieces) ^ swizzle<T>(r & 15)) << 4);
    const uint32_t to = __builtin_amdgcn_readfirstlane(base + c * 1024);
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(from), "s"(to) : "memory", "m0");
  }
  if (tid == 0) s_dead = 0;
  __syncthreads();
  for (int r = tid; r < tiles * 32; r += kFewWaves * 64) {
    int head, token;
    order.at(0, min(r, total - 1), head, token);
    const float lse = a.lse[(s * g + head) * a.n_q + token];
    const int limit = r < total ? n - a.n_q + token + 1 : 0;
    const bool none = lse == -__builtin_inff() || limit <= 0;
    s_lse[r] = none ? -__builtin_inff() : (float)(-lse * a.per_lse);
    s_limit[r] = none ? 0 : limit;
    if (none) s_dead = 1;
  }
  uint32_t q_at[8];
  keys.addresses(base, q_at);
  keys.arrive();
  sync_stage();
  const bool dead = __builtin_amdgcn_readfirstlane(s_dead) != 0;
  while (at < g1) {
    const int key = min(keys.first + (lane & 31), n - 1);
    float* weight = a.weights + s * a.key_rows + key;
    const float before = *weight;
#pragma unroll 1
    for (int t = 0; t < tiles; ++t) {
      const int most = n - 32 * t / g, least = n - min(32 * t + 31, total - 1) / g;
      if (keys.first < most)
        keys.weigh(q_at, t * 32 * kRow, s_lse + 32 * t, s_limit + 32 * t, least, dead, a.scale);
    }
    keys.each_sum(n, [&](int, float y) { *weight = before + y; });
    at += kFewWaves;
    if (at < g1) keys.load(a.keys, s * a.key_rows, at * kTile, n);
  }
}

// The parts' sums, four keys a thread.
__global__ __launch_bounds__(256)
void add_weights_kernel(const WeightArgs a, int blocks_per_slice) {
  const int64_t s = blockIdx.x / blocks_per_slice;
  const int i = (int)(blockIdx.x % blocks_per_slice) * 256 + threadIdx.x;
  if (i >= length_of(a.n_keys, s, a.key_rows)) return;
  float y = 0.f;
#pragma unroll 4
  for (int c = 0; c < a.splits; ++c) y += a.part[((int64_t)c * a.n_slices + s) * a.key_rows + i];
  a.weights[s * a.key_rows + i] += y;
}

// How a call is cut: two key tiles a wave where a block has many stages of queries, and the
// queries in parts until there are two rounds of blocks, the longer ones first (a block's first
// keys are seen by the most queries).
// Few queries stay in LDS, and the keys are cut instead (split of the keys).
struct WeightCut { int key_tiles, splits; int64_t key_blocks; bool few; };
WeightCut weight_cut(int64_t n_slices, int group_size, int n_q, int64_t key_rows, int dtype) {
  WeightCut c{};
  const int64_t rows = (int64_t)group_size * n_q;
  if (rows <= (dtype == LOUISKV_BF16 ? kFewQueries<uint16_t> : kFewQueries<float>)) {
    c.few = true;
    c.key_tiles = 1;
    c.key_blocks = 1;
    const int64_t groups = (key_rows + kTile - 1) / kTile;
    c.splits = (int)std::max<int64_t>(1, std::min((groups + kFewWaves - 1) / kFewWaves, 512 / n_slices));
    return c;
  }
  const int64_t stages = ((int64_t)group_size * n_q + kQueries - 1) / kQueries;
  c.key_tiles = dtype == LOUISKV_BF16 && stages >= 32 ? 2 : 1;
  c.key_blocks = (key_rows + block_keys(c.key_tiles) - 1) / block_keys(c.key_tiles);
  const int64_t blocks = std::max<int64_t>(1, n_slices * c.key_blocks);
  c.splits = (int)std::max<int64_t>(1, std::min({(1536 + blocks - 1) / blocks, stages / 4, (int64_t)16}));
  return c;
}

size_t weight_bytes(int64_t n_slices, int group_size, int n_q, int64_t key_rows) {
  auto splits = [&](int dtype) {
    const WeightCut c = weight_cut(n_slices, group_size, n_q, key_rows, dtype);
    return c.few ? 1 : c.splits;
  };
  const int most = std::max(splits(LOUISKV_BF16), splits(LOUISKV_F32));
  return most > 1 ? align_up((size_t)most * n_slices * key_rows * sizeof(float), 256) : 0;
}

// Whether the launches of launch_weights fit (of 256 threads a block, twice kMaxGrid do; the blocks of
// 512 are a slice's, and a few more).
bool weights_fit(int64_t n_slices, int group_size, int n_q, int64_t key_rows, int dtype) {
  const WeightCut c = weight_cut(n_slices, group_size, n_q, key_rows, dtype);
  return n_slices * c.key_blocks * c.splits <= 2 * kMaxGrid && (c.few || n_slices * ((key_rows + 255) / 256) <= 2 * kMaxGrid);
}

// Logits and lse are brought to base 2 by one factor, scale * log2(e) rounded once, so that its
// rounding is relative to their difference, which decides, and not to their size.
int launch_weights(WeightArgs a, float scale, int dtype, void* workspace, hipStream_t hs) {
  a.scale = scale * kLog2E;
  a.per_lse = a.scale != 0.f ? (double)a.scale / (double)scale : 1.4426950408889634;
  const WeightCut c = weight_cut(a.n_slices, a.group_size, a.n_q, a.key_rows, dtype);
  a.splits = c.splits;
  a.part = static_cast<float*>(workspace);
  const int64_t grid = a.n_slices * c.key_blocks * c.splits;
  if (c.few) {
    if (dtype == LOUISKV_BF16) weights_few_kernel<uint16_t><<<(unsigned)grid, kFewWaves * 64, 0, hs>>>(a);
    else weights_few_kernel<float><<<(unsigned)grid, kFewWaves * 64, 0, hs>>>(a);
    LKV_CHECK_LAUNCH();
    return LOUISKV_OK;
  }
  if (dtype == LOUISKV_F32) weights_kernel<float, 1><<<(unsigned)grid, kBlockWaves * 64, 0, hs>>>(a);
  else if (c.key_tiles == 1) weights_kernel<uint16_t, 1><<<(unsigned)grid, kBlockWaves * 64, 0, hs>>>(a);
  else weights_kernel<uint16_t, 2><<<(unsigned)grid, kBlockWaves * 64, 0, hs>>>(a);
  LKV_CHECK_LAUNCH();
  if (a.splits == 1) return LOUISKV_OK;
  const int per = (a.key_rows + 255) / 256;
  add_weights_kernel<<<(unsigned)(a.n_slices * per), 256, 0, hs>>>(a, per);
  LKV_CHECK_LAUNCH();
  return LOUISKV_OK;
}

// Results of queries cut into parts, and weights of own rows from the logits that the
// attention left.
struct FinishArgs {
  const float* part;
  int n_parts;
  int64_t n_rows;
  void* out;
  float* lse_out;
  int64_t merge_blocks;
  int wide;                       // a block a query
  const float* logits;
  int logit_stride, per_slice;    // queries of a slice, at most 32
  const int32_t* n_own;
  int own_rows, chunks;           // blocks of a slice's rows
  float* weights;
};
constexpr int kFinishKeys = 1024;   // of a block, four a thread
constexpr int64_t kWideRows = 1024; // queries that a block each fills the chip with

// merge_blocks blocks of four queries, a wave each, or (wide) of one, whose parts the waves
// share; then `chunks` of each slice's rows.
template <class TO>
__global__ __launch_bounds__(256)
void finish_kernel(const FinishArgs a) {
  __shared__ float s_lse[32], s_o[4][kHeadDim], s_m[4], s_l[4];
  int64_t id = blockIdx.x;
  const int w = threadIdx.x >> 6;
  if (id < a.merge_blocks && !a.wide) {
    const int64_t row = id * 4 + w;
    if (row < a.n_rows) merge_row(a.part, a.n_parts, row, static_cast<TO*>(a.out), a.lse_out);
    return;
  }
  if (id < a.merge_blocks) {
    const int c0 = a.n_parts * w / 4, c1 = a.n_parts * (w + 1) / 4, tid = threadIdx.x;
    float m, l, o0, o1;
    join_parts(a.part + (id * a.n_parts + c0) * kPartFloats, c1 - c0, m, l, o0, o1);
    *reinterpret_cast<float2*>(&s_o[w][2 * (tid & 63)]) = make_float2(o0, o1);
    s_m[w] = m;
    s_l[w] = l;
    __syncthreads();
    if (tid >= kHeadDim) return;
    m = fmaxf(fmaxf(s_m[0], s_m[1]), fmaxf(s_m[2], s_m[3]));
    l = 0.f;
    float o = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float e = __builtin_amdgcn_exp2f(s_m[i] - max_base(m));
      l += s_l[i] * e;
      o += s_o[i][tid] * e;
    }
    store_from_f32(static_cast<TO*>(a.out) + id * kHeadDim, tid, o * inv_sum(l));
    if (a.lse_out && tid == 0) a.lse_out[id] = lse_of(m, l);
    return;
  }
  id -= a.merge_blocks;
  const int64_t s = id / a.chunks;
  const int i = (int)(id - s * a.chunks) * kFinishKeys + 4 * threadIdx.x;
  const int n = length_of(a.n_own, s, a.own_rows), r = threadIdx.x >> 3, j = threadIdx.x & 7;
  // eight threads a query: its base-2 lse, infinite where it sees nothing
  if (r < a.per_slice) {
    float m = -__builtin_inff(), l = 0.f;
    const float* p = a.part + (s * a.per_slice + r) * a.n_parts * kPartFloats;
    for (int c = j; c < a.n_parts; c += 8) {
      const float2 ml = *reinterpret_cast<const float2*>(p + (size_t)c * kPartFloats);
      const float mm = fmaxf(m, ml.x);
      l = l * __builtin_amdgcn_exp2f(m - max_base(mm)) + ml.y * __builtin_amdgcn_exp2f(ml.x - max_base(mm));
      m = mm;
    }
    for (int o = 1; o < 8; o <<= 1) {
      const float m1 = __shfl_xor(m, o, kWave), l1 = __shfl_xor(l, o, kWave), mm = fmaxf(m, m1);
      l = l * __builtin_amdgcn_exp2f(m - max_base(mm)) + l1 * __builtin_amdgcn_exp2f(m1 - max_base(mm));
      m = mm;
    }
    if (j == 0) s_lse[r] = l == 0.f ? __builtin_inff() : max_base(m) + log2f(l);
  }
  __syncthreads();
  if (i < n)
    add_weights(a.logits + s * a.per_slice * a.logit_stride, a.logit_stride, a.per_slice, s_lse, n, i,
                a.weights + s * a.own_rows);
}

int check_types(int dtype, int out_dtype) {
  for (int t : {dtype, out_dtype})
    if (t != LOUISKV_F32 && t != LOUISKV_BF16) return fail(LOUISKV_ERR_DTYPE, "unknown dtype %d", t);
  return LOUISKV_OK;
}

// Sizes that both calls share.
int check_sizes(int64_t n_slices, int32_t n_kv_heads, int32_t group_size, int32_t n_q, int32_t d, int64_t rows) {
  if (d != kHeadDim) return fail(LOUISKV_ERR_UNSUPPORTED, "head dim %d not supported (only 128)", d);
  if (n_kv_heads < 1 || n_slices < 1 || n_slices % n_kv_heads != 0)
    return fail(LOUISKV_ERR_SHAPE, "n_slices=%lld must be a positive multiple of n_kv_heads=%d", (long long)n_slices,
                n_kv_heads);
  if (group_size < 1 || group_size > 8) return fail(LOUISKV_ERR_UNSUPPORTED, "group_size=%d must be 1 to 8", group_size);
  if (n_q < 1 || rows < 0 || rows > kMaxRows)
    return fail(LOUISKV_ERR_SHAPE, "n_q=%d must be positive, rows=%lld at most %lld", n_q, (long long)rows,
                (long long)kMaxRows);
  if (n_slices > kMaxGrid || n_slices * group_size > kMaxQueries / n_q)
    return fail(LOUISKV_ERR_SHAPE, "%lld slices of %d heads and n_q=%d are too many queries for one call",
                (long long)n_slices, group_size, n_q);
  return LOUISKV_OK;
}

bool served(int64_t n_slices, int32_t group_size, int32_t n_q, int64_t rows) {
  return n_slices >= 1 && n_slices <= kMaxGrid && group_size >= 1 && group_size <= 8 && n_q >= 1 && rows >= 0 &&
         rows <= kMaxRows && n_slices * group_size <= kMaxQueries / n_q;
}

// Own rows' weights take the logits that the attention leaves where a slice has up to 32
// queries (8 bytes a row and query, written and read, against its key read again), and the
// keys anew where it has more.
int logit_stride(int64_t own_rows) { return (int)align_up((size_t)own_rows, kTile); }
bool keeps_logits(int group_size, int n_q) { return (int64_t)group_size * n_q <= 32; }
size_t weight_space(int64_t n_slices, int group_size, int n_q, int64_t own_rows) {
  const size_t rows = (size_t)n_slices * group_size * n_q;
  return align_up(rows * sizeof(float), 256) +
         (keeps_logits(group_size, n_q) ? align_up(rows * logit_stride(own_rows) * sizeof(float), 256) : weight_bytes(n_slices, group_size, n_q, own_rows));
}

size_t attn_bytes(int64_t n_slices, int64_t n_prefix_slices, int group_size, int n_q, int64_t prefix_rows, int64_t own_rows,
                  bool with_weights) {
  auto parts = [&](int dtype) { return cut_of(n_slices, n_prefix_slices, group_size, n_q, prefix_rows, own_rows, dtype).n_parts(); };
  return part_bytes(n_slices * group_size * n_q, std::max(parts(LOUISKV_BF16), parts(LOUISKV_F32))) +
         (with_weights ? weight_space(n_slices, group_size, n_q, own_rows) : 0);
}

// Whether the attention's launches fit (blocks of 256 threads).
bool attn_fits(const Cut& c, int64_t n_slices, int group_size, int n_q, int64_t own_rows, bool with_weights, int dtype) {
  if (c.blocks_p + c.blocks_o > 2 * kMaxGrid) return false;
  if (!with_weights || own_rows == 0) return true;
  if (!keeps_logits(group_size, n_q)) return weights_fit(n_slices, group_size, n_q, own_rows, dtype);
  return (n_slices * group_size * n_q + 3) / 4 + n_slices * ((own_rows + kFinishKeys - 1) / kFinishKeys) <= 2 * kMaxGrid;
}

// Neither a prefix nor own rows: every query sees nothing.
__global__ void no_rows_kernel(void* out, int out_bf16, float* lse_out, int64_t n_rows) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;   // four channels
  if (i >= n_rows * (kHeadDim / 4)) return;
  if (out_bf16) static_cast<uint2*>(out)[i] = make_uint2(0, 0);
  else static_cast<uint4*>(out)[i] = make_uint4(0, 0, 0, 0);
  if (lse_out && i % (kHeadDim / 4) == 0) lse_out[i / (kHeadDim / 4)] = -__builtin_inff();
}

int no_rows(const AttnArgs& a, int64_t n_rows, hipStream_t hs) {
  no_rows_kernel<<<(unsigned)((n_rows * (kHeadDim / 4) + 255) / 256), 256, 0, hs>>>(a.out, a.out_bf16, a.lse_out, n_rows);
  LKV_CHECK_LAUNCH();
  return LOUISKV_OK;
}

}  // namespace
}  // namespace louiskv

using namespace louiskv;

extern "C" size_t louiskv_shared_prefix_attn_workspace_size(int64_t n_slices, int64_t n_prefix_slices,
                                                            int32_t group_size, int32_t n_q, int32_t d,
                                                            int64_t prefix_rows, int64_t own_rows,
                                                            int32_t with_weights) {
  (void)d;
  if (!served(n_slices, group_size, n_q, own_rows) || prefix_rows < 0 || prefix_rows > kMaxRows ||
      (prefix_rows > 0 && (n_prefix_slices < 1 || n_slices % n_prefix_slices != 0)))
    return 0;
  auto fits = [&](int dtype) {
    return attn_fits(cut_of(n_slices, n_prefix_slices, group_size, n_q, prefix_rows, own_rows, dtype), n_slices, group_size, n_q,
                     own_rows, with_weights, dtype);
  };
  if (!fits(LOUISKV_BF16) && !fits(LOUISKV_F32)) return 0;
  return attn_bytes(n_slices, n_prefix_slices, group_size, n_q, prefix_rows, own_rows, with_weights);
}

extern "C" int louiskv_shared_prefix_attn(const void* q, int32_t dtype, int64_t n_slices, int32_t n_kv_heads,
                                          int32_t group_size, int32_t n_q, int32_t d, float scale,
                                          const void* k_prefix, const void* v_prefix, int64_t n_prefix_slices,
                                          int64_t prefix_rows, const int32_t* n_prefix, const void* k_own,
                                          const void* v_own, int64_t own_rows, const int32_t* n_own, float* weights,
                                          void* out, int32_t out_dtype, float* lse_out, void* workspace,
                                          size_t workspace_bytes, void* stream) {
  if (!q || !out || (prefix_rows > 0 && (!k_prefix || !v_prefix)) || (own_rows > 0 && (!k_own || !v_own)))
    return fail(LOUISKV_ERR_NULL, "q, out, and the keys and values of the prefix and the own rows are required");
  int st = check_types(dtype, out_dtype);
  if (st || (st = check_sizes(n_slices, n_kv_heads, group_size, n_q, d, own_rows))) return st;
  if (prefix_rows < 0 || prefix_rows > kMaxRows)
    return fail(LOUISKV_ERR_SHAPE, "prefix_rows=%lld must be in [0, %lld]", (long long)prefix_rows, (long long)kMaxRows);
  if (prefix_rows > 0 && (n_prefix_slices < 1 || n_slices % n_prefix_slices != 0 || n_prefix_slices % n_kv_heads != 0))
    return fail(LOUISKV_ERR_SHAPE, "n_prefix_slices=%lld must be a multiple of n_kv_heads=%d and divide n_slices=%lld",
                (long long)n_prefix_slices, n_kv_heads, (long long)n_slices);
  if (!aligned16(q, out, k_prefix, v_prefix, k_own, v_own))
    return fail(LOUISKV_ERR_UNSUPPORTED, "q, out, keys and values must be 16-byte aligned");
  const size_t need = attn_bytes(n_slices, n_prefix_slices, group_size, n_q, prefix_rows, own_rows, weights != nullptr);
  if ((st = check_workspace(workspace, workspace_bytes, need))) return st;
  const Cut c = cut_of(n_slices, n_prefix_slices, group_size, n_q, prefix_rows, own_rows, dtype);
  const int64_t n_rows = n_slices * group_size * n_q, chunks = (own_rows + kFinishKeys - 1) / kFinishKeys;
  const bool with_logits = weights && own_rows > 0 && keeps_logits(group_size, n_q);
  if (!attn_fits(c, n_slices, group_size, n_q, own_rows, weights != nullptr, dtype))
    return fail(LOUISKV_ERR_SHAPE, "problem too large for one launch");
  const size_t parts = part_bytes(n_rows, c.n_parts());
  AttnArgs a{};
  a.q = q; a.group_size = group_size; a.n_q = n_q; a.scale = scale;
  a.n_prefix_slices = prefix_rows ? n_prefix_slices : n_slices;
  a.n_seqs = (int)(n_slices / a.n_prefix_slices);
  a.prefix = {k_prefix, v_prefix, n_prefix, (int)prefix_rows, c.groups_p, c.splits_p};
  a.own = {k_own, v_own, n_own, (int)own_rows, c.groups_o, c.splits_o};
  a.prefix_blocks = c.blocks_p; a.n_parts = c.n_parts(); a.part = static_cast<float*>(workspace);
  a.stream = (a.n_prefix_slices * prefix_rows + n_slices * own_rows) * 2 * kHeadDim * (dtype == LOUISKV_BF16 ? 2 : 4) > kCacheBytes;
  a.out = out; a.out_bf16 = out_dtype == LOUISKV_BF16;
  a.lse_out = lse_out ? lse_out : weights ? reinterpret_cast<float*>(static_cast<char*>(workspace) + parts) : nullptr;
  hipStream_t hs = as_stream(stream);
  if (a.n_parts == 0) return no_rows(a, n_rows, hs);
  char* rest = static_cast<char*>(workspace) + parts + align_up((size_t)n_rows * sizeof(float), 256);
  if (with_logits) {
    a.logits = reinterpret_cast<float*>(rest);
    a.logit_stride = logit_stride(own_rows);
    a.weights = weights;
  }
  if (dtype == LOUISKV_BF16) launch_attn<uint16_t>(a, c, hs);
  else launch_attn<float>(a, c, hs);
  LKV_CHECK_LAUNCH();
  if (a.n_parts > 1) {
    FinishArgs f{};
    f.part = a.part; f.n_parts = a.n_parts; f.n_rows = n_rows; f.out = out; f.lse_out = a.lse_out;
    f.wide = a.n_parts >= 16 && n_rows <= kWideRows;
    f.merge_blocks = f.wide ? n_rows : (n_rows + 3) / 4;
    if (with_logits) {
      f.logits = a.logits; f.logit_stride = a.logit_stride; f.per_slice = group_size * n_q; f.n_own = n_own;
      f.own_rows = (int)own_rows; f.chunks = (int)chunks; f.weights = weights;
    }
    const int64_t grid = f.merge_blocks + n_slices * f.chunks;
    if (a.out_bf16) finish_kernel<uint16_t><<<(unsigned)grid, 256, 0, hs>>>(f);
    else finish_kernel<float><<<(unsigned)grid, 256, 0, hs>>>(f);
    LKV_CHECK_LAUNCH();
  }
  if (with_logits) return LOUISKV_OK;
  if (!weights || own_rows == 0) return LOUISKV_OK;
  WeightArgs wa{};
  wa.q = q; wa.group_size = group_size; wa.n_q = n_q; wa.keys = k_own; wa.key_rows = (int)own_rows;
  wa.n_keys = n_own; wa.lse = a.lse_out; wa.weights = weights; wa.n_slices = n_slices;
  return launch_weights(wa, scale, dtype, rest, hs);
}

extern "C" size_t louiskv_attn_weights_workspace_size(int64_t n_slices, int32_t group_size, int32_t n_q, int32_t d,
                                                      int64_t key_rows) {
  (void)d;
  auto fits = [&](int dtype) { return weights_fit(n_slices, group_size, n_q, key_rows, dtype); };
  return served(n_slices, group_size, n_q, key_rows) && (fits(LOUISKV_BF16) || fits(LOUISKV_F32))
             ? weight_bytes(n_slices, group_size, n_q, key_rows) : 0;
}

extern "C" int louiskv_attn_weights(const void* q, int32_t dtype, int64_t n_slices, int32_t n_kv_heads,
                                    int32_t group_size, int32_t n_q, int32_t d, float scale, const void* keys,
                                    int64_t key_rows, const int32_t* n_keys, const float* lse, float* weights,
                                    void* workspace, size_t workspace_bytes, void* stream) {
  if (!q || !keys || !lse || !weights) return fail(LOUISKV_ERR_NULL, "q, keys, lse and weights are required");
  int st = check_types(dtype, dtype);
  if (st || (st = check_sizes(n_slices, n_kv_heads, group_size, n_q, d, key_rows))) return st;
  if (key_rows < 1) return fail(LOUISKV_ERR_SHAPE, "key_rows=%lld must be positive", (long long)key_rows);
  if (!aligned16(q, keys)) return fail(LOUISKV_ERR_UNSUPPORTED, "q and keys must be 16-byte aligned");
  if (!weights_fit(n_slices, group_size, n_q, key_rows, dtype)) return fail(LOUISKV_ERR_SHAPE, "problem too large for one launch");
  const size_t need = weight_bytes(n_slices, group_size, n_q, key_rows);
  if ((st = check_workspace(workspace, workspace_bytes, need))) return st;
  WeightArgs a{};
  a.q = q; a.group_size = group_size; a.n_q = n_q; a.keys = keys; a.key_rows = (int)key_rows;
  a.n_keys = n_keys; a.lse = lse; a.weights = weights; a.n_slices = n_slices;
  return launch_weights(a, scale, dtype, workspace, as_stream(stream));
}
