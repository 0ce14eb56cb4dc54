// The prompt's attention over selected blocks of its keys: the selection of each
// query tile's blocks by their index vectors, and the causal attention over them.
#include <type_traits>

#include "common.h"
#include "merge.h"

namespace louiskv {
namespace {

constexpr int kMaxBlocks = 8192;    // key blocks a tile's selection ranks
constexpr int kMaxTile = 128;       // queries of a tile
constexpr int kMaxKeys = 1 << 30;   // of a sequence, and of a list

// ------------------------------------------------------------------ selection

struct SelectArgs {
  const void* q;
  int group_size, n_q;
  const float* reps;
  int units_cap, n_keys, q_start, q_block, log_block, n_first, n_recent, n_top;
  int32_t* sel;
  int sel_cap;
  int32_t* n_sel;
  int n_tiles;
};

// A float64 as an unsigned integer of the same order; NaN below every number, -0
// as 0.
__device__ __forceinline__ uint64_t ordered(double x) {
  if (x != x) return 0;
  const uint64_t u = (uint64_t)__double_as_longlong(x + 0.0);
  return (u >> 63) ? ~u : u | (1ull << 63);
}

// Eight channels of a query as they are stored.
template <class T> struct Eight;
template <> struct Eight<uint16_t> {
  uint4 v;
  __device__ __forceinline__ void load(const uint16_t* p) { v = *reinterpret_cast<const uint4*>(p); }
  __device__ __forceinline__ float at(int e) const {
    const uint32_t w = (&v.x)[e >> 1];
    return __uint_as_float(e & 1 ? w & 0xffff0000u : w << 16);
  }
};
template <> struct Eight<float> {
  float4 v[2];
  __device__ __forceinline__ void load(const float* p) {
    v[0] = reinterpret_cast<const float4*>(p)[0];
    v[1] = reinterpret_cast<const float4*>(p)[1];
  }
  __device__ __forceinline__ float at(int e) const { return (&v[e >> 2].x)[e & 3]; }
};

constexpr int kSelThreads = 256;
constexpr int kSelWaves = kSelThreads / 64;

// Block (slice, tile): the sum of the tile's queries in float64 (16 lanes a row, the
// waves share the rows), the scores of the ranked blocks (four lanes a block, each
// with 32 of the sum's channels in registers), then the first wave finds the
// n_top-th largest key by radix selection (8 bits a pass, only the keys that share
// the digits found so far are counted) and writes the list in block order.  Bound
// by the read of the queries where there are many tiles (a layer of 32K tokens:
// 68 us, 4.0 TB/s; four tiles to a block, whose index vectors pass through LDS once
// for all of them, 123 us: the phases of fewer waves overlap less) and by trips
// to memory where there are few.
template <class T>
__global__ __launch_bounds__(kSelThreads)
void select_blocks_kernel(const SelectArgs a) {
  extern __shared__ uint64_t s_key[];            // one per ranked block
  __shared__ double s_q[kSelWaves][kHeadDim];
  __shared__ int s_hist[256];
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  const int64_t s = blockIdx.x / a.n_tiles;
  const int t = (int)(blockIdx.x - s * a.n_tiles);
  const int i0 = t * a.q_block, n_tok = min(a.q_block, a.n_q - i0);
  // blocks [first, lo) are ranked; those before and lo..hi are taken
  const int hi = (a.q_start + i0 + n_tok - 1) >> a.log_block;
  const int lo = max(0, ((a.q_start + i0) >> a.log_block) - a.n_recent), first = min(a.n_first, lo);
  const int ranked = lo - first, n_pick = min(a.n_top, ranked);
  if (n_pick > 0 && n_pick < ranked) {           // block-uniform
    {
      const int sub = lane & 15, n_rows = n_tok * a.group_size;
      const T* q = static_cast<const T*>(a.q) + ((size_t)s * a.group_size * a.n_q + i0) * kHeadDim + 8 * sub;
      constexpr int kFlight = sizeof(T) == 2 ? 16 : 8, kGroups = 4 * kSelWaves;   // rows in flight of a 16-lane group
      double sum[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) sum[e] = 0.0;
      const int r0 = w * 4 + (lane >> 4);
      int head = 0, tok = r0;                    // of row r: r = head * n_tok + tok
      for (int r = r0; r < n_rows; r += kGroups * kFlight) {
        Eight<T> v[kFlight];
#pragma unroll
        for (int i = 0; i < kFlight; ++i) {
          if (r + kGroups * i < n_rows) {
            while (tok >= n_tok) {
              tok -= n_tok;
              ++head;
            }
            v[i].load(q + ((size_t)head * a.n_q + tok) * kHeadDim);
          }
          tok += kGroups;
        }
#pragma unroll
        for (int i = 0; i < kFlight; ++i)
          if (r + kGroups * i < n_rows) {
#pragma unroll
            for (int e = 0; e < 8; ++e) sum[e] += (double)v[i].at(e);
          }
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        double y = sum[e] + __shfl_xor(sum[e], 16, kWave);
        y += __shfl_xor(y, 32, kWave);
        if (lane < 16) s_q[w][8 * sub + e] = y;
      }
    }
    __syncthreads();
    // lane j of a quad: channels 16 k + 4 j + 0..3
    double sum[8][4];
    const int j = lane & 3;
#pragma unroll
    for (int k = 0; k < 8; ++k)
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        double y = 0.0;
#pragma unroll
        for (int p = 0; p < kSelWaves; ++p) y += s_q[p][16 * k + 4 * j + c];
        sum[k][c] = y;
      }
    const float* reps = a.reps + (size_t)s * a.units_cap * kHeadDim + 4 * j;
#pragma unroll 2
    for (int b = first + (tid >> 2); b < lo; b += kSelThreads / 4) {
      float4 v[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = *reinterpret_cast<const float4*>(reps + (size_t)b * kHeadDim + 16 * k);
      double acc = 0.0;
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        acc = fma(sum[k][0], (double)v[k].x, acc);
        acc = fma(sum[k][1], (double)v[k].y, acc);
        acc = fma(sum[k][2], (double)v[k].z, acc);
        acc = fma(sum[k][3], (double)v[k].w, acc);
      }
      acc += __shfl_xor(acc, 1, kWave);
      acc += __shfl_xor(acc, 2, kWave);
      if (j == 0) s_key[b - first] = ordered(acc);
    }
    __syncthreads();
  }
  if (w > 0) return;
  int32_t* sel = a.sel + ((size_t)s * a.n_tiles + t) * a.sel_cap;
  if (lane == 0) a.n_sel[(size_t)s * a.n_tiles + t] = first + n_pick + hi - lo + 1;
  for (int b = lane; b < first; b += kWave) sel[b] = b;
  for (int b = lo + lane; b <= hi; b += kWave) sel[first + n_pick + b - lo] = b;
  if (n_pick == 0) return;
  if (n_pick == ranked) {
    for (int b = lane; b < ranked; b += kWave) sel[first + b] = first + b;
    return;
  }
  uint64_t prefix = 0, mask = 0;
  int need = n_pick;              // still to take among the keys that match the prefix
  for (int shift = 56; shift >= 0; shift -= 8) {
#pragma unroll
    for (int e = 0; e < 4; ++e) s_hist[lane + 64 * e] = 0;
    __builtin_amdgcn_wave_barrier();
    for (int b = lane; b < ranked; b += kWave) {
      const uint64_t k = s_key[b];
      if ((k & mask) == prefix) atomicAdd(&s_hist[(int)((k >> shift) & 255)], 1);
    }
    __builtin_amdgcn_wave_barrier();
    // the digit at which the count from the top reaches `need`
    int c[4], mine = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      c[e] = s_hist[255 - (4 * lane + e)];
      mine += c[e];
    }
    int before = mine;
    for (int o = 1; o < kWave; o <<= 1) {
      const int y = __shfl_up(before, o, kWave);
      if (lane >= o) before += y;
    }
    before -= mine;
    int digit = 0, above = 0, equal = 0;
    bool here = false;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (before < need && before + c[e] >= need) {
        digit = 255 - (4 * lane + e);
        above = before;
        equal = c[e];
        here = true;
      }
      before += c[e];
    }
    const int src = __ffsll((unsigned long long)__ballot(here)) - 1;   // exactly one lane: need <= keys counted
    digit = __shfl(digit, src, kWave);
    need -= __shfl(above, src, kWave);
    prefix |= (uint64_t)digit << shift;
    mask |= 255ull << shift;
    if (__shfl(equal, src, kWave) == need) break;      // every key with this prefix is taken
  }
  // taken: keys above the prefix, and the first `need` that match it
  int taken = 0, equal = 0;
  for (int b0 = 0; b0 < ranked; b0 += kWave) {
    const int b = b0 + lane;
    const uint64_t k = b < ranked ? s_key[b] & mask : 0;
    const bool above = b < ranked && k > prefix, eq = b < ranked && k == prefix;
    const uint64_t abv = __ballot(above), eqs = __ballot(eq), below = (1ull << lane) - 1;
    const int my_above = taken + __popcll(abv & below), my_eq = equal + __popcll(eqs & below);
    if (above || (eq && my_eq < need)) sel[first + my_above + min(my_eq, need)] = first + b;
    taken += __popcll(abv);
    equal += __popcll(eqs);
  }
}

// ------------------------------------------------------------------ attention

struct PrefillArgs {
  const void* q;
  int group_size, n_q;
  float scale;
  const void* keys;
  const void* values;
  int64_t key_rows;
  int n_keys, q_start, q_block, log_block;
  const int32_t* sel;
  int sel_cap;
  const int32_t* n_sel;
  int n_tiles, n_split;
  float* part;
  void* out;
  int out_bf16;
  float* lse_out;
};

// The waves' products are on the matrix cores.

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

// Waits for every copy and LDS access of the wave, then for the block's waves.
__device__ __forceinline__ void sync_stage() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// 64 lanes copy 16 bytes each from base + off (per lane) to LDS lds + 16 * lane.  The
// copy reads M0 one wait state after its write at the earliest.
__device__ __forceinline__ void copy_to_lds(const void* base, uint32_t off, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(off), "s"(base), "s"(lds)
               : "memory", "m0");
}

typedef __attribute__((address_space(3))) char* lds_ptr;
__device__ __forceinline__ uint32_t lds_addr(const void* p) { return (uint32_t)(uintptr_t)(lds_ptr)p; }

// Rows lie in LDS with their 16-byte pieces permuted, piece c of row r at
// c ^ swizzle(r).  Sixteen consecutive rows put a piece in sixteen different places
// (the key reads, a lane a row).  bfloat16, 16 pieces: four consecutive rows put a
// run of four pieces in four different ones (the transposing value reads).
// float32, 32 pieces: rows four apart put a run of eight in different halves of the
// banks (the value reads of the two halves of a wave).
template <class T>
__device__ __forceinline__ int swizzle(int r) {
  if constexpr (sizeof(T) == 2) return ((r & 3) << 2) | ((r >> 2) & 3);
  else return (r & 3) | ((r >> 3) & 1) << 2 | ((r >> 2) & 1) << 3;
}

constexpr float kGrow = 8.0f;   // base-2 logits may pass the base by this much before the sums are rescaled

// Block (slice, tile, row group, split): rows r of the tile are (token r / g, head
// r % g), 32 of them a wave, WR waves of rows by WK waves that share the keys.
// Keys and values of 64 list positions at a time are copied to LDS (two stages,
// one in flight; two in flight were no faster, 1.14 against 1.12 ms for a layer of
// 32K tokens).  A wave computes S^T = K Q^T for 32 keys, so that a lane holds
// 16 scores of one query row; their exponentials are, unmoved, the B operand of
// O^T += V^T P^T, whose A operand comes from LDS through transposing reads.  The
// running base, sum and the rescale are then a lane's own; the sums are rescaled
// only where a score passes the base by 2^8.  The exponentials are rounded to bfloat16
// for that product, 2^-8 of each at most, while their sum takes them unrounded: unlike in
// the decode attention no column of the product is idle, and what the rounding leaves
// would cost a second one, half as many products again (results are off by 2.0e-3 of
// their size; the rounding of a bfloat16 result alone is 1.7e-3 of it).
// float32: the same with 32 positions a stage and products of two channels or keys
// at a time, k index = half of the wave; the weights need no rounding.  The kernels for
// 256 and 128 rows keep 26 and 30 registers in scratch memory; the loop's reloads wait for
// the copies in flight as well (vmcnt counts in order), which undoes the overlap of
// copies and products in part.
//
// A layer of 32K tokens (8 slices x 512 tiles of 256 rows, 30 blocks of 64 keys, 985
// GFLOP): 1.10 to 1.19 ms, 0.89 to 0.83 PFLOP/s, on parts where a large product reaches
// 1.35 and 1.30; in float32 a layer of 8192 tokens 1.92 ms, 117 TFLOP/s of 154.  For each
// 32 rows by 32 keys a wave has 16 products (512 cycles), 16 exponentials and 80 other
// vector operations, and reads 16 KB of LDS.  Two waves of a SIMD alternate between them,
// and overlap in part: where the layer took 1.10 ms, the same instructions without a
// dependency between the pairs took 1.02, the products and LDS reads alone 0.74.  64 rows
// a wave would halve the LDS reads, but its accumulators do not fit beside the rest (copies
// between the register files: 1.60 ms); phases kept apart by barriers 1.35 ms, a maximum
// over 64 keys at a time 1.16, the next 32 keys' scores between the exponentials 1.11 to
// 1.13.
constexpr int kStageBytes = 16384;   // of the keys, and of the values

template <class T, int WR, int WK>
__global__ __launch_bounds__(WR * WK * 64, 2)
void prefill_kernel(const PrefillArgs a, int row_groups, int64_t n_blocks) {
  constexpr int NW = WR * WK;
  constexpr bool kBf16 = sizeof(T) == 2;
  constexpr int kRowBytes = kHeadDim * sizeof(T), kPieces = kRowBytes / 16;
  constexpr int kStageKeys = kStageBytes / kRowBytes, kHalves = kStageKeys / 32;
  constexpr int kCopyRows = 1024 / kRowBytes;             // rows of one copy of 64 x 16 bytes
  constexpr int kCopies = kStageBytes / 1024 / NW;        // copies of a wave, of keys and of values
  static_assert(kStageBytes % (1024 * NW) == 0 && kHalves % WK == 0, "waves share a stage evenly");
  __shared__ __align__(256) char s_ring[2][2 * kStageBytes];
  __shared__ int s_bad;
  const int tid = threadIdx.x, lane = tid & 63, h = lane >> 5, n = lane & 31;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6), wr = w % WR, wk = w / WR;
  // Neighbouring tiles of a slice, which share blocks, go to one XCD (blocks are
  // dealt to the eight in turn).
  int64_t id = blockIdx.x;
  if (n_blocks >= 64) {
    const int64_t per = n_blocks >> 3, rest = n_blocks & 7, x = id & 7;
    id = x * per + min<int64_t>(x, rest) + (id >> 3);
  }
  const int split = (int)(id % a.n_split);
  id /= a.n_split;
  const int rgrp = (int)(id % row_groups);
  id /= row_groups;
  const int64_t s = id / a.n_tiles;
  const int t = (int)(id - s * a.n_tiles);
  const int lg = 31 - __builtin_clz(a.group_size);
  const int i0 = t * a.q_block, n_tok = min(a.q_block, a.n_q - i0), n_rows = n_tok << lg;
  const int row0 = (rgrp * WR + wr) * 32;    // of this wave, in the tile
  if (rgrp * WR * 32 >= n_rows) return;      // the tile is shorter than the others (block-uniform)

  // this lane's row: 16-byte pieces 2 c + h (bfloat16) or 16 h + c (float32)
  constexpr int kQ = kPieces / 2;
  typename std::conditional<kBf16, bf16x8, f32x4>::type q[kQ];
  const float qs = a.scale * kLog2E;
  const uint32_t flip = qs < 0.f ? (kBf16 ? 0x80008000u : 0x80000000u) : 0u;     // |scale| multiplies the scores of -q
  const int r = min(row0 + n, n_rows - 1), qpos = a.q_start + i0 + (r >> lg);
  const size_t row = ((size_t)s * a.group_size + (r & (a.group_size - 1))) * a.n_q + i0 + (r >> lg);
  const uint4* src = reinterpret_cast<const uint4*>(static_cast<const T*>(a.q) + row * kHeadDim);
#pragma unroll
  for (int c = 0; c < kQ; ++c) {
    uint4 v = src[kBf16 ? 2 * c + h : 16 * h + c];
    v.x ^= flip; v.y ^= flip; v.z ^= flip; v.w ^= flip;
    q[c] = __builtin_bit_cast(typename std::remove_reference<decltype(q[c])>::type, v);
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");       // the queries are in before the copies start
#pragma unroll
  for (int c = 0; c < kQ; ++c) asm volatile("" : "+v"(q[c]));
  const float mult = fabsf(qs);
  const int first_pos = a.q_start + i0 + (min(row0, n_rows - 1) >> lg);
  const int last_pos = a.q_start + i0 + (min(row0 + 31, n_rows - 1) >> lg);
  const int block_first = a.q_start + i0 + ((rgrp * WR * 32) >> lg);   // first token of the block

  const int64_t list = s * a.n_tiles + t;
  const int32_t* sel = a.sel + (size_t)list * a.sel_cap;
  const int n_list = max(0, min(a.n_sel[list], a.sel_cap));
  const int e0 = (int)((int64_t)n_list * split / a.n_split), e1 = (int)((int64_t)n_list * (split + 1) / a.n_split);
  const int last_block = (a.n_keys - 1) >> a.log_block;
  const int n_groups = (e1 - e0) << (a.log_block - 4);           // of 16 keys
  const int n_stages = (n_groups + kStageKeys / 16 - 1) / (kStageKeys / 16);
  // Entries e0 + 64 c + lane of the list, and the next 64.
  int cur = 0, nxt = 0, cur_base = 0;
  auto entries = [&](int at) { return min(max(sel[min(e0 + at + lane, max(e1 - 1, 0))], 0), last_block); };
  if (n_list > 0 && e1 > e0) {
    cur = entries(0);
    nxt = entries(64);
  }
  asm volatile("s_waitcnt vmcnt(0)" : "+v"(cur), "+v"(nxt));
  // token of the first key of 16-key group gi (below n_groups)
  auto group_pos = [&](int gi) -> int {
    const int e = (gi >> (a.log_block - 4)) - cur_base;
    const int v = __builtin_amdgcn_readlane(e < 64 ? cur : nxt, e & 63);
    return (v << a.log_block) + ((gi & ((1 << (a.log_block - 4)) - 1)) << 4);
  };
  struct StagePos { int at[kStageKeys / 16]; };   // of a stage's groups; no token where the list has ended
  constexpr int kNoToken = INT32_MAX - 16;
  auto stage_pos = [&](int st) {
    StagePos p;
#pragma unroll
    for (int x = 0; x < kStageKeys / 16; ++x) {
      const int gi = st * (kStageKeys / 16) + x;
      p.at[x] = gi < n_groups ? group_pos(gi) : kNoToken;
    }
    return p;
  };
  const char* kb = static_cast<const char*>(a.keys) + (size_t)s * a.key_rows * kRowBytes;
  const char* vb = static_cast<const char*>(a.values) + (size_t)s * a.key_rows * kRowBytes;
  // a wave's share of stage st to LDS; a group past the list repeats its last
  auto copy_stage = [&](int st, char* buf) {
    constexpr int kOfGroup = 16 / kCopyRows, kPer = kCopies < kOfGroup ? kCopies : kOfGroup;   // copies of a 16-row group
#pragma unroll
    for (int x = 0; x < kCopies / kPer; ++x) {
      const int c0 = w * kCopies + x * kPer, g16 = c0 / kOfGroup;
      const int pos = group_pos(min(st * (kStageKeys / 16) + g16, n_groups - 1));
      const int from = min(pos, a.n_keys - 1);                          // rows behind the last key repeat it
      const char* kg = kb + (size_t)from * kRowBytes;
      const char* vg = vb + (size_t)from * kRowBytes;
      const uint32_t dst = __builtin_amdgcn_readfirstlane(lds_addr(buf) + c0 * 1024);
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        const int r16 = (c0 % kOfGroup + i) * kCopyRows + lane / kPieces;   // row of the group
        const int r = min(r16, a.n_keys - 1 - from);
        const uint32_t off = r * kRowBytes + (((lane % kPieces) ^ swizzle<T>(r16)) << 4);
        copy_to_lds(kg, off, dst + i * 1024);
        copy_to_lds(vg, off, dst + kStageBytes + i * 1024);
      }
    }
  };

  f32x16 o[4];
  float base = 0.f, grow_at = -__builtin_inff(), sum = 0.f;
#pragma unroll
  for (int dt = 0; dt < 4; ++dt)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[dt][i] = 0.f;
  // LDS addresses of this lane's reads in 32 keys of a stage.  bfloat16: pieces
  // 2 c + h of key n, and of the values rows 4 h + 0..3 and, in the second, those + 8
  // (the same swizzle but for bit 1) of channels 32 dt + 0..31.  float32: pieces
  // 16 h + c of key n, and channel n % 4 of piece n / 4 (+ 8 dt) of rows 4 h + i.
  uint32_t k_at[8], v_at[4][2];
  {
    const uint32_t k0 = lds_addr(s_ring) + n * kRowBytes, v0 = lds_addr(s_ring) + kStageBytes;
    if constexpr (kBf16) {
      const uint32_t kp = (h ^ swizzle<T>(n & 15)) << 4;
      const int j4 = (lane & 15) >> 2, xp = (((lane >> 4) & 1) << 1) | ((lane & 3) >> 1);
      const uint32_t v1 = v0 + (4 * h + j4) * kRowBytes + ((lane & 1) << 3), vp = ((j4 << 2) | (xp ^ h)) << 4;
#pragma unroll
      for (int c = 0; c < 8; ++c) k_at[c] = k0 + (kp ^ (c << 5));
#pragma unroll
      for (int dt = 0; dt < 4; ++dt) {
        v_at[dt][0] = v1 + (vp ^ (dt << 6));
        v_at[dt][1] = v1 + 8 * kRowBytes + (vp ^ (dt << 6) ^ 32);
      }
    } else {
#pragma unroll
      for (int c = 0; c < 8; ++c) k_at[c] = k0 + h * 256 + ((c ^ swizzle<T>(n & 15)) << 4);    // and ^ 128 for c + 8
      // row (i & 3) + 8 (i >> 2) + 4 h: its swizzle is (i & 3) | (i >> 2 & 1) << 2 | h << 3
#pragma unroll
      for (int dt = 0; dt < 4; ++dt)
        v_at[dt][0] = v0 + 4 * h * kRowBytes + (((8 * dt + (n >> 2)) ^ (h << 3)) << 4) + ((n & 3) << 2);
    }
  }
  typedef const __attribute__((address_space(3))) bf16x8* lds_bf16x8;
  typedef const __attribute__((address_space(3))) f32x4* lds_f32x4;
  typedef const __attribute__((address_space(3))) float* lds_f32;
  typedef __attribute__((address_space(3))) s16x4* lds_s16x4;
  // Keys 32 sub .. + 31 of the stage `off` bytes into the ring, and their values
  // (float32: read where they are used).
  typedef typename std::conditional<kBf16, bf16x8[8], int>::type Keys;
  typedef typename std::conditional<kBf16, s16x8[2][4], int>::type Values;
  typedef typename std::conditional<kBf16, bf16x8[2], f32x16>::type Weights;
  auto load_keys = [&](uint32_t off, int sub, Keys& kf) {
    if constexpr (kBf16) {
#pragma unroll
      for (int c = 0; c < 8; ++c) kf[c] = *(lds_bf16x8)(uintptr_t)(k_at[c] + off + sub * 32 * kRowBytes);
    }
  };
  auto load_values = [&](uint32_t off, int sub, Values& vf) {
    if constexpr (kBf16) {
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int dt = 0; dt < 4; ++dt) {
          const uint32_t at = off + (sub * 32 + 16 * k) * kRowBytes;
          const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(uintptr_t)(v_at[dt][0] + at));
          const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(uintptr_t)(v_at[dt][1] + at));
          vf[k][dt] = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        }
    }
  };
  auto scores = [&](uint32_t off, const Keys& kf) {
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
  };
  // Masks scores of keys from tokens p0 and p1 on (16 each).
  auto mask = [&](f32x16& sc, int p0, int p1) {
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int key = (i < 8 ? p0 : p1) + (i & 3) + 8 * ((i >> 2) & 1) + 4 * h;
      sc[i] = key <= qpos ? sc[i] * mult : -__builtin_inff();
    }
  };
  auto largest = [&](const f32x16& sc) {
    float top = sc[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) top = fmaxf(top, sc[i]);
    return top;
  };
  // Raises the base where a lane's scores pass it.
  auto rebase = [&](float top) {
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
  };
  auto weights = [&](const f32x16& sc, float m, Weights& pb) {
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const float p = __builtin_amdgcn_exp2f(fmaf(sc[i], m, -base));
      sum += p;
      if constexpr (kBf16) pb[i >> 3][i & 7] = (__bf16)p;
      else pb[i] = p;
    }
  };
  auto add_values = [&](uint32_t off, const Values& vf, const Weights& pb) {
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
          const uint32_t at = v_at[dt][0] + ((i & 3) + 8 * (i >> 2)) * kRowBytes;
          const float v = *(lds_f32)(uintptr_t)((at ^ (((i & 3) | ((i >> 2) & 1) << 2) << 4)) + off);
          o[dt] = __builtin_amdgcn_mfma_f32_32x32x2f32(v, pb[i], o[dt], 0, 0, 0);
        }
    }
  };
  auto soften = [&](f32x16& sc, int p0, int p1, Weights& pb) {
    float m = mult;
    if (max(p0, p1) + 15 > first_pos) {
      mask(sc, p0, p1);
      m = 1.f;
    }
    rebase(largest(sc) * m);
    weights(sc, m, pb);
  };

  // Values that a query may not see must not reach it: 0 * inf is NaN.  In a stage
  // that holds keys behind the block's first query, values that are not finite
  // become 0; after the loop they are added to the queries that do see them.
  auto holds_later_keys = [&](const StagePos& p) {   // block-uniform
    int top = 0;
#pragma unroll
    for (int x = 0; x < kStageKeys / 16; ++x) top = max(top, p.at[x]);
    return top + 15 > block_first;
  };
  // Of the rows that this wave copied.
  auto clear_not_finite = [&](char* buf) {
#pragma unroll
    for (int i = 0; i < kCopies; ++i) {
      uint4* v = reinterpret_cast<uint4*>(buf + kStageBytes + (w * kCopies + i) * 1024) + lane;
      uint4 u = *v;
      uint32_t* e = &u.x;
      bool bad = false;
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const bool b0 = kBf16 && (e[c] & 0x7f80u) == 0x7f80u, b1 = (e[c] & 0x7f800000u) == 0x7f800000u;
        e[c] &= (b0 ? 0xffff0000u : ~0u) & (b1 ? (kBf16 ? 0x0000ffffu : 0u) : ~0u);
        bad |= b0 | b1;
      }
      if (bad) {
        *v = u;
        s_bad = 1;
      }
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  };
  // the list's next 64 entries, once stage st begins among them
  auto refill = [&](int st) {
    if (((st * (kStageKeys / 16)) >> (a.log_block - 4)) - cur_base < 64) return;
    cur = nxt;
    cur_base += 64;
    nxt = entries(cur_base + 64);
    asm volatile("s_waitcnt vmcnt(0)" : "+v"(nxt));   // now, not at a use that copies are in flight at
  };

  if (tid == 0) s_bad = 0;
  __syncthreads();
  StagePos pos{};
  // Stage st, which lies at place `at` of the ring (a constant where it is inlined).
  auto stage = [&](int st, int at) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    const StagePos p = pos;
    if (holds_later_keys(p)) clear_not_finite(s_ring[at]);
    sync_stage();                               // stage st is in LDS; the other place is free
    if (st + 1 < n_stages) {
      refill(st + 1);
      copy_stage(st + 1, s_ring[at ^ 1]);
      pos = stage_pos(st + 1);
    }
    const uint32_t off = at * 2 * kStageBytes;
    Keys kf;
    Values vf;
    Weights pb;
    auto half = [&](int sub, int p0, int p1, bool more) {
      f32x16 sc = scores(off, kf);
      load_values(off, sub, vf);
      if (more) load_keys(off, 1, kf);
      __builtin_amdgcn_sched_barrier(0);
      soften(sc, p0, p1, pb);
      add_values(off, vf, pb);
    };
    if constexpr (kHalves == 1) {
      if (min(p.at[0], p.at[1]) <= last_pos) half(0, p.at[0], p.at[1], false);
    } else if constexpr (WK == 1) {
      const bool see0 = min(p.at[0], p.at[1]) <= last_pos, see1 = min(p.at[2], p.at[3]) <= last_pos;
      load_keys(off, see0 ? 0 : 1, kf);
      if (see0) half(0, p.at[0], p.at[1], true);
      if (see1) half(1, p.at[2], p.at[3], false);
    } else {
      const int p0 = wk ? p.at[2] : p.at[0], p1 = wk ? p.at[3] : p.at[1];
      if (min(p0, p1) > last_pos) return;
      load_keys(off, wk, kf);
      half(wk, p0, p1, false);
    }
  };
  if (n_stages > 0) {
    copy_stage(0, s_ring[0]);
    pos = stage_pos(0);
  }
  for (int st = 0; st < n_stages; st += 2) {
    stage(st, 0);
    if (st + 1 < n_stages) stage(st + 1, 1);
  }
  sync_stage();
  if (s_bad) {                                  // block-uniform, rare
    if (n_list > 0 && e1 > e0) {
      cur_base = 0;
      cur = entries(0);
      nxt = entries(64);
    }
#pragma unroll 1
    for (int gi = 0; gi < n_groups; ++gi) {
      if ((gi >> (a.log_block - 4)) - cur_base >= 64) {
        cur = nxt;
        cur_base += 64;
        nxt = entries(cur_base + 64);
      }
      if (gi / 2 % WK != wk || !holds_later_keys(stage_pos(gi / (kStageKeys / 16)))) continue;
      const int p0 = group_pos(gi);
#pragma unroll 1
      for (int pos = p0; pos < min(p0 + 16, last_pos + 1); ++pos) {
        const T* v = reinterpret_cast<const T*>(vb) + (size_t)pos * kHeadDim;
#pragma unroll
        for (int dt = 0; dt < 4; ++dt)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const float f = load_as_f32(v, 32 * dt + (i & 3) + 8 * (i >> 2) + 4 * h);
            o[dt][i] += pos <= qpos && !__builtin_isfinite(f) ? f : 0.f;
          }
      }
    }
  }

  // the waves that shared the keys: wk = 1 leaves its sums in LDS, wk = 0 adds them
  float m = grow_at == -__builtin_inff() ? -__builtin_inff() : base;
  if constexpr (WK > 1) {
    static_assert(WK == 2 && WR * 34 * 256 <= 2 * kStageBytes, "half of a wave's sums fit a stage");
    float* s0 = reinterpret_cast<float*>(s_ring[0]) + wr * 34 * 64 + lane;
    float* s1 = reinterpret_cast<float*>(s_ring[1]) + wr * 34 * 64 + lane;
    if (wk == 1) {
#pragma unroll
      for (int i = 0; i < 32; ++i) {
        s0[i * 64] = o[i >> 4][i & 15];
        s1[i * 64] = o[2 + (i >> 4)][i & 15];
      }
      s0[32 * 64] = m;
      s1[32 * 64] = sum;
    }
    __syncthreads();
    if (wk == 1) return;
    const float m1 = s0[32 * 64], mm = fmaxf(m, m1);
    const float f0 = __builtin_amdgcn_exp2f(m - max_base(mm)), f1 = __builtin_amdgcn_exp2f(m1 - max_base(mm));
    m = mm;
    sum = sum * f0 + s1[32 * 64] * f1;
#pragma unroll
    for (int i = 0; i < 32; ++i) {
      o[i >> 4][i & 15] = o[i >> 4][i & 15] * f0 + s0[i * 64] * f1;
      o[2 + (i >> 4)][i & 15] = o[2 + (i >> 4)][i & 15] * f0 + s1[i * 64] * f1;
    }
  }
  const float total = sum + __shfl_xor(sum, 32, kWave);
  if (row0 + n >= n_rows) return;
  if (a.n_split > 1) {
    float* p = a.part + (row * a.n_split + split) * kPartFloats;
    if (h == 0) *reinterpret_cast<float2*>(p) = make_float2(m, total);
#pragma unroll
    for (int dt = 0; dt < 4; ++dt)
#pragma unroll
      for (int i = 0; i < 16; i += 2)
        *reinterpret_cast<float2*>(p + 2 + 32 * dt + (i & 3) + 8 * (i >> 2) + 4 * h) =
            make_float2(o[dt][i], o[dt][i + 1]);
    return;
  }
  const float inv = inv_sum(total);
  if (a.lse_out && h == 0) a.lse_out[row] = lse_of(m, total);
#pragma unroll
  for (int dt = 0; dt < 4; ++dt)
#pragma unroll
    for (int i = 0; i < 16; i += 4) {
      const size_t at = row * kHeadDim + 32 * dt + 2 * i + 4 * h;
      const float y0 = o[dt][i] * inv, y1 = o[dt][i + 1] * inv, y2 = o[dt][i + 2] * inv, y3 = o[dt][i + 3] * inv;
      if (a.out_bf16) {
        *reinterpret_cast<uint2*>(static_cast<uint16_t*>(a.out) + at) =
            make_uint2(f32_to_bf16(y0) | (uint32_t)f32_to_bf16(y1) << 16, f32_to_bf16(y2) | (uint32_t)f32_to_bf16(y3) << 16);
      } else {
        *reinterpret_cast<float4*>(static_cast<float*>(a.out) + at) = make_float4(y0, y1, y2, y3);
      }
    }
}

int check_dtype(int dtype) {
  if (dtype != LOUISKV_F32 && dtype != LOUISKV_BF16) return fail(LOUISKV_ERR_DTYPE, "unknown dtype %d", dtype);
  return LOUISKV_OK;
}

// How a call is cut into blocks of waves.  A block takes all rows of a tile, up to
// 256, as long as there are 256 blocks for the chip (8 slices in tiles of 64 tokens
// by 4 heads: of 8192 tokens 256 rows a block 276 us, 64 rows 343; of 1024 tokens 256
// rows and lists in four parts 76 us, 64 rows and whole lists 49).  Where that is
// not enough the lists are split for 512 blocks (256 tokens: 28.7 us; 256 blocks
// 30.7, 1024 blocks 35.6), into parts of two stages or more, so that the next one is
// under way (one token, 2112 keys: 9.6 us; one stage 10.7, four 11.2), and of four
// keys a row (two in float32), so that writing and reading the partials moves half
// of the keys' bytes at most (64 tokens, 2112 keys: 17.5 us; half 22.4, twice 19.1).
// 256 slices of one token stay whole: 53 us; split in two 50, but the same
// rule takes 141 us for 75 with 2048 tokens.
struct Cut {
  int rows;         // rows (tokens by heads) of a tile that a block takes: 64, 128 or 256
  int row_groups;   // blocks of a tile
  int splits;       // parts of a tile's list
  int64_t blocks;
};
constexpr int kFullGrid = 256, kSplitGrid = 512;
Cut cut_of(int64_t n_slices, int group_size, int n_q, int q_block, int block_len, int sel_cap, int dtype) {
  const int rows = std::min(q_block, n_q) * group_size, stage_keys = dtype == LOUISKV_BF16 ? 64 : 32;
  const int64_t tiles = n_slices * (((int64_t)n_q + q_block - 1) / q_block);
  Cut c;
  auto take = [&](int per) {
    c.rows = per;
    c.row_groups = (rows + per - 1) / per;
    c.blocks = tiles * c.row_groups;
  };
  take(rows > 128 ? 256 : rows > 64 ? 128 : 64);
  while (c.rows > 64 && c.blocks < kFullGrid) take(c.rows / 2);
  const int part_keys = std::max(2 * stage_keys, std::min(rows, c.rows) * stage_keys / 16);
  const int64_t by_keys = std::max<int64_t>(1, (int64_t)sel_cap * block_len / part_keys);
  c.splits = c.blocks >= kFullGrid ? 1 : (int)std::min<int64_t>(by_keys, kSplitGrid / c.blocks);
  c.blocks *= c.splits;
  return c;
}

template <class T, int WR, int WK>
void launch_prefill(const PrefillArgs& a, const Cut& c, hipStream_t s) {
  prefill_kernel<T, WR, WK><<<(unsigned)c.blocks, WR * WK * 64, 0, s>>>(a, c.row_groups, c.blocks);
}

int log2_block(int block_len) {
  switch (block_len) {
    case 16: return 4;
    case 32: return 5;
    case 64: return 6;
    case 128: return 7;
    case 256: return 8;
    default: return -1;
  }
}

// Sizes that both calls share.
int check_sizes(int64_t n_slices, int32_t n_kv_heads, int32_t n_q, int32_t d, int32_t n_keys, int32_t q_start,
                int32_t q_block, int32_t block_len) {
  if (d != kHeadDim) return fail(LOUISKV_ERR_UNSUPPORTED, "head dim %d not supported (only 128)", d);
  if (n_kv_heads < 1 || n_slices < 1 || n_slices % n_kv_heads != 0)
    return fail(LOUISKV_ERR_SHAPE, "n_slices=%lld must be a positive multiple of n_kv_heads=%d", (long long)n_slices,
                n_kv_heads);
  if (q_block < 1 || q_block > kMaxTile || log2_block(block_len) < 0)
    return fail(LOUISKV_ERR_UNSUPPORTED, "q_block=%d must be in [1, %d], block_len=%d one of 16, 32, 64, 128, 256",
                q_block, kMaxTile, block_len);
  if (n_keys > kMaxKeys) return fail(LOUISKV_ERR_SHAPE, "n_keys=%d exceeds %d", n_keys, kMaxKeys);
  if (n_q < 1 || n_keys < 1 || q_start < 0 || (int64_t)q_start + n_q > n_keys)
    return fail(LOUISKV_ERR_SHAPE, "queries q_start=%d .. +%d must be among the n_keys=%d tokens", q_start, n_q, n_keys);
  if (n_slices > kMaxGrid || n_slices * (((int64_t)n_q + q_block - 1) / q_block) > kMaxGrid)
    return fail(LOUISKV_ERR_SHAPE, "problem too large for one launch");
  return LOUISKV_OK;
}

}  // namespace
}  // namespace louiskv

using namespace louiskv;

extern "C" size_t louiskv_retrieve_blocks_cap(int32_t n_keys, int32_t q_block, int32_t block_len, int32_t n_first,
                                              int32_t n_recent, int32_t n_top) {
  if (n_keys < 1 || q_block < 1 || q_block > kMaxTile || log2_block(block_len) < 0 || n_first < 0 || n_recent < 0 ||
      n_top < 0)
    return 0;
  const int64_t blocks = ((int64_t)n_keys + block_len - 1) / block_len;
  const int64_t own = (q_block + block_len - 2) / block_len + 1;
  return (size_t)std::min(blocks, (int64_t)n_first + n_recent + n_top + own);
}

extern "C" int louiskv_retrieve_blocks(const void* q, int32_t dtype, int64_t n_slices, int32_t n_kv_heads,
                                       int32_t group_size, int32_t n_q, int32_t d, const float* reps,
                                       int32_t units_cap, int32_t n_keys, int32_t q_start, int32_t q_block,
                                       int32_t block_len, int32_t n_first, int32_t n_recent, int32_t n_top,
                                       int32_t* sel_blocks, int32_t sel_cap, int32_t* n_sel_blocks, void* stream) {
  if (!q || !reps || !sel_blocks || !n_sel_blocks)
    return fail(LOUISKV_ERR_NULL, "q, reps, sel_blocks and n_sel_blocks are required");
  int st = check_dtype(dtype);
  if (st) return st;
  if ((st = check_sizes(n_slices, n_kv_heads, n_q, d, n_keys, q_start, q_block, block_len))) return st;
  if (group_size < 1 || group_size > 8) return fail(LOUISKV_ERR_UNSUPPORTED, "group_size=%d must be 1 to 8", group_size);
  if (!aligned16(q, reps)) return fail(LOUISKV_ERR_UNSUPPORTED, "q and reps must be 16-byte aligned");
  if (n_first < 0 || n_recent < 0 || n_top < 0)
    return fail(LOUISKV_ERR_SHAPE, "n_first=%d n_recent=%d n_top=%d", n_first, n_recent, n_top);
  const int blocks = (int)(((int64_t)n_keys + block_len - 1) / block_len);
  if (blocks > kMaxBlocks || blocks > units_cap)
    return fail(LOUISKV_ERR_SHAPE, "%d blocks exceed units_cap=%d or %d", blocks, units_cap, kMaxBlocks);
  const size_t cap = louiskv_retrieve_blocks_cap(n_keys, q_block, block_len, n_first, n_recent, n_top);
  if (sel_cap < 1 || (size_t)sel_cap < cap) return fail(LOUISKV_ERR_SHAPE, "sel_cap=%d, a list can need %zu", sel_cap, cap);
  SelectArgs a;
  a.q = q; a.group_size = group_size; a.n_q = n_q; a.reps = reps; a.units_cap = units_cap; a.n_keys = n_keys;
  a.q_start = q_start; a.q_block = q_block; a.log_block = log2_block(block_len);
  a.n_first = n_first; a.n_recent = std::min(n_recent, blocks); a.n_top = n_top;
  a.sel = sel_blocks; a.sel_cap = sel_cap; a.n_sel = n_sel_blocks; a.n_tiles = (n_q - 1) / q_block + 1;
  const size_t lds = (size_t)blocks * sizeof(uint64_t);
  const void* kernel = dtype == LOUISKV_BF16 ? (const void*)select_blocks_kernel<uint16_t>
                                             : (const void*)select_blocks_kernel<float>;
  if ((st = check_lds(kernel, lds))) return st;
  const unsigned grid = (unsigned)(n_slices * a.n_tiles);
  if (dtype == LOUISKV_BF16) select_blocks_kernel<uint16_t><<<grid, kSelThreads, lds, as_stream(stream)>>>(a);
  else select_blocks_kernel<float><<<grid, kSelThreads, lds, as_stream(stream)>>>(a);
  LKV_CHECK_LAUNCH();
  return LOUISKV_OK;
}

extern "C" size_t louiskv_sparse_prefill_attn_workspace_size(int64_t n_slices, int32_t group_size, int32_t n_q,
                                                             int32_t d, int32_t q_block, int32_t block_len,
                                                             int32_t sel_cap) {
  (void)d;
  if (n_slices < 1 || n_slices > kMaxGrid || group_size < 1 || group_size > 8 || n_q < 1 || q_block < 1 ||
      q_block > kMaxTile || log2_block(block_len) < 0 || sel_cap < 1)
    return 0;
  auto parts = [&](int dtype) { return cut_of(n_slices, group_size, n_q, q_block, block_len, sel_cap, dtype).splits; };
  return part_bytes(n_slices * group_size * n_q, std::max(parts(LOUISKV_BF16), parts(LOUISKV_F32)));
}

extern "C" int louiskv_sparse_prefill_attn(const void* q, int32_t dtype, int64_t n_slices, int32_t n_kv_heads,
                                           int32_t group_size, int32_t n_q, int32_t d, float scale, const void* keys,
                                           const void* values, int64_t key_rows, int32_t n_keys, int32_t q_start,
                                           int32_t q_block, int32_t block_len, const int32_t* sel_blocks,
                                           int32_t sel_cap, const int32_t* n_sel_blocks, void* out, int32_t out_dtype,
                                           float* lse_out, void* workspace, size_t workspace_bytes, void* stream) {
  if (!q || !keys || !values || !sel_blocks || !n_sel_blocks || !out)
    return fail(LOUISKV_ERR_NULL, "q, keys, values, sel_blocks, n_sel_blocks and out are required");
  int st = check_dtype(dtype);
  if (st || (st = check_dtype(out_dtype))) return st;
  if ((st = check_sizes(n_slices, n_kv_heads, n_q, d, n_keys, q_start, q_block, block_len))) return st;
  if (group_size != 1 && group_size != 2 && group_size != 4 && group_size != 8)
    return fail(LOUISKV_ERR_UNSUPPORTED, "group_size=%d must be 1, 2, 4 or 8", group_size);
  if (!aligned16(q, keys, values, out))
    return fail(LOUISKV_ERR_UNSUPPORTED, "q, keys, values and out must be 16-byte aligned");
  if (key_rows < n_keys || sel_cap < 1 || (int64_t)sel_cap * block_len > kMaxKeys)
    return fail(LOUISKV_ERR_SHAPE, "key_rows=%lld n_keys=%d sel_cap=%d", (long long)key_rows, n_keys, sel_cap);
  PrefillArgs a;
  a.q = q; a.group_size = group_size; a.n_q = n_q; a.scale = scale; a.keys = keys; a.values = values;
  a.key_rows = key_rows; a.n_keys = n_keys; a.q_start = q_start; a.q_block = q_block; a.log_block = log2_block(block_len);
  a.sel = sel_blocks; a.sel_cap = sel_cap; a.n_sel = n_sel_blocks; a.n_tiles = (n_q - 1) / q_block + 1; a.n_split = 1;
  a.part = nullptr; a.out = out; a.out_bf16 = out_dtype == LOUISKV_BF16; a.lse_out = lse_out;
  const int64_t n_rows = n_slices * group_size * n_q;
  const Cut c = cut_of(n_slices, group_size, n_q, q_block, block_len, sel_cap, dtype);
  const size_t need =
      louiskv_sparse_prefill_attn_workspace_size(n_slices, group_size, n_q, d, q_block, block_len, sel_cap);
  if (need > 0 && (!workspace || workspace_bytes < need || !aligned16(workspace)))
    return fail(LOUISKV_ERR_WORKSPACE, "workspace needs %zu bytes, 16-byte aligned, got %zu", need, workspace_bytes);
  hipStream_t hs = as_stream(stream);
  a.n_split = c.splits;
  a.part = static_cast<float*>(workspace);
  if (c.blocks > kMaxGrid) return fail(LOUISKV_ERR_SHAPE, "problem too large for one launch");
  if (dtype == LOUISKV_BF16) {
    switch (c.rows) {
      case 256: launch_prefill<uint16_t, 8, 1>(a, c, hs); break;
      case 128: launch_prefill<uint16_t, 4, 1>(a, c, hs); break;
      default: launch_prefill<uint16_t, 2, 2>(a, c, hs); break;
    }
  } else {
    switch (c.rows) {
      case 256: launch_prefill<float, 8, 1>(a, c, hs); break;
      case 128: launch_prefill<float, 4, 1>(a, c, hs); break;
      default: launch_prefill<float, 2, 1>(a, c, hs); break;
    }
  }
  LKV_CHECK_LAUNCH();
  if (c.splits == 1) return LOUISKV_OK;
  return merge_parts(a.part, c.splits, n_rows, out, out_dtype, lse_out, hs);
}
