// A cache that keeps the rows of most attention weight: which rows stay, and the
// moves that leave them in the cache's first rows.
#include "common.h"
#include "merge.h"

namespace louiskv {
namespace {

struct PlanArgs {
  const float* weights;
  const int32_t* pos;        // NULL: row numbers
  const int32_t* n_rows;     // NULL: rows
  const int32_t* n_seen;
  int rows, n_keep, n_first, n_recent;
  int32_t* map;              // [slices][n_keep]: the row that each row is taken from
  int32_t* movers;           // [slices][n_keep]: the staying rows from m on, ascending (slices of more than kPlanRows)
  int32_t* kept;             // [slices]: m
};

// A float32 as an unsigned integer of the same order; NaN below every number, -0 as 0.
__device__ __forceinline__ uint32_t ordered(float x) {
  if (x != x) return 0;
  const uint32_t u = __float_as_uint(x + 0.f);
  return (u >> 31) ? ~u : u | 0x80000000u;
}
constexpr uint32_t kProtected = 0xffffffffu;   // above every ordered float

// ------------------------------------------------------------------- which rows stay

// Rows of a slice as order keys: in registers, kValues a lane (a wave's rows are consecutive,
// 64 at a time: row 64 (kValues w + j) + lane), or recomputed from memory where kValues
// is 0 and a slice has more rows than that.
template <int kThreads, int kValues>
struct Rows {
  static constexpr int kWaves = kThreads / 64;
  const float* w;
  const int32_t* pos;
  int n, n_first, steps;
  int64_t recent;
  uint32_t key[kValues > 0 ? kValues : 1];

  __device__ __forceinline__ uint32_t key_of(int p, float x) const {
    return p < n_first || p >= recent ? kProtected : ordered(x);
  }
  __device__ __forceinline__ int row(int j) const {
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    return 64 * ((kValues > 0 ? kValues : steps) * wave + j) + lane;
  }
  __device__ __forceinline__ uint32_t get(int j) const {
    if constexpr (kValues > 0) return key[j];
    const int i = row(j);
    return i < n ? key_of(pos ? pos[i] : i, w[i]) : 0;
  }
  // f(j, row, key) for the lane's rows
  template <class F>
  __device__ __forceinline__ void each(F&& f) const {
    if constexpr (kValues > 0) {
#pragma unroll
      for (int j = 0; j < kValues; ++j) f(j, row(j), key[j]);
    } else {
      for (int j = 0; j < steps; ++j) f(j, row(j), get(j));
    }
  }
  // The slice's rows; all loads are on their way together where they stay in registers.
  __device__ __forceinline__ void load(const PlanArgs& a, int64_t s, int n_, int64_t seen) {
    n = n_;
    n_first = a.n_first;
    w = a.weights + s * a.rows;
    pos = a.pos ? a.pos + s * a.rows : nullptr;
    recent = seen - a.n_recent;
    steps = (n + 64 * kWaves - 1) / (64 * kWaves);
    if constexpr (kValues > 0) {
      constexpr int kAtOnce = kValues < 16 ? kValues : 16;
#pragma unroll
      for (int j0 = 0; j0 < kValues; j0 += kAtOnce) {
        float x[kAtOnce];
        int p[kAtOnce];
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) {
          const int i = min(row(j0 + j), n - 1);
          x[j] = w[i];
          p[j] = pos ? pos[i] : i;
        }
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) key[j0 + j] = key_of(p[j], x[j]);
      }
    }
  }
};

// 32 bits in digits of 11, 11 and 10: the first tells exponents apart.  (More counts a bin, so
// that lanes whose weights are alike meet less often, took as long: 6.4 us for 32768 rows with
// one, two, eight or sixteen.)
constexpr int kDigit = 11, kBins = 1 << kDigit;
template <int kThreads>
struct Scratch {
  alignas(8) int hist[kBins];   // also a wave's least key each, 8 bytes
  int part[kThreads / 64], part2[kThreads / 64];
  int digit, need, equal;
};

// Sum of x over the waves before this one; every lane gives its wave's x.  (The next call begins
// with a barrier, behind which `part` is free.)
template <int kThreads>
__device__ __forceinline__ int waves_before(int x, int* part) {
  const int wave = threadIdx.x >> 6;
  __syncthreads();
  if ((threadIdx.x & 63) == 0) part[wave] = x;
  __syncthreads();
  int before = 0;
#pragma unroll
  for (int i = 0; i < kThreads / 64; ++i) before += i < wave ? part[i] : 0;
  return before;
}

// The m-th largest key of n (1 <= m <= n), how many rows have it and how many of those stay.
template <int kThreads, int kValues>
__device__ __forceinline__ uint32_t limit_key(const Rows<kThreads, kValues>& rows, int m, Scratch<kThreads>& x, int& need,
                                              int& equal) {
  constexpr int kPer = kBins / kThreads;
  const int tid = threadIdx.x, lane = tid & 63;
  uint32_t prefix = 0, mask = 0;
  need = m;
  for (int shift = 32 - kDigit;; shift = max(0, shift - kDigit)) {
#pragma unroll
    for (int e = 0; e < kPer; ++e) x.hist[tid + e * kThreads] = 0;
    __syncthreads();
    // the digit's bits that the mask does not hold already
    rows.each([&](int, int i, uint32_t k) {
      if (i < rows.n && (k & mask) == prefix) atomicAdd(&x.hist[(k >> shift) & (kBins - 1)], 1);
    });
    __syncthreads();
    // bins from the top, kPer a thread; the digit at which the count reaches `need`
    int c[kPer], mine = 0;
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
      c[e] = x.hist[kBins - 1 - (tid * kPer + e)];
      mine += c[e];
    }
    int before = mine;
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
      const int y = __shfl_up(before, o, kWave);
      if (lane >= o) before += y;
    }
    const int wave_total = __shfl(before, 63, kWave);
    before += waves_before<kThreads>(wave_total, x.part) - mine;
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
      if (before < need && before + c[e] >= need) {   // exactly one bin
        x.digit = kBins - 1 - (tid * kPer + e);
        x.need = need - before;
        x.equal = c[e];
      }
      before += c[e];
    }
    __syncthreads();
    prefix |= (uint32_t)x.digit << shift;
    mask |= (uint32_t)(kBins - 1) << shift;
    need = x.need;
    equal = x.equal;
    __syncthreads();
    if (shift == 0) return prefix;
    if (equal == need) return prefix;                  // all rows from this prefix on stay: the lowest key that has it
  }
}

// A row's fate, by rank among those at the limit where only some of them stay: f(j, row, stays)
// for the lane's rows, every lane in step.
template <int kThreads, int kValues, class F>
__device__ __forceinline__ void each_fate(const Rows<kThreads, kValues>& rows, uint32_t limit, int need, int equal,
                                          Scratch<kThreads>& x, F&& f) {
  const int lane = threadIdx.x & 63;
  const uint64_t below = (1ull << lane) - 1;
  int rank = 0;
  if (need < equal) {                                  // block-uniform
    int mine = 0;
    rows.each([&](int, int i, uint32_t k) { mine += __popcll(__ballot(i < rows.n && k == limit)); });
    rank = waves_before<kThreads>(mine, x.part2);
  }
  rows.each([&](int j, int i, uint32_t k) {
    bool stays = i < rows.n && k >= limit;
    if (need < equal) {
      const uint64_t eq = __ballot(i < rows.n && k == limit);
      if (k == limit && rank + __popcll(eq & below) < equal - need) stays = false;
      rank += __popcll(eq);
    }
    f(j, i, stays);
  });
}

// Block: a slice.  Writes the row that each of the m rows is taken from.
//
// 64 slices of 32768 rows, 2048 kept: 21.4 us, a block each, so that its own steps bound it:
// some 3 us until the weights are there, 6.5 for the first digit (32768 atomic additions in LDS),
// 2.4 for each other one, mostly barriers, and 4 for the words.
template <int kThreads, int kValues>
__global__ __launch_bounds__(kThreads)
void plan_kernel(const PlanArgs a) {
  __shared__ Scratch<kThreads> x;
  const int64_t s = blockIdx.x;
  const int lane = threadIdx.x & 63;
  const int n = a.n_rows ? max(0, min(a.n_rows[s], a.rows)) : a.rows, m = min(n, a.n_keep);
  if (threadIdx.x == 0) a.kept[s] = m;
  int32_t* map = a.map + s * a.n_keep;
  if (m == n) {                                        // none leaves
    for (int i = threadIdx.x; i < m; i += kThreads) map[i] = i;
    return;
  }
  if (m == 0) return;
  Rows<kThreads, kValues> rows;
  rows.load(a, s, n, a.pos ? a.n_seen[s] : n);
  int need, equal;
  const uint32_t limit = limit_key(rows, m, x, need, equal);
  const uint64_t below = (1ull << lane) - 1;
  if constexpr (kValues > 0) {
    // which rows stay, a word 64 of them; a thread a word counts those from m on and the gaps below
    constexpr int kWords = kThreads / 64 * kValues;
    __shared__ uint64_t s_word[kWords];
    __shared__ uint16_t s_gaps[kWords], s_mover[kWords * 32];
    const int tid = threadIdx.x;
    uint64_t word = 0;
    each_fate(rows, limit, need, equal, x, [&](int j, int, bool stays) {
      const uint64_t b = __ballot(stays);
      if (lane == j) word = b;
    });
    if (lane < kValues) s_word[(tid >> 6) * kValues + lane] = word;
    __syncthreads();
    uint64_t late = 0;
    int mine = 0;                                      // staying rows from m on, and gaps below m in the upper half
    if (tid < kWords) {
      const int lows = max(0, min(64, m - 64 * tid));
      const uint64_t low = lows == 64 ? ~0ull : (1ull << lows) - 1;
      late = s_word[tid] & ~low;
      mine = __popcll(late) + (__popcll(~s_word[tid] & low) << 16);
    }
    int before = mine;
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
      const int y = __shfl_up(before, o, kWave);
      if (lane >= o) before += y;
    }
    const int wave_total = __shfl(before, 63, kWave);
    before += waves_before<kThreads>(wave_total, x.part) - mine;
    if (tid < kWords) s_gaps[tid] = (uint16_t)(before >> 16);
    for (int at = before & 0xffff; late; late &= late - 1) s_mover[at++] = (uint16_t)(64 * tid + __ffsll((unsigned long long)late) - 1);
    __syncthreads();
    for (int i = tid; i < m; i += kThreads) {
      const uint64_t u = s_word[i >> 6];
      map[i] = u >> (i & 63) & 1 ? i : s_mover[s_gaps[i >> 6] + __popcll(~u & ((1ull << (i & 63)) - 1))];
    }
  } else {
    int32_t* movers = a.movers + s * a.n_keep;
    int late = 0, gone = 0;                            // staying rows from m on, and leaving ones below m, of the wave
    each_fate(rows, limit, need, equal, x, [&](int, int i, bool stays) {
      late += __popcll(__ballot(stays && i >= m));
      gone += __popcll(__ballot(!stays && i < m));
    });
    late = waves_before<kThreads>(late, x.part);
    gone = waves_before<kThreads>(gone, x.part);
    each_fate(rows, limit, need, equal, x, [&](int, int i, bool stays) {
      const uint64_t l = __ballot(stays && i >= m);
      if (stays && i >= m) movers[late + __popcll(l & below)] = i;
      late += __popcll(l);
    });
    __threadfence_block();
    __syncthreads();
    each_fate(rows, limit, need, equal, x, [&](int, int i, bool stays) {
      const uint64_t g = __ballot(!stays && i < m);
      if (i < m) map[i] = stays ? i : movers[gone + __popcll(g & below)];
      gone += __popcll(g);
    });
  }
}

constexpr int kPlanRows = 32768;   // that a block holds in registers
int launch_plan(const PlanArgs& p, int64_t n_slices, hipStream_t hs) {
  const unsigned grid = (unsigned)n_slices;
  if (p.rows <= 2048) plan_kernel<256, 8><<<grid, 256, 0, hs>>>(p);
  else if (p.rows <= 8192) plan_kernel<1024, 8><<<grid, 1024, 0, hs>>>(p);
  else if (p.rows <= kPlanRows) plan_kernel<1024, 32><<<grid, 1024, 0, hs>>>(p);
  else plan_kernel<1024, 0><<<grid, 1024, 0, hs>>>(p);
  LKV_CHECK_LAUNCH();
  return LOUISKV_OK;
}

// ------------------------------------------------------------------- moves

struct MoveArgs {
  const void* k;
  const void* v;
  void* k_to;
  void* v_to;
  const float* weights;
  float* weights_to;
  const int32_t* pos;
  int32_t* pos_to;
  int rows, rows_to, n_keep;
  const int32_t* map;
  const int32_t* kept;
  int32_t* n_rows_to;
};

// Rows 8 a wave, their keys' and values' 16-byte pieces all on their way together.  kStream: the
// rows come past the caches (64 slices' 2048 bfloat16 rows out of 32768: 25.8 us; through them
// 31.6.  24 slices' 777 float32 rows 9.6 and 8.3 us).
constexpr int kMoveRows = 8;
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
template <int kRowBytes, bool kStream>
__global__ __launch_bounds__(256)
void move_kernel(const MoveArgs a, int blocks_per_slice) {
  constexpr int kPieces = kRowBytes / 16, kAtOnce = 64 / kPieces, kSteps = kMoveRows / kAtOnce;   // of keys, as of values
  const int64_t s = blockIdx.x / blocks_per_slice;
  const int i0 = ((int)(blockIdx.x % blocks_per_slice) * 4 + (threadIdx.x >> 6)) * kMoveRows, lane = threadIdx.x & 63;
  const int m = a.kept[s];
  if (i0 == 0 && lane == 0 && a.n_rows_to) a.n_rows_to[s] = m;
  if (i0 >= m) return;
  // lane j < 8: row i0 + j
  const int mine = i0 + min(lane, kMoveRows - 1), from = a.map[s * a.n_keep + min(mine, m - 1)];
  const int64_t src = s * a.rows, dst = s * a.rows_to;
  const int piece = lane % kPieces * 16;
  u32x4 k[kSteps] = {}, v[kSteps] = {};
#pragma unroll
  for (int j = 0; j < kSteps; ++j) {
    const int r = j * kAtOnce + lane / kPieces, at = __shfl(from, r, kWave);
    const bool there = i0 + r < m, moved = at != i0 + r;
    const int64_t x = (src + at) * kRowBytes + piece;
    const u32x4* kx = reinterpret_cast<const u32x4*>(static_cast<const char*>(a.k) + x);
    const u32x4* vx = reinterpret_cast<const u32x4*>(static_cast<const char*>(a.v) + x);
    if (there && (moved || a.k_to != a.k)) k[j] = kStream ? __builtin_nontemporal_load(kx) : *kx;
    if (there && (moved || a.v_to != a.v)) v[j] = kStream ? __builtin_nontemporal_load(vx) : *vx;
  }
#pragma unroll
  for (int j = 0; j < kSteps; ++j) {
    const int r = j * kAtOnce + lane / kPieces, at = __shfl(from, r, kWave);
    const bool there = i0 + r < m, moved = at != i0 + r;
    const int64_t y = (dst + i0 + r) * kRowBytes + piece;
    if (there && (moved || a.k_to != a.k)) *reinterpret_cast<u32x4*>(static_cast<char*>(a.k_to) + y) = k[j];
    if (there && (moved || a.v_to != a.v)) *reinterpret_cast<u32x4*>(static_cast<char*>(a.v_to) + y) = v[j];
  }
  if (lane >= kMoveRows || mine >= m) return;
  if (a.weights_to && (from != mine || a.weights_to != a.weights)) a.weights_to[dst + mine] = a.weights[src + from];
  if (a.pos_to && (from != mine || a.pos_to != a.pos)) a.pos_to[dst + mine] = a.pos ? a.pos[src + from] : from;
}

struct StoreArgs {
  const void* k_new;
  const void* v_new;
  void* k;
  void* v;
  float* weights;
  int32_t* pos;
  int32_t* n_rows;
  int32_t* n_seen;
  int n_new;
  const int32_t* kept;
};

// The new rows behind the m that stay.  Block: a slice.
template <int kRowBytes>
__global__ __launch_bounds__(256)
void append_kernel(const StoreArgs a, int rows) {
  constexpr int kPieces = kRowBytes / 16;
  const int64_t s = blockIdx.x;
  const int m = a.kept[s], seen = a.n_seen[s];
  const int64_t dst = s * rows + m, src = s * a.n_new;
  for (int64_t c = threadIdx.x; c < (int64_t)a.n_new * kPieces; c += 256) {
    reinterpret_cast<uint4*>(static_cast<char*>(a.k) + dst * kRowBytes)[c] =
        reinterpret_cast<const uint4*>(static_cast<const char*>(a.k_new) + src * kRowBytes)[c];
    reinterpret_cast<uint4*>(static_cast<char*>(a.v) + dst * kRowBytes)[c] =
        reinterpret_cast<const uint4*>(static_cast<const char*>(a.v_new) + src * kRowBytes)[c];
  }
  for (int i = threadIdx.x; i < a.n_new; i += 256) {
    a.weights[dst + i] = 0.f;
    a.pos[dst + i] = seen + i;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    a.n_rows[s] = m + a.n_new;
    a.n_seen[s] = seen + a.n_new;
  }
}

// A store that at most 64 rows leave for, in one launch.  Block: a slice.  What a row
// that moves, and a new one, holds is read beside the weights; the rows that leave are
// found (one: the least key; more: by digits), and the staying rows among the last go
// to their places in order.  8 slices of 2048 rows 4.5 us (three launches 36), 1024 slices
// and five new rows each 11 to 14 us (317): dependent trips to memory and barriers.
constexpr int kMostGone = 64;
template <int kRowBytes, int kThreads, int kValues>
__global__ __launch_bounds__(kThreads)
void store_kernel(const PlanArgs a, const StoreArgs t) {
  constexpr int kPieces = kRowBytes / 16;
  __shared__ Scratch<kThreads> x;
  __shared__ int s_gone[kMostGone], s_n_gone, s_hole[kMostGone], s_to[kMostGone];
  const int64_t s = blockIdx.x;
  const int tid = threadIdx.x, lane = tid & 63;
  const int seen = t.n_seen[s], n = max(0, min(t.n_rows[s], a.rows)), m = min(n, a.n_keep), gone = n - m;
  const int64_t row0 = s * a.rows;
  Rows<kThreads, kValues> rows;
  if (gone > 0) rows.load(a, s, n, seen);
  // piece c of the last rows: of their keys, then of their values, row by row
  auto last = [&](int c) -> uint4 {
    const int r = c / (2 * kPieces), p = c % (2 * kPieces);
    const char* from = static_cast<const char*>(p < kPieces ? t.k : t.v);
    return *reinterpret_cast<const uint4*>(from + (row0 + m + r) * kRowBytes + p % kPieces * 16);
  };
  auto fresh = [&](int c) -> uint4 {
    const int r = c / (2 * kPieces), p = c % (2 * kPieces);
    const char* from = static_cast<const char*>(p < kPieces ? t.k_new : t.v_new);
    return *reinterpret_cast<const uint4*>(from + (s * t.n_new + r) * kRowBytes + p % kPieces * 16);
  };
  auto put = [&](int row, int c, const uint4& u) {
    const int p = c % (2 * kPieces);
    char* to = static_cast<char*>(p < kPieces ? t.k : t.v);
    *reinterpret_cast<uint4*>(to + (row0 + row) * kRowBytes + p % kPieces * 16) = u;
  };
  const int moves = gone * 2 * kPieces, news = t.n_new * 2 * kPieces;
  uint4 move0 = make_uint4(0, 0, 0, 0), new0 = make_uint4(0, 0, 0, 0);
  float w0 = 0.f;
  int p0 = 0;
  if (tid < moves) move0 = last(tid);
  if (tid < news) new0 = fresh(tid);
  if (tid < gone) {
    w0 = t.weights[row0 + m + tid];
    p0 = t.pos[row0 + m + tid];
  }
  if (gone > 0) {
    if (tid == 0) s_n_gone = 0;
    if (gone == 1) {
      // the least key, of equal ones the lowest row
      uint64_t least = ~0ull;
      rows.each([&](int, int i, uint32_t k) {
        if (i < n) least = min(least, (uint64_t)k << 32 | (uint32_t)i);
      });
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) least = min(least, (uint64_t)__shfl_xor((unsigned long long)least, o, kWave));
      uint64_t* s_least = reinterpret_cast<uint64_t*>(x.hist);
      if (lane == 0) s_least[tid >> 6] = least;
      __syncthreads();
#pragma unroll
      for (int i = 0; i < kThreads / 64; ++i) least = min(least, s_least[i]);
      if (tid == 0) s_gone[0] = (int)(uint32_t)least;
    } else if (m > 0) {
      int need, equal;
      const uint32_t limit = limit_key(rows, m, x, need, equal);
      each_fate(rows, limit, need, equal, x, [&](int, int i, bool stays) {
        if (i < n && !stays) s_gone[atomicAdd(&s_n_gone, 1)] = i;
      });
    } else if (tid < gone) {
      s_gone[tid] = tid;                               // all leave
    }
    __syncthreads();
    if (tid < 64) {
      // lane: a row that leaves, and a row of the last ones
      const int e = lane < gone ? s_gone[lane] : INT32_MAX, c = m + lane;
      int rank = 0;
      bool leaves = false;
      for (int j = 0; j < gone; ++j) {
        const int y = __builtin_amdgcn_readlane(e, j);
        rank += y < e;
        leaves |= y == c;
      }
      if (e < m) s_hole[rank] = e;
      const bool stays = lane < gone && !leaves;
      const uint64_t b = __ballot(stays);
      __builtin_amdgcn_wave_barrier();
      if (lane < gone) s_to[lane] = stays ? s_hole[__popcll(b & ((1ull << lane) - 1))] : -1;
    }
    __syncthreads();
    for (int c = tid; c < moves; c += kThreads) {
      const int to = s_to[c / (2 * kPieces)];
      if (to < 0) continue;
      put(to, c, c == tid ? move0 : last(c));
    }
    if (tid < gone && s_to[tid] >= 0) {
      t.weights[row0 + s_to[tid]] = w0;
      t.pos[row0 + s_to[tid]] = p0;
    }
  }
  __syncthreads();                                     // what is replaced below has been read, the counts too
  for (int c = tid; c < news; c += kThreads) put(m + c / (2 * kPieces), c, c == tid ? new0 : fresh(c));
  for (int i = tid; i < t.n_new; i += kThreads) {
    t.weights[row0 + m + i] = 0.f;
    t.pos[row0 + m + i] = seen + i;
  }
  if (tid == 0) {
    t.n_rows[s] = m + t.n_new;
    t.n_seen[s] = seen + t.n_new;
  }
}

// The rows that can leave at once where a slice's buffer is full; whether one launch does.
bool stores_at_once(int64_t rows, int64_t budget, int64_t n_new) {
  return rows <= kPlanRows && rows - (budget - n_new) <= kMostGone;
}

template <int kRowBytes>
int launch_store(const PlanArgs& p, const StoreArgs& t, int64_t n_slices, hipStream_t hs) {
  const unsigned grid = (unsigned)n_slices;
  if (p.rows <= 2048) store_kernel<kRowBytes, 256, 8><<<grid, 256, 0, hs>>>(p, t);
  else if (p.rows <= 8192) store_kernel<kRowBytes, 1024, 8><<<grid, 1024, 0, hs>>>(p, t);
  else store_kernel<kRowBytes, 1024, 32><<<grid, 1024, 0, hs>>>(p, t);
  LKV_CHECK_LAUNCH();
  return LOUISKV_OK;
}

size_t plan_bytes(int64_t n_slices, int64_t rows, int64_t n_keep) {
  return align_up((size_t)n_slices * 4, 256) + (rows > kPlanRows ? 2 : 1) * align_up((size_t)n_slices * n_keep * 4, 256);
}

void carve(PlanArgs& p, void* workspace, int64_t n_slices) {
  Carver c(workspace);
  p.kept = c.take<int32_t>(n_slices);
  p.map = c.take<int32_t>((size_t)n_slices * p.n_keep);
  p.movers = p.rows > kPlanRows ? c.take<int32_t>((size_t)n_slices * p.n_keep) : nullptr;
}

// Blocks that the moves of a slice's n_keep rows take.
int64_t move_blocks(int64_t n_keep) { return std::max<int64_t>(1, (n_keep + 4 * kMoveRows - 1) / (4 * kMoveRows)); }

// Whether the launches fit: a block a slice that plans or stores (of 1024 threads where it has more
// than 2048 rows, half as many as kMaxGrid then), and where rows move in a launch of their own its
// blocks of 256 threads, of which twice kMaxGrid fit.
bool fits_launch(int64_t n_slices, int64_t rows, int64_t n_keep, bool moves) {
  return n_slices <= (rows > 2048 ? kMaxGrid / 2 : kMaxGrid) && (!moves || n_slices * move_blocks(n_keep) <= 2 * kMaxGrid);
}

int check_sizes(int dtype, int64_t n_slices, int32_t d, int64_t rows, int64_t n_keep, int32_t n_first,
                int32_t n_recent, bool moves) {
  if (dtype != LOUISKV_F32 && dtype != LOUISKV_BF16) return fail(LOUISKV_ERR_DTYPE, "unknown dtype %d", dtype);
  if (d != kHeadDim) return fail(LOUISKV_ERR_UNSUPPORTED, "head dim %d not supported (only 128)", d);
  if (n_slices < 1 || n_slices > kMaxGrid || rows < 1 || rows > kMaxRows)
    return fail(LOUISKV_ERR_SHAPE, "n_slices=%lld must be in [1, %lld], rows=%lld in [1, %lld]", (long long)n_slices,
                (long long)kMaxGrid, (long long)rows, (long long)kMaxRows);
  if (n_first < 0 || n_recent < 0 || (int64_t)n_first + n_recent > n_keep || n_keep > rows)
    return fail(LOUISKV_ERR_SHAPE, "n_first=%d and n_recent=%d must fit the %lld rows kept of %lld", n_first, n_recent,
                (long long)n_keep, (long long)rows);
  if (!fits_launch(n_slices, rows, n_keep, moves)) return fail(LOUISKV_ERR_SHAPE, "problem too large for one launch");
  return LOUISKV_OK;
}

int launch_move(const MoveArgs& a, int64_t n_slices, int dtype, hipStream_t hs) {
  const int per = (int)move_blocks(a.n_keep);
  const unsigned grid = (unsigned)(n_slices * per);
  const bool bf16 = dtype == LOUISKV_BF16, stream = n_slices * a.n_keep * 2 * kHeadDim * (bf16 ? 2 : 4) > kCacheBytes;
  if (bf16 && stream) move_kernel<256, true><<<grid, 256, 0, hs>>>(a, per);
  else if (bf16) move_kernel<256, false><<<grid, 256, 0, hs>>>(a, per);
  else if (stream) move_kernel<512, true><<<grid, 256, 0, hs>>>(a, per);
  else move_kernel<512, false><<<grid, 256, 0, hs>>>(a, per);
  LKV_CHECK_LAUNCH();
  return LOUISKV_OK;
}

bool overlap(const void* a, size_t na, const void* b, size_t nb) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return a && b && x < y + nb && y < x + na;
}

}  // namespace
}  // namespace louiskv

using namespace louiskv;

extern "C" size_t louiskv_evict_rows_workspace_size(int64_t n_slices, int64_t rows, int64_t n_keep) {
  if (n_slices < 1 || n_slices > kMaxGrid || rows < 1 || rows > kMaxRows || n_keep < 1 ||
      !fits_launch(n_slices, rows, std::min(rows, n_keep), true))
    return 0;
  return plan_bytes(n_slices, rows, std::min(rows, n_keep));
}

extern "C" int louiskv_evict_rows(const float* weights, const int32_t* pos, const int32_t* n_rows,
                                  const int32_t* n_seen, int32_t dtype, int64_t n_slices, int32_t d, int64_t rows,
                                  int64_t n_keep, int32_t n_first, int32_t n_recent, const void* k, const void* v,
                                  void* k_to, void* v_to, float* weights_to, int32_t* pos_to, int64_t rows_to,
                                  int32_t* n_rows_to, void* workspace, size_t workspace_bytes, void* stream) {
  if (!weights || !k || !v || !k_to || !v_to || !n_rows_to)
    return fail(LOUISKV_ERR_NULL, "weights, k, v, k_to, v_to and n_rows_to are required");
  if (!pos != !n_seen) return fail(LOUISKV_ERR_NULL, "pos and n_seen go together");
  const int64_t keep = std::min(n_keep, rows);   // more rows than there are: all stay
  int st = check_sizes(dtype, n_slices, d, rows, keep, 0, 0, true);
  if (st) return st;
  if (n_keep < 1 || n_keep > rows_to || rows_to > kMaxRows || n_first < 0 || n_recent < 0 ||
      (int64_t)n_first + n_recent > n_keep)
    return fail(LOUISKV_ERR_SHAPE, "n_first=%d + n_recent=%d <= n_keep=%lld <= rows_to=%lld does not hold", n_first,
                n_recent, (long long)n_keep, (long long)rows_to);
  if (!aligned16(k, v, k_to, v_to)) return fail(LOUISKV_ERR_UNSUPPORTED, "k, v, k_to and v_to must be 16-byte aligned");
  const int row_bytes = kHeadDim * (dtype == LOUISKV_BF16 ? 2 : 4);
  // each output is its input or overlaps nothing
  const size_t ns = (size_t)n_slices, big = ns * rows * row_bytes, big_to = ns * rows_to * row_bytes;
  const struct { const void* p; size_t bytes; } in[] = {
      {k, big}, {v, big}, {weights, ns * rows * 4}, {pos, ns * rows * 4}, {n_rows, ns * 4}, {n_seen, ns * 4}};
  const struct { const void* p; size_t bytes; int of; } outs[] = {{k_to, big_to, 0}, {v_to, big_to, 1},
      {weights_to, ns * rows_to * 4, 2}, {pos_to, ns * rows_to * 4, 3}, {n_rows_to, ns * 4, 4}};
  for (int o = 0; o < 5; ++o) {
    for (int i = 0; i < 6; ++i) {
      if (!overlap(outs[o].p, outs[o].bytes, in[i].p, in[i].bytes)) continue;
      if (i != outs[o].of || in[i].p != outs[o].p || (o < 4 && rows_to != rows))
        return fail(LOUISKV_ERR_SHAPE, "an output must be the buffer that it is taken from, of as many rows, or overlap none");
    }
    for (int i = 0; i < o; ++i)
      if (overlap(outs[o].p, outs[o].bytes, outs[i].p, outs[i].bytes))
        return fail(LOUISKV_ERR_SHAPE, "outputs overlap");
  }
  const size_t need = louiskv_evict_rows_workspace_size(n_slices, rows, n_keep);
  if ((st = check_workspace(workspace, workspace_bytes, need))) return st;
  PlanArgs p;
  p.weights = weights; p.pos = pos; p.n_rows = n_rows; p.n_seen = n_seen; p.rows = (int)rows; p.n_keep = (int)keep;
  p.n_first = n_first; p.n_recent = n_recent;
  carve(p, workspace, n_slices);
  hipStream_t hs = as_stream(stream);
  if ((st = launch_plan(p, n_slices, hs))) return st;
  MoveArgs mv;
  mv.k = k; mv.v = v; mv.k_to = k_to; mv.v_to = v_to; mv.weights = weights; mv.weights_to = weights_to; mv.pos = pos;
  mv.pos_to = pos_to; mv.rows = (int)rows; mv.rows_to = (int)rows_to; mv.n_keep = (int)keep;
  mv.map = p.map; mv.kept = p.kept; mv.n_rows_to = n_rows_to;
  return launch_move(mv, n_slices, dtype, hs);
}

extern "C" size_t louiskv_store_evict_workspace_size(int64_t n_slices, int64_t rows, int32_t n_new, int64_t budget) {
  if (n_slices < 1 || n_slices > kMaxGrid || rows < 1 || rows > kMaxRows || n_new < 1 || budget < n_new || budget > rows)
    return 0;
  return stores_at_once(rows, budget, n_new) || !fits_launch(n_slices, rows, budget - n_new, true)
             ? 0 : plan_bytes(n_slices, rows, budget - n_new);
}

extern "C" int louiskv_store_evict(const void* k_new, const void* v_new, int32_t dtype, int64_t n_slices, int32_t n_new,
                                   int32_t d, void* k, void* v, float* weights, int32_t* pos, int32_t* n_rows,
                                   int32_t* n_seen, int64_t rows, int64_t budget, int32_t n_first, int32_t n_recent,
                                   void* workspace, size_t workspace_bytes, void* stream) {
  if (!k_new || !v_new || !k || !v || !weights || !pos || !n_rows || !n_seen)
    return fail(LOUISKV_ERR_NULL, "k_new, v_new, k, v, weights, pos, n_rows and n_seen are required");
  if (n_new < 1 || budget < n_new || budget > rows)
    return fail(LOUISKV_ERR_SHAPE, "n_new=%d, budget=%lld and rows=%lld must be 1 <= n_new <= budget <= rows", n_new,
                (long long)budget, (long long)rows);
  int st = check_sizes(dtype, n_slices, d, rows, budget - n_new, n_first, n_recent, !stores_at_once(rows, budget, n_new));
  if (st) return st;
  if (!aligned16(k_new, v_new, k, v)) return fail(LOUISKV_ERR_UNSUPPORTED, "k_new, v_new, k and v must be 16-byte aligned");
  const size_t need = louiskv_store_evict_workspace_size(n_slices, rows, n_new, budget);
  if ((st = check_workspace(workspace, workspace_bytes, need))) return st;
  // what changes overlaps nothing else
  const size_t ns = (size_t)n_slices, row_bytes = kHeadDim * (dtype == LOUISKV_BF16 ? 2 : 4);
  const struct { const void* p; size_t bytes; } bufs[] = {
      {k, ns * rows * row_bytes}, {v, ns * rows * row_bytes}, {weights, ns * rows * 4}, {pos, ns * rows * 4},
      {n_rows, ns * 4}, {n_seen, ns * 4}, {k_new, ns * n_new * row_bytes}, {v_new, ns * n_new * row_bytes}};
  for (int i = 0; i < 6; ++i)
    for (int j = i + 1; j < 8; ++j)
      if (overlap(bufs[i].p, bufs[i].bytes, bufs[j].p, bufs[j].bytes)) return fail(LOUISKV_ERR_SHAPE, "buffers overlap");
  PlanArgs p;
  p.weights = weights; p.pos = pos; p.n_rows = n_rows; p.n_seen = n_seen; p.rows = (int)rows;
  p.n_keep = (int)(budget - n_new); p.n_first = n_first; p.n_recent = n_recent;
  StoreArgs t;
  t.k_new = k_new; t.v_new = v_new; t.k = k; t.v = v; t.weights = weights; t.pos = pos; t.n_rows = n_rows;
  t.n_seen = n_seen; t.n_new = n_new; t.kept = nullptr;
  hipStream_t hs = as_stream(stream);
  const bool bf16 = dtype == LOUISKV_BF16;
  if (stores_at_once(rows, budget, n_new)) {
    p.map = p.movers = p.kept = nullptr;
    return bf16 ? launch_store<256>(p, t, n_slices, hs) : launch_store<512>(p, t, n_slices, hs);
  }
  carve(p, workspace, n_slices);
  if ((st = launch_plan(p, n_slices, hs))) return st;
  MoveArgs mv;
  mv.k = k; mv.v = v; mv.k_to = k; mv.v_to = v; mv.weights = weights; mv.weights_to = weights; mv.pos = pos;
  mv.pos_to = pos; mv.rows = (int)rows; mv.rows_to = (int)rows; mv.n_keep = p.n_keep;
  mv.map = p.map; mv.kept = p.kept; mv.n_rows_to = nullptr;
  if ((st = launch_move(mv, n_slices, dtype, hs))) return st;
  t.kept = p.kept;
  if (bf16) append_kernel<256><<<(unsigned)n_slices, 256, 0, hs>>>(t, (int)rows);
  else append_kernel<512><<<(unsigned)n_slices, 256, 0, hs>>>(t, (int)rows);
  LKV_CHECK_LAUNCH();
  return LOUISKV_OK;
}
