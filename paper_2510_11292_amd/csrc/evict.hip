// A cache that keeps the rows of most attention weight: which rows stay, and the
// moves that leave them in the cache's first rows.
#include "common.h"
#include "merge.h"

namespace louiskv {
namespace {

constexpr int64_t kMaxRows = 1 << 30;   // of a slice

struct PlanArgs {
  const float* weights;
  const int32_t* pos;        // NULL: row numbers
  const int32_t* n_rows;     // NULL: rows
  const int32_t* n_seen;
  int rows, n_keep, n_first, n_recent;
  int32_t* map;              // [slices][n_keep]: the row that each row is taken from
  int32_t* movers;           // [slices][n_keep]: the staying rows from m on, ascending
  int32_t* kept;             // [slices]: m
};

// A float32 as an unsigned integer of the same order; NaN below every number, -0 as 0.
__device__ __forceinline__ uint32_t ordered(float x) {
  if (x != x) return 0;
  const uint32_t u = __float_as_uint(x + 0.f);
  return (u >> 31) ? ~u : u | 0x80000000u;
}
constexpr uint32_t kProtected = 0xffffffffu;   // above every ordered float

constexpr int kPlanThreads = 256;

// Sum of x over the threads before this one; *total that of all.  Ends with a barrier.
__device__ __forceinline__ int block_before(int x, int* total, int* s_part) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  int v = x;
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1) {
    const int y = __shfl_up(v, o, kWave);
    if (lane >= o) v += y;
  }
  if (lane == 63) s_part[w] = v;
  __syncthreads();
  int before = 0, all = 0;
  for (int i = 0; i < kPlanThreads / 64; ++i) {
    if (i < w) before += s_part[i];
    all += s_part[i];
  }
  __syncthreads();
  *total = all;
  return before + v - x;
}

// Block: a slice.  The m-th largest key by digits of eight bits, then the rows above
// it and the last of those that equal it stay.
__global__ __launch_bounds__(kPlanThreads)
void plan_kernel(const PlanArgs a) {
  __shared__ int s_hist[256], s_part[kPlanThreads / 64], s_digit, s_need, s_equal;
  const int64_t s = blockIdx.x;
  const int tid = threadIdx.x;
  const int n = a.n_rows ? max(0, min(a.n_rows[s], a.rows)) : a.rows;
  const int m = min(n, a.n_keep);
  const float* w = a.weights + s * a.rows;
  const int32_t* pos = a.pos ? a.pos + s * a.rows : nullptr;
  const int64_t recent = (int64_t)(a.pos ? a.n_seen[s] : n) - a.n_recent;
  auto key = [&](int i) -> uint32_t {
    const int p = pos ? pos[i] : i;
    return p < a.n_first || p >= recent ? kProtected : ordered(w[i]);
  };
  if (tid == 0) a.kept[s] = m;
  if (m == 0) return;
  uint32_t prefix = 0, mask = 0;
  int need = m, equal = 0;
  for (int shift = 24; shift >= 0; shift -= 8) {
    s_hist[tid] = 0;
    __syncthreads();
    for (int i = tid; i < n; i += kPlanThreads) {
      const uint32_t k = key(i);
      if ((k & mask) == prefix) atomicAdd(&s_hist[(k >> shift) & 255], 1);
    }
    __syncthreads();
    int total;
    const int c = s_hist[255 - tid], above = block_before(c, &total, s_part);
    if (above < need && above + c >= need) {   // exactly one thread
      s_digit = 255 - tid;
      s_need = need - above;
      s_equal = c;
    }
    __syncthreads();
    prefix |= (uint32_t)s_digit << shift;
    mask |= 255u << shift;
    need = s_need;
    equal = s_equal;
    __syncthreads();
  }
  // of `equal` rows at the limit the first equal - need leave
  int32_t* map = a.map + s * a.n_keep;
  int32_t* movers = a.movers + s * a.n_keep;
  for (int pass = 0; pass < 2; ++pass) {
    int seen = 0, found = 0;   // rows at the limit so far; movers (pass 0) or holes (pass 1) so far
    for (int i0 = 0; i0 < n; i0 += kPlanThreads) {
      const int i = i0 + tid;
      const uint32_t k = i < n ? key(i) : 0;
      const bool eq = i < n && k == prefix;
      int total;
      const int rank = seen + block_before(eq, &total, s_part);
      seen += total;
      const bool stays = i < n && (k > prefix || (eq && rank >= equal - need));
      const bool hit = pass == 0 ? stays && i >= m : i < m && !stays;
      const int at = found + block_before(hit, &total, s_part);
      found += total;
      if (pass == 0 && hit) movers[at] = i;
      if (pass == 1 && i < m) map[i] = hit ? movers[at] : i;
    }
    __threadfence_block();
    __syncthreads();
  }
}

struct MoveArgs {
  const void* k;
  const void* v;
  void* k_to;
  void* v_to;
  const float* weights;
  float* weights_to;
  const int32_t* pos;
  int32_t* pos_to;
  int rows, rows_to, n_keep, row_bytes;
  const int32_t* map;
  const int32_t* kept;
  int32_t* n_rows_to;
};

// A wave a row: 16-byte pieces of its key, then of its value.
__global__ __launch_bounds__(256)
void move_kernel(const MoveArgs a, int blocks_per_slice) {
  const int64_t s = blockIdx.x / blocks_per_slice;
  const int i = (int)(blockIdx.x % blocks_per_slice) * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int m = a.kept[s];
  if (i == 0 && lane == 0 && a.n_rows_to) a.n_rows_to[s] = m;
  if (i >= m) return;
  const int from = a.map[s * a.n_keep + i];
  const int64_t src = s * a.rows + from, dst = s * a.rows_to + i;
  const bool moved = from != i;
  const int pieces = a.row_bytes / 16;
  for (int c = lane; c < 2 * pieces; c += kWave) {
    const bool val = c >= pieces;
    const int p = val ? c - pieces : c;
    const char* x = static_cast<const char*>(val ? a.v : a.k);
    char* y = static_cast<char*>(val ? a.v_to : a.k_to);
    if (moved || x != y)
      *reinterpret_cast<uint4*>(y + dst * a.row_bytes + 16 * p) =
          *reinterpret_cast<const uint4*>(x + src * a.row_bytes + 16 * p);
  }
  if (lane == 0 && a.weights_to && (moved || a.weights_to != a.weights)) a.weights_to[dst] = a.weights[src];
  if (lane == 0 && a.pos_to && (moved || a.pos_to != a.pos)) a.pos_to[dst] = a.pos ? a.pos[src] : from;
}

struct AppendArgs {
  const void* k_new;
  const void* v_new;
  void* k;
  void* v;
  float* weights;
  int32_t* pos;
  int32_t* n_rows;
  int32_t* n_seen;
  int n_new, rows, row_bytes;
  const int32_t* kept;
};

// Block: a slice.
__global__ __launch_bounds__(256)
void append_kernel(const AppendArgs a) {
  const int64_t s = blockIdx.x;
  const int m = a.kept[s], seen = a.n_seen[s], pieces = a.row_bytes / 16;
  const int64_t dst = s * a.rows + m, src = s * a.n_new;
  for (int64_t c = threadIdx.x; c < (int64_t)a.n_new * pieces; c += 256) {
    reinterpret_cast<uint4*>(static_cast<char*>(a.k) + dst * a.row_bytes)[c] =
        reinterpret_cast<const uint4*>(static_cast<const char*>(a.k_new) + src * a.row_bytes)[c];
    reinterpret_cast<uint4*>(static_cast<char*>(a.v) + dst * a.row_bytes)[c] =
        reinterpret_cast<const uint4*>(static_cast<const char*>(a.v_new) + src * a.row_bytes)[c];
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

size_t plan_bytes(int64_t n_slices, int64_t n_keep) {
  return align_up((size_t)n_slices * 4, 256) + 2 * align_up((size_t)n_slices * n_keep * 4, 256);
}

void carve(PlanArgs& p, void* workspace, int64_t n_slices) {
  Carver c(workspace);
  p.kept = c.take<int32_t>(n_slices);
  p.map = c.take<int32_t>((size_t)n_slices * p.n_keep);
  p.movers = c.take<int32_t>((size_t)n_slices * p.n_keep);
}

int check_sizes(int dtype, int64_t n_slices, int32_t d, int64_t rows, int64_t n_keep, int32_t n_first,
                int32_t n_recent) {
  if (dtype != LOUISKV_F32 && dtype != LOUISKV_BF16) return fail(LOUISKV_ERR_DTYPE, "unknown dtype %d", dtype);
  if (d != kHeadDim) return fail(LOUISKV_ERR_UNSUPPORTED, "head dim %d not supported (only 128)", d);
  if (n_slices < 1 || n_slices > kMaxGrid || rows < 1 || rows > kMaxRows)
    return fail(LOUISKV_ERR_SHAPE, "n_slices=%lld must be in [1, %lld], rows=%lld in [1, %lld]", (long long)n_slices,
                (long long)kMaxGrid, (long long)rows, (long long)kMaxRows);
  if (n_first < 0 || n_recent < 0 || (int64_t)n_first + n_recent > n_keep || n_keep > rows)
    return fail(LOUISKV_ERR_SHAPE, "n_first=%d and n_recent=%d must fit the %lld rows kept of %lld", n_first, n_recent,
                (long long)n_keep, (long long)rows);
  if (n_slices * ((n_keep + 3) / 4) > kMaxGrid) return fail(LOUISKV_ERR_SHAPE, "problem too large for one launch");
  return LOUISKV_OK;
}

int check_workspace(const void* workspace, size_t bytes, size_t need) {
  if (need > 0 && (!workspace || bytes < need || !aligned16(workspace)))
    return fail(LOUISKV_ERR_WORKSPACE, "workspace needs %zu bytes, 16-byte aligned, got %zu", need, bytes);
  return LOUISKV_OK;
}

int launch_move(const MoveArgs& a, int64_t n_slices, hipStream_t hs) {
  const int per = std::max(1, (a.n_keep + 3) / 4);
  move_kernel<<<(unsigned)(n_slices * per), 256, 0, hs>>>(a, per);
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
  if (n_slices < 1 || n_slices > kMaxGrid || rows < 1 || rows > kMaxRows || n_keep < 1) return 0;
  return plan_bytes(n_slices, std::min(rows, n_keep));
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
  int st = check_sizes(dtype, n_slices, d, rows, keep, 0, 0);
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
  plan_kernel<<<(unsigned)n_slices, kPlanThreads, 0, hs>>>(p);
  LKV_CHECK_LAUNCH();
  MoveArgs mv;
  mv.k = k; mv.v = v; mv.k_to = k_to; mv.v_to = v_to; mv.weights = weights; mv.weights_to = weights_to; mv.pos = pos;
  mv.pos_to = pos_to; mv.rows = (int)rows; mv.rows_to = (int)rows_to; mv.n_keep = (int)keep; mv.row_bytes = row_bytes;
  mv.map = p.map; mv.kept = p.kept; mv.n_rows_to = n_rows_to;
  return launch_move(mv, n_slices, hs);
}

extern "C" size_t louiskv_store_evict_workspace_size(int64_t n_slices, int64_t rows, int32_t n_new, int64_t budget) {
  if (n_slices < 1 || n_slices > kMaxGrid || rows < 1 || rows > kMaxRows || n_new < 1 || budget < n_new || budget > rows)
    return 0;
  return plan_bytes(n_slices, budget - n_new);
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
  int st = check_sizes(dtype, n_slices, d, rows, budget - n_new, n_first, n_recent);
  if (st) return st;
  if (!aligned16(k_new, v_new, k, v)) return fail(LOUISKV_ERR_UNSUPPORTED, "k_new, v_new, k and v must be 16-byte aligned");
  const size_t need = louiskv_store_evict_workspace_size(n_slices, rows, n_new, budget);
  if ((st = check_workspace(workspace, workspace_bytes, need))) return st;
  PlanArgs p;
  p.weights = weights; p.pos = pos; p.n_rows = n_rows; p.n_seen = n_seen; p.rows = (int)rows;
  p.n_keep = (int)(budget - n_new); p.n_first = n_first; p.n_recent = n_recent;
  carve(p, workspace, n_slices);
  hipStream_t hs = as_stream(stream);
  plan_kernel<<<(unsigned)n_slices, kPlanThreads, 0, hs>>>(p);
  LKV_CHECK_LAUNCH();
  const int row_bytes = kHeadDim * (dtype == LOUISKV_BF16 ? 2 : 4);
  MoveArgs mv;
  mv.k = k; mv.v = v; mv.k_to = k; mv.v_to = v; mv.weights = weights; mv.weights_to = weights; mv.pos = pos;
  mv.pos_to = pos; mv.rows = (int)rows; mv.rows_to = (int)rows; mv.n_keep = p.n_keep; mv.row_bytes = row_bytes;
  mv.map = p.map; mv.kept = p.kept; mv.n_rows_to = nullptr;
  if ((st = launch_move(mv, n_slices, hs))) return st;
  AppendArgs ap;
  ap.k_new = k_new; ap.v_new = v_new; ap.k = k; ap.v = v; ap.weights = weights; ap.pos = pos; ap.n_rows = n_rows;
  ap.n_seen = n_seen; ap.n_new = n_new; ap.rows = (int)rows; ap.row_bytes = row_bytes; ap.kept = p.kept;
  append_kernel<<<(unsigned)n_slices, 256, 0, hs>>>(ap);
  LKV_CHECK_LAUNCH();
  return LOUISKV_OK;
}
