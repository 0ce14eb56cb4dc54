// The prompt's attention over selected blocks of its keys: the selection of each
// query tile's blocks by their index vectors, and the causal attention over them.
#include "common.h"
#include "merge.h"

namespace louiskv {
namespace {

constexpr int kMaxBlocks = 8192;    // key blocks a tile's selection ranks
constexpr int kMaxTile = 128;       // queries of a tile

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

__device__ __forceinline__ double elem(const uint16_t* p) { return (double)bf16_to_f32(*p); }
__device__ __forceinline__ double elem(const float* p) { return (double)*p; }

constexpr int kSelThreads = 256;

// Block (slice, tile): the sum of the tile's queries in float64, the score of
// every ranked block, then the n_top-th largest key by radix selection (8 bits a
// pass, only the keys that share the digits found so far are counted) and the
// list in block order.
template <class T>
__global__ __launch_bounds__(kSelThreads)
void select_blocks_kernel(const SelectArgs a) {
  extern __shared__ uint64_t s_key[];   // one per ranked block
  __shared__ double s_q[kHeadDim], s_half[kHeadDim];
  __shared__ int s_hist[256];
  __shared__ int s_wave[kSelThreads / 64][2];
  __shared__ int s_digit, s_above, s_equal;
  const int64_t s = blockIdx.x / a.n_tiles;
  const int t = (int)(blockIdx.x - s * a.n_tiles), tid = threadIdx.x;
  const int i0 = t * a.q_block, i1 = min(i0 + a.q_block, a.n_q);
  const int p0 = a.q_start + i0, p1 = a.q_start + i1 - 1;
  const int hi = p1 >> a.log_block, lo = max(0, (p0 >> a.log_block) - a.n_recent);
  const int first = min(a.n_first, lo), ranked = lo - first;
  int32_t* sel = a.sel + ((size_t)s * a.n_tiles + t) * a.sel_cap;
  const int n_pick = min(a.n_top, ranked);
  const int n_total = first + n_pick + hi - lo + 1;
  if (tid == 0) a.n_sel[(size_t)s * a.n_tiles + t] = n_total;
  for (int b = tid; b < first; b += kSelThreads) sel[b] = b;
  for (int b = lo + tid; b <= hi; b += kSelThreads) sel[first + n_pick + b - lo] = b;
  if (n_pick == 0) return;
  if (n_pick == ranked) {
    for (int b = tid; b < ranked; b += kSelThreads) sel[first + b] = first + b;
    return;
  }
  {
    const int c = tid & 127, part = tid >> 7;
    double x = 0.0;
    for (int j = 0; j < a.group_size; ++j) {
      const T* q = static_cast<const T*>(a.q) + (((size_t)s * a.group_size + j) * a.n_q) * kHeadDim + c;
      for (int i = i0 + part; i < i1; i += 2) x += elem(q + (size_t)i * kHeadDim);
    }
    if (part) s_half[c] = x;
    __syncthreads();
    if (!part) s_q[c] = x + s_half[c];
    __syncthreads();
  }
  for (int b = tid; b < ranked; b += kSelThreads) {
    const float4* rep = reinterpret_cast<const float4*>(a.reps + ((size_t)s * a.units_cap + first + b) * kHeadDim);
    double x = 0.0;
    for (int k = 0; k < kHeadDim / 4; ++k) {
      const float4 f = rep[k];
      x += s_q[4 * k] * (double)f.x;
      x += s_q[4 * k + 1] * (double)f.y;
      x += s_q[4 * k + 2] * (double)f.z;
      x += s_q[4 * k + 3] * (double)f.w;
    }
    s_key[b] = ordered(x);
  }
  uint64_t prefix = 0, mask = 0;
  int need = n_pick;              // still to take among the keys that match the prefix
  for (int shift = 56; shift >= 0; shift -= 8) {
    s_hist[tid] = 0;
    __syncthreads();
    for (int b = tid; b < ranked; b += kSelThreads) {
      const uint64_t k = s_key[b];
      if ((k & mask) == prefix) atomicAdd(&s_hist[(int)((k >> shift) & 255)], 1);
    }
    __syncthreads();
    if (tid < 64) {               // the digit at which the count from the top reaches `need`
      int c[4], sum = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        c[e] = s_hist[255 - (4 * tid + e)];
        sum += c[e];
      }
      int before = sum;
      for (int o = 1; o < 64; o <<= 1) {
        const int y = __shfl_up(before, o, kWave);
        if (tid >= o) before += y;
      }
      before -= sum;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if (before < need && before + c[e] >= need) {
          s_digit = 255 - (4 * tid + e);
          s_above = before;
          s_equal = c[e];
        }
        before += c[e];
      }
    }
    __syncthreads();
    prefix |= (uint64_t)s_digit << shift;
    mask |= 255ull << shift;
    need -= s_above;
    const bool all = s_equal == need;
    __syncthreads();
    if (all) break;               // every key with this prefix is taken
  }
  // taken: keys above the prefix, and the first `need` that match it
  int taken = 0, equal = 0;
  for (int b0 = 0; b0 < ranked; b0 += kSelThreads) {
    const int b = b0 + tid, w = tid >> 6, lane = tid & 63;
    const uint64_t k = b < ranked ? s_key[b] & mask : 0;
    const bool above = b < ranked && k > prefix, eq = b < ranked && k == prefix;
    const uint64_t eqs = __ballot(eq), abv = __ballot(above), below = (1ull << lane) - 1;
    if (lane == 0) {
      s_wave[w][0] = __popcll(abv);
      s_wave[w][1] = __popcll(eqs);
    }
    __syncthreads();
    int my_above = taken + __popcll(abv & below), my_eq = equal + __popcll(eqs & below);
    for (int x = 0; x < kSelThreads / 64; ++x) {
      if (x < w) {
        my_above += s_wave[x][0];
        my_eq += s_wave[x][1];
      }
      taken += s_wave[x][0];
      equal += s_wave[x][1];
    }
    if (above || (eq && my_eq < need)) sel[first + my_above + min(my_eq, need)] = first + b;
    __syncthreads();
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

template <class T>
__device__ __forceinline__ void row8(const T* p, float (&x)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] = load_as_f32(p, e);
}

// Sixteen lanes per (query, head), lane sub with channels 8 sub..+7: one pass over
// the keys of the tile's blocks.
template <class T>
__global__ __launch_bounds__(256)
void prefill_attn_kernel(const PrefillArgs a, int64_t n_rows) {
  const int64_t row = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4);
  if (row >= n_rows) return;
  const int sub = threadIdx.x & 15;
  const int64_t sh = row / a.n_q, s = sh / a.group_size;
  const int i = (int)(row - sh * a.n_q), pos = a.q_start + i;
  const int64_t list = s * a.n_tiles + i / a.q_block;
  const int n = max(0, min(a.n_sel[list], a.sel_cap));
  float q[8], acc[8];
  row8(static_cast<const T*>(a.q) + (size_t)row * kHeadDim + 8 * sub, q);
  const float qs = a.scale * kLog2E;
  float m = -__builtin_inff(), l = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    q[e] *= qs;
    acc[e] = 0.f;
  }
  const int last = min(a.n_keys - 1, pos);
  for (int x = 0; x < n; ++x) {
    const int b = min(max(a.sel[list * a.sel_cap + x], 0), (a.n_keys - 1) >> a.log_block);
    const int k0 = b << a.log_block, k1 = min(k0 + (1 << a.log_block) - 1, last);
    for (int k = k0; k <= k1; ++k) {
      const size_t o = ((size_t)s * a.key_rows + k) * kHeadDim + 8 * sub;
      float kv[8], vv[8];
      row8(static_cast<const T*>(a.keys) + o, kv);
      row8(static_cast<const T*>(a.values) + o, vv);
      float d = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) d = fmaf(q[e], kv[e], d);
      d = row16_add(d);
      const float mn = fmaxf(m, d), base = max_base(mn);
      const float c = __builtin_amdgcn_exp2f(m - base), p = __builtin_amdgcn_exp2f(d - base);
      m = mn;
      l = l * c + p;
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[e] = fmaf(acc[e], c, p * vv[e]);
    }
  }
  const float inv = inv_sum(l);
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const size_t o = (size_t)row * kHeadDim + 8 * sub + e;
    if (a.out_bf16) static_cast<uint16_t*>(a.out)[o] = f32_to_bf16(acc[e] * inv);
    else static_cast<float*>(a.out)[o] = acc[e] * inv;
  }
  if (a.lse_out && sub == 0) a.lse_out[row] = lse_of(m, l);
}

int check_dtype(int dtype) {
  if (dtype != LOUISKV_F32 && dtype != LOUISKV_BF16) return fail(LOUISKV_ERR_DTYPE, "unknown dtype %d", dtype);
  return LOUISKV_OK;
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
  if (n_q < 1 || n_keys < 1 || q_start < 0 || (int64_t)q_start + n_q > n_keys)
    return fail(LOUISKV_ERR_SHAPE, "queries q_start=%d .. +%d must be among the n_keys=%d tokens", q_start, n_q, n_keys);
  if (n_slices * (((int64_t)n_q + q_block - 1) / q_block) > INT32_MAX)
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
  (void)n_slices; (void)group_size; (void)n_q; (void)d; (void)q_block; (void)block_len; (void)sel_cap;
  return 0;
}

extern "C" int louiskv_sparse_prefill_attn(const void* q, int32_t dtype, int64_t n_slices, int32_t n_kv_heads,
                                           int32_t group_size, int32_t n_q, int32_t d, float scale, const void* keys,
                                           const void* values, int64_t key_rows, int32_t n_keys, int32_t q_start,
                                           int32_t q_block, int32_t block_len, const int32_t* sel_blocks,
                                           int32_t sel_cap, const int32_t* n_sel_blocks, void* out, int32_t out_dtype,
                                           float* lse_out, void* workspace, size_t workspace_bytes, void* stream) {
  (void)workspace; (void)workspace_bytes;
  if (!q || !keys || !values || !sel_blocks || !n_sel_blocks || !out)
    return fail(LOUISKV_ERR_NULL, "q, keys, values, sel_blocks, n_sel_blocks and out are required");
  int st = check_dtype(dtype);
  if (st || (st = check_dtype(out_dtype))) return st;
  if ((st = check_sizes(n_slices, n_kv_heads, n_q, d, n_keys, q_start, q_block, block_len))) return st;
  if (group_size != 1 && group_size != 2 && group_size != 4 && group_size != 8)
    return fail(LOUISKV_ERR_UNSUPPORTED, "group_size=%d must be 1, 2, 4 or 8", group_size);
  if (key_rows < n_keys || sel_cap < 1)
    return fail(LOUISKV_ERR_SHAPE, "key_rows=%lld n_keys=%d sel_cap=%d", (long long)key_rows, n_keys, sel_cap);
  PrefillArgs a;
  a.q = q; a.group_size = group_size; a.n_q = n_q; a.scale = scale; a.keys = keys; a.values = values;
  a.key_rows = key_rows; a.n_keys = n_keys; a.q_start = q_start; a.q_block = q_block; a.log_block = log2_block(block_len);
  a.sel = sel_blocks; a.sel_cap = sel_cap; a.n_sel = n_sel_blocks; a.n_tiles = (n_q - 1) / q_block + 1; a.n_split = 1;
  a.part = nullptr; a.out = out; a.out_bf16 = out_dtype == LOUISKV_BF16; a.lse_out = lse_out;
  const int64_t n_rows = n_slices * group_size * n_q;
  if ((n_rows + 15) / 16 > INT32_MAX) return fail(LOUISKV_ERR_SHAPE, "problem too large for one launch");
  const unsigned grid = (unsigned)((n_rows + 15) / 16);
  if (dtype == LOUISKV_BF16) prefill_attn_kernel<uint16_t><<<grid, 256, 0, as_stream(stream)>>>(a, n_rows);
  else prefill_attn_kernel<float><<<grid, 256, 0, as_stream(stream)>>>(a, n_rows);
  LKV_CHECK_LAUNCH();
  return LOUISKV_OK;
}
