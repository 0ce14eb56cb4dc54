// Attention of sequences that share a prefix (or of caches of bounded size), and the
// weight that queries give to each key.
#include "common.h"
#include "merge.h"

namespace louiskv {
namespace {

constexpr int64_t kMaxRows = 1 << 30;   // rows of a slice, queries of a prefix slice

struct AttnArgs {
  const void* q;
  int group_size, n_q;
  float scale;
  const void* k_prefix;
  const void* v_prefix;
  int64_t n_prefix_slices;
  int prefix_rows;
  const int32_t* n_prefix;
  const void* k_own;
  const void* v_own;
  int own_rows;
  const int32_t* n_own;
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

// Block: one query.  Its waves take every fourth 64 rows, a row a lane for the
// scores, two channels a lane for the sums.
template <class T>
__global__ __launch_bounds__(256)
void attn_kernel(const AttnArgs a) {
  __shared__ float s_q[kHeadDim];
  __shared__ float s_o[4][kHeadDim], s_m[4], s_l[4];
  const int64_t row = blockIdx.x, s = row / (a.group_size * a.n_q);
  const int t = (int)(row % a.n_q), lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  if (threadIdx.x < kHeadDim) s_q[threadIdx.x] = at<T>(a.q, row, threadIdx.x) * (a.scale * kLog2E);
  __syncthreads();
  const int64_t ps = a.prefix_rows ? s % a.n_prefix_slices : 0;
  const int np = a.prefix_rows ? length_of(a.n_prefix, ps, a.prefix_rows) : 0;
  const int own = max(0, length_of(a.n_own, s, a.own_rows) - a.n_q + t + 1);
  float m = -__builtin_inff(), l = 0.f, o0 = 0.f, o1 = 0.f;
  for (int part = 0; part < 2; ++part) {
    const int n = part ? own : np;
    const void* k = part ? a.k_own : a.k_prefix;
    const void* v = part ? a.v_own : a.v_prefix;
    const int64_t r0 = part ? s * a.own_rows : ps * a.prefix_rows;
    for (int i0 = 64 * w; i0 < n; i0 += 256) {
      const int i = min(i0 + lane, n - 1);
      float x = 0.f;
      for (int c = 0; c < kHeadDim; ++c) x += s_q[c] * at<T>(k, r0 + i, c);
      if (i0 + lane >= n) x = -__builtin_inff();
      const float mm = fmaxf(m, wave_max(x)), f = exp2f(max_base(m) - max_base(mm));
      const float p = exp2f(x - max_base(mm));
      m = mm;
      l = l * f + p;
      o0 *= f;
      o1 *= f;
      for (int j = 0; j < min(64, n - i0); ++j) {
        const float pj = __shfl(p, j, kWave);
        o0 += pj * at<T>(v, r0 + i0 + j, 2 * lane);
        o1 += pj * at<T>(v, r0 + i0 + j, 2 * lane + 1);
      }
    }
  }
  l = wave_sum(l);
  s_m[w] = m;
  s_l[w] = l;
  s_o[w][2 * lane] = o0;
  s_o[w][2 * lane + 1] = o1;
  __syncthreads();
  if (threadIdx.x >= kHeadDim) return;
  m = fmaxf(fmaxf(s_m[0], s_m[1]), fmaxf(s_m[2], s_m[3]));
  float o = 0.f;
  l = 0.f;
  for (int i = 0; i < 4; ++i) {
    const float f = exp2f(s_m[i] - max_base(m));
    l += s_l[i] * f;
    o += s_o[i][threadIdx.x] * f;
  }
  o *= inv_sum(l);
  if (a.out_bf16) store_from_f32(static_cast<uint16_t*>(a.out) + row * kHeadDim, threadIdx.x, o);
  else store_from_f32(static_cast<float*>(a.out) + row * kHeadDim, threadIdx.x, o);
  if (a.lse_out && threadIdx.x == 0) a.lse_out[row] = lse_of(m, l);
}

struct WeightArgs {
  const void* q;
  int group_size, n_q;
  float scale;
  const void* keys;
  int key_rows;
  const int32_t* n_keys;
  const float* lse;
  float* weights;
};

// A thread a key.
template <class T>
__global__ __launch_bounds__(256)
void weights_kernel(const WeightArgs a, int blocks_per_slice) {
  const int64_t s = blockIdx.x / blocks_per_slice;
  const int i = (int)(blockIdx.x % blocks_per_slice) * 256 + threadIdx.x;
  const int n = length_of(a.n_keys, s, a.key_rows);
  if (i >= n) return;
  float total = 0.f;
  for (int j = 0; j < a.group_size; ++j)
    for (int t = max(0, i - (n - a.n_q)); t < a.n_q; ++t) {
      const int64_t row = (s * a.group_size + j) * a.n_q + t;
      const float lse = a.lse[row];
      if (lse == -__builtin_inff()) continue;
      float x = 0.f;
      for (int c = 0; c < kHeadDim; ++c) x += at<T>(a.q, row, c) * at<T>(a.keys, s * a.key_rows + i, c);
      total += exp2f(x * (a.scale * kLog2E) - lse * kLog2E);
    }
  a.weights[s * a.key_rows + i] += total;
}

int launch_weights(const WeightArgs& a, int64_t n_slices, int dtype, hipStream_t hs) {
  const int per = (a.key_rows + 255) / 256;
  const unsigned grid = (unsigned)(n_slices * per);
  if (dtype == LOUISKV_BF16) weights_kernel<uint16_t><<<grid, 256, 0, hs>>>(a, per);
  else weights_kernel<float><<<grid, 256, 0, hs>>>(a, per);
  LKV_CHECK_LAUNCH();
  return LOUISKV_OK;
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
  if (n_slices > kMaxGrid || n_slices * group_size > kMaxRows / n_q)
    return fail(LOUISKV_ERR_SHAPE, "%lld slices of %d heads and n_q=%d are too many queries for one call",
                (long long)n_slices, group_size, n_q);
  return LOUISKV_OK;
}

bool served(int64_t n_slices, int32_t group_size, int32_t n_q, int64_t rows) {
  return n_slices >= 1 && n_slices <= kMaxGrid && group_size >= 1 && group_size <= 8 && n_q >= 1 && rows >= 0 &&
         rows <= kMaxRows && n_slices * group_size <= kMaxRows / n_q;
}

int check_workspace(const void* workspace, size_t bytes, size_t need) {
  if (need > 0 && (!workspace || bytes < need || !aligned16(workspace)))
    return fail(LOUISKV_ERR_WORKSPACE, "workspace needs %zu bytes, 16-byte aligned, got %zu", need, bytes);
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
  return with_weights ? align_up((size_t)n_slices * group_size * n_q * sizeof(float), 256) : 0;
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
  const size_t need = louiskv_shared_prefix_attn_workspace_size(n_slices, n_prefix_slices, group_size, n_q, d,
                                                                prefix_rows, own_rows, weights != nullptr);
  if ((st = check_workspace(workspace, workspace_bytes, need))) return st;
  AttnArgs a;
  a.q = q; a.group_size = group_size; a.n_q = n_q; a.scale = scale;
  a.k_prefix = k_prefix; a.v_prefix = v_prefix; a.n_prefix_slices = prefix_rows ? n_prefix_slices : n_slices;
  a.prefix_rows = (int)prefix_rows; a.n_prefix = n_prefix;
  a.k_own = k_own; a.v_own = v_own; a.own_rows = (int)own_rows; a.n_own = n_own;
  a.out = out; a.out_bf16 = out_dtype == LOUISKV_BF16;
  a.lse_out = lse_out ? lse_out : weights ? static_cast<float*>(workspace) : nullptr;
  hipStream_t hs = as_stream(stream);
  const unsigned grid = (unsigned)(n_slices * group_size * n_q);
  if (dtype == LOUISKV_BF16) attn_kernel<uint16_t><<<grid, 256, 0, hs>>>(a);
  else attn_kernel<float><<<grid, 256, 0, hs>>>(a);
  LKV_CHECK_LAUNCH();
  if (!weights || own_rows == 0) return LOUISKV_OK;
  WeightArgs wa;
  wa.q = q; wa.group_size = group_size; wa.n_q = n_q; wa.scale = scale; wa.keys = k_own; wa.key_rows = (int)own_rows;
  wa.n_keys = n_own; wa.lse = a.lse_out; wa.weights = weights;
  return launch_weights(wa, n_slices, dtype, hs);
}

extern "C" size_t louiskv_attn_weights_workspace_size(int64_t n_slices, int32_t group_size, int32_t n_q, int32_t d,
                                                      int64_t key_rows) {
  (void)d;
  if (!served(n_slices, group_size, n_q, key_rows)) return 0;
  return 0;
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
  const size_t need = louiskv_attn_weights_workspace_size(n_slices, group_size, n_q, d, key_rows);
  if ((st = check_workspace(workspace, workspace_bytes, need))) return st;
  WeightArgs a;
  a.q = q; a.group_size = group_size; a.n_q = n_q; a.scale = scale; a.keys = keys; a.key_rows = (int)key_rows;
  a.n_keys = n_keys; a.lse = lse; a.weights = weights;
  return launch_weights(a, n_slices, dtype, as_stream(stream));
}
