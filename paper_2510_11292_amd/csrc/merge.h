// Softmax partials of rows that several blocks attend parts of, and their merge.
#pragma once

#include "common.h"

namespace louiskv {

constexpr float kLn2 = 0.6931471805599453f;
constexpr float kLog2E = 1.4426950408889634f;

// Blocks of up to 512 threads that one launch can hold: 2^32 - 1 threads.
constexpr int64_t kMaxGrid = (1 << 23) - 1;

constexpr int64_t kMaxRows = 1 << 30;      // of a slice of a shared prefix or a cache of bounded size
constexpr int64_t kCacheBytes = 32 << 20;  // the L2s: what such a call reads beyond them goes past them

// Whether kernels may read (or write) these in 16-byte pieces.
template <class... P>
bool aligned16(const P*... p) { return ((reinterpret_cast<uintptr_t>(p) | ...) & 15) == 0; }

inline int check_workspace(const void* workspace, size_t bytes, size_t need) {
  if (need > 0 && (!workspace || bytes < need || !aligned16(workspace)))
    return fail(LOUISKV_ERR_WORKSPACE, "workspace needs %zu bytes, 16-byte aligned, got %zu", need, bytes);
  return LOUISKV_OK;
}

// A partial: the maximum of its base-2 logits (-inf: no key), the sum of
// 2^(logit - max) and the weighted sum of the value rows.  Partials of row r are
// part[r][0..n_parts-1].
constexpr int kPartFloats = 2 + kHeadDim;

inline size_t part_bytes(int64_t n_rows, int n_parts) {
  return n_parts <= 1 ? 0 : align_up((size_t)n_rows * n_parts * kPartFloats * sizeof(float), 256);
}

// What a maximum is subtracted as: a row without a finite score (no key, or scores
// of -inf) keeps 0, so that its weights are 2^-inf = 0.  A NaN score does not move
// the maximum; it makes the sum NaN.
__device__ __forceinline__ float max_base(float m) { return m == -__builtin_inff() ? 0.f : m; }
// 1 / sum; 0 for a row without any weight, NaN stays
__device__ __forceinline__ float inv_sum(float l) { return l == 0.f ? 0.f : 1.f / l; }
// base-2 maximum and sum -> natural log of the softmax denominator
__device__ __forceinline__ float lse_of(float m, float l) { return kLn2 * (max_base(m) + log2f(l)); }

// A wave joins n_parts parts of a row (at least one): their maximum m, and the sum l and, in
// lane k, dims 2k and 2k + 1 of the weighted sums against it.  Lane c loads the maximum and sum
// of part c; a batch of parts' weighted sums is on its way meanwhile (32 rows of 17
// parts: 3.6 us, most of it the trips to memory; four loads at a time, 4.2).
constexpr int kMergeParts = 16;
__device__ __forceinline__ void join_parts(const float* __restrict__ p, int n_parts, float& m, float& l, float& a0, float& a1) {
  const int lane = threadIdx.x & 63;
  float2 x[kMergeParts];
  auto load = [&](int c0) {
#pragma unroll
    for (int b = 0; b < kMergeParts; ++b)
      x[b] = *reinterpret_cast<const float2*>(p + (size_t)min(c0 + b, n_parts - 1) * kPartFloats + 2 + 2 * lane);
  };
  float2 ml = *reinterpret_cast<const float2*>(p + (size_t)min(lane, n_parts - 1) * kPartFloats);
  load(0);
  m = ml.x;
  for (int c = kWave + lane; c < n_parts; c += kWave) m = fmaxf(m, p[(size_t)c * kPartFloats]);
  m = wave_max(m);
  const float base = max_base(m);
  l = 0.f, a0 = 0.f, a1 = 0.f;
  for (int c0 = 0; c0 < n_parts; c0 += kMergeParts) {
    if (c0 > 0) {
      load(c0);
      if (c0 % kWave == 0) ml = *reinterpret_cast<const float2*>(p + (size_t)min(c0 + lane, n_parts - 1) * kPartFloats);
    }
    const float e = __builtin_amdgcn_exp2f(ml.x - base);
#pragma unroll
    for (int b = 0; b < kMergeParts; ++b)
      if (c0 + b < n_parts) {
        const int src = (c0 + b) % kWave;
        const float w = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(e), src));
        l += __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(ml.y), src)) * w;
        a0 += x[b].x * w;
        a1 += x[b].y * w;
      }
  }
}

template <class TO>
__device__ __forceinline__ void merge_row(const float* __restrict__ part, int n_parts, int64_t row,
                                          TO* __restrict__ out, float* __restrict__ lse_out) {
  const int lane = threadIdx.x & 63;
  float m, l, a0, a1;
  join_parts(part + (size_t)row * n_parts * kPartFloats, n_parts, m, l, a0, a1);
  const float inv = inv_sum(l);
  store_from_f32(out + (size_t)row * kHeadDim, 2 * lane, a0 * inv);
  store_from_f32(out + (size_t)row * kHeadDim, 2 * lane + 1, a1 * inv);
  if (lse_out && lane == 0) lse_out[row] = lse_of(m, l);
}

template <class TO>
__global__ __launch_bounds__(256)
void merge_parts_kernel(const float* __restrict__ part, int n_parts, int64_t n_rows, TO* __restrict__ out,
                        float* __restrict__ lse_out) {
  const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (row < n_rows) merge_row(part, n_parts, row, out, lse_out);
}

inline int merge_parts(const float* part, int n_parts, int64_t n_rows, void* out, int out_dtype, float* lse_out,
                       hipStream_t s) {
  const unsigned grid = (unsigned)((n_rows + 3) / 4);
  if (out_dtype == LOUISKV_BF16)
    merge_parts_kernel<uint16_t><<<grid, 256, 0, s>>>(part, n_parts, n_rows, static_cast<uint16_t*>(out), lse_out);
  else
    merge_parts_kernel<float><<<grid, 256, 0, s>>>(part, n_parts, n_rows, static_cast<float*>(out), lse_out);
  LKV_CHECK_LAUNCH();
  return LOUISKV_OK;
}

// Sum over the 16 lanes of a DPP row, result in every lane of the row.
__device__ __forceinline__ float row16_add(float x) {
  x += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), 0xB1, 0xF, 0xF, false));
  x += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), 0x4E, 0xF, 0xF, false));
  x += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), 0x141, 0xF, 0xF, false));
  x += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), 0x140, 0xF, 0xF, false));
  return x;
}

}  // namespace louiskv
