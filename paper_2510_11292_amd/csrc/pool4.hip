// The KV pool in 4-bit floating point: its writes (prompt and evicted segments),
// dense reads, and decode attention over listed rows.
//
// Format (include/louiskv.h): blocks of 32 channels, a power-of-two scale 2^E with
// the smallest E in [-125, 125] such that max|x| <= 7 * 2^E, elements rounded to
// 0, .5, 1, 1.5, 2, 3, 4, 6 scales, ties to the even code.  Everything about it is
// exact: E comes from the bits of the maximum (1.m <= 1.75 or not), x * 2^-E and
// code * 2^E are products with powers of two, and the conversion instructions
// round once.  The range of E keeps every held value a normal, finite number of
// bfloat16.
#include "common.h"
#include "merge.h"

namespace louiskv {
namespace {

constexpr int kCodeBytes = 128;   // a row's key and value codes
constexpr int kScaleBytes = 8;    // and their scales
constexpr uint32_t kNotFinite = 255;

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

// The scale byte E + 127 of a block whose largest |x| has these float32 bits.
__device__ __forceinline__ uint32_t scale_byte(uint32_t amax) {
  if (amax >= 0x7f800000u) return kNotFinite;
  const int b = (int)(amax >> 23) - 2 + ((amax & 0x7fffffu) > 0x600000u ? 1 : 0);
  return (uint32_t)min(max(b, 2), 252);
}

// 2^(byte - 127) for a byte as stored; 255 (0x7f800000, an infinite scale) makes every
// element NaN in the conversion instructions.
__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float(byte << 23); }

// Eight consecutive channels of a row as float32.
__device__ __forceinline__ void load8(const uint16_t* p, float (&x)[8]) {
  const uint4 v = *reinterpret_cast<const uint4*>(p);
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(w[i] << 16);
    x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ void load8(const float* p, float (&x)[8]) {
  const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
  x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
}

// The four lanes of a quad hold a block of 32 channels, eight each: the block's
// scale byte and this lane's eight codes.
__device__ __forceinline__ uint32_t quantise8(const float (&x)[8], uint32_t& byte) {
  uint32_t top = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(x[e]) & 0x7fffffffu);
  top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0xB1, 0xF, 0xF, false));
  top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0x4E, 0xF, 0xF, false));
  byte = scale_byte(top);
  if (byte == kNotFinite) return 0;
  const float inv = __uint_as_float((254u - byte) << 23);   // 2^-E, a normal number for bytes 2..252
  uint32_t c = 0;
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[0] * inv, x[1] * inv, 1.0f, 0);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[2] * inv, x[3] * inv, 1.0f, 1);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[4] * inv, x[5] * inv, 1.0f, 2);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[6] * inv, x[7] * inv, 1.0f, 3);
  return c;
}

// The eight channels of a code word.
__device__ __forceinline__ void expand8(uint32_t c, float scale, float (&x)[8]) {
  const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, scale, 0);
  const f32x2 b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, scale, 1);
  const f32x2 d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, scale, 2);
  const f32x2 e = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, scale, 3);
  x[0] = a[0]; x[1] = a[1]; x[2] = b[0]; x[3] = b[1]; x[4] = d[0]; x[5] = d[1]; x[6] = e[0]; x[7] = e[1];
}

// float32 -> bfloat16 bits of a value that bfloat16 holds exactly, or NaN
__device__ __forceinline__ uint32_t exact_bf16(float x) { return __float_as_uint(x) >> 16; }

__device__ __forceinline__ void store8(uint16_t* p, const float (&x)[8]) {
  uint4 v;
  v.x = exact_bf16(x[0]) | exact_bf16(x[1]) << 16;
  v.y = exact_bf16(x[2]) | exact_bf16(x[3]) << 16;
  v.z = exact_bf16(x[4]) | exact_bf16(x[5]) << 16;
  v.w = exact_bf16(x[6]) | exact_bf16(x[7]) << 16;
  *reinterpret_cast<uint4*>(p) = v;
}
__device__ __forceinline__ void store8(float* p, const float (&x)[8]) {
  reinterpret_cast<float4*>(p)[0] = make_float4(x[0], x[1], x[2], x[3]);
  reinterpret_cast<float4*>(p)[1] = make_float4(x[4], x[5], x[6], x[7]);
}

// ------------------------------------------------------------------ pool writes and dense reads

// Rows are taken 32 to a block: 32 lanes a row, 16 for its key and 16 for its
// value, eight channels each, so that a wave's code stores are two whole 128-byte
// rows.  A block takes one (slice, 32 rows) chunk; blocks that stride over several
// lose their loads' time in between (64 slices of 32768 bfloat16 rows, written and
// read back, 2.73 GB: 498 us, 5.5 TB/s; eight blocks a compute unit 540, 64 of them
// 511).  Both are bound by memory: a copy of that size reaches 4.8 to 5.2 TB/s.
constexpr int kRowsPerChunk = 32;
constexpr int kRowsInFlight = 4;   // of a wave's lane half

template <class T>
__global__ __launch_bounds__(256)
void pack_q4_kernel(const T* __restrict__ keys, const T* __restrict__ values, const int32_t* __restrict__ perm,
                    int n_tokens, int64_t n_chunks, int chunks_per_slice, uint8_t* __restrict__ codes,
                    uint8_t* __restrict__ scales, int64_t pool_rows) {
  const int lane = threadIdx.x & 31, rg = threadIdx.x >> 5, sub = lane & 15;
  const T* src = lane < 16 ? keys : values;
  for (int64_t ch = blockIdx.x; ch < n_chunks; ch += gridDim.x) {
    const int64_t s = ch / chunks_per_slice;
    const int r0 = (int)(ch - s * chunks_per_slice) * kRowsPerChunk;
    float x[kRowsInFlight][8];
    bool live[kRowsInFlight];
#pragma unroll
    for (int i = 0; i < kRowsInFlight; ++i) {
      const int r = r0 + 8 * i + rg;
      live[i] = r < n_tokens;
      const int rr = min(r, n_tokens - 1);
      const int tok = perm ? min(max(perm[s * n_tokens + rr], 0), n_tokens - 1) : rr;
      load8(src + ((size_t)s * n_tokens + tok) * kHeadDim + 8 * sub, x[i]);
    }
#pragma unroll
    for (int i = 0; i < kRowsInFlight; ++i) {
      uint32_t byte;
      const uint32_t c = quantise8(x[i], byte);
      if (!live[i]) continue;
      const size_t row = (size_t)s * pool_rows + r0 + 8 * i + rg;
      *reinterpret_cast<uint32_t*>(codes + row * kCodeBytes + 4 * lane) = c;
      if ((lane & 3) == 0) scales[row * kScaleBytes + (lane >> 2)] = (uint8_t)byte;
    }
  }
}

template <class T>
__global__ __launch_bounds__(256)
void gather_q4_kernel(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales, int64_t pool_rows,
                      const int32_t* __restrict__ rows, const int32_t* __restrict__ n_sel, int buf_rows,
                      int64_t n_chunks, int chunks_per_slice, T* __restrict__ k_buf, T* __restrict__ v_buf) {
  const int lane = threadIdx.x & 31, rg = threadIdx.x >> 5, sub = lane & 15;
  T* dst = lane < 16 ? k_buf : v_buf;
  for (int64_t ch = blockIdx.x; ch < n_chunks; ch += gridDim.x) {
    const int64_t s = ch / chunks_per_slice;
    const int r0 = (int)(ch - s * chunks_per_slice) * kRowsPerChunk;
    const int n = n_sel ? max(0, min(n_sel[s], buf_rows)) : buf_rows;
    uint32_t c[kRowsInFlight], b[kRowsInFlight];
#pragma unroll
    for (int i = 0; i < kRowsInFlight; ++i) {
      const int r = min(r0 + 8 * i + rg, buf_rows - 1);   // entries behind n are not read: the row of the last is
      const int64_t src = rows ? min<int64_t>(max(r < n ? rows[(size_t)s * buf_rows + r] : 0, 0), pool_rows - 1) : r;
      const size_t row = (size_t)s * pool_rows + src;
      c[i] = *reinterpret_cast<const uint32_t*>(codes + row * kCodeBytes + 4 * lane);
      b[i] = scales[row * kScaleBytes + (lane >> 2)];
    }
#pragma unroll
    for (int i = 0; i < kRowsInFlight; ++i) {
      const int r = r0 + 8 * i + rg;
      if (r >= n) continue;
      float x[8];
      expand8(c[i], scale_of(b[i]), x);
      store8(dst + ((size_t)s * buf_rows + r) * kHeadDim + 8 * sub, x);
    }
  }
}

// ------------------------------------------------------------------ decode store

// The words of a slice's segment state that louiskv_segment_state_init lays out:
// units, first token of the window, head and count of the ring of segment
// starts, overflow flag; the ring begins at kRing.
constexpr int kNUnits = 0, kWinFirst = 1, kHead = 2, kCount = 3, kOverflow = 4, kRing = 8;

// A block of 256 per slice: 32 lanes a row (16 its key, 16 its value), eight rows at
// a time.  The rows of the segment that leaves go to the pool and into eight
// float64 partial means per channel, then the new token enters its slot, which
// is the first of the rows that left: the barrier and the wait before it keep
// every wave's reads ahead of that write.  Bound by latency: a lane group's rows, four of
// a segment of 32, are read one after another, each read behind the stores of the row
// before (8 slices with a segment of 32 tokens 4.4 us, 1024 slices, 22 MB, 6.9 us).
template <class T, bool kSeg>
__global__ __launch_bounds__(256)
void store_q4_kernel(const T* __restrict__ k_new, const T* __restrict__ v_new, T* __restrict__ k_local,
                     T* __restrict__ v_local, int window, int step, int seg_len, int evict_seg,
                     const uint8_t* __restrict__ fire, int n_kv_heads, int32_t* __restrict__ state,
                     float* __restrict__ reps, int32_t* __restrict__ unit_start, int32_t* __restrict__ unit_size,
                     int units_cap, int n_clusters, uint8_t* __restrict__ codes, uint8_t* __restrict__ scales,
                     int64_t pool_rows, int prompt_len) {
  __shared__ double s_sum[8][kHeadDim];
  const int64_t s = blockIdx.x;
  const int tid = threadIdx.x, lane = tid & 31, rg = tid >> 5, sub = lane & 15;
  const size_t lbase = (size_t)s * window * kHeadDim;
  T* ring_rows = (lane < 16 ? k_local : v_local) + lbase + 8 * sub;
  float nx[8];
  load8((lane < 16 ? k_new : v_new) + (size_t)s * kHeadDim + 8 * sub, nx);

  bool evict, room = true, opens = false;
  int a, len, unit;
  int32_t* st = nullptr;
  int n_units = 0, win_first = 0, head = 0, count = 0, overflow = 0;
  if constexpr (kSeg) {
    st = state + s * (kRing + window);
    n_units = st[kNUnits];
    win_first = st[kWinFirst];
    head = st[kHead];
    count = st[kCount];
    overflow = st[kOverflow];
    const int32_t* ring = st + kRing;
    const bool fired = fire && fire[s / n_kv_heads] != 0;
    const int open_first = count > 0 ? ring[(head + count - 1) % window] : -1;
    opens = count == 0 || fired || step - open_first >= seg_len;
    evict = step - win_first >= window && count > 0;
    a = evict ? ring[head] : 0;
    len = evict ? (count > 1 ? ring[(head + 1) % window] : step) - a : 0;
    unit = n_units;
    room = n_units < units_cap && (!codes || (int64_t)prompt_len + a + len <= pool_rows);
    __syncthreads();   // every thread has read the state before one rewrites it
  } else {
    evict = evict_seg >= 0;
    a = evict ? evict_seg * seg_len : 0;
    len = evict ? seg_len : 0;
    unit = n_clusters + evict_seg;
  }
  if (evict) {
    const int64_t prow = (int64_t)prompt_len + a;
    double sum[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) sum[e] = 0.0;
    for (int r = rg; r < len; r += 8) {
      float x[8];
      load8(ring_rows + (size_t)((a + r) % window) * kHeadDim, x);
#pragma unroll
      for (int e = 0; e < 8; ++e) sum[e] += (double)x[e];
      if (codes && room) {
        uint32_t byte;
        const uint32_t c = quantise8(x, byte);
        const size_t row = (size_t)s * pool_rows + prow + r;
        *reinterpret_cast<uint32_t*>(codes + row * kCodeBytes + 4 * lane) = c;
        if ((lane & 3) == 0) scales[row * kScaleBytes + (lane >> 2)] = (uint8_t)byte;
      }
    }
    if (lane < 16) {
#pragma unroll
      for (int e = 0; e < 8; ++e) s_sum[rg][8 * sub + e] = sum[e];
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (room && tid < kHeadDim) {
      double t = 0.0;
#pragma unroll
      for (int g = 0; g < 8; ++g) t += s_sum[g][tid];
      reps[((size_t)s * units_cap + unit) * kHeadDim + tid] = (float)(t / (double)len);
    }
    if (room && tid == 0) {
      unit_start[s * units_cap + unit] = (int32_t)prow;
      unit_size[s * units_cap + unit] = len;
    }
  }
  if (rg == 0) {
    T* p = ring_rows + (size_t)(step % window) * kHeadDim;
    if constexpr (sizeof(T) == 2) store8(reinterpret_cast<uint16_t*>(p), nx);
    else store8(reinterpret_cast<float*>(p), nx);
  }
  if constexpr (kSeg) {
    if (tid == 0) {
      if (evict) {
        if (room) ++n_units;
        else overflow = 1;   // no room for the unit: its tokens are no longer attended
        head = (head + 1) % window;
        --count;
        win_first = a + len;
      }
      if (opens) {
        st[kRing + (head + count) % window] = step;
        ++count;
      }
      st[kNUnits] = n_units;
      st[kWinFirst] = win_first;
      st[kHead] = head;
      st[kCount] = count;
      st[kOverflow] = overflow;
    }
  }
}

// ------------------------------------------------------------------ decode attention

struct AttnQ4 {
  const void* q;
  float scale;
  const uint8_t* codes;
  const uint8_t* scales;
  int64_t pool_rows;
  const int32_t* rows;
  const int32_t* n_sel;
  int budget;
  const void* k_local;
  const void* v_local;
  int window, local_start, n_local;
  const int32_t* seg_state;
  int n_tokens;
  int n_chunks;
  float* part;
  void* out;
  int out_bf16;
  float* lse_out;
};

// Window of slice s: the arguments, or with a segment state its own tokens from
// its first to n_tokens - 1.
__device__ __forceinline__ void window_of(const AttnQ4& a, int64_t s, int& start, int& n) {
  start = a.local_start;
  n = a.n_local;
  if (!a.seg_state) return;
  const int first = a.seg_state[s * (kRing + a.window) + kWinFirst];
  n = min(max(a.n_tokens - first, 0), a.window);
  start = first >= 0 ? first % a.window : 0;
}

// The waves' maxima, sums and weighted sums of a block to its output rows, or to
// its partials where a slice has several blocks.
template <int G, int NW>
__device__ __forceinline__ void merge_waves(const AttnQ4& a, const float (*s_m)[G], const float (*s_l)[G],
                                            const float (*s_acc)[G][kHeadDim], int64_t s, int chunk, int tid) {
  for (int i = tid; i < G * kHeadDim; i += NW * 64) {
    const int j = i / kHeadDim, k = i % kHeadDim;
    float mm = -__builtin_inff();
#pragma unroll
    for (int x = 0; x < NW; ++x) mm = fmaxf(mm, s_m[x][j]);
    const float base = max_base(mm);
    float ll = 0.f, o = 0.f;
#pragma unroll
    for (int x = 0; x < NW; ++x) {
      const float c = __builtin_amdgcn_exp2f(s_m[x][j] - base);
      ll += s_l[x][j] * c;
      o += s_acc[x][j][k] * c;
    }
    const size_t row = (size_t)s * G + j;
    if (a.n_chunks > 1) {
      float* p = a.part + (row * a.n_chunks + chunk) * kPartFloats;
      p[2 + k] = o;
      if (k == 0) {
        p[0] = mm;
        p[1] = ll;
      }
      continue;
    }
    o *= inv_sum(ll);
    if (a.out_bf16) static_cast<uint16_t*>(a.out)[row * kHeadDim + k] = f32_to_bf16(o);
    else static_cast<float*>(a.out)[row * kHeadDim + k] = o;
    if (a.lse_out && k == 0) a.lse_out[row] = lse_of(mm, ll);
  }
}

// ---- float32: vector ALUs

// a's lower and b's upper halves (32) of the wave, or even and odd quarters (16), are
// added to the others: a's sums in the lower half (even quarters), b's in the upper.
template <int kLanes>
__device__ __forceinline__ float swap_add(float a, float b) {
  typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
  u32x2 r;
  if constexpr (kLanes == 32) r = __builtin_amdgcn_permlane32_swap(__float_as_uint(a), __float_as_uint(b), false, false);
  else r = __builtin_amdgcn_permlane16_swap(__float_as_uint(a), __float_as_uint(b), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// Block (slice, chunk): softmax over the chunk's share of the slice's rows, one
// pass, 16 lanes a row (lane sub owns channels 8 sub..+7), four rows of a group on
// their way.  Every 16-lane group keeps its own running maximum, sum and weighted
// sum; they are joined at the end.  Two rows share a rescale (one each: 256 slices of
// 2148 rows, 4 heads, 71 us; two 48; four 47, but more idle work where rows are few).
// Bound by the vector ALUs, 27 operations a row and head and lane, where there are many
// rows; by trips to memory where few (8 slices of 1300 rows, 8 heads: 12.1 us with the
// merge; the wave's groups joined by shuffles 17.5).
constexpr int kAttnWaves = 8;

template <int G>
__global__ __launch_bounds__(kAttnWaves * 64)
void attn_q4_kernel(const AttnQ4 a) {
  constexpr int kGroups = kAttnWaves * 4;
  __shared__ float s_m[kAttnWaves][G], s_l[kAttnWaves][G];
  __shared__ __align__(16) float s_acc[kAttnWaves][G][kHeadDim];
  const int64_t s = blockIdx.x / a.n_chunks;
  const int chunk = (int)(blockIdx.x - s * a.n_chunks);
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, sub = tid & 15, grp = tid >> 4;
  int local_start, n_local;
  window_of(a, s, local_start, n_local);
  const int nsel = max(0, min(a.n_sel[s], a.budget));
  const int total = nsel + n_local;
  const int r0 = (int)((int64_t)total * chunk / a.n_chunks), r1 = (int)((int64_t)total * (chunk + 1) / a.n_chunks);
  const float qs = a.scale * kLog2E;
  float q[G][8];
#pragma unroll
  for (int j = 0; j < G; ++j) {
    load8(static_cast<const float*>(a.q) + ((size_t)s * G + j) * kHeadDim + 8 * sub, q[j]);
#pragma unroll
    for (int e = 0; e < 8; ++e) q[j][e] *= qs;
  }
  float m[G], l[G], acc[G][8];
#pragma unroll
  for (int j = 0; j < G; ++j) {
    m[j] = -__builtin_inff();
    l[j] = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[j][e] = 0.f;
  }
  // Two of a group's rows, of which n are there (the other repeats one of them): their
  // scores, one rescale for both, and their values.
  auto attend = [&](const float (&k)[2][8], const float (&v)[2][8], int n) {
#pragma unroll
    for (int j = 0; j < G; ++j) {
      float p[2], mn = m[j];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        float d = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) d = fmaf(q[j][e], k[u][e], d);
        p[u] = u < n ? row16_add(d) : -__builtin_inff();
        mn = fmaxf(mn, p[u]);
      }
      const float base = max_base(mn), c = __builtin_amdgcn_exp2f(m[j] - base);
      m[j] = mn;
      l[j] *= c;
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[j][e] *= c;
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const float y = __builtin_amdgcn_exp2f(p[u] - base);
        l[j] += y;
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[j][e] = fmaf(y, v[u][e], acc[j][e]);
      }
    }
  };
  // kRows of a group's rows are on their way together: list entries, then codes
  constexpr int kRows = 4;
  const int p1 = min(r1, nsel);
  for (int r = r0 + grp; r < p1; r += kRows * kGroups) {
    size_t row[kRows];
#pragma unroll
    for (int u = 0; u < kRows; ++u)
      row[u] = (size_t)s * a.pool_rows +
               min<int64_t>(max(a.rows[(size_t)s * a.budget + min(r + u * kGroups, p1 - 1)], 0), a.pool_rows - 1);
    uint32_t kc[kRows], vc[kRows], ks[kRows], vs[kRows];
#pragma unroll
    for (int u = 0; u < kRows; ++u) {
      kc[u] = *reinterpret_cast<const uint32_t*>(a.codes + row[u] * kCodeBytes + 4 * sub);
      vc[u] = *reinterpret_cast<const uint32_t*>(a.codes + row[u] * kCodeBytes + 64 + 4 * sub);
      ks[u] = a.scales[row[u] * kScaleBytes + (sub >> 2)];
      vs[u] = a.scales[row[u] * kScaleBytes + 4 + (sub >> 2)];
    }
    const int n = (p1 - r + kGroups - 1) / kGroups;
#pragma unroll
    for (int u = 0; u < kRows; u += 2) {
      if (u >= n) break;
      float k[2][8], v[2][8];
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        expand8(kc[u + x], scale_of(ks[u + x]), k[x]);
        expand8(vc[u + x], scale_of(vs[u + x]), v[x]);
      }
      attend(k, v, n - u);
    }
  }
  for (int r = max(r0, nsel) + grp; r < r1; r += 2 * kGroups) {
    float k[2][8], v[2][8];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      int slot = local_start + (min(r + u * kGroups, r1 - 1) - nsel);
      slot -= slot >= a.window ? a.window : 0;
      const size_t o = ((size_t)s * a.window + slot) * kHeadDim + 8 * sub;
      load8(static_cast<const float*>(a.k_local) + o, k[u]);
      load8(static_cast<const float*>(a.v_local) + o, v[u]);
      // a repeated row weighs 0, and 0 times an infinity would be NaN
#pragma unroll
      for (int e = 0; e < 8; ++e) v[u][e] = r + u * kGroups < r1 ? v[u][e] : 0.f;
    }
    attend(k, v, (r1 - r + kGroups - 1) / kGroups);
  }
  // the wave's four groups, then its totals into LDS
#pragma unroll
  for (int j = 0; j < G; ++j) {
    float mm = fmaxf(m[j], __shfl_xor(m[j], 16, kWave));
    mm = fmaxf(mm, __shfl_xor(mm, 32, kWave));
    const float c = __builtin_amdgcn_exp2f(m[j] - max_base(mm));
    float ll = l[j] * c;
    ll += __shfl_xor(ll, 16, kWave);
    ll += __shfl_xor(ll, 32, kWave);
    // halves, then quarters of the wave change places with another channel's: what is
    // left of eight sums over four lanes is channels 2 h and 2 h + 1 in lane 16 h + sub
    float x[4], y[2];
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = swap_add<32>(acc[j][e] * c, acc[j][e + 4] * c);
#pragma unroll
    for (int e = 0; e < 2; ++e) y[e] = swap_add<16>(x[e], x[e + 2]);
    *reinterpret_cast<float2*>(&s_acc[w][j][8 * sub + 2 * (lane >> 4)]) = make_float2(y[0], y[1]);
    if (lane == 0) {
      s_m[w][j] = mm;
      s_l[w][j] = ll;
    }
  }
  __syncthreads();
  merge_waves<G, kAttnWaves>(a, s_m, s_l, s_acc, s, chunk, tid);
}

// ---- bf16: matrix cores

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

// The eight channels of a code word as four bfloat16 pairs.
__device__ __forceinline__ uint4 expand8_bf16(uint32_t c, float scale) {
  uint4 v;
  v.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 0));
  v.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 1));
  v.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 2));
  v.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 3));
  return v;
}

constexpr float kGrow = 8.0f;   // base-2 logits may pass the base by this much before the sums are rescaled

// Block (slice, chunk), eight waves, each with tiles of 32 rows.  Lane (c = l % 16,
// h = l / 16).
//   scores  S^T = K Q^T, 16 rows at a time: the lane holds 32 channels (a block of
//           the format, one scale) of key row c as the A operand, and as the B
//           operand the same channels of head c % G, so that it receives the
//           scores of head c for rows 4 h + 0..3 and 16 + 4 h + 0..3.
//   values  O = P V: those eight weights, unmoved, are the lane's part of the A
//           operand (k index = its eight rows), and its part of the B operand is
//           one channel of the same eight rows.  It has word c (eight channels, in
//           one block of the format) of each of them; the i-th channel of all of
//           them, paired by byte permutes, is the operand of the i-th product, whose
//           columns are channels 8 c + i.
// Rows are loaded 16 bytes a lane, five loads a tile; the values' words and the
// scales change lanes through LDS (loaded where they are used, in twenty loads of
// 1 and 4 bytes, the time was the same).  The second product takes a weight as the sum
// of two bfloat16, off by 2^-16 of it at most: rows c < 8 of its A operand hold the
// weights of head c % G rounded to bfloat16, rows c + 8, whose heads are the same, what
// that rounding left, and the two results are added at the end.  The rounded weights
// alone (off by 2^-8, when the row-list attention over a full-precision pool has them in
// float32) would save 0.6 us of the time below.  The sum is of the unrounded ones.
// 256 slices of 2148 rows, 4 heads (86.5 MB): 20.6 us, 4.2 TB/s; of 4196 rows 32.9 us, so
// that some 8 us pass before the first rows arrive and after the last and the others come
// at 6.0 TB/s; of 8292 rows (307 MB, more than the last cache holds) 67 us.  Sixteen waves
// a block spill (61 us for 20.0, with the weights rounded once), the list staged in LDS
// is no faster (20.7).
template <int G>
__global__ __launch_bounds__(kAttnWaves * 64)
void attn_q4_mfma_kernel(const AttnQ4 a) {
  constexpr int NW = kAttnWaves;
  __shared__ float s_m[NW][G], s_l[NW][G];
  __shared__ __align__(16) float s_acc[NW][G][kHeadDim];
  __shared__ __align__(16) uint32_t s_v[NW][32 * 16 + 7 * 16], s_sc[NW][64];
  // word of a tile's row in s_v: 16 more after every four rows, so that a read of
  // rows 4 h + j by the four groups of lanes falls into different banks
  auto value_word = [](int r) { return r * 16 + (r >> 2) * 16; };
  const int64_t s = blockIdx.x / a.n_chunks;
  const int chunk = (int)(blockIdx.x - s * a.n_chunks);
  const int tid = threadIdx.x, lane = tid & 63, c = lane & 15, h = lane >> 4;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  int local_start, n_local;
  window_of(a, s, local_start, n_local);
  const int nsel = max(0, min(a.n_sel[s], a.budget));
  const int total = nsel + n_local;
  const int r0 = (int)((int64_t)total * chunk / a.n_chunks), r1 = (int)((int64_t)total * (chunk + 1) / a.n_chunks);
  const int p1 = min(r1, nsel), n_pool = max(p1 - r0, 0);               // pool rows r0..p1-1 of the chunk
  const int w0 = max(r0, nsel) - nsel, n_win = max(r1 - max(r0, nsel), 0);   // window rows w0.. of it
  const int n_pool_tiles = (n_pool + 31) / 32, n_win_tiles = (n_win + 31) / 32;

  bf16x8 q[4];
  const float qs = a.scale * kLog2E, mult = fabsf(qs);
  const uint32_t flip = qs < 0.f ? 0x80008000u : 0u;                    // |scale| multiplies the scores of -q
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    uint4 v = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(a.q) + ((size_t)s * G + c % G) * kHeadDim +
                                              32 * h + 8 * k);
    v.x ^= flip; v.y ^= flip; v.z ^= flip; v.w ^= flip;
    q[k] = __builtin_bit_cast(bf16x8, v);
  }
  const float rest = c < 8 ? 0.f : 1.f;                                 // this row's part of a weight: p - rest * rounded p
  float base = 0.f, grow_at = -__builtin_inff(), sum = 0.f;
  f32x4 o[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) o[i] = f32x4{0.f, 0.f, 0.f, 0.f};

  const uint8_t* codes = a.codes + (size_t)s * a.pool_rows * kCodeBytes;
  const uint8_t* scales = a.scales + (size_t)s * a.pool_rows * kScaleBytes;
  // A tile as it is loaded: 32 channels of rows c and 16 + c, and the four scales of
  // the keys (lanes 0..31) or values of row l % 32.
  struct Raw {
    uint4 k[2], v[2];
    uint32_t scale;
  };
  const uint8_t* kc = codes + 16 * h;
  const uint8_t* sc4 = scales + 4 * (lane >> 5);
  static_assert(kCodeBytes == 16 * kScaleBytes, "a row's scales are at a sixteenth of its codes' offset");
  // byte offsets of the codes of rows c, 16 + c and l % 32 of tile t; a row behind
  // the chunk's last is that one
  struct Rows { uint32_t at[2], own; };
  const int32_t* list = a.rows + (size_t)s * a.budget + r0;
  auto find = [&](int t, Rows& x) {
    auto row = [&](int r) {
      return (uint32_t)min(max(list[min(32 * t + r, n_pool - 1)], 0), (int)a.pool_rows - 1) * (uint32_t)kCodeBytes;
    };
    x.at[0] = row(c);
    x.at[1] = row(16 + c);
    x.own = row(lane & 31);
  };
  auto fetch = [&](const Rows& r, Raw& x) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      x.k[i] = *reinterpret_cast<const uint4*>(kc + r.at[i]);
      x.v[i] = *reinterpret_cast<const uint4*>(kc + r.at[i] + 64);
    }
    x.scale = *reinterpret_cast<const uint32_t*>(sc4 + (r.own >> 4));
  };
  // O += P V for the eight rows' values
  auto add_values = [&](const bf16x8& p, const uint4 (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      uint4 b;
      constexpr uint32_t kLow = 0x05040100, kHigh = 0x07060302;
#pragma unroll
      for (int t = 0; t < 4; ++t)
        (&b.x)[t] = __builtin_amdgcn_perm((&v[2 * t + 1].x)[i >> 1], (&v[2 * t].x)[i >> 1], i & 1 ? kHigh : kLow);
      o[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(p, __builtin_bit_cast(bf16x8, b), o[i], 0, 0, 0);
    }
  };
  // scores of 32 rows, of which n are there, and their values' pairs
  auto attend = [&](f32x4 (&sc)[2], uint4 (&v)[8], int n, bool window) {
    float m = mult;
    if (n < 32) {                                                        // wave-uniform
      m = 1.f;
#pragma unroll
      for (int j = 0; j < 8; ++j)
        sc[j >> 2][j & 3] = 16 * (j >> 2) + 4 * h + (j & 3) < n ? sc[j >> 2][j & 3] * mult : -__builtin_inff();
    }
    float top = sc[0][0];
#pragma unroll
    for (int j = 1; j < 8; ++j) top = fmaxf(top, sc[j >> 2][j & 3]);
    top *= m;
    if (__builtin_amdgcn_ballot_w64(top > grow_at)) {
      top = fmaxf(top, __shfl_xor(top, 16, kWave));
      top = fmaxf(top, __shfl_xor(top, 32, kWave));
      const bool grows = top > grow_at;
      // before the first finite score the sums are 0 (or NaN): any factor does
      const float f = grows && grow_at != -__builtin_inff() ? __builtin_amdgcn_exp2f(base - top) : 1.f;
      base = grows ? top : base;
      grow_at = grows ? top + kGrow : grow_at;
      sum *= f;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float fe = __shfl(f, 4 * h + e, kWave);                   // the factor of head 4 h + e
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i][e] *= fe;
      }
    }
    bf16x8 whole, p;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float y = __builtin_amdgcn_exp2f(fmaf(sc[j >> 2][j & 3], m, -base));
      sum += y;
      whole[j] = (__bf16)y;
      p[j] = (__bf16)fmaf(-rest, (float)whole[j], y);
    }
    if (window) {
      // What rounding left can be 0 or negative: an infinity must not meet it.  Where the
      // values hold any (0 times them is not 0), those that are not finite are added apart, by
      // the rounded weights.
      float zero[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int x = 0; x < 4; ++x)
          zero[x] = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, (&v[j].x)[x]), bf16x2{}, zero[x], false);
      const float all = (zero[0] + zero[1]) + (zero[2] + zero[3]);
      if (__builtin_amdgcn_ballot_w64(all != 0.f)) {
        uint4 apart[8];
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            uint32_t& e = (&v[j].x)[x];
            const uint32_t bad = ((e & 0x7f80u) == 0x7f80u ? 0xffffu : 0u) | ((e & 0x7f800000u) == 0x7f800000u ? 0xffff0000u : 0u);
            (&apart[j].x)[x] = e & bad;
            e &= ~bad;
          }
        add_values(whole, apart);
      }
    }
    add_values(p, v);
  };
  auto score = [&](const uint4 (&k)[4]) {
    f32x4 sc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < 4; ++i) sc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, k[i]), q[i], sc, 0, 0, 0);
    return sc;
  };

  auto tile = [&](int t, const Raw& x) {
    // through the wave's LDS: values to the lanes of their columns, scales to their rows'
#pragma unroll
    for (int i = 0; i < 2; ++i) *reinterpret_cast<uint4*>(&s_v[w][value_word(16 * i + c) + 4 * h]) = x.v[i];
    s_sc[w][lane] = x.scale;
    __builtin_amdgcn_wave_barrier();
    const uint8_t* sb = reinterpret_cast<const uint8_t*>(s_sc[w]);
    f32x4 sc[2];
    uint4 v[8];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const float f = scale_of(sb[4 * (16 * i + c) + h]);
      uint4 k[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) k[e] = expand8_bf16((&x.k[i].x)[e], f);
      sc[i] = score(k);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int r = 16 * (j >> 2) + 4 * h + (j & 3);
      v[j] = expand8_bf16(s_v[w][value_word(r) + c], scale_of(sb[128 + 4 * r + (c >> 2)]));
    }
    attend(sc, v, n_pool - 32 * t, false);
  };
  // a tile's rows are on their way while the one before is at hand, its list
  // entries while the one two before is
  Rows ra, rb;
  Raw xa, xb;
  if (w < n_pool_tiles) {
    find(w, ra);
    find(w + NW, rb);
    fetch(ra, xa);
  }
  const uint16_t* kl = static_cast<const uint16_t*>(a.k_local) + (size_t)s * a.window * kHeadDim;
  const uint16_t* vl = static_cast<const uint16_t*>(a.v_local) + (size_t)s * a.window * kHeadDim;
  // waves from the last on take the window's tiles, so that the shares even out
  for (int t = NW - 1 - w; t < n_win_tiles; t += NW) {
    auto slot = [&](int r) {
      const int y = local_start + w0 + min(32 * t + r, n_win - 1);
      return y >= a.window ? y - a.window : y;
    };
    uint4 v[8];
    f32x4 sc[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const uint4* src = reinterpret_cast<const uint4*>(kl + (size_t)slot(16 * i + c) * kHeadDim + 32 * h);
      uint4 k[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) k[e] = src[e];
      sc[i] = score(k);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j)
      v[j] = *reinterpret_cast<const uint4*>(vl + (size_t)slot(16 * (j >> 2) + 4 * h + (j & 3)) * kHeadDim + 8 * c);
    if (n_win - 32 * t < 32) {               // a repeated row weighs 0, and 0 times an infinity would be NaN
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (32 * t + 16 * (j >> 2) + 4 * h + (j & 3) >= n_win) v[j] = make_uint4(0, 0, 0, 0);
    }
    attend(sc, v, n_win - 32 * t, true);
  }
  for (int t = w; t < n_pool_tiles; t += 2 * NW) {
    if (t + NW < n_pool_tiles) fetch(rb, xb);
    if (t + 2 * NW < n_pool_tiles) find(t + 2 * NW, ra);
    __builtin_amdgcn_sched_barrier(0);
    tile(t, xa);
    if (t + NW >= n_pool_tiles) break;
    if (t + 2 * NW < n_pool_tiles) fetch(ra, xa);
    if (t + 3 * NW < n_pool_tiles) find(t + 3 * NW, rb);
    __builtin_amdgcn_sched_barrier(0);
    tile(t + NW, xb);
  }
  // the wave's sums: head c of lanes c < G, and rows 4 h + e of the channels 8 c + i.
  // Rows h and h + 2 change places with other channels': the sums of row 4 (h % 2) + e
  // are left for channels 8 c + 4 (h / 2) + 0..3.
  sum += __shfl_xor(sum, 16, kWave);
  sum += __shfl_xor(sum, 32, kWave);
  if (lane < G) {
    s_m[w][lane] = grow_at == -__builtin_inff() ? -__builtin_inff() : base;
    s_l[w][lane] = sum;
  }
#pragma unroll
  for (int e = 0; e < (G < 4 ? G : 4); ++e) {
    float x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = swap_add<32>(o[i][e], o[i + 4][e]);
    if (4 * (h & 1) < G)
      *reinterpret_cast<float4*>(&s_acc[w][4 * (h & 1) + e][8 * c + 4 * (h >> 1)]) = make_float4(x[0], x[1], x[2], x[3]);
  }
  __syncthreads();
  merge_waves<G, NW>(a, s_m, s_l, s_acc, s, chunk, tid);
}

// Chunks of a slice's rows: blocks for the chip, with the rows that a block has in
// flight at once: in bfloat16 a half tile a wave (8 slices of 2148 rows with the merge:
// 128 rows a block 8.9 us, 256 rows 9.3; 256 slices: one chunk 20.6 us, two and their
// merge 27.1), in float32 two rows a group (8 slices of 2148 rows with the merge: 64 rows
// a block 9.8 us, 128 rows 10.5).
constexpr int kTargetBlocks = 256;
int attn_q4_chunks(int64_t S, int budget, int window, int dtype) {
  const int min_rows = dtype == LOUISKV_BF16 ? 128 : 64;
  const int64_t cap = (int64_t)budget + window;
  const int64_t by_rows = std::max<int64_t>(1, (cap + min_rows - 1) / min_rows);
  const int64_t by_grid = std::max<int64_t>(1, kTargetBlocks / S);
  return (int)std::min(by_rows, by_grid);
}

void launch_attn_q4(const AttnQ4& a, int dtype, int group_size, unsigned grid, hipStream_t s) {
  if (dtype == LOUISKV_BF16) {
    switch (group_size) {
      case 1: attn_q4_mfma_kernel<1><<<grid, kAttnWaves * 64, 0, s>>>(a); break;
      case 2: attn_q4_mfma_kernel<2><<<grid, kAttnWaves * 64, 0, s>>>(a); break;
      case 4: attn_q4_mfma_kernel<4><<<grid, kAttnWaves * 64, 0, s>>>(a); break;
      default: attn_q4_mfma_kernel<8><<<grid, kAttnWaves * 64, 0, s>>>(a); break;
    }
    return;
  }
  switch (group_size) {
    case 1: attn_q4_kernel<1><<<grid, kAttnWaves * 64, 0, s>>>(a); break;
    case 2: attn_q4_kernel<2><<<grid, kAttnWaves * 64, 0, s>>>(a); break;
    case 4: attn_q4_kernel<4><<<grid, kAttnWaves * 64, 0, s>>>(a); break;
    default: attn_q4_kernel<8><<<grid, kAttnWaves * 64, 0, s>>>(a); break;
  }
}

int check_dtype(int dtype) {
  if (dtype != LOUISKV_F32 && dtype != LOUISKV_BF16) return fail(LOUISKV_ERR_DTYPE, "unknown dtype %d", dtype);
  return LOUISKV_OK;
}

int check_pool(const void* codes, const void* scales, int64_t pool_rows) {
  if (((uintptr_t)codes & 15) || ((uintptr_t)scales & 7))
    return fail(LOUISKV_ERR_UNSUPPORTED, "codes must be 16-byte and scales 8-byte aligned");
  if (pool_rows < 1 || pool_rows > LOUISKV_Q4_MAX_POOL_ROWS)
    return fail(LOUISKV_ERR_SHAPE, "pool_rows=%lld must be in [1, %d]", (long long)pool_rows, LOUISKV_Q4_MAX_POOL_ROWS);
  return LOUISKV_OK;
}

// Blocks of a launch over chunks of rows: one a chunk, as far as a launch holds them.
unsigned chunk_grid(int64_t n_chunks) { return (unsigned)std::min(n_chunks, kMaxGrid); }

int store_q4(const void* k_new, const void* v_new, int32_t dtype, int64_t n_slices, void* k_local, void* v_local,
             int32_t window, int32_t step, int32_t seg_len, int32_t evict, const uint8_t* fire, int32_t n_kv_heads,
             int32_t* seg_state, float* reps, int32_t* unit_start, int32_t* unit_size, int32_t units_cap,
             int32_t n_clusters, uint8_t* codes, uint8_t* scales, int64_t pool_rows, int32_t prompt_len,
             hipStream_t s) {
  auto launch = [&](auto kernel, auto type) {
    using T = decltype(type);
    kernel<<<(unsigned)n_slices, 256, 0, s>>>(
        static_cast<const T*>(k_new), static_cast<const T*>(v_new), static_cast<T*>(k_local), static_cast<T*>(v_local),
        window, step, seg_len, evict, fire, n_kv_heads, seg_state, reps, unit_start, unit_size, units_cap, n_clusters,
        codes, scales, pool_rows, prompt_len);
  };
  if (dtype == LOUISKV_BF16) {
    if (seg_state) launch(store_q4_kernel<uint16_t, true>, uint16_t{});
    else launch(store_q4_kernel<uint16_t, false>, uint16_t{});
  } else {
    if (seg_state) launch(store_q4_kernel<float, true>, float{});
    else launch(store_q4_kernel<float, false>, float{});
  }
  LKV_CHECK_LAUNCH();
  return LOUISKV_OK;
}

int attn_q4(const void* q, int32_t dtype, int64_t n_slices, int32_t n_kv_heads, int32_t group_size, int32_t d,
            float scale, const uint8_t* codes, const uint8_t* scales, int64_t pool_rows, const int32_t* sel_rows,
            const int32_t* n_sel, int32_t budget, const void* k_local, const void* v_local, int32_t window,
            int32_t local_start, int32_t n_local, const int32_t* seg_state, int32_t n_tokens, void* out,
            int32_t out_dtype, float* lse_out, void* workspace, size_t workspace_bytes, void* stream) {
  if (!q || !out || !n_sel) return fail(LOUISKV_ERR_NULL, "q, out and n_sel are required");
  if (budget > 0 && (!codes || !scales || !sel_rows))
    return fail(LOUISKV_ERR_NULL, "codes, scales and sel_rows required when budget > 0");
  if (n_local > 0 && (!k_local || !v_local)) return fail(LOUISKV_ERR_NULL, "k_local/v_local required when n_local > 0");
  int st = check_dtype(dtype);
  if (st || (st = check_dtype(out_dtype))) return st;
  if (d != kHeadDim) return fail(LOUISKV_ERR_UNSUPPORTED, "head dim %d not supported (only 128)", d);
  if (!aligned16(q, k_local, v_local)) return fail(LOUISKV_ERR_UNSUPPORTED, "q, k_local and v_local must be 16-byte aligned");
  if (n_kv_heads < 1 || n_slices < 1 || n_slices % n_kv_heads != 0)
    return fail(LOUISKV_ERR_SHAPE, "n_slices=%lld must be a positive multiple of n_kv_heads=%d", (long long)n_slices,
                n_kv_heads);
  if (group_size != 1 && group_size != 2 && group_size != 4 && group_size != 8)
    return fail(LOUISKV_ERR_UNSUPPORTED, "group_size=%d must be 1, 2, 4 or 8", group_size);
  if (budget < 0 || window < 0 || n_local < 0 || n_local > window ||
      (window > 0 && (local_start < 0 || local_start >= window)))
    return fail(LOUISKV_ERR_SHAPE, "budget=%d window=%d local_start=%d n_local=%d", budget, window, local_start, n_local);
  if (budget > 0 && (st = check_pool(codes, scales, pool_rows))) return st;
  const int n_chunks = attn_q4_chunks(n_slices, budget, window, dtype);
  if (n_slices > kMaxGrid || (int64_t)budget + window > LOUISKV_Q4_MAX_POOL_ROWS * 2)
    return fail(LOUISKV_ERR_SHAPE, "problem too large for one launch");
  const size_t need = louiskv_sparse_decode_attn_rows_q4_workspace_size(n_slices, group_size, d, budget, window);
  if (need > 0 && (!workspace || workspace_bytes < need || !aligned16(workspace)))
    return fail(LOUISKV_ERR_WORKSPACE, "workspace needs %zu bytes, 16-byte aligned, got %zu", need, workspace_bytes);
  AttnQ4 a;
  a.q = q; a.scale = scale; a.codes = codes; a.scales = scales; a.pool_rows = pool_rows;
  a.rows = sel_rows; a.n_sel = n_sel; a.budget = budget; a.k_local = k_local; a.v_local = v_local;
  a.window = std::max(window, 1); a.local_start = window > 0 ? local_start : 0; a.n_local = n_local;
  a.seg_state = seg_state; a.n_tokens = n_tokens; a.n_chunks = n_chunks; a.part = static_cast<float*>(workspace);
  a.out = out; a.out_bf16 = out_dtype == LOUISKV_BF16; a.lse_out = lse_out;
  const unsigned grid = (unsigned)(n_slices * n_chunks);
  hipStream_t s = as_stream(stream);
  launch_attn_q4(a, dtype, group_size, grid, s);
  LKV_CHECK_LAUNCH();
  if (n_chunks == 1) return LOUISKV_OK;
  return merge_parts(a.part, n_chunks, n_slices * group_size, out, out_dtype, lse_out, s);
}

}  // namespace
}  // namespace louiskv

using namespace louiskv;

extern "C" int louiskv_pack_pool_q4(const void* keys, const void* values, int32_t dtype, int64_t n_slices,
                                    int32_t n_tokens, int32_t d, const int32_t* perm, uint8_t* codes, uint8_t* scales,
                                    int64_t pool_rows, void* stream) {
  if (!keys || !values || !codes || !scales) return fail(LOUISKV_ERR_NULL, "keys, values, codes, scales required");
  int st = check_dtype(dtype);
  if (st) return st;
  if (d != kHeadDim) return fail(LOUISKV_ERR_UNSUPPORTED, "head dim %d not supported (only 128)", d);
  if (!aligned16(keys, values)) return fail(LOUISKV_ERR_UNSUPPORTED, "keys and values must be 16-byte aligned");
  if (n_slices < 1 || n_slices > INT32_MAX || n_tokens < 1)
    return fail(LOUISKV_ERR_SHAPE, "n_slices=%lld n_tokens=%d", (long long)n_slices, n_tokens);
  if ((st = check_pool(codes, scales, pool_rows))) return st;
  if (pool_rows < n_tokens)
    return fail(LOUISKV_ERR_SHAPE, "pool_rows=%lld < n_tokens=%d", (long long)pool_rows, n_tokens);
  const int per = (n_tokens + kRowsPerChunk - 1) / kRowsPerChunk;
  const int64_t n = n_slices * per;
  if (dtype == LOUISKV_BF16)
    pack_q4_kernel<uint16_t><<<chunk_grid(n), 256, 0, as_stream(stream)>>>(
        static_cast<const uint16_t*>(keys), static_cast<const uint16_t*>(values), perm, n_tokens, n, per, codes,
        scales, pool_rows);
  else
    pack_q4_kernel<float><<<chunk_grid(n), 256, 0, as_stream(stream)>>>(
        static_cast<const float*>(keys), static_cast<const float*>(values), perm, n_tokens, n, per, codes, scales,
        pool_rows);
  LKV_CHECK_LAUNCH();
  return LOUISKV_OK;
}

extern "C" int louiskv_gather_rows_q4(const uint8_t* codes, const uint8_t* scales, int64_t n_slices, int64_t pool_rows,
                                      int32_t d, const int32_t* sel_rows, const int32_t* n_sel, int32_t buf_rows,
                                      void* k_buf, void* v_buf, int32_t dtype, void* stream) {
  if (!codes || !scales || !k_buf || !v_buf) return fail(LOUISKV_ERR_NULL, "codes, scales, k_buf, v_buf required");
  int st = check_dtype(dtype);
  if (st) return st;
  if (d != kHeadDim) return fail(LOUISKV_ERR_UNSUPPORTED, "head dim %d not supported (only 128)", d);
  if (!aligned16(k_buf, v_buf)) return fail(LOUISKV_ERR_UNSUPPORTED, "k_buf and v_buf must be 16-byte aligned");
  if (n_slices < 1 || n_slices > INT32_MAX || buf_rows < 1)
    return fail(LOUISKV_ERR_SHAPE, "n_slices=%lld buf_rows=%d", (long long)n_slices, buf_rows);
  if ((st = check_pool(codes, scales, pool_rows))) return st;
  if (!sel_rows && buf_rows > pool_rows)
    return fail(LOUISKV_ERR_SHAPE, "buf_rows=%d > pool_rows=%lld", buf_rows, (long long)pool_rows);
  const int per = (int)(((int64_t)buf_rows + kRowsPerChunk - 1) / kRowsPerChunk);
  const int64_t n = n_slices * per;
  if (dtype == LOUISKV_BF16)
    gather_q4_kernel<uint16_t><<<chunk_grid(n), 256, 0, as_stream(stream)>>>(
        codes, scales, pool_rows, sel_rows, n_sel, buf_rows, n, per, static_cast<uint16_t*>(k_buf),
        static_cast<uint16_t*>(v_buf));
  else
    gather_q4_kernel<float><<<chunk_grid(n), 256, 0, as_stream(stream)>>>(
        codes, scales, pool_rows, sel_rows, n_sel, buf_rows, n, per, static_cast<float*>(k_buf),
        static_cast<float*>(v_buf));
  LKV_CHECK_LAUNCH();
  return LOUISKV_OK;
}

extern "C" int louiskv_segment_output_q4(const void* k_new, const void* v_new, int32_t dtype, int64_t n_slices,
                                         int32_t d, void* k_local, void* v_local, int32_t window, int32_t step,
                                         int32_t seg_len, float* reps, int32_t* unit_start, int32_t* unit_size,
                                         int32_t units_cap, int32_t n_clusters, uint8_t* codes, uint8_t* scales,
                                         int64_t pool_rows, int32_t prompt_len, void* stream) {
  if (!k_new || !v_new || !k_local || !v_local) return fail(LOUISKV_ERR_NULL, "k_new, v_new, k_local, v_local required");
  if (!codes != !scales) return fail(LOUISKV_ERR_NULL, "codes and scales go together");
  int st = check_dtype(dtype);
  if (st) return st;
  if (d != kHeadDim) return fail(LOUISKV_ERR_UNSUPPORTED, "head dim %d not supported (only 128)", d);
  if (!aligned16(k_new, v_new, k_local, v_local))
    return fail(LOUISKV_ERR_UNSUPPORTED, "k_new, v_new, k_local and v_local must be 16-byte aligned");
  if (n_slices < 1 || n_slices > kMaxGrid) return fail(LOUISKV_ERR_SHAPE, "n_slices=%lld", (long long)n_slices);
  if (codes && (st = check_pool(codes, scales, pool_rows))) return st;
  int32_t ev = -1;
  if ((st = louiskv_window_info(step, window, seg_len, &ev, nullptr, nullptr, nullptr))) return st;
  if (ev >= 0) {
    if (!reps || !unit_start || !unit_size) return fail(LOUISKV_ERR_NULL, "unit tables required for an eviction");
    if (n_clusters < 0 || (int64_t)n_clusters + ev >= units_cap)
      return fail(LOUISKV_ERR_SHAPE, "unit %lld exceeds units_cap=%d", (long long)n_clusters + ev, units_cap);
    if (prompt_len < 0 || (codes && (int64_t)prompt_len + (int64_t)(ev + 1) * seg_len > pool_rows))
      return fail(LOUISKV_ERR_SHAPE, "segment rows exceed pool_rows=%lld", (long long)pool_rows);
  }
  return store_q4(k_new, v_new, dtype, n_slices, k_local, v_local, window, step, seg_len, ev, nullptr, 1, nullptr, reps,
                  unit_start, unit_size, units_cap, n_clusters, codes, scales, pool_rows, prompt_len,
                  as_stream(stream));
}

extern "C" int louiskv_segment_output_boundary_q4(const void* k_new, const void* v_new, int32_t dtype,
                                                  int64_t n_slices, int32_t n_kv_heads, int32_t d, void* k_local,
                                                  void* v_local, int32_t window, int32_t step, int32_t seg_max,
                                                  const uint8_t* fire, int32_t* seg_state, float* reps,
                                                  int32_t* unit_start, int32_t* unit_size, int32_t units_cap,
                                                  int32_t n_clusters, uint8_t* codes, uint8_t* scales,
                                                  int64_t pool_rows, int32_t prompt_len, void* stream) {
  if (!k_new || !v_new || !k_local || !v_local || !seg_state)
    return fail(LOUISKV_ERR_NULL, "k_new, v_new, k_local, v_local and seg_state are required");
  if (!reps || !unit_start || !unit_size) return fail(LOUISKV_ERR_NULL, "unit tables are required");
  if (!codes != !scales) return fail(LOUISKV_ERR_NULL, "codes and scales go together");
  int st = check_dtype(dtype);
  if (st) return st;
  if (d != kHeadDim) return fail(LOUISKV_ERR_UNSUPPORTED, "head dim %d not supported (only 128)", d);
  if (!aligned16(k_new, v_new, k_local, v_local))
    return fail(LOUISKV_ERR_UNSUPPORTED, "k_new, v_new, k_local and v_local must be 16-byte aligned");
  if (n_kv_heads < 1 || n_slices < 1 || n_slices % n_kv_heads != 0 || n_slices > kMaxGrid)
    return fail(LOUISKV_ERR_SHAPE, "n_slices=%lld must be a positive multiple of n_kv_heads=%d", (long long)n_slices,
                n_kv_heads);
  if (window < 2 || seg_max < 1 || seg_max >= window)
    return fail(LOUISKV_ERR_SHAPE, "need 1 <= seg_max=%d < window=%d", seg_max, window);
  if (step < 0) return fail(LOUISKV_ERR_SHAPE, "step=%d < 0", step);
  if (n_clusters < 1 || n_clusters > units_cap)
    return fail(LOUISKV_ERR_SHAPE, "n_clusters=%d must be in [1, units_cap=%d]", n_clusters, units_cap);
  if (codes && (st = check_pool(codes, scales, pool_rows))) return st;
  if (prompt_len < 0 || (codes && pool_rows < prompt_len))
    return fail(LOUISKV_ERR_SHAPE, "prompt_len=%d pool_rows=%lld", prompt_len, (long long)pool_rows);
  return store_q4(k_new, v_new, dtype, n_slices, k_local, v_local, window, step, seg_max, -1, fire, n_kv_heads,
                  seg_state, reps, unit_start, unit_size, units_cap, n_clusters, codes, scales, pool_rows, prompt_len,
                  as_stream(stream));
}

extern "C" size_t louiskv_sparse_decode_attn_rows_q4_workspace_size(int64_t n_slices, int32_t group_size, int32_t d,
                                                                    int32_t budget, int32_t window) {
  (void)d;
  if (n_slices < 1 || n_slices > kMaxGrid || group_size < 1 || group_size > 8 || budget < 0 || window < 0) return 0;
  const int parts = std::max(attn_q4_chunks(n_slices, budget, window, LOUISKV_BF16),
                             attn_q4_chunks(n_slices, budget, window, LOUISKV_F32));
  return part_bytes(n_slices * group_size, parts);
}

extern "C" int louiskv_sparse_decode_attn_rows_q4(const void* q, int32_t dtype, int64_t n_slices, int32_t n_kv_heads,
                                                  int32_t group_size, int32_t d, float scale, const uint8_t* codes,
                                                  const uint8_t* scales, int64_t pool_rows, const int32_t* sel_rows,
                                                  const int32_t* n_sel, int32_t budget, const void* k_local,
                                                  const void* v_local, int32_t window, int32_t local_start,
                                                  int32_t n_local, void* out, int32_t out_dtype, float* lse_out,
                                                  void* workspace, size_t workspace_bytes, void* stream) {
  return attn_q4(q, dtype, n_slices, n_kv_heads, group_size, d, scale, codes, scales, pool_rows, sel_rows, n_sel,
                 budget, k_local, v_local, window, local_start, n_local, nullptr, 0, out, out_dtype, lse_out,
                 workspace, workspace_bytes, stream);
}

extern "C" int louiskv_sparse_decode_attn_rows_q4_seg(const void* q, int32_t dtype, int64_t n_slices,
                                                      int32_t n_kv_heads, int32_t group_size, int32_t d, float scale,
                                                      const uint8_t* codes, const uint8_t* scales, int64_t pool_rows,
                                                      const int32_t* sel_rows, const int32_t* n_sel, int32_t budget,
                                                      const void* k_local, const void* v_local, int32_t window,
                                                      const int32_t* seg_state, int32_t n_tokens, void* out,
                                                      int32_t out_dtype, float* lse_out, void* workspace,
                                                      size_t workspace_bytes, void* stream) {
  if (!seg_state) return fail(LOUISKV_ERR_NULL, "seg_state is required");
  if (window < 2) return fail(LOUISKV_ERR_SHAPE, "window=%d must be at least 2 for segment states", window);
  if (!k_local || !v_local) return fail(LOUISKV_ERR_NULL, "k_local and v_local are required");
  if (n_tokens < 1) return fail(LOUISKV_ERR_SHAPE, "n_tokens=%d must be >= 1", n_tokens);
  return attn_q4(q, dtype, n_slices, n_kv_heads, group_size, d, scale, codes, scales, pool_rows, sel_rows, n_sel,
                 budget, k_local, v_local, window, 0, 0, seg_state, n_tokens, out, out_dtype, lse_out, workspace,
                 workspace_bytes, stream);
}
