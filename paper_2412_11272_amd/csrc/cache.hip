// Key / value caches of the token-by-token part: rows written as they come or quantised to e4m3, and read back.  The formats and
// rules are stated with the declarations in include/wf_encoder.h.
//
// Quantisation of a head's 64 values x: e = min{whole e >= -127 : max|x| <= 448 2^e}, q = round(x 2^-e) in e4m3.  A power of two keeps
// the product x 2^-e exact, so that q has one rounding (to nearest even, half a step of 2^-4 relative to the value).  A reader gets q 2^e
// exactly in fp32, and in bf16 from e = -124 on (q's smallest step is 2^-9, bf16's 2^-133; below, a bf16 reader rounds once more).  At the other end
// 256 * 2^120 would be 2^128: kMostF8 = 240 * 2^120 is the largest value that a code and an exponent stand for, and finite values end there.
#include "cache_device.h"
#include "host_runtime.h"

namespace wf {

namespace {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// Both kernels are bound by memory: a wave has one token, eight lanes a vector of 64 values, so that a load is 512 bytes of
// keys and 512 of values and a store of the 8-bit cache 512 consecutive bytes.  Up to kBatch vectors a lane are in flight before
// the first is used (20 heads: the whole token).  51 000 tokens of 20 heads between bf16 and 8 bits, 389 MB: written in 81 us, read in 73, 4.7
// and 5.2 TB/s (a copy of 4 GiB: 4.7); with a wave for each vector of 64 values it was 940 and 806.  320 tokens: 4.9 us on the GPU.
constexpr int kBatch = 5;

// The sequence of token t: the largest s with cu[s] <= t, found 64 ways at a time.  The same in all lanes.
__device__ __forceinline__ int wave_find_stream(const int32_t *cu, int B, int t) {
  const int lane = threadIdx.x & 63;
  int lo = 0, len = B;
  while (len > 1) {
    const int stride = (len + 63) >> 6, at = lane * stride;
    const int c = __popcll(__ballot(at < len && cu[lo + at] <= t));
    const int skip = c > 1 ? (c - 1) * stride : 0;
    lo += skip;
    len = stride < len - skip ? stride : len - skip;
  }
  return lo;
}

// The cache row of token t: -1 outside the cache, -2 behind the last sequence.
__device__ __forceinline__ int64_t token_row(const int32_t *cu, const int32_t *row, int B, int64_t n_rows, int t) {
  const int end = cu[B], s = wave_find_stream(cu, B, t);
  if (t >= end) return -2;
  const int64_t at = (int64_t)t - cu[s], r = row[s] + at;
  return at >= 0 && r >= 0 && r < n_rows ? r : -1;
}

// Eight values of a vector as a lane has them.
template <typename T> struct Eight { u32x4 d[sizeof(T) / 2]; };
template <typename T>
__device__ __forceinline__ Eight<T> load8(const T *p) {
  Eight<T> e;
#pragma unroll
  for (int i = 0; i < (int)sizeof(T) / 2; ++i) e.d[i] = ((const u32x4 *)p)[i];
  return e;
}
template <typename T>
__device__ __forceinline__ void store8(T *p, const Eight<T> &e) {
#pragma unroll
  for (int i = 0; i < (int)sizeof(T) / 2; ++i) ((u32x4 *)p)[i] = e.d[i];
}
__device__ __forceinline__ void to_floats(const Eight<__bf16> &e, float (&x)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t u = e.d[0][i];
    x[2 * i] = __builtin_bit_cast(float, u << 16);
    x[2 * i + 1] = __builtin_bit_cast(float, u & 0xffff0000u);
  }
}
__device__ __forceinline__ void to_floats(const Eight<float> &e, float (&x)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t u = e.d[i >> 2][i & 3];      // a bit cast of the vector's element itself reads its first
    x[i] = __builtin_bit_cast(float, u);
  }
}
__device__ __forceinline__ void from_floats(const float (&x)[8], Eight<float> &e) {
#pragma unroll
  for (int i = 0; i < 8; ++i) e.d[i >> 2][i & 3] = __builtin_bit_cast(uint32_t, x[i]);
}
__device__ __forceinline__ void from_floats(const float (&x)[8], Eight<__bf16> &e) {
  bf16x8 b;
#pragma unroll
  for (int i = 0; i < 8; ++i) b[i] = (__bf16)x[i];
  e.d[0] = __builtin_bit_cast(u32x4, b);
}

// The maximum over the eight lanes of a vector: neighbours, pairs, halves of four.
template <int CTRL>
__device__ __forceinline__ float dpp(float v) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xF, 0xF, true));
}
__device__ __forceinline__ float max_of_8_lanes(float v) {
  v = fmaxf(v, dpp<0xB1>(v));
  v = fmaxf(v, dpp<0x4E>(v));
  return fmaxf(v, dpp<0x141>(v));
}

constexpr float kMostF8 = 0x1.ep127f;

template <int CACHE> struct Stored { typedef __bf16 type; };
template <> struct Stored<WF_DTYPE_F32> { typedef float type; };

template <typename T, int CACHE>
__global__ void __launch_bounds__(256) cache_write_kernel(CacheView c, const T *k, const T *v, int64_t ld, const int32_t *cu, const int32_t *row, int B,
                                                          int n_tokens) {
  const int64_t t = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (t >= n_tokens) return;
  const int lane = threadIdx.x & 63, part = (lane & 7) * 8, units = 2 * c.n_heads;
  int64_t r = -1;
  for (int u0 = 0; u0 < units; u0 += 8 * kBatch) {
    Eight<T> x[kBatch];
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const int u = u0 + 8 * i + (lane >> 3);
      if (u < units) x[i] = load8((u & 1 ? v : k) + t * ld + (u >> 1) * 64 + part);
    }
    if (u0 == 0) {                          // behind the loads: they do not wait for it
      r = token_row(cu, row, B, c.n_rows, (int)t);
      if (r < 0) return;
    }
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const int u = u0 + 8 * i + (lane >> 3);
      if (u >= units) continue;             // whole groups of eight lanes
      if constexpr (CACHE == WF_DTYPE_F8) {
        float f[8], largest = 0.0f;
        to_floats(x[i], f);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const bool fine = (__builtin_bit_cast(uint32_t, f[e]) & 0x7f800000u) != 0x7f800000u;
          largest = fmaxf(largest, fine ? fabsf(f[e]) : 0.0f);
          f[e] = fine ? __builtin_amdgcn_fmed3f(f[e], -kMostF8, kMostF8) : __builtin_nanf("");
        }
        const uint32_t biased = f8_exponent(max_of_8_lanes(largest));
        const float factor = __builtin_bit_cast(float, (254u - biased) << 23);
        u32x2 q;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int low = __builtin_amdgcn_cvt_pk_fp8_f32(f[4 * e] * factor, f[4 * e + 1] * factor, 0, false);
          q[e] = __builtin_amdgcn_cvt_pk_fp8_f32(f[4 * e + 2] * factor, f[4 * e + 3] * factor, low, true);
        }
        *(u32x2 *)((uint8_t *)c.data + (r * units + u) * 64 + part) = q;
        if ((lane & 7) == 0) c.exps[u * c.n_rows + r] = (uint8_t)biased;
      } else {
        typedef typename Stored<CACHE>::type S;
        S *dst = (S *)c.data + (r * 2 + (u & 1)) * c.n_heads * 64 + (u >> 1) * 64 + part;
        if constexpr (sizeof(S) == sizeof(T)) {
          store8((T *)dst, x[i]);
        } else {
          float f[8];
          Eight<S> y;
          to_floats(x[i], f);
          from_floats(f, y);
          store8(dst, y);
        }
      }
    }
  }
}

template <typename T, int CACHE>
__global__ void __launch_bounds__(256) cache_read_kernel(CacheView c, T *out, const int32_t *cu, const int32_t *row, int B, int n_tokens) {
  const int64_t t = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (t >= n_tokens) return;
  const int lane = threadIdx.x & 63, part = (lane & 7) * 8, units = 2 * c.n_heads;
  const int64_t r = token_row(cu, row, B, c.n_rows, (int)t);
  if (r == -2) return;
  typedef typename Stored<CACHE>::type S;
  for (int u0 = 0; u0 < units; u0 += 8 * kBatch) {
    Eight<S> x[kBatch];
    u32x2 q[kBatch];
    uint32_t biased[kBatch];
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const int u = u0 + 8 * i + (lane >> 3);
      if (u >= units || r < 0) continue;
      if constexpr (CACHE == WF_DTYPE_F8) {
        q[i] = *(const u32x2 *)((const uint8_t *)c.data + (r * units + u) * 64 + part);
        biased[i] = c.exps[u * c.n_rows + r];
      } else {
        x[i] = load8((const S *)c.data + (r * 2 + (u & 1)) * c.n_heads * 64 + (u >> 1) * 64 + part);
      }
    }
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const int u = u0 + 8 * i + (lane >> 3);
      if (u >= units) continue;
      float f[8];
      if (r < 0) {
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = 0.0f;
      } else if constexpr (CACHE == WF_DTYPE_F8) {
        const float factor = f8_factor(biased[i]);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          f[4 * e] = __builtin_amdgcn_cvt_f32_fp8(q[i][e], 0) * factor;
          f[4 * e + 1] = __builtin_amdgcn_cvt_f32_fp8(q[i][e], 1) * factor;
          f[4 * e + 2] = __builtin_amdgcn_cvt_f32_fp8(q[i][e], 2) * factor;
          f[4 * e + 3] = __builtin_amdgcn_cvt_f32_fp8(q[i][e], 3) * factor;
        }
      } else {
        to_floats(x[i], f);
      }
      Eight<T> y;
      from_floats(f, y);
      store8(out + (t * 2 + (u & 1)) * c.n_heads * 64 + (u >> 1) * 64 + part, y);
    }
  }
}

}  // namespace

namespace host {

int check_cache(const wf_cache *c) {
  if (!c) return fail(WF_E_INVALID_ARG, "cache is NULL");
  if (c->dtype != WF_DTYPE_F32 && c->dtype != WF_DTYPE_BF16 && c->dtype != WF_DTYPE_F8) return fail(WF_E_INVALID_ARG, "cache dtype = %d", c->dtype);
  if (c->n_heads < 1 || c->n_heads > 1024) return fail(WF_E_INVALID_ARG, "cache n_heads = %d (supported: 1 .. 1024)", c->n_heads);
  if (c->n_rows < 1 || c->n_rows > INT32_MAX) return fail(WF_E_INVALID_ARG, "cache n_rows = %lld", (long long)c->n_rows);
  return WF_OK;
}

int check_cache_memory(const wf_cache *c) {
  if (!c->data_dev) return fail(WF_E_INVALID_ARG, "cache data_dev is NULL");
  if ((uintptr_t)c->data_dev % 16) return fail(WF_E_INVALID_ARG, "cache data_dev is not aligned to 16 bytes");
  if ((c->dtype == WF_DTYPE_F8) != (c->exps_dev != nullptr)) return fail(WF_E_INVALID_ARG, "exps_dev goes with WF_DTYPE_F8 and with no other type");
  return WF_OK;
}

}  // namespace host

namespace {

int check_tokens(const wf_cache *c, const int32_t *cu, const int32_t *row, int32_t dtype, int32_t B, int32_t n_tokens) {
  int rc = host::check_cache(c);
  if (rc) return rc;
  if (dtype != WF_DTYPE_F32 && dtype != WF_DTYPE_BF16) return host::fail(WF_E_INVALID_ARG, "dtype = %d", dtype);
  if (B < 1) return host::fail(WF_E_INVALID_ARG, "B = %d, need B >= 1", B);
  if (n_tokens < 0) return host::fail(WF_E_INVALID_ARG, "n_tokens = %d", n_tokens);
  if (n_tokens >= 1 << 25) return host::fail(WF_E_CAPACITY, "n_tokens = %d (supported: below 2^25 a call)", n_tokens);      // 64 threads each, fewer than 2^32 in all
  if (n_tokens == 0) return WF_OK;
  if (!cu || !row) return host::fail(WF_E_INVALID_ARG, "cu_dev or row_dev is NULL");
  return host::check_cache_memory(c);
}

template <typename F>
int launch_checked(const char *what, F &&launch) {
  launch();
  const hipError_t err = hipGetLastError();
  return err == hipSuccess ? WF_OK : host::fail(WF_E_HIP, "%s launch: %s", what, hipGetErrorString(err));
}

template <typename T>
void launch_write(const CacheView &c, int cache_dtype, const void *k, const void *v, int64_t ld, const int32_t *cu, const int32_t *row, int B, int n_tokens,
                  hipStream_t s) {
  const dim3 grid((uint32_t)(((int64_t)n_tokens + 3) / 4));
  switch (cache_dtype) {
    case WF_DTYPE_F8: cache_write_kernel<T, WF_DTYPE_F8><<<grid, 256, 0, s>>>(c, (const T *)k, (const T *)v, ld, cu, row, B, n_tokens); break;
    case WF_DTYPE_BF16: cache_write_kernel<T, WF_DTYPE_BF16><<<grid, 256, 0, s>>>(c, (const T *)k, (const T *)v, ld, cu, row, B, n_tokens); break;
    default: cache_write_kernel<T, WF_DTYPE_F32><<<grid, 256, 0, s>>>(c, (const T *)k, (const T *)v, ld, cu, row, B, n_tokens);
  }
}

template <typename T>
void launch_read(const CacheView &c, int cache_dtype, void *out, const int32_t *cu, const int32_t *row, int B, int n_tokens, hipStream_t s) {
  const dim3 grid((uint32_t)(((int64_t)n_tokens + 3) / 4));
  switch (cache_dtype) {
    case WF_DTYPE_F8: cache_read_kernel<T, WF_DTYPE_F8><<<grid, 256, 0, s>>>(c, (T *)out, cu, row, B, n_tokens); break;
    case WF_DTYPE_BF16: cache_read_kernel<T, WF_DTYPE_BF16><<<grid, 256, 0, s>>>(c, (T *)out, cu, row, B, n_tokens); break;
    default: cache_read_kernel<T, WF_DTYPE_F32><<<grid, 256, 0, s>>>(c, (T *)out, cu, row, B, n_tokens);
  }
}

}  // namespace
}  // namespace wf

using namespace wf;
using namespace wf::host;

extern "C" {

int wf_op_cache_write(const wf_cache *cache, const void *k_dev, const void *v_dev, int32_t dtype, int64_t ld, const int32_t *cu_dev,
                      const int32_t *row_dev, int32_t B, int32_t n_tokens, void *hip_stream) {
  int rc = check_tokens(cache, cu_dev, row_dev, dtype, B, n_tokens);
  if (rc) return rc;
  const int es = dtype == WF_DTYPE_BF16 ? 2 : 4;
  if (ld < 64 * (int64_t)cache->n_heads) return fail(WF_E_INVALID_ARG, "ld = %lld, need at least 64 * n_heads", (long long)ld);
  if (n_tokens == 0) return WF_OK;
  if (!k_dev || !v_dev) return fail(WF_E_INVALID_ARG, "k_dev or v_dev is NULL");
  if ((uintptr_t)k_dev % 16 || (uintptr_t)v_dev % 16 || ld * es % 16) return fail(WF_E_INVALID_ARG, "k_dev, v_dev and the row stride must be multiples of 16 bytes");
  const CacheView c = view_of(*cache);
  const hipStream_t s = (hipStream_t)hip_stream;
  return launch_checked("cache_write", [&] {
    if (dtype == WF_DTYPE_BF16) launch_write<__bf16>(c, cache->dtype, k_dev, v_dev, ld, cu_dev, row_dev, B, n_tokens, s);
    else launch_write<float>(c, cache->dtype, k_dev, v_dev, ld, cu_dev, row_dev, B, n_tokens, s);
  });
}

int wf_op_cache_read(const wf_cache *cache, const int32_t *cu_dev, const int32_t *row_dev, int32_t B, void *out_dev, int32_t dtype,
                     int32_t n_tokens, void *hip_stream) {
  int rc = check_tokens(cache, cu_dev, row_dev, dtype, B, n_tokens);
  if (rc) return rc;
  if (n_tokens == 0) return WF_OK;
  if (!out_dev) return fail(WF_E_INVALID_ARG, "out_dev is NULL");
  if ((uintptr_t)out_dev % 16) return fail(WF_E_INVALID_ARG, "out_dev is not aligned to 16 bytes");
  const CacheView c = view_of(*cache);
  const hipStream_t s = (hipStream_t)hip_stream;
  return launch_checked("cache_read", [&] {
    if (dtype == WF_DTYPE_BF16) launch_read<__bf16>(c, cache->dtype, out_dev, cu_dev, row_dev, B, n_tokens, s);
    else launch_read<float>(c, cache->dtype, out_dev, cu_dev, row_dev, B, n_tokens, s);
  });
}

}  // extern "C"
