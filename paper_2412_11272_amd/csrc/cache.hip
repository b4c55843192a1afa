// Key / value caches of the token-by-token part: rows written as they come or quantised to e4m3, and read back.  The formats and
// rules are stated with the declarations in include/wf_encoder.h.
//
// Quantisation of a head's 64 values x: e = min{whole e >= -127 : max|x| <= 448 2^e}, q = round(x 2^-e) in e4m3.  A power of two keeps
// the product x 2^-e exact, so that q has one rounding (to nearest even, half a step of 2^-4 relative to the value) and a reader gets
// q 2^e exactly in bf16 or fp32.
#include "cache_device.h"
#include "host_runtime.h"

namespace wf {

namespace {

__device__ __forceinline__ float load_act(const float *p) { return *p; }
__device__ __forceinline__ float load_act(const __bf16 *p) { return (float)*p; }

// The cache row of token t, -1 if it has none.
__device__ __forceinline__ int64_t token_row(const int32_t *cu, const int32_t *row, int B, int64_t n_rows, int t, bool *live) {
  *live = t < cu[B];
  if (!*live) return -1;
  const int s = find_stream(cu, B, t);
  const int64_t at = (int64_t)t - cu[s], r = row[s] + at;
  return at >= 0 && r >= 0 && r < n_rows ? r : -1;
}

template <typename T, int CACHE>
__global__ void __launch_bounds__(256) cache_write_kernel(CacheView c, const T *k, const T *v, int64_t ld, const int32_t *cu, const int32_t *row, int B,
                                                          int n_tokens) {
  const int64_t unit = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);      // (token, head, keys | values)
  const int lane = threadIdx.x & 63, units = 2 * c.n_heads;
  const int64_t t = unit / units;
  if (t >= n_tokens) return;
  const int u = (int)(unit % units), h = u >> 1, kv = u & 1;
  bool live;
  const int64_t r = token_row(cu, row, B, c.n_rows, (int)t, &live);
  if (r < 0) return;
  float x = load_act((kv ? v : k) + t * ld + h * 64 + lane);
  if constexpr (CACHE == WF_DTYPE_F8) {
    const bool fine = (__builtin_bit_cast(uint32_t, x) & 0x7f800000u) != 0x7f800000u;
    const uint32_t biased = f8_exponent(wave_max(fine ? fabsf(x) : 0.0f));
    x = fine ? x * __builtin_bit_cast(float, (254u - biased) << 23) : __builtin_nanf("");
    ((uint8_t *)c.data)[(r * units + u) * 64 + lane] = (uint8_t)__builtin_amdgcn_cvt_pk_fp8_f32(x, x, 0, false);
    if (lane == 0) c.exps[u * c.n_rows + r] = (uint8_t)biased;
  } else if constexpr (CACHE == WF_DTYPE_BF16) {
    ((__bf16 *)c.data)[r * units * 64 + (kv * c.n_heads + h) * 64 + lane] = (__bf16)x;
  } else {
    ((float *)c.data)[r * units * 64 + (kv * c.n_heads + h) * 64 + lane] = x;
  }
}

template <typename T, int CACHE>
__global__ void __launch_bounds__(256) cache_read_kernel(CacheView c, T *out, const int32_t *cu, const int32_t *row, int B, int n_tokens) {
  const int64_t unit = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int lane = threadIdx.x & 63, units = 2 * c.n_heads;
  const int64_t t = unit / units;
  if (t >= n_tokens) return;
  const int u = (int)(unit % units), h = u >> 1, kv = u & 1;
  bool live;
  const int64_t r = token_row(cu, row, B, c.n_rows, (int)t, &live);
  if (!live) return;
  float x = 0.0f;
  if (r >= 0) {
    if constexpr (CACHE == WF_DTYPE_F8)
      x = __builtin_amdgcn_cvt_f32_fp8(((const uint8_t *)c.data)[(r * units + u) * 64 + lane], 0) * f8_factor(c.exps[u * c.n_rows + r]);
    else if constexpr (CACHE == WF_DTYPE_BF16)
      x = (float)((const __bf16 *)c.data)[r * units * 64 + (kv * c.n_heads + h) * 64 + lane];
    else
      x = ((const float *)c.data)[r * units * 64 + (kv * c.n_heads + h) * 64 + lane];
  }
  out[(t * units + kv * c.n_heads + h) * 64 + lane] = (T)x;
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
  const dim3 grid((uint32_t)(((int64_t)n_tokens * 2 * c.n_heads + 3) / 4));
  switch (cache_dtype) {
    case WF_DTYPE_F8: cache_write_kernel<T, WF_DTYPE_F8><<<grid, 256, 0, s>>>(c, (const T *)k, (const T *)v, ld, cu, row, B, n_tokens); break;
    case WF_DTYPE_BF16: cache_write_kernel<T, WF_DTYPE_BF16><<<grid, 256, 0, s>>>(c, (const T *)k, (const T *)v, ld, cu, row, B, n_tokens); break;
    default: cache_write_kernel<T, WF_DTYPE_F32><<<grid, 256, 0, s>>>(c, (const T *)k, (const T *)v, ld, cu, row, B, n_tokens);
  }
}

template <typename T>
void launch_read(const CacheView &c, int cache_dtype, void *out, const int32_t *cu, const int32_t *row, int B, int n_tokens, hipStream_t s) {
  const dim3 grid((uint32_t)(((int64_t)n_tokens * 2 * c.n_heads + 3) / 4));
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
