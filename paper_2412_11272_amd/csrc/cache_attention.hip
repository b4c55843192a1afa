// Attention of a few queries per sequence over a key / value cache (one new token, the beams of a stream, a tree of drafted tokens).  The
// definition is stated with wf_op_cache_attention in include/wf_encoder.h.
#include "cache_device.h"
#include "host_runtime.h"

#include <cmath>

namespace wf {

namespace {

struct AttendArgs {
  CacheView c;
  const void *q;
  void *out;
  int64_t ldq, ldo;
  const int32_t *cu_q, *row, *len;
  const uint32_t *mask;
  const int32_t *mask_from;
  int32_t n_heads, n_seqs, n_q_rows, max_q, max_len, mask_words;
  float scale;
};

template <int CACHE>
__device__ __forceinline__ float cache_value(const CacheView &c, int64_t r, int h, int kv, int i) {
  if constexpr (CACHE == WF_DTYPE_F8)
    return __builtin_amdgcn_cvt_f32_fp8(((const uint8_t *)c.data)[((r * c.n_heads + h) * 2 + kv) * 64 + i], 0) * f8_factor(c.exps[(2 * h + kv) * c.n_rows + r]);
  else if constexpr (CACHE == WF_DTYPE_BF16)
    return (float)((const __bf16 *)c.data)[(r * 2 + kv) * c.n_heads * 64 + h * 64 + i];
  else
    return ((const float *)c.data)[(r * 2 + kv) * c.n_heads * 64 + h * 64 + i];
}

// One wave per (sequence, query, head): 64 keys at a time, first a lane per key, then a lane per value.
template <typename T, int CACHE>
__global__ void __launch_bounds__(64) cache_attention_kernel(AttendArgs p) {
  __shared__ float sq[64], sw[64];
  const int lane = threadIdx.x;
  const int h = blockIdx.x % p.n_heads, i = (blockIdx.x / p.n_heads) % p.max_q, s = blockIdx.x / (p.n_heads * p.max_q);
  const int64_t r = (int64_t)p.cu_q[s] + i;
  if (r >= p.cu_q[s + 1] || r < 0 || r >= p.n_q_rows) return;
  const int hk = h / (p.n_heads / p.c.n_heads);
  const int64_t row0 = p.row[s];
  int64_t n = p.len[s];
  n = n < p.max_len ? n : p.max_len;
  if (row0 < 0) n = 0;
  n = n < p.c.n_rows - row0 ? n : p.c.n_rows - row0;
  const int64_t from = !p.mask ? n : p.mask_from ? p.mask_from[s] : 0;
  sq[lane] = (float)((const T *)p.q)[r * p.ldq + h * 64 + lane];
  __syncthreads();
  const float c = p.scale * 1.4426950408889634f;
  float m = -INFINITY, l = 0.0f, o = 0.0f;
  for (int64_t k0 = 0; k0 < n; k0 += 64) {
    const int64_t k = k0 + lane;
    bool seen = k < n;
    if (seen && k >= from) {
      const int64_t at = k - from;
      seen = at < 32 * (int64_t)p.mask_words && (p.mask[r * p.mask_words + at / 32] >> (at & 31) & 1);
    }
    float x = -INFINITY;
    if (seen) {
      x = 0.0f;
      for (int d = 0; d < 64; ++d) x += sq[d] * cache_value<CACHE>(p.c, row0 + k, hk, 0, d);
      x *= c;
    }
    const uint64_t some = __ballot(seen);
    if (!some) continue;
    const float m_new = fmaxf(m, wave_max(x)), base = m_new == -INFINITY ? 0.0f : m_new;
    const float w = seen ? exp2f(x - base) : 0.0f, keep = exp2f(m - base);
    l = l * keep + wave_sum(w);
    m = m_new;
    o *= keep;
    sw[lane] = w;
    __syncthreads();
    for (int j = 0; j < 64; ++j)
      if (some >> j & 1) o += sw[j] * cache_value<CACHE>(p.c, row0 + k0 + j, hk, 1, lane);
    __syncthreads();
  }
  ((T *)p.out)[r * p.ldo + h * 64 + lane] = (T)(l != 0.0f ? o / l : 0.0f);
}

}  // namespace
}  // namespace wf

using namespace wf;
using namespace wf::host;

namespace {

int check_query(const wf_cache *c, const wf_cache_query *a) {
  int rc = check_cache(c);
  if (rc) return rc;
  if (!a) return fail(WF_E_INVALID_ARG, "query is NULL");
  if (a->dtype != WF_DTYPE_F32 && a->dtype != WF_DTYPE_BF16) return fail(WF_E_INVALID_ARG, "query dtype = %d", a->dtype);
  if (c->dtype != WF_DTYPE_F8 && c->dtype != a->dtype) return fail(WF_E_INVALID_ARG, "queries of type %d over a cache of type %d", a->dtype, c->dtype);
  if (a->n_heads < 1 || a->n_heads % c->n_heads || a->n_heads > 65536)
    return fail(WF_E_INVALID_ARG, "n_heads = %d must be a multiple of the cache's %d", a->n_heads, c->n_heads);
  if (a->n_seqs < 1 || a->n_q_rows < 0 || a->max_q < 1 || a->max_len < 0)
    return fail(WF_E_INVALID_ARG, "n_seqs = %d, n_q_rows = %d, max_q = %d, max_len = %d", a->n_seqs, a->n_q_rows, a->max_q, a->max_len);
  if (!std::isfinite(a->scale)) return fail(WF_E_INVALID_ARG, "scale is not finite");
  if ((int64_t)a->n_seqs * std::min(a->max_q, std::max(a->n_q_rows, 1)) * a->n_heads >= ((int64_t)1 << 31))
    return fail(WF_E_CAPACITY, "%d sequences of up to %d queries of %d heads: more than 2^31 rows", a->n_seqs, a->max_q, a->n_heads);
  return WF_OK;
}

}  // namespace

extern "C" {

int64_t wf_cache_attention_workspace(const wf_cache *cache, const wf_cache_query *query) { return check_query(cache, query); }

int wf_op_cache_attention(const wf_cache *cache, const wf_cache_query *query, void *hip_stream) {
  int rc = check_query(cache, query);
  if (rc) return rc;
  const wf_cache_query &a = *query;
  const int es = a.dtype == WF_DTYPE_BF16 ? 2 : 4;
  if (a.ldq < 64 * (int64_t)a.n_heads || a.ldo < 64 * (int64_t)a.n_heads) return fail(WF_E_INVALID_ARG, "ldq = %lld, ldo = %lld, need at least 64 * n_heads", (long long)a.ldq, (long long)a.ldo);
  if (a.mask_dev ? a.mask_words < 1 : a.mask_from_dev != nullptr) return fail(WF_E_INVALID_ARG, "mask_words = %d with mask_dev %s", a.mask_words, a.mask_dev ? "set" : "NULL");
  if (a.n_q_rows == 0) return WF_OK;
  if (!a.q_dev || !a.out_dev || !a.cu_q_dev || !a.row_dev || !a.len_dev) return fail(WF_E_INVALID_ARG, "q_dev, out_dev, cu_q_dev, row_dev or len_dev is NULL");
  if ((rc = check_cache_memory(cache))) return rc;
  if ((uintptr_t)a.q_dev % 16 || (uintptr_t)a.out_dev % 16 || a.ldq * es % 16 || a.ldo * es % 16)
    return fail(WF_E_INVALID_ARG, "q_dev, out_dev and their row strides must be multiples of 16 bytes");
  const AttendArgs p{view_of(*cache), a.q_dev, a.out_dev, a.ldq, a.ldo, a.cu_q_dev, a.row_dev, a.len_dev, a.mask_dev, a.mask_from_dev,
                     a.n_heads, a.n_seqs, a.n_q_rows, std::min(a.max_q, a.n_q_rows), a.max_len, a.mask_words, a.scale};
  const dim3 grid((uint32_t)((int64_t)p.n_seqs * p.max_q * p.n_heads));
  const hipStream_t s = (hipStream_t)hip_stream;
  if (a.dtype == WF_DTYPE_BF16) {
    if (cache->dtype == WF_DTYPE_F8) cache_attention_kernel<__bf16, WF_DTYPE_F8><<<grid, 64, 0, s>>>(p);
    else cache_attention_kernel<__bf16, WF_DTYPE_BF16><<<grid, 64, 0, s>>>(p);
  } else {
    if (cache->dtype == WF_DTYPE_F8) cache_attention_kernel<float, WF_DTYPE_F8><<<grid, 64, 0, s>>>(p);
    else cache_attention_kernel<float, WF_DTYPE_F32><<<grid, 64, 0, s>>>(p);
  }
  const hipError_t err = hipGetLastError();
  return err == hipSuccess ? WF_OK : fail(WF_E_HIP, "cache_attention launch: %s", hipGetErrorString(err));
}

}  // extern "C"
