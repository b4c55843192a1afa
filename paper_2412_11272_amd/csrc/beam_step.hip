// One step of a beam search over many streams: the best continuations over beams and vocabulary, and the beams' states
// moved behind their new owners.  The rules are stated with wf_op_beam_select and wf_op_beam_reorder in include/wf_encoder.h.
#include "device_utils.h"
#include "host_runtime.h"

namespace wf {

namespace {

constexpr int kMaxBeams = 32;

// Values as whole numbers of the same order (finite ones: > 0), so that (value, lowest token) is one comparison of 64 bits.
__device__ __forceinline__ uint32_t order_of(float x) {
  const uint32_t u = __builtin_bit_cast(uint32_t, x + 0.0f);      // -0 is 0
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t order) {
  return __builtin_bit_cast(float, order & 0x80000000u ? order & 0x7fffffffu : ~order);
}
__device__ __forceinline__ bool is_finite(float x) { return (__builtin_bit_cast(uint32_t, x) & 0x7f800000u) != 0x7f800000u; }

__device__ __forceinline__ uint64_t wave_max_u64(uint64_t v) {
  for (int m = 32; m; m >>= 1) {
    const uint64_t o = __shfl_xor((unsigned long long)v, m);
    v = v > o ? v : o;
  }
  return v;
}
__device__ __forceinline__ double wave_sum_f64(double v) {
  for (int m = 32; m; m >>= 1) v += __shfl_xor(v, m);
  return v;
}
__device__ __forceinline__ double wave_max_f64(double v) {
  for (int m = 32; m; m >>= 1) v = fmax(v, __shfl_xor(v, m));
  return v;
}

// What a beam offers: its candidates by logit and then the lowest token (token < 0: no more), and the log of its sum.
struct RowBest {
  double log_sum;
  int32_t token[kMaxBeams];
  float logit[kMaxBeams];
};

struct SelectArgs {
  const void *logits;
  int64_t ld;
  const int32_t *n_in, *n_out;
  const float *score_in;
  const uint8_t *done_in;
  int32_t *token_out, *parent_out;
  float *score_out;
  uint8_t *done_out;
  RowBest *rows;
  int32_t B, width, n_vocab, eos, keep_slots;
};

__device__ __forceinline__ int clamped(const int32_t *n, int s, int width) {
  if (!n) return width;
  return n[s] < 0 ? 0 : n[s] < width ? n[s] : width;
}

// One workgroup per beam.
template <typename T>
__global__ void __launch_bounds__(256) beam_rows_kernel(SelectArgs p) {
  const int s = blockIdx.x / p.width, b = blockIdx.x % p.width;
  if (b >= clamped(p.n_in, s, p.width)) return;
  RowBest &row = p.rows[blockIdx.x];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  if (p.done_in && p.done_in[blockIdx.x]) {
    if (tid == 0) row.log_sum = 0.0;
    if (tid < p.width) { row.token[tid] = tid == 0 ? p.eos : -1; row.logit[tid] = 0.0f; }
    return;
  }
  __shared__ uint64_t best_of[4];
  __shared__ double sum_of[4];
  const T *x = (const T *)p.logits + (int64_t)blockIdx.x * p.ld;
  uint64_t last = ~0ull;
  for (int k = 0; k < p.width; ++k) {
    uint64_t best = 0;
    for (int t = tid; t < p.n_vocab; t += 256) {
      const float v = (float)x[t];
      const uint64_t key = is_finite(v) ? (uint64_t)order_of(v) << 32 | (uint32_t)~t : 0;
      if (key < last && key > best) best = key;
    }
    best = wave_max_u64(best);
    if (lane == 0) best_of[wave] = best;
    __syncthreads();
    for (int w = 0; w < 4; ++w) best = best > best_of[w] ? best : best_of[w];
    __syncthreads();
    if (tid == 0) { row.token[k] = best ? (int32_t)~(uint32_t)best : -1; row.logit[k] = best ? value_of((uint32_t)(best >> 32)) : 0.0f; }
    if (k == 0 && best) {
      const float top = value_of((uint32_t)(best >> 32));
      double sum = 0.0;
      for (int t = tid; t < p.n_vocab; t += 256) {
        const float v = (float)x[t];
        if (is_finite(v)) sum += expf(v - top);
      }
      sum = wave_sum_f64(sum);
      if (lane == 0) sum_of[wave] = sum;
      __syncthreads();
      if (tid == 0) row.log_sum = top + log(sum_of[0] + sum_of[1] + sum_of[2] + sum_of[3]);
    }
    last = best;
  }
}

// One wave per stream: the beams' sorted candidates are merged, lane b holding the first of beam b that is not taken yet.
__global__ void __launch_bounds__(64) beam_merge_kernel(SelectArgs p) {
  __shared__ int32_t s_token[kMaxBeams], s_parent[kMaxBeams], s_slot[kMaxBeams];
  __shared__ float s_score[kMaxBeams];
  const int s = blockIdx.x, lane = threadIdx.x, W = p.width;
  const int n_in = clamped(p.n_in, s, W), n_out = clamped(p.n_out, s, W);
  const RowBest *row = p.rows + (int64_t)s * W + lane;
  const float start = lane < n_in ? p.score_in[(int64_t)s * W + lane] : -INFINITY;
  const bool live = lane < n_in && is_finite(start);
  const bool was_done = live && p.done_in && p.done_in[(int64_t)s * W + lane];
  int at = 0, token = live ? row->token[0] : -1;
  double total = token >= 0 ? (double)start + ((double)row->logit[0] - row->log_sum) : -INFINITY;
  int n = 0;
  for (; n < n_out; ++n) {
    const double best = wave_max_f64(total);
    const uint64_t who = __ballot(token >= 0 && total == best);
    if (!who) break;
    const int b = __ffsll((unsigned long long)who) - 1;
    if (lane == b) {
      s_token[n] = was_done || token == p.eos ? token | 1 << 31 : token;       // the top bit: done
      s_parent[n] = b;
      s_score[n] = (float)total;
      ++at;
      token = at < W ? row->token[at] : -1;
      total = token >= 0 ? (double)start + ((double)row->logit[at] - row->log_sum) : -INFINITY;
    }
  }
  __syncthreads();
  if (lane == 0) {
    for (int j = 0; j < W; ++j) s_slot[j] = !p.keep_slots && j < n ? j : -1;
    if (p.keep_slots) {
      uint32_t placed = 0;
      for (int j = 0; j < n; ++j)
        if (s_parent[j] < n_out && s_slot[s_parent[j]] < 0) { s_slot[s_parent[j]] = j; placed |= 1u << j; }
      int free = 0;
      for (int j = 0; j < n; ++j) {
        if (placed >> j & 1) continue;
        while (s_slot[free] >= 0) ++free;
        s_slot[free] = j;
      }
    }
  }
  __syncthreads();
  if (lane < W) {
    const int64_t o = (int64_t)s * W + lane;
    const int j = s_slot[lane];
    p.token_out[o] = j < 0 ? -1 : s_token[j] & 0x7fffffff;
    p.parent_out[o] = j < 0 ? -1 : s_parent[j];
    p.score_out[o] = j < 0 ? -INFINITY : s_score[j];
    if (p.done_out) p.done_out[o] = j >= 0 && s_token[j] < 0;
  }
}

struct ReorderArgs {
  void *dst;
  const void *src;
  const int32_t *parent, *len;
  int32_t B, width;
  int64_t n_pos, pos_bytes, slot_bytes, chunks;
};

// A thread holds one column of V bytes of all of a stream's slots, so that a slot is read before any is written.
template <typename V, int MAXW>
__global__ void __launch_bounds__(256) beam_reorder_kernel(ReorderArgs p) {
  const int64_t ls = blockIdx.x / p.chunks, chunk = blockIdx.x % p.chunks;      // (layer, stream)
  const int s = (int)(ls % p.B);
  int64_t n = p.len ? p.len[s] : p.n_pos;
  n = n < 0 ? 0 : n < p.n_pos ? n : p.n_pos;
  const int64_t at = (chunk * 256 + threadIdx.x) * sizeof(V);
  if (at >= n * p.pos_bytes) return;
  const char *src = (const char *)p.src + ls * p.width * p.slot_bytes + at;
  char *dst = (char *)p.dst + ls * p.width * p.slot_bytes + at;
  V v[MAXW];
  int from[MAXW];
#pragma unroll
  for (int j = 0; j < MAXW; ++j) {
    from[j] = j < p.width ? p.parent[(int64_t)s * p.width + j] : -1;
    if (from[j] >= p.width || (p.src == p.dst && from[j] == j)) from[j] = -1;
    if (from[j] >= 0) v[j] = *(const V *)(src + from[j] * p.slot_bytes);
  }
#pragma unroll
  for (int j = 0; j < MAXW; ++j)
    if (from[j] >= 0) *(V *)(dst + j * p.slot_bytes) = v[j];
}

template <typename V>
void launch_reorder(ReorderArgs p, int64_t layers_streams, hipStream_t s) {
  const dim3 grid((uint32_t)(layers_streams * p.chunks));
  if (p.width <= 4) beam_reorder_kernel<V, 4><<<grid, 256, 0, s>>>(p);
  else if (p.width <= 8) beam_reorder_kernel<V, 8><<<grid, 256, 0, s>>>(p);
  else if (p.width <= 16) beam_reorder_kernel<V, 16><<<grid, 256, 0, s>>>(p);
  else beam_reorder_kernel<V, 32><<<grid, 256, 0, s>>>(p);
}

}  // namespace
}  // namespace wf

using namespace wf;
using namespace wf::host;

namespace {

int check_step(const wf_beam_step *a) {
  if (!a) return fail(WF_E_INVALID_ARG, "step is NULL");
  if (a->dtype != WF_DTYPE_F32 && a->dtype != WF_DTYPE_BF16) return fail(WF_E_INVALID_ARG, "logits dtype = %d", a->dtype);
  if (a->B < 1) return fail(WF_E_INVALID_ARG, "B = %d, need B >= 1", a->B);
  if (a->width < 1 || a->width > kMaxBeams) return fail(WF_E_INVALID_ARG, "width = %d (supported: 1 .. %d)", a->width, kMaxBeams);
  if (a->n_vocab < 1) return fail(WF_E_INVALID_ARG, "n_vocab = %d", a->n_vocab);
  if ((int64_t)a->B * a->width >= 1 << 22) return fail(WF_E_CAPACITY, "B * width = %lld beams (supported: below 2^22)", (long long)a->B * a->width);
  return WF_OK;
}

}  // namespace

extern "C" {

int64_t wf_beam_select_workspace(const wf_beam_step *a) {
  const int rc = check_step(a);
  return rc ? rc : (int64_t)a->B * a->width * (int64_t)sizeof(RowBest);
}

int wf_op_beam_select(const wf_beam_step *a, void *hip_stream) {
  const int64_t need = wf_beam_select_workspace(a);
  if (need < 0) return (int)need;
  if (!a->logits_dev || !a->score_in_dev || !a->token_out_dev || !a->parent_out_dev || !a->score_out_dev)
    return fail(WF_E_INVALID_ARG, "logits_dev, score_in_dev or one of the outputs is NULL");
  if (a->ld < a->n_vocab) return fail(WF_E_INVALID_ARG, "ld = %lld, need at least n_vocab = %d", (long long)a->ld, a->n_vocab);
  if ((a->done_in_dev != nullptr) != (a->done_out_dev != nullptr)) return fail(WF_E_INVALID_ARG, "done_in_dev and done_out_dev go together");
  if (a->done_in_dev && (a->eos < 0 || a->eos >= a->n_vocab)) return fail(WF_E_INVALID_ARG, "eos = %d outside [0, %d)", a->eos, a->n_vocab);
  if (!a->workspace_dev || (uintptr_t)a->workspace_dev % 16) return fail(WF_E_INVALID_ARG, "workspace_dev is NULL or not aligned to 16 bytes");
  if (a->workspace_bytes < need) return fail(WF_E_CAPACITY, "workspace of %lld bytes, need %lld", (long long)a->workspace_bytes, (long long)need);
  const SelectArgs p{a->logits_dev, a->ld, a->n_in_dev, a->n_out_dev, a->score_in_dev, a->done_in_dev, a->token_out_dev, a->parent_out_dev, a->score_out_dev,
                     a->done_out_dev, (RowBest *)a->workspace_dev, a->B, a->width, a->n_vocab, a->done_in_dev ? a->eos : -1, a->keep_slots};
  const hipStream_t s = (hipStream_t)hip_stream;
  if (a->dtype == WF_DTYPE_BF16) beam_rows_kernel<__bf16><<<a->B * a->width, 256, 0, s>>>(p);
  else beam_rows_kernel<float><<<a->B * a->width, 256, 0, s>>>(p);
  beam_merge_kernel<<<a->B, 64, 0, s>>>(p);
  const hipError_t err = hipGetLastError();
  return err == hipSuccess ? WF_OK : fail(WF_E_HIP, "beam_select launch: %s", hipGetErrorString(err));
}

int wf_op_beam_reorder(void *dst_dev, const void *src_dev, const int32_t *parent_dev, const int32_t *len_dev, int32_t B, int32_t width,
                       int32_t n_layers, int64_t n_pos, int64_t pos_bytes, void *hip_stream) {
  if (B < 1) return fail(WF_E_INVALID_ARG, "B = %d, need B >= 1", B);
  if (width < 1 || width > kMaxBeams) return fail(WF_E_INVALID_ARG, "width = %d (supported: 1 .. %d)", width, kMaxBeams);
  if (n_layers < 0 || n_pos < 0 || pos_bytes < 1) return fail(WF_E_INVALID_ARG, "n_layers = %d, n_pos = %lld, pos_bytes = %lld", n_layers, (long long)n_pos, (long long)pos_bytes);
  if (n_layers == 0 || n_pos == 0) return WF_OK;
  if (!dst_dev || !src_dev || !parent_dev) return fail(WF_E_INVALID_ARG, "dst_dev, src_dev or parent_dev is NULL");
  int64_t slot, all;
  if (__builtin_mul_overflow(n_pos, pos_bytes, &slot) || __builtin_mul_overflow(slot, (int64_t)B * width, &all) || __builtin_mul_overflow(all, (int64_t)n_layers, &all))
    return fail(WF_E_INVALID_ARG, "n_pos = %lld, pos_bytes = %lld: too large", (long long)n_pos, (long long)pos_bytes);
  const uintptr_t d = (uintptr_t)dst_dev, f = (uintptr_t)src_dev;
  if (d != f && d < f + (uintptr_t)all && f < d + (uintptr_t)all) return fail(WF_E_INVALID_ARG, "dst_dev and src_dev overlap");
  const int vec = (d | f | (uintptr_t)slot | (uintptr_t)pos_bytes) % 16 == 0 ? 16 : (d | f | (uintptr_t)slot | (uintptr_t)pos_bytes) % 4 == 0 ? 4 : 1;
  ReorderArgs p{dst_dev, src_dev, parent_dev, len_dev, B, width, n_pos, pos_bytes, slot, (slot + 256 * vec - 1) / (256 * vec)};
  if ((int64_t)n_layers * B * (double)p.chunks >= 2147483648.0) return fail(WF_E_CAPACITY, "%lld bytes in %d layers: more than 2^31 workgroups", (long long)all, n_layers);
  const int64_t ls = (int64_t)n_layers * B;
  const hipStream_t s = (hipStream_t)hip_stream;
  if (vec == 16) launch_reorder<uint4>(p, ls, s);
  else if (vec == 4) launch_reorder<uint32_t>(p, ls, s);
  else launch_reorder<uint8_t>(p, ls, s);
  const hipError_t err = hipGetLastError();
  return err == hipSuccess ? WF_OK : fail(WF_E_HIP, "beam_reorder launch: %s", hipGetErrorString(err));
}

}  // extern "C"
