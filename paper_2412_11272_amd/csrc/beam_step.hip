// One step of a beam search over many streams: the best continuations over beams and vocabulary, and the beams' states
// moved behind their new owners.  The rules are stated with wf_op_beam_select and wf_op_beam_reorder in include/wf_encoder.h.
#include "device_utils.h"
#include "host_runtime.h"

namespace wf {

namespace {

constexpr int kMaxBeams = 32;
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// Values as whole numbers of the same order (finite ones: > 0), so that (value, lowest token) is one comparison of 64 bits.
__device__ __forceinline__ uint32_t order_of(float x) {
  const uint32_t u = __builtin_bit_cast(uint32_t, x + 0.0f);      // -0 is 0
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t order) {
  return __builtin_bit_cast(float, order & 0x80000000u ? order & 0x7fffffffu : ~order);
}
__device__ __forceinline__ bool is_finite(float x) { return fabsf(x) < INFINITY; }

// Between a wave's writes to the LDS and its other lanes' reads: the LDS works in order, so only the compiler has to keep it.
__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// Maxima and sums over a wave by the same lane moves as device_utils.h's, on two registers.
template <typename U, int N>
__device__ __forceinline__ U row_rotate64(U v) {
  const u32x2 u = __builtin_bit_cast(u32x2, v);
  const uint32_t lo = u[0], hi = u[1];
  const u32x2 r = {(uint32_t)__builtin_amdgcn_update_dpp(0, (int)lo, 0x120 + N, 0xF, 0xF, true), (uint32_t)__builtin_amdgcn_update_dpp(0, (int)hi, 0x120 + N, 0xF, 0xF, true)};
  return __builtin_bit_cast(U, r);
}
template <typename U, typename F>
__device__ __forceinline__ U wave_reduce64(U v, F f) {
  v = f(v, row_rotate64<U, 8>(v));
  v = f(v, row_rotate64<U, 4>(v));
  v = f(v, row_rotate64<U, 2>(v));
  v = f(v, row_rotate64<U, 1>(v));
  u32x2 u = __builtin_bit_cast(u32x2, v);
  uint32_t lo = u[0], hi = u[1];
  const auto l16 = __builtin_amdgcn_permlane16_swap(lo, lo, false, false), h16 = __builtin_amdgcn_permlane16_swap(hi, hi, false, false);
  const u32x2 a = {(uint32_t)l16[0], (uint32_t)h16[0]}, b = {(uint32_t)l16[1], (uint32_t)h16[1]};
  u = __builtin_bit_cast(u32x2, f(__builtin_bit_cast(U, a), __builtin_bit_cast(U, b)));
  lo = u[0]; hi = u[1];
  const auto l32 = __builtin_amdgcn_permlane32_swap(lo, lo, false, false), h32 = __builtin_amdgcn_permlane32_swap(hi, hi, false, false);
  const u32x2 c = {(uint32_t)l32[0], (uint32_t)h32[0]}, d = {(uint32_t)l32[1], (uint32_t)h32[1]};
  return f(__builtin_bit_cast(U, c), __builtin_bit_cast(U, d));
}
template <typename U>
__device__ __forceinline__ U max64(U a, U b) { return a > b ? a : b; }
template <typename U>
__device__ __forceinline__ U wave_max64(U v) { return wave_reduce64(v, max64<U>); }
__device__ __forceinline__ double wave_sum_f64(double v) { return wave_reduce64(v, [](double a, double b) { return a + b; }); }

// Part of a beam's row: the sum of 2^(x kLog2e - base) over its values x (no finite one: base = -infinity), and its best candidates as keys (0: no
// more).  kLog2e is the fp32 value and the sum's logarithm is divided by that very number, so that its rounding, 1.3e-8, costs the entropy times that
// much, and not the logits.
struct PartSum {
  double sum, base;
};
constexpr float kLog2e = 1.4426950408889634f;

struct SelectArgs {
  const void *logits;
  int64_t ld;
  const int32_t *n_in, *n_out;
  const float *score_in;
  const uint8_t *done_in;
  int32_t *token_out, *parent_out;
  float *score_out;
  uint8_t *done_out;
  PartSum *sums;             // [beam][part]
  uint64_t *keys;            // [beam][part][width]
  int32_t B, width, n_vocab, eos, keep_slots, parts;
};

__device__ __forceinline__ int clamped(const int32_t *n, int s, int width) {
  if (!n) return width;
  return n[s] < 0 ? 0 : n[s] < width ? n[s] : width;
}

__device__ __forceinline__ uint64_t key_of(float x, int t) { return is_finite(x) ? (uint64_t)order_of(x) << 32 | (uint32_t)~t : 0; }

constexpr int kPart = 2048;      // tokens of a part: 32 values a lane

// A part's values as the lanes of its wave hold them: value e of chunk i is token first + i * 64 * N + lane * N + e, N = 16 bytes.  Rows start anywhere.
template <typename T> struct Values;
template <> struct Values<float> {
  static constexpr int N = 4;
  typedef float __attribute__((ext_vector_type(4), aligned(4))) vec;
};
template <> struct Values<__bf16> {
  static constexpr int N = 8;
  typedef __bf16 __attribute__((ext_vector_type(8), aligned(2))) vec;
};

// One wave per part: read once, into registers.  The width best are among the values that reach the width-th largest of the 64 lanes'
// maxima (so many lanes do, each with one value at least); a bisection over the upper half of the bits finds a bound just below it,
// usually a handful of values pass, and these are ranked by comparing each with each.  Where more than 64 pass (equal values, few finite
// ones) the best are taken out one by one.  64 x 5 beams over 51 866 tokens, 66 MB of fp32: 15 us here and 6 for the merge (scanning a row once for each
// candidate took 418).  The memory's share would be 11, some 460 vector instructions a part take the rest; bf16 logits take 18 us in all.
template <typename T>
__global__ void __launch_bounds__(256) beam_parts_kernel(SelectArgs p) {
  constexpr int N = Values<T>::N, CH = 32 / N;
  __shared__ uint64_t s_keys[4][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int row = blockIdx.x, part = blockIdx.y * 4 + wave;
  if (part >= p.parts) return;
  const int s = row / p.width, b = row % p.width;
  if (b >= clamped(p.n_in, s, p.width) || (p.done_in && p.done_in[row])) return;
  const int64_t id = (int64_t)row * p.parts + part;
  const T *x = (const T *)p.logits + (int64_t)row * p.ld + (int64_t)part * kPart;
  const int left = p.n_vocab - part * kPart;
  float v[32];
  if (left >= kPart) {
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      const auto w = *(const typename Values<T>::vec *)(x + (i * 64 + lane) * N);
#pragma unroll
      for (int e = 0; e < N; ++e) v[i * N + e] = (float)w[e];
    }
  } else {
#pragma unroll
    for (int i = 0; i < CH; ++i)
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const int at = (i * 64 + lane) * N + e;
        v[i * N + e] = at < left ? (float)x[at] : -INFINITY;
      }
  }
  float mine = -INFINITY;
#pragma unroll
  for (int i = 0; i < 32; ++i) {
    v[i] = is_finite(v[i]) ? v[i] : -INFINITY;
    mine = fmaxf(mine, v[i]);
  }
  const float top = wave_max(mine);
  const int W = p.width;
  uint64_t *keys = p.keys + id * W;
  if (top == -INFINITY) {
    if (lane < W) keys[lane] = 0;
    if (lane == 0) p.sums[id] = PartSum{0.0, -(double)INFINITY};
    return;
  }
  // The sum: eight values in 32 bits, the rest in 64 (each in 64 costs two instructions a value where the vector unit is what bounds the kernel).
  // What it is off by, relative to itself and so absolute in the logarithm: the argument's rounding, 2^-24 ln 2 of its size, whose mean by weight stays
  // below log2 n_vocab <= 28 (2^-20 at most); the exponential, 2^-23; seven additions, 2^-21.2; the entropy times kLog2e's 2^-26.2 (2^-21.9): less than 2^-19
  // in all.
  // (the fused form's base is off from top * kLog2e by up to 2^-24 of it, which enters every exponential: harmless for ordinary logits, but 2^440 in a
  // part at -1e10.  Differences from large maxima are exact wherever their exponential is not zero.)
  const bool huge = fabsf(top) > 0x1p16f;
  const float base = top * kLog2e;
  double sum = 0.0;
  if (!huge) {
#pragma unroll
    for (int i = 0; i < 32; i += 8) {
      float f = 0.0f;
#pragma unroll
      for (int e = 0; e < 8; ++e) f += __builtin_amdgcn_exp2f(__builtin_fmaf(v[i + e], kLog2e, -base));
      sum += f;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 32; ++i) sum += __builtin_amdgcn_exp2f((v[i] - top) * kLog2e);
  }
  sum = wave_sum_f64(sum);
  if (lane == 0) p.sums[id] = PartSum{sum, huge ? (double)top * kLog2e : (double)base};

  const uint32_t order = mine == -INFINITY ? 0 : order_of(mine);
  uint32_t bound = 0;
#pragma unroll
  for (int bit = 31; bit >= 16; --bit) {
    const uint32_t higher = bound | 1u << bit;
    if (__popcll(__ballot(order >= higher)) >= W) bound = higher;
  }
  const float least = bound > order_of(-3.4028234664e38f) ? value_of(bound) : -3.4028234664e38f;
  int n = 0;
#pragma unroll
  for (int i = 0; i < 32; ++i) {
    const uint64_t who = __ballot(v[i] >= least);
    if (!who) continue;
    const int at = n + __popcll(who & ((1ull << lane) - 1));
    if ((who >> lane & 1) && at < 64) s_keys[wave][at] = key_of(v[i], part * kPart + ((i / N) * 64 + lane) * N + i % N);
    n += __popcll(who);
  }
  if (n <= 64) {
    wave_sync();
    const uint64_t key = lane < n ? s_keys[wave][lane] : 0;
    const uint32_t lo = (uint32_t)key, hi = (uint32_t)(key >> 32);
    int rank = 0;
    for (int j = 0; j < n; ++j) {
      const uint64_t other = (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)hi, j) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)lo, j);
      rank += other > key;
    }
    if (lane < n && rank < W) keys[rank] = key;
    if (lane >= n && lane < W) keys[lane] = 0;
  } else {
    uint64_t last = ~0ull;
    for (int k = 0; k < W; ++k) {
      uint64_t best = 0;
#pragma unroll
      for (int i = 0; i < 32; ++i) {
        const uint64_t key = key_of(v[i], part * kPart + ((i / N) * 64 + lane) * N + i % N);
        if (key < last && key > best) best = key;
      }
      last = wave_max64(best);
      if (lane == 0) keys[k] = last;
    }
  }
}

// One workgroup per stream.  One wave joins the sums of a beam's parts, another takes the best of the parts' candidates.  Then the first wave merges
// the beams' sorted candidates, lane b holding the first of beam b that is not taken yet.
constexpr int kHeld = 4;      // keys of a beam that a lane keeps in registers
__global__ void __launch_bounds__(1024) beam_merge_kernel(SelectArgs p) {
  __shared__ uint64_t s_key[kMaxBeams][kMaxBeams];
  __shared__ double s_log[kMaxBeams];
  __shared__ int32_t s_token[kMaxBeams], s_parent[kMaxBeams], s_slot[kMaxBeams];
  __shared__ float s_score[kMaxBeams];
  const int s = blockIdx.x, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6, W = p.width;
  const int n_in = clamped(p.n_in, s, W), n_out = clamped(p.n_out, s, W);
  const float start = lane < n_in ? p.score_in[(int64_t)s * W + lane] : -INFINITY;      // read before any output is written: it may be the same memory
  const bool live = lane < n_in && is_finite(start);
  const bool was_done = live && p.done_in && p.done_in[(int64_t)s * W + lane];
  for (int job = wave; job < 2 * n_in; job += waves) {
    const int b = job >> 1;
    const int64_t row = (int64_t)s * W + b;
    const bool done = p.done_in && p.done_in[row];
    if (job & 1) {
      const PartSum *sums = p.sums + row * p.parts;
      double base = -INFINITY, sum = 0.0;
      if (!done) {
        for (int i = lane; i < p.parts; i += 64) base = max64(base, sums[i].base);
        base = wave_max64(base);
        for (int i = lane; i < p.parts; i += 64)
          if (sums[i].base != -INFINITY) sum += sums[i].sum * exp2(sums[i].base - base);
        sum = wave_sum_f64(sum);
      }
      if (lane == 0) s_log[b] = done ? 0.0 : (base + log2(sum)) / (double)kLog2e;
      continue;
    }
    if (done) {
      if (lane < W) s_key[b][lane] = lane == 0 ? key_of(0.0f, p.eos) : 0;
      continue;
    }
    const uint64_t *keys = p.keys + row * p.parts * W;
    const int n = p.parts * W;
    uint64_t held[kHeld];
#pragma unroll
    for (int i = 0; i < kHeld; ++i) held[i] = lane + 64 * i < n ? keys[lane + 64 * i] : 0;
    uint64_t last = ~0ull;
    for (int k = 0; k < W; ++k) {
      uint64_t best = 0;
#pragma unroll
      for (int i = 0; i < kHeld; ++i)
        if (held[i] < last && held[i] > best) best = held[i];
      for (int i = lane + 64 * kHeld; i < n; i += 64) {
        const uint64_t key = keys[i];
        if (key < last && key > best) best = key;
      }
      last = wave_max64(best);
      if (lane == 0) s_key[b][k] = last;
    }
  }
  __syncthreads();
  if (wave > 0) return;
  const double log_sum = live ? s_log[lane] : 0.0;
  int at = 0;
  uint64_t key = live ? s_key[lane][0] : 0;
  auto total_of = [&] { return key ? (double)start + ((double)value_of((uint32_t)(key >> 32)) - log_sum) : -(double)INFINITY; };
  double total = total_of();
  int n = 0;
  for (; n < n_out; ++n) {
    const double best = wave_max64(total);
    const uint64_t who = __ballot(key != 0 && total == best);
    if (!who) break;
    const int b = __ffsll((unsigned long long)who) - 1;
    if (lane == b) {
      const int token = (int)~(uint32_t)key;
      s_token[n] = was_done || token == p.eos ? token | (int)0x80000000 : token;       // the top bit: done
      s_parent[n] = b;
      s_score[n] = (float)total;
      ++at;
      key = at < W ? s_key[lane][at] : 0;
      total = total_of();
    }
  }
  wave_sync();
  if (p.keep_slots) {
    if (lane == 0) {
      for (int j = 0; j < W; ++j) s_slot[j] = -1;
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
    wave_sync();
  }
  if (lane < W) {
    const int64_t o = (int64_t)s * W + lane;
    const int j = p.keep_slots ? s_slot[lane] : lane < n ? lane : -1;
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

// A thread holds COLS columns of V bytes of all of a stream's slots that take over another's, so that a slot is read before any is written.  Two columns
// keep twice the reads in flight (64 x 5 slots of 90 .. 320 positions of 5 KB, two layers: 207 us with one, 84 with two, 85 with four).
template <typename V, int MAXW, int COLS>
__global__ void __launch_bounds__(256) beam_reorder_kernel(ReorderArgs p) {
  const int64_t ls = blockIdx.x / p.chunks, chunk = blockIdx.x % p.chunks;      // (layer, stream)
  const int s = (int)(ls % p.B);
  int64_t n = p.len ? p.len[s] : p.n_pos;
  n = (n < 0 ? 0 : n < p.n_pos ? n : p.n_pos) * p.pos_bytes;
  const int64_t at = (chunk * 256 * COLS + threadIdx.x) * sizeof(V);
  if (chunk * 256 * COLS * (int64_t)sizeof(V) >= n) return;
  const char *src = (const char *)p.src + ls * p.width * p.slot_bytes + at;
  char *dst = (char *)p.dst + ls * p.width * p.slot_bytes + at;
  V v[MAXW][COLS];
  int from[MAXW];
#pragma unroll
  for (int j = 0; j < MAXW; ++j) {
    from[j] = j < p.width ? p.parent[(int64_t)s * p.width + j] : -1;
    if (from[j] >= p.width || (p.src == p.dst && from[j] == j)) from[j] = -1;
  }
#pragma unroll
  for (int j = 0; j < MAXW; ++j)
    if (from[j] >= 0)
#pragma unroll
      for (int c = 0; c < COLS; ++c)
        if (at + c * 256 * (int64_t)sizeof(V) < n) v[j][c] = *(const V *)(src + from[j] * p.slot_bytes + c * 256 * sizeof(V));
#pragma unroll
  for (int j = 0; j < MAXW; ++j)
    if (from[j] >= 0)
#pragma unroll
      for (int c = 0; c < COLS; ++c)
        if (at + c * 256 * (int64_t)sizeof(V) < n) *(V *)(dst + j * p.slot_bytes + c * 256 * sizeof(V)) = v[j][c];
}

template <typename V, int MAXW, int COLS>
void launch_reorder(ReorderArgs p, int64_t layers_streams, hipStream_t s) {
  p.chunks = (p.slot_bytes + 256 * COLS * (int64_t)sizeof(V) - 1) / (256 * COLS * (int64_t)sizeof(V));
  beam_reorder_kernel<V, MAXW, COLS><<<dim3((uint32_t)(layers_streams * p.chunks)), 256, 0, s>>>(p);
}

template <typename V>
void launch_reorder(const ReorderArgs &p, int64_t layers_streams, hipStream_t s) {
  if (p.width <= 4) launch_reorder<V, 4, 2>(p, layers_streams, s);
  else if (p.width <= 8) launch_reorder<V, 8, 2>(p, layers_streams, s);
  else if (p.width <= 16) launch_reorder<V, 16, 2>(p, layers_streams, s);
  else launch_reorder<V, 32, 1>(p, layers_streams, s);
}

}  // namespace
}  // namespace wf

using namespace wf;
using namespace wf::host;

namespace {

int parts_of(int32_t n_vocab) { return (int)(((int64_t)n_vocab + kPart - 1) / kPart); }

int check_step(const wf_beam_step *a) {
  if (!a) return fail(WF_E_INVALID_ARG, "step is NULL");
  if (a->dtype != WF_DTYPE_F32 && a->dtype != WF_DTYPE_BF16) return fail(WF_E_INVALID_ARG, "logits dtype = %d", a->dtype);
  if (a->B < 1) return fail(WF_E_INVALID_ARG, "B = %d, need B >= 1", a->B);
  if (a->width < 1 || a->width > kMaxBeams) return fail(WF_E_INVALID_ARG, "width = %d (supported: 1 .. %d)", a->width, kMaxBeams);
  if (a->n_vocab < 1) return fail(WF_E_INVALID_ARG, "n_vocab = %d", a->n_vocab);
  if ((int64_t)a->B * a->width >= 1 << 22) return fail(WF_E_CAPACITY, "B * width = %lld beams (supported: below 2^22)", (long long)a->B * a->width);
  if (a->n_vocab > 1 << 28 || (int64_t)a->B * a->width * parts_of(a->n_vocab) >= (int64_t)1 << 32)
    return fail(WF_E_CAPACITY, "%d streams of %d beams over %d tokens: too many parts", a->B, a->width, a->n_vocab);
  return WF_OK;
}

}  // namespace

extern "C" {

int64_t wf_beam_select_workspace(const wf_beam_step *a) {
  const int rc = check_step(a);
  return rc ? rc : (int64_t)a->B * a->width * parts_of(a->n_vocab) * (int64_t)(sizeof(PartSum) + 8 * a->width);
}

int wf_op_beam_select(const wf_beam_step *a, void *hip_stream) {
  const int64_t need = wf_beam_select_workspace(a);
  if (need < 0) return (int)need;
  if (!a->logits_dev || !a->score_in_dev || !a->token_out_dev || !a->parent_out_dev || !a->score_out_dev)
    return fail(WF_E_INVALID_ARG, "logits_dev, score_in_dev or one of the outputs is NULL");
  if ((uintptr_t)a->logits_dev % (a->dtype == WF_DTYPE_BF16 ? 2 : 4)) return fail(WF_E_INVALID_ARG, "logits_dev is not aligned to its type");
  if (a->ld < a->n_vocab) return fail(WF_E_INVALID_ARG, "ld = %lld, need at least n_vocab = %d", (long long)a->ld, a->n_vocab);
  if ((a->done_in_dev != nullptr) != (a->done_out_dev != nullptr)) return fail(WF_E_INVALID_ARG, "done_in_dev and done_out_dev go together");
  if (a->done_in_dev && (a->eos < 0 || a->eos >= a->n_vocab)) return fail(WF_E_INVALID_ARG, "eos = %d outside [0, %d)", a->eos, a->n_vocab);
  if (!a->workspace_dev || (uintptr_t)a->workspace_dev % 16) return fail(WF_E_INVALID_ARG, "workspace_dev is NULL or not aligned to 16 bytes");
  if (a->workspace_bytes < need) return fail(WF_E_CAPACITY, "workspace of %lld bytes, need %lld", (long long)a->workspace_bytes, (long long)need);
  const int parts = parts_of(a->n_vocab);
  const int64_t waves = (int64_t)a->B * a->width * parts;
  PartSum *const sums = (PartSum *)a->workspace_dev;
  const SelectArgs p{a->logits_dev, a->ld, a->n_in_dev, a->n_out_dev, a->score_in_dev, a->done_in_dev, a->token_out_dev, a->parent_out_dev, a->score_out_dev,
                     a->done_out_dev, sums, (uint64_t *)(sums + waves), a->B, a->width, a->n_vocab, a->done_in_dev ? a->eos : -1, a->keep_slots, parts};
  const hipStream_t s = (hipStream_t)hip_stream;
  const dim3 grid(a->B * a->width, (parts + 3) / 4);
  if (a->dtype == WF_DTYPE_BF16) beam_parts_kernel<__bf16><<<grid, 256, 0, s>>>(p);
  else beam_parts_kernel<float><<<grid, 256, 0, s>>>(p);
  beam_merge_kernel<<<a->B, 64 * std::min(2 * a->width, 16), 0, s>>>(p);
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
  ReorderArgs p{dst_dev, src_dev, parent_dev, len_dev, B, width, n_pos, pos_bytes, slot, (slot - 1) / (256 * vec) + 1};      // the most workgroups of any form
  if ((int64_t)n_layers * B * (double)p.chunks >= (double)(1 << 24))
    return fail(WF_E_CAPACITY, "%lld bytes in %d layers, moved %d at a time: more than 2^32 threads", (long long)all, n_layers, vec);
  const int64_t ls = (int64_t)n_layers * B;
  const hipStream_t s = (hipStream_t)hip_stream;
  if (vec == 16) launch_reorder<u32x4>(p, ls, s);
  else if (vec == 4) launch_reorder<uint32_t>(p, ls, s);
  else launch_reorder<uint8_t>(p, ls, s);
  const hipError_t err = hipGetLastError();
  return err == hipSuccess ? WF_OK : fail(WF_E_HIP, "beam_reorder launch: %s", hipGetErrorString(err));
}

}  // extern "C"
