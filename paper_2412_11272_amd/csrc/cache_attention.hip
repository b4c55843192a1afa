// Attention of a few queries per sequence over a key / value cache (one new token, the beams of a stream, a tree of drafted tokens).  The
// definition is stated with wf_op_cache_attention in include/wf_encoder.h.
//
// Bound by memory: a key / value pair of a head is 256 bytes in bf16 (130 in 8 bits) and serves only the query rows that share the
// head (queries of the sequence times query heads per key head), so the cache goes from memory straight to registers, once,
// and nothing of it through the LDS.  A workgroup has one key / value head of one sequence, up to 16 * NQ of its query rows and a range of keys; its
// waves take tiles of 32 keys in turn, each with a running maximum and sum of its own, and join in the LDS at the end.  Measured on one MI355X (reading
// alone reaches 6.2 TB/s): 320 sequences of 512 keys of 20 heads 6.1 TB/s in bf16, 5.5 in 8 bits, 6.2 in fp32; five beams each of 64 streams of
// 51 .. 1525 keys 4.4, 3.6 and 4.5 (57, 36 and 111 us): 1280 workgroups on 768 or, in 8 bits, 1024 places leave a last round partly filled (720 keys each:
// 4.9, 4.0 and 4.7), and the uneven lengths cost the rest; trees of 68 .. 160 rows are held up by the softmax's and the weights' instructions, 2.1 TB/s and
// 260 TFLOP/s.  fp32 queries over 8 bits are bound by the fp32 matrix instructions, 64 of 32 cycles a tile whatever it weighs: 3.0 TB/s, and 67 us for
// the beams; such trees 520 us over fp32, 640 over 8 bits.
//
// A tile's products, on the 16 x 16 matrix instructions, run transposed like those of the prefill attention: S^T = K Q^T, O^T = V^T P^T.
// A lane (n = lane % 16, g = lane / 16) then holds
//   K as loaded       key 16 s + n of the tile (s = 0, 1), values 16 g .. 16 g + 15: consecutive bytes; which values meet in one instruction is
//                     free as long as the queries' registers follow (value 16 g + 8 f + i at place i of the f-th instruction)
//   S^T               query n, keys 16 s + 4 g + i, i = 0 .. 3, so that a query's maximum is four registers, twice, and two exchanges
//   P^T               the same registers: place 4 s + i of the lane's share of the second product's reduction is key 16 s + 4 g + i
//   V as loaded       values 4 n .. 4 n + 3 of those same eight keys: consecutive bytes, 16 lanes a whole row of the head
//   O^T               query n, values 16 g + 4 i + t from the t-th of four instructions (which takes value 4 n + t of each lane's keys)
// What remains between loading V and multiplying is to pair two keys' values in a register: one byte permutation for two of them.
//
// Rounding: logits, statistics and sums are fp32.  Next to bf16 the weights enter as the sum of two bf16 parts (2^-18 of a weight is lost, where
// one part would lose 2^-9, and the output's rounding 2^-9 of the result): twice the second product's instructions.  A third part would keep all 24 bits; it
// leaves the error against 64 bits as it is (trees, relative: 1.66440e-3 either way) and takes 156 us for the trees instead of 138, 35.5 for beams instead
// of 33.5.  Values of the 8-bit caches with their
// powers of two are exact as fp32 operands, and as bf16 operands from 2^-124 on.
#include "cache_device.h"
#include "host_runtime.h"

#include <cmath>
#include <type_traits>

namespace wf {

namespace {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

constexpr int kTile = 32;      // keys
constexpr int kMaxSplits = 64;

struct AttendArgs {
  CacheView c;
  const void *q;
  void *out;
  int64_t ldq, ldo;
  const int32_t *cu_q, *row, *len;
  const uint32_t *mask;
  const int32_t *mask_from;
  float *part;                       // [sequence][key head][row][split][64], then the maxima and sums [..][split][2]
  float *part_ml;
  int32_t n_heads, group, n_seqs, n_q_rows, max_q, max_len, mask_words;
  int32_t chunks, n_split, split_keys;      // query row chunks of a head, ranges of split_keys keys
  float scale;
};

// Ranges of split_keys keys that n >= 1 keys take; n + split_keys may pass 2^31.
__host__ __device__ constexpr int ranges_of(int n, int split_keys) { return (n - 1) / split_keys + 1; }
static_assert(ranges_of(1, kTile) == 1 && ranges_of(kTile + 1, kTile) == 2 && ranges_of((1 << 30) + 1, 1 << 30) == 2 && ranges_of(INT32_MAX, 1 << 30) == 2, "");

// The keys of sequence s: their number and the first row.
__device__ __forceinline__ int sequence_keys(const AttendArgs &p, int s, int64_t *row0) {
  *row0 = p.row[s];
  int64_t n = p.len[s];
  n = n < p.max_len ? n : p.max_len;
  if (*row0 < 0) n = 0;
  n = n < p.c.n_rows - *row0 ? n : p.c.n_rows - *row0;
  return n > 0 ? (int)n : 0;
}
__device__ __forceinline__ int sequence_queries(const AttendArgs &p, int s, int *first) {
  const int a = p.cu_q[s], b = p.cu_q[s + 1];
  *first = a;
  if (a < 0 || b <= a) return 0;
  int64_t n = (int64_t)b - a;
  n = n < p.max_q ? n : p.max_q;
  n = n < (int64_t)p.n_q_rows - a ? n : (int64_t)p.n_q_rows - a;
  return n > 0 ? (int)n : 0;
}

template <int CACHE> struct Format;
template <> struct Format<WF_DTYPE_BF16> { static constexpr int es = 2; };
template <> struct Format<WF_DTYPE_F32> { static constexpr int es = 4; };
template <> struct Format<WF_DTYPE_F8> { static constexpr int es = 1; };

// What a lane holds of a tile (see above), and of the masks and exponents that go with it.
template <int CACHE, int NQ, bool MASK>
struct Tile {
  static constexpr int KD = 4 * Format<CACHE>::es, VD = Format<CACHE>::es;      // registers a key sub-tile, a value row
  uint32_t k[2][KD], v[8][VD];
  uint32_t ke[CACHE == WF_DTYPE_F8 ? 2 : 1], ve[CACHE == WF_DTYPE_F8 ? 2 : 1];      // exponents: of the lane's keys, of four of its value rows
  uint32_t word[MASK ? NQ : 1][2];
};

// N registers from `at` bytes on: of memory, or of a buffer (zero past its end).
template <int N>
__device__ __forceinline__ void load_dwords(uint32_t (&d)[N], const unsigned char *base, uint32_t at) {
#pragma unroll
  for (int i = 0; i < N; i += 4) {
    const u32x4 x = *(const u32x4 *)(base + at + 4 * i);
    d[i] = x[0]; d[i + 1] = x[1]; d[i + 2] = x[2]; d[i + 3] = x[3];
  }
}
template <int N>
__device__ __forceinline__ void load_dwords(uint32_t (&d)[N], __amdgpu_buffer_rsrc_t base, uint32_t at) {
  if constexpr (N >= 4) {
#pragma unroll
    for (int i = 0; i < N; i += 4) {
      const u32x4 x = __builtin_amdgcn_raw_buffer_load_b128(base, at + 4 * i, 0, 0);
      d[i] = x[0]; d[i + 1] = x[1]; d[i + 2] = x[2]; d[i + 3] = x[3];
    }
  } else if constexpr (N == 2) {
    const u32x2 x = __builtin_amdgcn_raw_buffer_load_b64(base, at, 0, 0);
    d[0] = x[0]; d[1] = x[1];
  } else {
    d[0] = __builtin_amdgcn_raw_buffer_load_b32(base, at, 0, 0);
  }
}

__device__ __forceinline__ uint32_t pack(bf16x2 x) { return __builtin_bit_cast(uint32_t, x); }
// Two e4m3 values times a power of two, exactly; of `factor` only the exponent's bits 23 .. 30 count (0: 2^-127), whatever stands beside them.
__device__ __forceinline__ uint32_t f8_pair(uint32_t x, uint32_t factor, bool high) {
  const float f = __builtin_bit_cast(float, factor);
  return pack(high ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, f, true) : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, f, false));
}
__device__ __forceinline__ f32x2 f8_pair_f32(uint32_t x, uint32_t factor, bool high) {
  const float f = __builtin_bit_cast(float, factor);
  return high ? __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(x, f, true) : __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(x, f, false);
}
// Byte i of four exponents where a factor has it
__device__ __forceinline__ uint32_t exponent_of(uint32_t four, int i) { return i < 3 ? four << (23 - 8 * i) : four >> 1; }
__device__ __forceinline__ bool is_finite(float x) { return (__builtin_bit_cast(uint32_t, x) & 0x7f800000u) != 0x7f800000u; }

__device__ __forceinline__ f32x4 mma(const uint32_t (&a)[4], const uint32_t (&b)[4], f32x4 c) {
  const u32x4 x = {a[0], a[1], a[2], a[3]}, y = {b[0], b[1], b[2], b[3]};
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x), __builtin_bit_cast(bf16x8, y), c, 0, 0, 0);
}

// A product that is rounded, whatever is added to it: the largest logit is its reference then, of any size.  (fp32, where an instruction more
// costs nothing next to the matrix instructions.)
__device__ __forceinline__ float rounded_product(float a, float b) {
#pragma clang fp contract(off)
  return a * b;
}

// A wave's running state for 16 query rows: lane (n, g) has row n's reference (in powers of two), its share of the sum, and values 16 g + 4 i + t.
struct State {
  float m, l;
  f32x4 o[4];
};

// One row by one wave, 64 keys at a time, first a lane per key, then a lane per value: what a row does not see is not touched.
struct RowState {
  float m, l, o;
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
template <typename T, int CACHE>
__device__ __forceinline__ RowState one_row(const AttendArgs &p, int64_t r, int hq, int h, int64_t row0, int k_from, int k_to, int from) {
  const int lane = threadIdx.x & 63;
  const T *q = (const T *)p.q + r * p.ldq + hq * 64;
  const float c = p.scale * 1.4426950408889634f;
  RowState w{-INFINITY, 0.0f, 0.0f};
#pragma unroll 1
  for (int64_t k0 = k_from; k0 < k_to; k0 += 64) {
    const int64_t k = k0 + lane;
    bool seen = k < k_to;
    if (seen && k >= from) {
      const int64_t at = k - from;
      seen = at < 32 * (int64_t)p.mask_words && (p.mask[r * p.mask_words + at / 32] >> (at & 31) & 1);
    }
    float x = -INFINITY;
    if (seen) {
      x = 0.0f;
#pragma unroll 1
      for (int d = 0; d < 64; ++d) x += (float)q[d] * cache_value<CACHE>(p.c, row0 + k, h, 0, d);
      x *= c;
    }
    const uint64_t some = __ballot(seen);
    if (!some) continue;
    const float m = fmaxf(w.m, wave_max(x)), base = m == -INFINITY ? 0.0f : m;
    const float e = seen ? __builtin_amdgcn_exp2f(x - base) : 0.0f, keep = __builtin_amdgcn_exp2f(w.m - base);
    w.l = w.l * keep + wave_sum(e);
    w.o *= keep;
    w.m = m;
#pragma unroll 1
    for (int j = 0; j < 64; ++j)
      if (some >> j & 1) w.o += __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, e), j)) * cache_value<CACHE>(p.c, row0 + k0 + j, h, 1, lane);
  }
  return w;
}

template <typename T, int CACHE, int NQ, int NW, bool MASK>
__global__ void __launch_bounds__(64 * NW, NQ == 1 && sizeof(T) == 2 ? 3 : 2) cache_attention_kernel(AttendArgs p) {
  constexpr bool BF = sizeof(T) == 2;
  constexpr int es = Format<CACHE>::es;
  typedef Tile<CACHE, NQ, MASK> Tile;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n16 = lane & 15, g = lane >> 4;
  const int H = p.c.n_heads;
  // Workgroups go to the 8 XCDs in turn: those that read the same keys for other rows come 8 behind each other, to the same L2.  The heads are
  // turned by one from one sequence to the next: with 8 or 16 of them, every XCD would read the same few of them only, whose rows lie at the same
  // places of the memory's channels (five beams of 64 streams, 20 heads: bf16 60.7 -> 56.2 us, fp32 110 -> 103; drafted trees, 8 heads: 146 -> 140).
  int id = blockIdx.x, chunk = 0;
  if (p.chunks > 1) {
    chunk = id / 8 % p.chunks;
    id = id / (8 * p.chunks) * 8 + id % 8;
  }
  const int h = (id % H + id / H) % H; id /= H;
  const int s = id % p.n_seqs, z = id / p.n_seqs;
  if (z >= p.n_split) return;

  int q_first;
  const int rows = sequence_queries(p, s, &q_first) * p.group - chunk * 16 * NQ;      // of this chunk on
  if (rows <= 0) return;
  int64_t row0;
  const int n = sequence_keys(p, s, &row0);
  const int64_t split_from = (int64_t)z * p.split_keys;
  if (z > 0 && split_from >= n) return;
  const int t_end = (int)(((split_from + p.split_keys < n ? split_from + p.split_keys : n) + kTile - 1) / kTile);      // split_keys is a multiple of a tile
  const int t_first = (int)(split_from / kTile) + wave;
  const int n_tiles_q = rows >= 16 * NQ ? NQ : (rows + 15) / 16;

  const uint32_t row_bytes = H * 128u * es;
  const unsigned char *seq = (const unsigned char *)p.c.data + row0 * row_bytes + (CACHE == WF_DTYPE_F8 ? h * 128 : h * 64 * es);
  const uint32_t v_off = CACHE == WF_DTYPE_F8 ? 64u : H * 64u * es;
  const uint8_t *k_exps = CACHE == WF_DTYPE_F8 ? p.c.exps + 2 * h * p.c.n_rows + row0 : nullptr;
  const uint8_t *v_exps = CACHE == WF_DTYPE_F8 ? k_exps + p.c.n_rows : nullptr;

  // The lane's query of each of the 16-row tiles: in registers, or, for several tiles, in the LDS in the order the lanes read it
  constexpr int QD = BF ? 8 : 16;
  __shared__ u32x4 s_q[NQ > 1 ? NQ : 1][NQ > 1 ? QD / 4 : 1][64];
  uint32_t q_one[QD];
  const uint32_t *words[MASK ? NQ : 1];
  (void)words;
#pragma unroll
  for (int t = 0; t < NQ; ++t) {
    const int local = t * 16 + n16;
    const bool have = local < rows;
    const int row = chunk * 16 * NQ + (have ? local : 0);
    const int64_t r = q_first + row / p.group;
    if constexpr (MASK) words[t] = p.mask + r * p.mask_words;
    if (NQ > 1 && t % NW != wave) continue;
    load_dwords(q_one, (const unsigned char *)p.q + (r * p.ldq + (h * p.group + row % p.group) * 64 + 16 * g) * sizeof(T), 0);
    if (!have)
#pragma unroll
      for (int i = 0; i < QD; ++i) q_one[i] = 0;
    if (p.scale < 0.0f)               // so that the largest product is the largest logit
#pragma unroll
      for (int i = 0; i < QD; ++i) q_one[i] ^= BF ? 0x80008000u : 0x80000000u;
    if constexpr (NQ > 1)
#pragma unroll
      for (int i = 0; i < QD / 4; ++i) s_q[t][i][lane] = u32x4{q_one[4 * i], q_one[4 * i + 1], q_one[4 * i + 2], q_one[4 * i + 3]};
  }
  if constexpr (NQ > 1) __syncthreads();
  const int from = MASK && p.mask_from ? p.mask_from[s] : 0;

  // Sub-tiles of 16 keys go through buffers that end behind the sequence's last key: rows past it read as zero.
  const uint32_t k_lane = n16 * row_bytes + g * 16 * es, v_lane = 4 * g * row_bytes + v_off + n16 * 4 * es;
  auto load = [&](Tile &a, int tile) {
    const int left = n - tile * kTile;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int keys = left - 16 * u < 16 ? left - 16 * u : 16;
      const auto buffer = __builtin_amdgcn_make_buffer_rsrc((void *)(seq + ((int64_t)tile * kTile + 16 * u) * row_bytes), 0,
                                                            keys > 0 ? (keys - 1) * row_bytes + v_off + 64 * es : 0, 0x00027000);
      load_dwords(a.k[u], buffer, k_lane);
#pragma unroll
      for (int j = 0; j < 4; ++j) load_dwords(a.v[4 * u + j], buffer, v_lane + j * row_bytes);
    }
    if constexpr (CACHE == WF_DTYPE_F8) {
      const uint8_t *ke = k_exps + (int64_t)tile * kTile, *ve = v_exps + (int64_t)tile * kTile;
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        if (left >= kTile) {
          a.ke[u] = ke[16 * u + n16];
          __builtin_memcpy(&a.ve[u], ve + 16 * u + 4 * g, 4);
        } else {
          a.ke[u] = ke[16 * u + n16 < left ? 16 * u + n16 : left - 1];
          a.ve[u] = 0;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int key = 16 * u + 4 * g + i;
            a.ve[u] |= (uint32_t)ve[key < left ? key : left - 1] << (8 * i);
          }
        }
      }
    }
    if constexpr (MASK) {             // the two words that hold the tile's 32 bits
      const int64_t at = (int64_t)tile * kTile - from;
      const int64_t w = at >> 5;
      if (at > -kTile) {
#pragma unroll
        for (int t = 0; t < NQ; ++t)
#pragma unroll
          for (int i = 0; i < 2; ++i) a.word[t][i] = w + i >= 0 && w + i < p.mask_words ? words[t][w + i] : w + i < 0 ? ~0u : 0u;
      }
    }
  };
  // Bit k: the lane's query of tile t sees key k of the tile
  auto seen_keys = [&](const Tile &a, int tile, int t) -> uint32_t {
    const int left = n - tile * kTile;
    uint32_t w = left >= kTile ? ~0u : (1u << left) - 1;
    if constexpr (MASK) {
      const int64_t at = (int64_t)tile * kTile - from;
      if (at > -kTile) w &= (uint32_t)((((uint64_t)a.word[t][1] << 32) | a.word[t][0]) >> (at & 31));
    }
    return w;
  };

  State st[NQ];
  // exp(s scale) = exp2(s c); never 0, so that a key that is not seen stays at -infinity
  const float c = fmaxf(fabsf(p.scale) * 1.4426950408889634f, 0x1p-149f);

  // The values with pairs of keys next to each other, as the second product takes them
  auto values = [&](const Tile &a, uint32_t (&vt)[4][BF ? 4 : 8]) {
    if constexpr (BF) {
      uint32_t v[8][2];
#pragma unroll
      for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          if constexpr (CACHE == WF_DTYPE_F8) v[j][i] = f8_pair(a.v[j][0], exponent_of(a.ve[j >> 2], j & 3), i == 1);
          else v[j][i] = a.v[j][i];
        }
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          vt[2 * i][j] = __builtin_amdgcn_perm(v[2 * j + 1][i], v[2 * j][i], 0x05040100);
          vt[2 * i + 1][j] = __builtin_amdgcn_perm(v[2 * j + 1][i], v[2 * j][i], 0x07060302);
        }
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if constexpr (CACHE == WF_DTYPE_F8) {
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const f32x2 x = f8_pair_f32(a.v[j][0], exponent_of(a.ve[j >> 2], j & 3), i == 1);
            const float x0 = x[0], x1 = x[1];
            vt[2 * i][j] = __builtin_bit_cast(uint32_t, x0);
            vt[2 * i + 1][j] = __builtin_bit_cast(uint32_t, x1);
          }
        } else {
#pragma unroll
          for (int t = 0; t < 4; ++t) vt[t][j] = a.v[j][t];
        }
      }
    }
  };
  // FREE: every row sees every key of the tile.
  auto compute = [&](const Tile &a, int tile, auto free) {
    constexpr bool FREE = decltype(free)::value;
    uint32_t vt[4][BF ? 4 : 8];
    if constexpr (NQ > 1) values(a, vt);
    // ---- keys
    uint32_t kt[2][QD];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      if constexpr (CACHE == WF_DTYPE_F8) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            if constexpr (BF) {
              kt[u][2 * i + e] = f8_pair(a.k[u][i], a.ke[u] << 23, e == 1);
            } else {
              const f32x2 x = f8_pair_f32(a.k[u][i], a.ke[u] << 23, e == 1);
              const float x0 = x[0], x1 = x[1];
              kt[u][4 * i + 2 * e] = __builtin_bit_cast(uint32_t, x0);
              kt[u][4 * i + 2 * e + 1] = __builtin_bit_cast(uint32_t, x1);
            }
          }
      } else {
#pragma unroll
        for (int i = 0; i < QD; ++i) kt[u][i] = a.k[u][i];
      }
    }
    // Two query tiles side by side: one's matrix instructions beside the other's exponentials.  (Behind an odd number of tiles an empty one is computed.)
    constexpr int GT = NQ < 2 ? NQ : 2;
#pragma unroll
    for (int t0 = 0; t0 < NQ; t0 += GT) {
      if (t0 > 0 && t0 >= n_tiles_q) break;
      float x[GT][8];
      bool rise = false;
#pragma unroll
      for (int k = 0; k < GT; ++k) {
        const int t = t0 + k;
        uint32_t qa[QD];
#pragma unroll
        for (int i = 0; i < QD; ++i) qa[i] = q_one[i];
        if constexpr (NQ > 1)
#pragma unroll
          for (int i = 0; i < QD / 4; ++i) {
            const u32x4 y = s_q[t][i][lane];
            qa[4 * i] = y[0]; qa[4 * i + 1] = y[1]; qa[4 * i + 2] = y[2]; qa[4 * i + 3] = y[3];
          }
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          f32x4 d{0.0f, 0.0f, 0.0f, 0.0f};
          if constexpr (BF) {
#pragma unroll
            for (int f = 0; f < 2; ++f) {
              const uint32_t ka[4] = {kt[u][4 * f], kt[u][4 * f + 1], kt[u][4 * f + 2], kt[u][4 * f + 3]};
              const uint32_t qb[4] = {qa[4 * f], qa[4 * f + 1], qa[4 * f + 2], qa[4 * f + 3]};
              d = mma(ka, qb, d);
            }
          } else {
#pragma unroll
            for (int i = 0; i < 16; ++i)
              d = __builtin_amdgcn_mfma_f32_16x16x4f32(__builtin_bit_cast(float, kt[u][i]), __builtin_bit_cast(float, qa[i]), d, 0, 0, 0);
          }
#pragma unroll
          for (int i = 0; i < 4; ++i) x[k][4 * u + i] = d[i];
        }
        if constexpr (!FREE) {
          const uint32_t mine = seen_keys(a, tile, t) >> (4 * g);
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (!(mine >> (16 * (j >> 2) + (j & 3)) & 1)) x[k][j] = -INFINITY;
        }
        float top = x[k][0];
#pragma unroll
        for (int j = 1; j < 8; ++j) top = fmaxf(top, x[k][j]);
        rise |= (top > -INFINITY) & (top * c > st[t].m + 8.0f);
      }
      // A row's reference follows its maximum only where that is 2^8 above it: weights of up to 2^8 lose nothing in fp32.  The reference stays
      // finite: against one of infinity even the largest logit's weight would be 0, and a row of logits beyond fp32 would look like one that sees nothing.
      if (__ballot(rise)) {
#pragma unroll
        for (int k = 0; k < GT; ++k) {
          State &w = st[t0 + k];
          float top = x[k][0];
#pragma unroll
          for (int j = 1; j < 8; ++j) top = fmaxf(top, x[k][j]);
          const Pair rp = row_pair(top);
          top = half_max(fmaxf(rp.a, rp.b));
          top = top == -INFINITY ? w.m : fmaxf(w.m, fminf(top * c, 3.4028234664e38f));
          const float keep = top == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(w.m - top);
          w.l *= keep;
#pragma unroll
          for (int i = 0; i < 4; ++i) w.o[i] *= keep;
          w.m = top;
        }
      }
#pragma unroll
      for (int k = 0; k < GT; ++k) {
        State &w = st[t0 + k];
        const float base = w.m == -INFINITY ? 0.0f : w.m;
#pragma unroll
        for (int j = 0; j < 8; ++j) x[k][j] = __builtin_amdgcn_exp2f(BF ? __builtin_fmaf(x[k][j], c, -base) : rounded_product(x[k][j], c) - base);
        w.l += ((x[k][0] + x[k][1]) + (x[k][2] + x[k][3])) + ((x[k][4] + x[k][5]) + (x[k][6] + x[k][7]));
        if constexpr (NQ == 1) values(a, vt);      // once the keys' registers are free
        if constexpr (BF) {
          uint32_t hi[4], lo[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            hi[j] = pack(__builtin_convertvector(f32x2{x[k][2 * j], x[k][2 * j + 1]}, bf16x2));
            const f32x2 rest = {x[k][2 * j] - __builtin_bit_cast(float, hi[j] << 16), x[k][2 * j + 1] - __builtin_bit_cast(float, hi[j] & 0xffff0000u)};
            lo[j] = pack(__builtin_convertvector(rest, bf16x2));
          }
#pragma unroll
          for (int i = 0; i < 4; ++i) w.o[i] = mma(vt[i], hi, mma(vt[i], lo, w.o[i]));
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) w.o[i] = __builtin_amdgcn_mfma_f32_16x16x4f32(__builtin_bit_cast(float, vt[i][j]), x[k][j], w.o[i], 0, 0, 0);
        }
      }
    }
  };
#pragma unroll
  for (int t = 0; t < NQ; ++t) {
    st[t].m = -INFINITY;
    st[t].l = 0.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i) st[t].o[i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  }
  // One tile is in use, one on its way (two on their way gain nothing: 39.4 us against 38.4 with five beams of 64 streams in 8 bits).
  // The two change places by an unrolled index: written out one after the other, the same steps leave the compiler short of registers (355 us against
  // 138 with the drafted trees).
  Tile ring[2];
  int tile = t_first;
  if (tile < t_end) load(ring[0], tile);
  const int t_free = MASK ? (from < n ? from > 0 ? from : 0 : n) / kTile : n / kTile;      // tiles before it are free
  while (tile < t_end && tile < t_free) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      if (tile + NW < t_end) load(ring[1 - i], tile + NW);
      compute(ring[i], tile, std::true_type{});
      tile += NW;
      if (tile >= t_end || tile >= t_free) {
        if (i == 0) ring[0] = ring[1];
        break;
      }
    }
  }
  while (tile < t_end) {
    if (tile + NW < t_end) load(ring[1], tile + NW);
    compute(ring[0], tile, std::false_type{});
    ring[0] = ring[1];
    tile += NW;
  }
  const bool whole = p.n_split == 1 || n <= p.split_keys;      // no other workgroup has keys of this sequence
  const int64_t part_at = (((int64_t)s * H + h) * p.chunks + chunk) * 16 * NQ * p.n_split + z;      // of row 0 of the chunk; a row on: n_split

  // 0 x infinity and 0 x NaN of values that a row does not see, and infinity x the two parts of a weight, leave the result not finite, whatever
  // follows.  Next to a reference of 2^30 and more, rounded to whole numbers and coarser, products that are not rounded (bf16) give weights of 0 or
  // infinity.  Then, and only then, the rows are computed one by one: all of the workgroup, since what one row does not see spoils every other that shares
  // the tile, and slowly, a lane a key (one key of NaN in each head: 64 x 5 beams of 20 heads where it is in one stream's cache 57 -> 261 us,
  // in 8 bits 36 -> 467; hidden in one of four trees 166 us -> 9 ms).
  if constexpr (BF || MASK) {
    bool fine = true;
#pragma unroll
    for (int t = 0; t < NQ; ++t)
      if (t * 16 + n16 < rows) {
        if constexpr (BF) fine = fine && (fabsf(st[t].m) < 0x1p30f || st[t].m == -INFINITY);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) fine = fine && is_finite(st[t].o[i][e]);
      }
    if (__syncthreads_or(!fine)) {
      const int to = (int)(split_from + p.split_keys < n ? split_from + p.split_keys : n);
      for (int local = wave; local < rows && local < 16 * NQ; local += NW) {
        const int row = chunk * 16 * NQ + local;
        const int64_t r = q_first + row / p.group;
        const int hq = h * p.group + row % p.group;
        const RowState w = one_row<T, CACHE>(p, r, hq, h, row0, (int)split_from, to, MASK ? from : INT32_MAX);
        if (whole) {
          ((T *)p.out)[r * p.ldo + hq * 64 + lane] = (T)(w.l != 0.0f ? w.o / w.l : 0.0f);
        } else {
          const int64_t at = part_at + (int64_t)local * p.n_split;
          p.part[at * 64 + lane] = w.o;
          if (lane == 0) { p.part_ml[2 * at] = w.m; p.part_ml[2 * at + 1] = w.l; }
        }
      }
      return;
    }
  }

  // ---- the waves' parts meet
  constexpr int kRow = 68;       // floats of a row in the LDS: 64 and room against bank conflicts
  __shared__ __attribute__((aligned(16))) float s_o[NW][16][kRow];
  __shared__ float s_m[NW][16], s_l[NW][16];
#pragma unroll
  for (int t = 0; t < NQ; ++t) {
    if (t > 0 && t >= n_tiles_q) break;
    if (t > 0) __syncthreads();
    const Pair rp = row_pair(st[t].l);
    const float l = half_sum(rp.a + rp.b);
    if (g == 0) { s_m[wave][n16] = st[t].m; s_l[wave][n16] = l; }
#pragma unroll
    for (int i = 0; i < 4; ++i) *(f32x4 *)&s_o[wave][n16][16 * g + 4 * i] = f32x4{st[t].o[0][i], st[t].o[1][i], st[t].o[2][i], st[t].o[3][i]};
    __syncthreads();
    for (int e = threadIdx.x; e < 256; e += 64 * NW) {
      const int q = e >> 4, d = (e & 15) * 4;
      float m = s_m[0][q];
#pragma unroll
      for (int w = 1; w < NW; ++w) m = fmaxf(m, s_m[w][q]);
      const float base = m == -INFINITY ? 0.0f : m;
      f32x4 o{0.0f, 0.0f, 0.0f, 0.0f};
      float l_all = 0.0f;
#pragma unroll
      for (int w = 0; w < NW; ++w) {
        if (s_l[w][q] == 0.0f) continue;                       // saw nothing
        const float f = __builtin_amdgcn_exp2f(s_m[w][q] - base);
        o += *(const f32x4 *)&s_o[w][q][d] * f;
        l_all += s_l[w][q] * f;
      }
      const int local = t * 16 + q;
      if (local >= rows) continue;
      const int row = chunk * 16 * NQ + local;
      if (whole) {
        const float inv = l_all != 0.0f ? 1.0f / l_all : 0.0f;
        o *= inv;
        T *dst = (T *)p.out + (int64_t)(q_first + row / p.group) * p.ldo + (h * p.group + row % p.group) * 64 + d;
        if constexpr (BF) *(bf16x4 *)dst = to_bf16x4(o);
        else *(f32x4 *)dst = o;
      } else {
        const int64_t at = part_at + (int64_t)local * p.n_split;
        *(f32x4 *)(p.part + at * 64 + d) = o;
        if (d == 0) { p.part_ml[2 * at] = m; p.part_ml[2 * at + 1] = l_all; }
      }
    }
  }
}

// The parts of the rows whose keys several workgroups shared: a wave a row.  Lane z has the maximum and sum of part z; the values are added by
// 16 lanes, four parts at a time.
template <typename T>
__global__ void __launch_bounds__(256) cache_attention_join_kernel(AttendArgs p, int rows_pad) {
  const int64_t unit = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lane = threadIdx.x & 63, d = (lane & 15) * 4, H = p.c.n_heads;
  const int64_t sh = unit / rows_pad;
  if (sh >= (int64_t)p.n_seqs * H) return;
  const int row = (int)(unit % rows_pad), s = (int)(sh / H), h = (int)(sh % H);
  int q_first;
  if (row >= sequence_queries(p, s, &q_first) * p.group) return;
  int64_t row0;
  const int n = sequence_keys(p, s, &row0);
  if (n <= p.split_keys) return;
  const int parts = ranges_of(n, p.split_keys);
  static_assert(kMaxSplits <= 64, "a lane per part");
  const f32x2 ml = lane < parts ? *(const f32x2 *)(p.part_ml + 2 * (unit * p.n_split + lane)) : f32x2{-INFINITY, 0.0f};
  const float m_one = ml[0], l_one = ml[1];
  const float m = wave_max(m_one), base = m == -INFINITY ? 0.0f : m;
  const float f_one = l_one == 0.0f ? 0.0f : __builtin_amdgcn_exp2f(m_one - base);      // no sum: saw nothing
  const float l = wave_sum(l_one * f_one);
  const float *part = p.part + unit * p.n_split * 64 + d;
  f32x4 o{0.0f, 0.0f, 0.0f, 0.0f};
  for (int z0 = 0; z0 < parts; z0 += 16) {
    f32x4 v[4];
    float f[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int z = z0 + 4 * i + (lane >> 4);
      f[i] = __shfl(f_one, z & 63);
      v[i] = z < parts ? *(const f32x4 *)(part + (int64_t)z * 64) : f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (z0 + 4 * i + (lane >> 4) < parts && f[i] != 0.0f) o += v[i] * f[i];
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float x = o[i];
    const Pair rp = row_pair(x);
    o[i] = half_sum(rp.a + rp.b);
  }
  if (lane >= 16) return;
  const float inv = l != 0.0f ? 1.0f / l : 0.0f;
  o *= inv;
  T *dst = (T *)p.out + (int64_t)(q_first + row / p.group) * p.ldo + (h * p.group + row % p.group) * 64 + d;
  if constexpr (sizeof(T) == 2) *(bf16x4 *)dst = to_bf16x4(o);
  else *(f32x4 *)dst = o;
}

struct Plan {
  int nq, nw, chunks, n_split, split_keys;
};

// Query rows of a workgroup: 16, 32 or 64.  Rows beyond that read the keys again, from the L2.  What decides is what the reading weighs:
//   bf16 over bf16: trees of 68 .. 160 rows over 20 000 .. 65 536 keys of 8 heads take 168 us with 64, 205 with 32; 16 x 64 rows over 1500 keys of 20
//     heads 41 and 44;
//   bf16 over 8 bits, half the bytes: 32 where two workgroups hold all rows (16 x 64 rows over 1500 keys of 20 heads 32 us with 32, 37 with 64;
//     64 x 64 over 51 .. 1525 62 and 69; 4 x 64 over 48 000 keys of 8 heads 78 and 92; but 64 x 64 over 1500 of 8 heads 43 and 39), and 64 beyond (132
//     rows over 4 x 40 000 keys of 8 heads 183 us with 32, 158 with 64; over 16 x 1500 26 and 32);
//   fp32 over fp32: 32 (16 x 64 rows over 1500 keys of 20 heads 90 us, 106 with 16; under a mask 97 and 109, though that kernel spills five registers;
//     64 do not fit);
//   fp32 over 8 bits: 16, its fp32 products outweigh a quarter of the bytes (16 x 64 rows over 1500 keys of 20 heads 79 us, 90 with 32; 32 over
//     4 x 20 000 of 8 heads 61 and 74; trees as above 627 and 623).
// Workgroups: keys are split where a chip of 256 compute units would not get four (eight, if they have more than 16 rows and so last long and unevenly)
// each: one token over 65 536 keys of 8 heads in 8 bits 23.2 us with 1024, 23.8 with 2048; the trees 163 and 147.  A part keeps 768 keys, between what short and
// what long sequences want: with 512, 1100 keys (then in two parts) of 20 heads take 12.4 us instead of 10.9, 30 sequences of them in 8 bits 27 instead of 24,
// 8192 keys of 20 heads 16.1 and 15.2; but 8 x 8192 keys of 8 heads 34.8 instead of 39.4, 16 x 4096 36.3 and 39.1.
// Waves: four share a sequence's tiles; where sequences are short and many, two or one (320 of them, 20 heads, 8 bits: 32 keys 26.5 us with four, 16.9 with
// two, 12.6 with one; 128 keys 37.1, 27.5, 25.5; 256 keys 47.7, 42.3, 43.2; 512 keys 75.9, 77.1, 80.4).
Plan plan_of(const wf_cache &c, const wf_cache_query &a) {
  Plan p{};
  const int64_t rows = (int64_t)std::min(a.max_q, std::max(a.n_q_rows, 1)) * (a.n_heads / c.n_heads);
  const bool f8 = c.dtype == WF_DTYPE_F8;
  p.nq = rows <= 16 || (f8 && a.dtype == WF_DTYPE_F32) ? 1 : rows <= (f8 ? 64 : 32) || a.dtype == WF_DTYPE_F32 ? 2 : 4;
  p.chunks = (int)((rows + 16 * p.nq - 1) / (16 * p.nq));
  const int64_t groups = (int64_t)a.n_seqs * c.n_heads * p.chunks, want = p.nq > 1 ? 2048 : 1024;
  int64_t n = groups >= want ? 1 : (want + groups - 1) / groups;
  n = std::min<int64_t>(std::min<int64_t>(n, std::max(1, a.max_len / 768)), kMaxSplits);
  p.split_keys = (int)std::min<int64_t>(host::round_up(std::max<int64_t>((a.max_len + n - 1) / n, kTile), kTile), INT32_MAX / kTile * kTile);
  p.n_split = (int)std::max<int64_t>(1, ((int64_t)a.max_len + p.split_keys - 1) / p.split_keys);
  p.nw = p.nq > 1 || groups < 1024 || a.max_len > 256 ? 4 : a.max_len > 64 ? 2 : 1;
  return p;
}

template <typename T, int CACHE, int NQ, int NW>
void launch_attend(const AttendArgs &p, dim3 grid, hipStream_t s) {
  if (p.mask) cache_attention_kernel<T, CACHE, NQ, NW, true><<<grid, 64 * NW, 0, s>>>(p);
  else cache_attention_kernel<T, CACHE, NQ, NW, false><<<grid, 64 * NW, 0, s>>>(p);
}

template <typename T, int CACHE>
void launch_attend(const AttendArgs &p, const Plan &plan, dim3 grid, hipStream_t s) {
  if (plan.nq == 1 && plan.nw == 1) launch_attend<T, CACHE, 1, 1>(p, grid, s);
  else if (plan.nq == 1 && plan.nw == 2) launch_attend<T, CACHE, 1, 2>(p, grid, s);
  else if (plan.nq == 1) launch_attend<T, CACHE, 1, 4>(p, grid, s);
  else if constexpr (sizeof(T) == 2 || CACHE == WF_DTYPE_F32) {
    if (plan.nq == 2) launch_attend<T, CACHE, 2, 4>(p, grid, s);
    else if constexpr (sizeof(T) == 2) launch_attend<T, CACHE, 4, 4>(p, grid, s);
  }
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
  if (!std::isfinite(a->scale * 1.4426950408889634f)) return fail(WF_E_INVALID_ARG, "scale = %g: it and log2(e) times it must be finite", a->scale);
  if ((double)a->n_seqs * std::min(a->max_q, std::max(a->n_q_rows, 1)) * a->n_heads >= (double)(1 << 30) || (double)a->n_seqs * c->n_heads >= (double)(1 << 24))
    return fail(WF_E_CAPACITY, "%d sequences of up to %d queries of %d heads: more than 2^30 rows or 2^24 heads", a->n_seqs, a->max_q, a->n_heads);
  return WF_OK;
}

// Floats of the parts and of their maxima and sums.
int64_t part_rows(const wf_cache &c, const wf_cache_query &a, const Plan &p) {
  return p.n_split == 1 ? 0 : (int64_t)a.n_seqs * c.n_heads * p.chunks * 16 * p.nq * p.n_split;
}

}  // namespace

extern "C" {

int64_t wf_cache_attention_workspace(const wf_cache *cache, const wf_cache_query *query) {
  const int rc = check_query(cache, query);
  return rc ? rc : part_rows(*cache, *query, plan_of(*cache, *query)) * 66 * 4;
}

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
  const Plan plan = plan_of(*cache, a);
  const int64_t parts = part_rows(*cache, a, plan);
  if (parts && (!a.workspace_dev || (uintptr_t)a.workspace_dev % 16)) return fail(WF_E_INVALID_ARG, "workspace_dev is NULL or not aligned to 16 bytes");
  if (a.workspace_bytes < parts * 66 * 4) return fail(WF_E_CAPACITY, "workspace of %lld bytes, need %lld", (long long)a.workspace_bytes, (long long)parts * 66 * 4);
  float *const part = (float *)a.workspace_dev;
  const AttendArgs p{view_of(*cache), a.q_dev, a.out_dev, a.ldq, a.ldo, a.cu_q_dev, a.row_dev, a.len_dev, a.mask_dev, a.mask_from_dev, part, part + parts * 64,
                     a.n_heads, a.n_heads / cache->n_heads, a.n_seqs, a.n_q_rows, a.max_q, a.max_len, a.mask_words, plan.chunks, plan.n_split, plan.split_keys, a.scale};
  int64_t groups = (int64_t)a.n_seqs * cache->n_heads * plan.n_split;
  if (plan.chunks > 1) groups = round_up(groups, 8) * plan.chunks;
  if (groups * plan.nw >= (int64_t)1 << 26) return fail(WF_E_CAPACITY, "%lld workgroups (supported: below 2^32 threads)", (long long)groups);
  const dim3 grid((uint32_t)groups);
  const hipStream_t s = (hipStream_t)hip_stream;
  if (a.dtype == WF_DTYPE_BF16) {
    if (cache->dtype == WF_DTYPE_F8) launch_attend<__bf16, WF_DTYPE_F8>(p, plan, grid, s);
    else launch_attend<__bf16, WF_DTYPE_BF16>(p, plan, grid, s);
  } else {
    if (cache->dtype == WF_DTYPE_F8) launch_attend<float, WF_DTYPE_F8>(p, plan, grid, s);
    else launch_attend<float, WF_DTYPE_F32>(p, plan, grid, s);
  }
  if (parts) {
    const int rows_pad = plan.chunks * 16 * plan.nq;
    const dim3 join((uint32_t)(((int64_t)a.n_seqs * cache->n_heads * rows_pad + 3) / 4));
    if (a.dtype == WF_DTYPE_BF16) cache_attention_join_kernel<__bf16><<<join, 256, 0, s>>>(p, rows_pad);
    else cache_attention_join_kernel<float><<<join, 256, 0, s>>>(p, rows_pad);
  }
  const hipError_t err = hipGetLastError();
  return err == hipSuccess ? WF_OK : fail(WF_E_HIP, "cache_attention launch: %s", hipGetErrorString(err));
}

}  // extern "C"
