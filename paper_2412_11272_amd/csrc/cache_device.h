// What the kernels over key / value caches share: the cache as they see it, and the e4m3 format's exponents.
#pragma once
#include "../../include/wf_encoder.h"

#include "device_utils.h"

namespace wf {

struct CacheView {
  void *data;
  uint8_t *exps;
  int64_t n_rows;
  int32_t n_heads;
};

inline CacheView view_of(const wf_cache &c) { return {c.data_dev, c.exps_dev, c.n_rows, c.n_heads}; }

// Biased exponent e + 127 of the smallest power of two 2^e, e >= -127, with largest <= 448 2^e = 1.75 * 2^(e + 8); `largest` finite, >= 0.
__device__ __forceinline__ uint32_t f8_exponent(float largest) {
  const uint32_t u = __builtin_bit_cast(uint32_t, largest);
  const int b = (int)(u >> 23) - 8 + ((u & 0x7fffffu) > 0x600000u);
  return b > 0 ? b : 0;
}
// 2^(biased - 127); 2^-127 is subnormal.
__device__ __forceinline__ float f8_factor(uint32_t biased) { return __builtin_bit_cast(float, biased ? biased << 23 : 1u << 22); }

namespace host {
int check_cache(const wf_cache *c);             // shape and type
int check_cache_memory(const wf_cache *c);      // pointers
}  // namespace host

}  // namespace wf
