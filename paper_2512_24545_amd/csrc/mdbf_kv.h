// The 4-bit cache in pages: layout and format, shared by the kernels that fill it and the attention over it.
#pragma once
#include "mdbf_internal.h"

namespace mdbf {

typedef uint32_t U32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t U32x4 __attribute__((ext_vector_type(4)));
typedef float F32x2 __attribute__((ext_vector_type(2)));
typedef float F32x4 __attribute__((ext_vector_type(4)));
typedef _Float16 F16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 Bf16x2 __attribute__((ext_vector_type(2)));

constexpr int kKvBlock = 32;              // channels that share a scale
constexpr uint32_t kKvNanScale = 255;
// scale bytes (2^(b - 127)) that a cache of fp16 resp. bf16 values uses: all of the block's values are numbers of that type; larger
// ones are read as NaN
constexpr uint32_t kKvScaleMin[2] = {104, 2}, kKvScaleMax[2] = {140, 252};

// bytes of one kv head's part of a page: key codes, value codes, key scales, value scales
__host__ __device__ inline int64_t kv_head_bytes(int page_size, int d) { return (int64_t)page_size * (d + d / 16); }
__host__ __device__ inline int64_t kv_page_bytes(const mdbf_kv_t& kv) {
  return (int64_t)kv.kv_heads * kv_head_bytes(kv.page_size, kv.head_dim);
}
// where the codes and scales of one token's key or value are
struct KvPlace {
  int64_t codes, scales;
};
__device__ __forceinline__ KvPlace kv_place(int64_t slot, int head, int value, int kv_heads, int page_shift, int d) {
  const int page_size = 1 << page_shift, tok = (int)(slot & (page_size - 1));
  const int64_t base = ((slot >> page_shift) * kv_heads + head) * kv_head_bytes(page_size, d);
  return {base + (int64_t)value * page_size * (d / 2) + (int64_t)tok * (d / 2),
          base + (int64_t)page_size * d + (int64_t)value * page_size * (d / 32) + tok * (d / 32)};
}
inline int kv_page_shift(int page_size) { return __builtin_ctz((unsigned)page_size); }

inline bool kv_aligned(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }
// a pool's description, and that the buffer holds it
int check_kv(const mdbf_kv_t* kv);
int check_kv_cache(const mdbf_kv_t* kv, const void* cache, size_t cache_bytes);

}  // namespace mdbf
