// Device helpers shared by the cache's kernels (cache.hip) and the attention
// over it (attend.hip): element types, the cache's addresses and the values of
// its 8-bit codes.  Not part of the public ABI.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <string>

#include "leech_internal.h"

namespace leech {

typedef uint32_t kv_u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t kv_u32x2 __attribute__((ext_vector_type(2)));
typedef float kv_f32x4 __attribute__((ext_vector_type(4)));
typedef float kv_f32x2 __attribute__((ext_vector_type(2)));

constexpr int kMaxHeadDim = 256;

__host__ __device__ constexpr int type_bytes(int type) {
  return type == LEECH_F32 ? 4 : (type == LEECH_F16 || type == LEECH_BF16) ? 2 : 1;
}
// Tokens whose values of one coordinate share sixteen bytes of the value pages.
__host__ __device__ constexpr int value_run(int type) { return 16 / type_bytes(type); }

__device__ __forceinline__ float half_value(uint32_t h) {
  return (float)__builtin_bit_cast(_Float16, (uint16_t)h);
}
__device__ __forceinline__ float bf16_value(uint32_t h) {
  return __builtin_bit_cast(float, h << 16);
}
__device__ __forceinline__ uint32_t half_bits(float v) {
  return __builtin_bit_cast(uint16_t, (_Float16)v);
}
// Rounded to nearest, ties to even; a NaN stays one.
__device__ __forceinline__ uint32_t bf16_bits(float v) {
  return __builtin_bit_cast(uint16_t, (__bf16)v);
}

// Where slot (a page and a place in it) of head h keeps its keys, its values
// and its scale; element offsets, 64 bits wide.
struct CacheShape {
  int64_t slots;          // pages · page_size
  int32_t heads, dim, log_page, type;
};
__device__ __forceinline__ int64_t scale_at(const CacheShape& c, int64_t slot, int h) {
  const int64_t page = slot >> c.log_page;
  return ((page * c.heads + h) << c.log_page) + (slot & ((1 << c.log_page) - 1));
}
__device__ __forceinline__ int64_t key_at(const CacheShape& c, int64_t slot, int h) {
  return scale_at(c, slot, h) * c.dim;
}
// of coordinate 0; coordinate d is d · value_run further
__device__ __forceinline__ int64_t value_at(const CacheShape& c, int64_t slot, int h) {
  const int64_t at = scale_at(c, slot, h);
  const int run = value_run(c.type);
  return (at & ~(int64_t)(run - 1)) * c.dim + (at & (run - 1));
}

// Host side: checks shared by the calls.
int check_cache(const leech_kv_cache* c, CacheShape* shape);
// Whether rows of dim elements, heads × T of them at these strides, share none.
bool rows_apart(int64_t token, int64_t head, int64_t T, int heads, int dim);
inline int hip_fail(const char* what, hipError_t e) {
  return set_error(LEECH_E_HIP, std::string(what) + ": " + hipGetErrorString(e));
}

}  // namespace leech
