// Types and small device functions shared by the kernels around the paged key/value cache.
#ifndef SP_CACHE_COMMON_H
#define SP_CACHE_COMMON_H
#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

#include "cache_index.h"

namespace {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(2))) float f32x2;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;

// f(integral_constant<int, G>) for G = FROM .. TO-1, expanded at compile time
template <int FROM, int TO, class F>
__device__ __forceinline__ void static_for(F &&f) {
  if constexpr (FROM < TO) {
    f(std::integral_constant<int, FROM>{});
    static_for<FROM + 1, TO>(f);
  }
}

__device__ __forceinline__ float bf_lo(uint32_t x) { return __builtin_bit_cast(float, x << 16); }
__device__ __forceinline__ float bf_hi(uint32_t x) { return __builtin_bit_cast(float, x & 0xffff0000u); }
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {  // round to nearest, ties to even
  f32x2 t = {a, b};
  bf16x2 r = __builtin_convertvector(t, bf16x2);
  return __builtin_bit_cast(uint32_t, r);
}
__device__ __forceinline__ bool any_lane(bool x) { return __builtin_amdgcn_ballot_w64(x) != 0ull; }
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

// inclusive prefix sum over the wavefront by lane moves inside the vector unit (shuffles through LDS take ten times as long)
template <int CTRL, int ROWS, int BANKS>
__device__ __forceinline__ uint32_t moved(uint32_t x) {  // zero where the move has no source or the mask leaves the lane out
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, ROWS, BANKS, false);
}
template <int CTRL, int ROWS, int BANKS>
__device__ __forceinline__ uint64_t moved(uint64_t x) {
  return moved<CTRL, ROWS, BANKS>((uint32_t)x) | (uint64_t)moved<CTRL, ROWS, BANKS>((uint32_t)(x >> 32)) << 32;
}
template <class T>
__device__ __forceinline__ T wave_prefix(T x) {
  x += moved<0x111, 0xf, 0xf>(x);  // 1 lane up in the row of 16
  x += moved<0x112, 0xf, 0xf>(x);  // 2
  x += moved<0x114, 0xf, 0xe>(x);  // 4
  x += moved<0x118, 0xf, 0xc>(x);  // 8
  x += moved<0x142, 0xa, 0xf>(x);  // the row's last lane to the next row
  x += moved<0x143, 0xc, 0xf>(x);  // the lower half's last lane to the upper half
  return x;
}

}  // namespace

#endif
