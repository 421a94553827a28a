// Vector types and bounded loads of the kernels for microscaled matrices.
#pragma once

#include "mx.h"

namespace coded {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2_t __attribute__((ext_vector_type(2)));
typedef unsigned int u32x4_t __attribute__((ext_vector_type(4)));
typedef short s16x4_t __attribute__((ext_vector_type(4)));
typedef f32x4_t f32x4_any __attribute__((aligned(4)));
typedef u32x2_t u32x2_any __attribute__((aligned(2)));

__host__ __device__ constexpr int64_t lesser(int64_t a, int64_t b) { return a < b ? a : b; }   // min() goes over doubles

// Loads within `bytes` of `base` (both the same for every lane); past them they give zeros and move nothing.
struct Window {
    __amdgpu_buffer_rsrc_t rsrc;
    __device__ __forceinline__ Window(const void* base, int64_t bytes)
        : rsrc(__builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), 0, static_cast<int>(bytes < 0 ? 0 : lesser(bytes, 0xFFFFFFFF)),
                                                 0x00027000)) {}
    // NTL: non-temporal, for what does not stay in the memory-side cache until it is read again
    template <bool NTL = false>
    __device__ __forceinline__ u32x4_t four(uint32_t at) const { return __builtin_amdgcn_raw_buffer_load_b128(rsrc, at, 0, NTL ? 2 : 0); }
    __device__ __forceinline__ u32x2_t two(uint32_t at) const { return __builtin_amdgcn_raw_buffer_load_b64(rsrc, at, 0, 0); }
    __device__ __forceinline__ uint32_t word(uint32_t at) const { return __builtin_amdgcn_raw_buffer_load_b32(rsrc, at, 0, 0); }
    __device__ __forceinline__ uint32_t two_bytes(uint32_t at) const { return __builtin_amdgcn_raw_buffer_load_b16(rsrc, at, 0, 0); }
    __device__ __forceinline__ uint32_t byte(uint32_t at) const { return __builtin_amdgcn_raw_buffer_load_b8(rsrc, at, 0, 0); }
};

}  // namespace
}  // namespace coded
