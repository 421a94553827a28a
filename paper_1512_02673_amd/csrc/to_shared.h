// Loads from memory straight into shared memory.
#pragma once

#include "mx_window.h"

namespace coded {
namespace {

// 16 or 4 bytes a lane from `from` bytes on, to `to` in shared memory (the wave's first lane's; the others' follow).
// NTL: non-temporal, for what does not stay in the memory-side cache until it is read again.
template <bool NTL = false>
__device__ __forceinline__ void sixteen_to_shared(const Window& w, char* to, uint32_t from) {
#ifdef __HIP_DEVICE_COMPILE__   // the host's pass knows no such load, and would drop the kernel
    __attribute__((address_space(3))) void* const at = (__attribute__((address_space(3))) void*)to;
    if constexpr (NTL)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(w.rsrc, at, 16, from, 0, 0, 2);
    else
        __builtin_amdgcn_raw_ptr_buffer_load_lds(w.rsrc, at, 16, from, 0, 0, 0);
#endif
}
__device__ __forceinline__ void four_to_shared(const Window& w, char* to, uint32_t from) {
#ifdef __HIP_DEVICE_COMPILE__
    __builtin_amdgcn_raw_ptr_buffer_load_lds(w.rsrc, (__attribute__((address_space(3))) void*)to, 4, from, 0, 0, 0);
#endif
}

}  // namespace
}  // namespace coded
