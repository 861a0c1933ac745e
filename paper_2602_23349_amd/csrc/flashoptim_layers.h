// Internal: what the device code of the layers (flashoptim_mx4.hip, flashoptim_norm.hip) shares.
#ifndef FLASHOPTIM_LAYERS_H
#define FLASHOPTIM_LAYERS_H

#include <hip/hip_runtime.h>

namespace fo {

using i32x4 = int __attribute__((ext_vector_type(4)));
using f32x4 = float __attribute__((ext_vector_type(4)));

template <typename T>
__device__ __forceinline__ T load_as(const void* p) {       // any alignment: the hardware takes global accesses at any byte
    T v;
    __builtin_memcpy(&v, p, sizeof(T));
    return v;
}
template <typename T>
__device__ __forceinline__ void store_as(void* p, T v) {
    __builtin_memcpy(p, &v, sizeof(T));
}

}  // namespace fo
#endif
