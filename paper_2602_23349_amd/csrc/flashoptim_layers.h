// Internal: what the device code of the layers (flashoptim_mx4.hip, flashoptim_norm.hip), of the losses and of the calls on gradients
// (flashoptim_loss.hip, flashoptim_clip.hip) shares.
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

// The FP64 sum of a wavefront whose lanes are all active, in every lane, in a fixed order: each step adds the value of another lane within the vector unit.
// (Exchanges through LDS instead: the policy loss of 12 rows of 1001 values, one sum for a row and three for the statistics, 7.0 us against 6.0.)
template <int CTRL, int ROWS = 0xf>
__device__ __forceinline__ double add_of_lane(double v) {
    const int low = __builtin_amdgcn_update_dpp(0, __double2loint(v), CTRL, ROWS, 0xf, false);
    const int high = __builtin_amdgcn_update_dpp(0, __double2hiint(v), CTRL, ROWS, 0xf, false);
    return v + __hiloint2double(high, low);             // (a lane without a source adds 0)
}
__device__ __forceinline__ double sum_of_wave(double v) {
    v = add_of_lane<0x111>(v);           // row_shr 1, 2, 4, 8: lane 15 of each row of 16 has the row's
    v = add_of_lane<0x112>(v);
    v = add_of_lane<0x114>(v);
    v = add_of_lane<0x118>(v);
    v = add_of_lane<0x142, 0xa>(v);      // row_bcast 15, into the second and the fourth row
    v = add_of_lane<0x143, 0xc>(v);      // row_bcast 31, into the upper half
    return __hiloint2double(__builtin_amdgcn_readlane(__double2hiint(v), 63), __builtin_amdgcn_readlane(__double2loint(v), 63));
}

}  // namespace fo
#endif
