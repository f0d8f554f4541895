// What the forms of serving attention (dense cross attention, attention over the 8-bit cache) share on the device.
#pragma once
#include <cuda_fp8.h>

#include "serving.cuh"

// Keys of sample b that can be seen at all: [0, n).
__device__ __forceinline__ int kv_length(const KvAttendArgs& a, int b) {
    return a.lengths == nullptr ? a.Tk : min(max(a.lengths[b], 0), a.Tk);
}
// Whether key n < length of a dense tensor is present.
__device__ __forceinline__ bool kv_present(int32_t id, uint32_t mask) { return id >= 0 && id < 32 && ((mask >> id) & 1u); }
// Head at position j of sample b's list; -1: not a head.
__device__ __forceinline__ int kv_head(const KvAttendArgs& a, int b, int j) {
    const int h = a.kept == nullptr ? j : a.kept[(size_t)b * a.k_h + j];
    return h >= 0 && h < a.Hq ? h : -1;
}
// What a code stands for, without its page's scale.
template <bool I8>
__device__ __forceinline__ float code_value(uint8_t c) {
    if constexpr (I8) return (float)(int8_t)c;
    else {
        const __half_raw h = __nv_cvt_fp8_to_halfraw(c, __NV_E4M3);
        return __half2float(__half(h));
    }
}
