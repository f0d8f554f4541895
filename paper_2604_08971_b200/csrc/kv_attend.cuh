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

// The positions of sample b's list whose head belongs to group g, in the list's order; by one warp.  With `first`, positions that hold no
// head get their zero rows here, and the status bit.
__device__ __forceinline__ int kv_group_heads(const KvAttendArgs& a, int b, int g, bool first, short* head, short* pos) {
    const int lane = threadIdx.x & 31, per = a.Hq / a.Hk;
    if (a.kept == nullptr) {
        for (int i = lane; i < per; i += 32) head[i] = pos[i] = (short)(g * per + i);
        return per;
    }
    int n = 0;
    for (int j0 = 0; j0 < a.k_h; j0 += 32) {
        const int j = j0 + lane, h = j < a.k_h ? kv_head(a, b, j) : -2;
        const unsigned mine = __ballot_sync(0xffffffffu, h >= 0 && h / per == g);
        if ((mine >> lane) & 1u) {
            const int at = n + __popc(mine & ((1u << lane) - 1u));
            head[at] = (short)h;
            pos[at] = (short)j;
        }
        n += __popc(mine);
        for (unsigned none = __ballot_sync(0xffffffffu, first && h == -1); none; none &= none - 1) {
            if (lane == 0) atomicOr(a.status, SENTRY_STATUS_BIT_BAD_INDEX);
            uint32_t* o = (uint32_t*)a.O + ((size_t)b * a.k_h + j0 + __ffs(none) - 1) * a.Tq * (a.d / 2);
            for (size_t e = lane; e < (size_t)a.Tq * (a.d / 2); e += 32) o[e] = 0u;
        }
    }
    return n;
}
__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
template <bool BF16>
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
    uint32_t v;
    if constexpr (BF16) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(v) : "f"(hi), "f"(lo));
    else asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(v) : "f"(hi), "f"(lo));
    return v;
}
// two codes in the low 16 bits of w -> fp16 pair
__device__ __forceinline__ uint32_t e4m3x2_to_f16x2(uint32_t w) {
    uint32_t r;
    asm("{\n\t.reg .b16 lo, hi;\n\tmov.b32 {lo, hi}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, lo;\n\t}" : "=r"(r) : "r"(w));
    return r;
}
__device__ __forceinline__ uint32_t e4m3x2_hi_to_f16x2(uint32_t w) {
    uint32_t r;
    asm("{\n\t.reg .b16 lo, hi;\n\tmov.b32 {lo, hi}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, hi;\n\t}" : "=r"(r) : "r"(w));
    return r;
}
// bytes (already + 128) -> fp16: 0x6400 | u is 1024 + u, exactly
__device__ __forceinline__ uint32_t biased_to_f16x2(uint32_t pair) {
    const uint32_t bias = 0x64806480u;   // 1152
    uint32_t r;
    asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(pair), "r"(bias));
    return r;
}
// four codes of a word, in order, as two fp16 pairs
template <bool I8>
__device__ __forceinline__ void codes_to_f16(uint32_t w, uint32_t& p01, uint32_t& p23) {
    if constexpr (I8) {
        const uint32_t u = w ^ 0x80808080u;
        p01 = biased_to_f16x2(__byte_perm(u, 0x64646464u, 0x4140));
        p23 = biased_to_f16x2(__byte_perm(u, 0x64646464u, 0x4342));
    } else {
        p01 = e4m3x2_to_f16x2(w);
        p23 = e4m3x2_hi_to_f16x2(w);
    }
}
