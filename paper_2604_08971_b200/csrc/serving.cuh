// Declarations shared by the serving operators (8-bit linear layer, cross attention, 8-bit cache): argument structs, launchers and
// the integer rounding that two of them use.
#pragma once
#include <atomic>

#include "common.cuh"

// Lets a kernel have `bytes` of dynamic shared memory; once per device (`done` is the caller's, one per kernel).
template <typename F>
static inline cudaError_t allow_smem(F* kernel, int bytes, int device, std::atomic<unsigned long long>& done) {
    const unsigned long long bit = device < 64 ? 1ull << device : 0ull;
    if (done.load(std::memory_order_acquire) & bit) return cudaSuccess;
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == cudaSuccess) done.fetch_or(bit, std::memory_order_release);
    return e;
}

constexpr int kServeMaxHeads = 256;

// Attention of packed rows over a dense tensor (format 0) or a paged 8-bit cache.
struct KvAttendArgs {
    int B, Tq, Tk;              // Tk: keys per sample (dense), or the capacity max_pages * page
    int Hq, Hk, d, k_h, dtype;
    long long qs[3], ks[3], vs[3];   // strides in elements: batch, head, token
    const void *Q, *K, *V;
    void* O;
    const int32_t *kept, *ids, *lengths;
    const uint32_t* masks;
    int format, page, n_pages, max_pages, causal;
    const float *k_scales, *v_scales;
    const int32_t* table;
    unsigned int* status;
    int sm_count;
};
int launch_kv_generic(sentry_ctx* ctx, const KvAttendArgs& a, cudaStream_t st);            // fp32 rows
size_t kv_rows_ws_bytes(const KvAttendArgs& a);
bool kv_tc_takes(const KvAttendArgs& a);                                                   // 16-bit rows, many of them
size_t kv_tc_ws_bytes(const KvAttendArgs& a);
int launch_kv_tc(sentry_ctx* ctx, const KvAttendArgs& a, WsAlloc& ws, cudaStream_t st);
int launch_kv_combine(sentry_ctx* ctx, const KvAttendArgs& a, const float* part, const float2* ml, int n_splits, cudaStream_t st);
int launch_kv_rows(sentry_ctx* ctx, const KvAttendArgs& a, WsAlloc& ws, cudaStream_t st);   // 16-bit rows, few of them

struct AppendArgs {
    sentry_kv_cache c;
    sentry_append_desc d;
    long long ks[3], vs[3];
    const void *K, *V;
    const int32_t *ids, *token_lengths, *lengths;
    const uint32_t* masks;
    int32_t* new_lengths;
    unsigned int* status;
};
int launch_cache_append(sentry_ctx* ctx, const AppendArgs& a, cudaStream_t st);

int launch_quantize_rows_i8(sentry_ctx* ctx, int M, int K, int dtype, const void* X, int8_t* codes, float* scales, cudaStream_t st);
struct LinearArgs {
    sentry_linear_desc d;
    const int8_t *X, *W;
    const float *xs, *ws, *bias;
    void* Y;
    unsigned int* status;
};
int launch_linear_i8(sentry_ctx* ctx, const LinearArgs& a, cudaStream_t st);

#ifdef __CUDACC__
// N values over s (positive): codes as words.  Adding 1.5 * 2^23 rounds x * inv to an integer and leaves it in the low bits, two values at a
// time; |x| <= 127 s (1 + 2^-22), s >= 2^-126.  The product with the rounded reciprocal is at most one off.  With CHECK the remainder
// x - r s (exact: a multiple of the smaller operand's last place, below s in size) says which neighbour is nearer, and an exact half goes
// to the even one.
// Without CHECK that cannot be (sure_i8).  Let x = m 2^i and top = t 2^j with whole m, t <= 2047, as 16-bit numbers are, s = top / 127 up to
// two roundings, and inv as reciprocal_i8 gives it: x * inv is 127 x / top = 127 m / (t 2^k) up to 2^-21 of itself (s 2^-23, 1 / s 2^-24, the
// move 2^-22 and its rounding 2^-24).  That fraction is a half of an odd number or at least 1 / (t 2^(k+1)) away from one, and 2^-21 of it
// is less, since 127 m < 2^20.  Where it is a half, x / s lies on the side to which s was rounded, and inv was moved there by more than its
// error; only where s was not rounded at all is it a half indeed.
__device__ __forceinline__ uint32_t pack_low_bytes(float a, float b, float c, float d) {
    return __byte_perm(__byte_perm(__float_as_uint(a), __float_as_uint(b), 0x0040), __byte_perm(__float_as_uint(c), __float_as_uint(d), 0x0040), 0x5410);
}
// 1 / s, moved by 2^-22 of itself to the side on which s was rounded from top / 127: a quotient that would be a half but for that
// rounding then falls where the exact one does.
__device__ __forceinline__ float reciprocal_i8(float s, float top) {
    const float inv = __fdiv_rn(1.0f, s), r = fmaf(-127.0f, s, top);
    return r < 0.0f ? inv * (1.0f - 2.38418579e-7f) : r > 0.0f ? inv * (1.0f + 2.38418579e-7f) : inv;
}
// Whether codes_i8 needs no check: values of a 16-bit type under the scale of the largest of them.
template <typename T>
__device__ __forceinline__ bool sure_i8(float s, float top) {
    return sizeof(T) == 2 && s > 1.17549435e-38f && fmaf(-127.0f, s, top) != 0.0f;
}
__device__ __forceinline__ uint64_t pair_f32(float lo, float hi) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ float2 pair_of(uint64_t p) {
    float2 f;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(f.x), "=f"(f.y) : "l"(p));
    return f;
}
__device__ __forceinline__ uint64_t fma_pair(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}
__device__ __forceinline__ uint64_t mul_pair(uint64_t a, uint64_t b) {
    uint64_t d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
template <bool CHECK, int N>
__device__ __forceinline__ void codes_i8(const float (&x)[N], float s, float inv, uint32_t (&w)[N / 4]) {
    constexpr float kMagic = 12582912.0f;
    const uint64_t magic = pair_f32(kMagic, kMagic), inv2 = pair_f32(inv, inv);
    float y[N];
#pragma unroll
    for (int i = 0; i < N; i += 2) {
        const float2 v = pair_of(fma_pair(pair_f32(x[i], x[i + 1]), inv2, magic));
        y[i] = v.x;
        y[i + 1] = v.y;
    }
    if constexpr (CHECK) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float e = fmaf(kMagic - y[i], s, x[i]), d = fmaf(2.0f, fabsf(e), -s);
            if (d > 0.0f || (d == 0.0f && (__float_as_uint(y[i]) & 1u))) y[i] += copysignf(1.0f, e);
        }
    }
#pragma unroll
    for (int i = 0; i < N / 4; ++i) w[i] = pack_low_bytes(y[4 * i], y[4 * i + 1], y[4 * i + 2], y[4 * i + 3]);
}
// (the product with 1/127 rounded to fp32, not the quotient: what the header defines)
__device__ __forceinline__ float scale_i8(float top) { return top > 0.0f ? fmaxf(__fmul_rn(top, 1.0f / 127.0f), 1.17549435e-38f) : 0.0f; }

// Sixteen bytes of a 16-bit or fp32 tensor as floats.
template <typename T> struct Vec16;
template <> struct Vec16<float> {
    static constexpr int N = 4;
    static __device__ __forceinline__ void get(const uint4& v, float* f) {
        f[0] = __uint_as_float(v.x); f[1] = __uint_as_float(v.y); f[2] = __uint_as_float(v.z); f[3] = __uint_as_float(v.w);
    }
};
template <> struct Vec16<__nv_bfloat16> {
    static constexpr int N = 8;
    static __device__ __forceinline__ void get(const uint4& v, float* f) {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) { f[2 * i] = __uint_as_float(w[i] << 16); f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
    }
};
template <> struct Vec16<__half> {
    static constexpr int N = 8;
    static __device__ __forceinline__ void get(const uint4& v, float* f) {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[2 * i] = __half2float(__ushort_as_half((unsigned short)(w[i] & 0xffffu)));
            f[2 * i + 1] = __half2float(__ushort_as_half((unsigned short)(w[i] >> 16)));
        }
    }
};

// The largest magnitude of a tensor's pieces, as bits (which order magnitudes, and infinities and NaNs above them).
template <typename T> struct AbsMax {
    uint32_t acc = 0;
    __device__ __forceinline__ void add(const uint4& v) {
        if constexpr (sizeof(T) == 4) {
            acc = max(acc, max(max(v.x & 0x7fffffffu, v.y & 0x7fffffffu), max(v.z & 0x7fffffffu, v.w & 0x7fffffffu)));
        } else {
            acc = __vimax3_u16x2(acc, v.x & 0x7fff7fffu, v.y & 0x7fff7fffu);
            acc = __vimax3_u16x2(acc, v.z & 0x7fff7fffu, v.w & 0x7fff7fffu);
        }
    }
    __device__ __forceinline__ uint32_t bits() const { return sizeof(T) == 4 ? acc : max(acc & 0xffffu, acc >> 16); }
};
// Those bits as a number; not a number for infinities too.
template <typename T>
__device__ __forceinline__ float magnitude(uint32_t bits) {
    float f;
    if constexpr (sizeof(T) == 4) f = __uint_as_float(bits);
    else f = to_f32<T>(*reinterpret_cast<const T*>(&bits));
    return f <= 3.4028234e38f ? f : __int_as_float(0x7fc00000);
}
#endif
