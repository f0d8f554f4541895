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
bool kv_tc_takes(const KvAttendArgs& a);                                                   // 16-bit dense, many rows
size_t kv_tc_ws_bytes(const KvAttendArgs& a);
int launch_kv_tc(sentry_ctx* ctx, const KvAttendArgs& a, WsAlloc& ws, cudaStream_t st);
int launch_kv_combine(sentry_ctx* ctx, const KvAttendArgs& a, const float* part, const float2* ml, const int2* plan, int n_splits, cudaStream_t st);
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
// x / s to the nearest integer, ties to even, of the exact quotient; |x| <= 127 s (1 + 2^-22), s >= 2^-126, inv = 1 / s rounded.
// The product with the rounded reciprocal is at most one off; x - r s is exact (a multiple of the smaller operand's last place, below
// s in size), and twice it against s says which neighbour is nearer.
__device__ __forceinline__ int round_quotient_i8(float x, float s, float inv) {
    float r = rintf(x * inv);
    const float e2 = 2.0f * fmaf(-r, s, x);
    const bool odd = ((int)r) & 1;
    if (e2 > s || (e2 == s && odd)) r += 1.0f;
    else if (e2 < -s || (e2 == -s && odd)) r -= 1.0f;
    return (int)fminf(fmaxf(r, -127.0f), 127.0f);
}
// N values over s (positive): codes as words.  Adding 1.5 * 2^23 rounds x * inv to an integer r and leaves it in the low bits, two values at a
// time.  The remainder x - r s is exact; where it is half of s or more, r may be the wrong neighbour, or the quotient an exact half, which
// has to go to the even side: round_quotient_i8 decides.  That would be common (two bf16 numbers' quotient is one of few fractions, a
// half often), but for reciprocal_i8.
__device__ __forceinline__ uint32_t pack_low_bytes(float a, float b, float c, float d) {
    return __byte_perm(__byte_perm(__float_as_uint(a), __float_as_uint(b), 0x0040), __byte_perm(__float_as_uint(c), __float_as_uint(d), 0x0040), 0x5410);
}
// 1 / s, moved by 2^-22 of itself to the side on which s was rounded from top / 127: a quotient that would be a half but for that
// rounding then falls where the exact one does.
__device__ __forceinline__ float reciprocal_i8(float s, float top) {
    const float inv = __fdiv_rn(1.0f, s), r = fmaf(-127.0f, s, top);
    return r < 0.0f ? inv * (1.0f - 2.38418579e-7f) : r > 0.0f ? inv * (1.0f + 2.38418579e-7f) : inv;
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
template <int N>
__device__ __forceinline__ void codes_i8(const float (&x)[N], float s, float inv, uint32_t (&w)[N / 4]) {
    constexpr float kMagic = 12582912.0f;
    const uint64_t magic = pair_f32(kMagic, kMagic), minus = pair_f32(-1.0f, -1.0f), inv2 = pair_f32(inv, inv), s2 = pair_f32(s, s);
    float y[N], far = 0.0f;
#pragma unroll
    for (int i = 0; i < N; i += 2) {
        const uint64_t xx = pair_f32(x[i], x[i + 1]), yy = fma_pair(xx, inv2, magic);
        const float2 e = pair_of(fma_pair(fma_pair(yy, minus, magic), s2, xx)), v = pair_of(yy);
        far = fmaxf(far, fmaxf(fabsf(e.x), fabsf(e.y)));
        y[i] = v.x;
        y[i + 1] = v.y;
    }
#pragma unroll
    for (int i = 0; i < N / 4; ++i) w[i] = pack_low_bytes(y[4 * i], y[4 * i + 1], y[4 * i + 2], y[4 * i + 3]);
    if (far + far >= s) {
        const float exact_inv = __fdiv_rn(1.0f, s);
#pragma unroll 1
        for (int i = 0; i < N; ++i) {
            float v = x[0];
#pragma unroll
            for (int j = 1; j < N; ++j) v = j == i ? x[j] : v;       // (no indexed registers)
            const uint32_t c = (uint32_t)(round_quotient_i8(v, s, exact_inv) & 255) << (8 * (i & 3)), keep = ~(255u << (8 * (i & 3)));
#pragma unroll
            for (int j = 0; j < N / 4; ++j) w[j] = j == i / 4 ? (w[j] & keep) | c : w[j];
        }
    }
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
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (sizeof(T) == 4) acc = max(acc, w[i] & 0x7fffffffu);
            else acc = __vmaxu2(acc, w[i] & 0x7fff7fffu);
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
