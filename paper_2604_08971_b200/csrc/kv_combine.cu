// Joins the parts of cross attention of many rows whose axis of keys was split over blocks.
#include "kv_attend.cuh"

namespace {

constexpr int kCombineThreads = 256;
constexpr int kMaxParts = 64;       // of a row

// A block per row: its warps take the parts in turn, with the loads of several on the way, and meet in shared memory.  (A warp per row, part
// after part: 37 us for 16 rows of 128 parts.)
template <bool BF16>
__global__ void __launch_bounds__(kCombineThreads) kv_combine_kernel(const KvAttendArgs a, const float* __restrict__ part, const float2* __restrict__ ml, int n) {
    __shared__ float s_weight[kMaxParts], s_acc[kCombineThreads / 32][128];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const size_t row = blockIdx.x, each = (size_t)a.k_h * a.Tq;      // rows of a sample
    grid_dependency_wait();
    const int b = (int)(row / each);
    const size_t in = row - (size_t)b * each;
    if (kv_head(a, b, (int)(in / a.Tq)) < 0) return;    // (its zero rows are written)
    // every warp by itself: the maximum, the total, and the weights of all parts
    const float2* x0 = ml + (size_t)b * n * each + in;
    float top = -INFINITY, total = 0.0f;
    float2 x[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) x[i] = i * 32 + lane < n ? x0[(i * 32 + lane) * each] : make_float2(-INFINITY, 0.0f);
#pragma unroll
    for (int i = 0; i < 2; ++i) top = fmaxf(top, x[i].x);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    const float ref = top == -INFINITY ? 0.0f : top;
    auto take = [&](int s, float2 v) {
        const float f = exp2_fast(v.x - ref);
        total += v.y * f;
        // (a part that saw nothing may not have been written)
        if (warp == 0) s_weight[s] = v.x == -INFINITY && v.y == 0.0f ? -1.0f : f;
    };
#pragma unroll
    for (int i = 0; i < 2; ++i)
        if (i * 32 + lane < n) take(i * 32 + lane, x[i]);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) total += __shfl_xor_sync(0xffffffffu, total, o);
    __syncthreads();
    // columns: four floats a lane, 16 to 128 of them; the lanes that are left over take further parts
    const int lanes = a.d / 4, sub = lane / lanes, subs = 32 / lanes, c = lane % lanes;
    float4 acc = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 8
    for (int s = warp * subs + sub; s < n; s += kCombineThreads / 32 * subs) {
        const float f = s_weight[s];
        if (f < 0.0f) continue;
        const float4 v = *reinterpret_cast<const float4*>(part + (((size_t)b * n + s) * each + in) * a.d + c * 4);
        acc.x += v.x * f; acc.y += v.y * f; acc.z += v.z * f; acc.w += v.w * f;
    }
    for (int o = lanes; o < 32; o <<= 1) {
        acc.x += __shfl_xor_sync(0xffffffffu, acc.x, o);
        acc.y += __shfl_xor_sync(0xffffffffu, acc.y, o);
        acc.z += __shfl_xor_sync(0xffffffffu, acc.z, o);
        acc.w += __shfl_xor_sync(0xffffffffu, acc.w, o);
    }
    if (sub == 0) *reinterpret_cast<float4*>(&s_acc[warp][c * 4]) = acc;
    __syncthreads();
    for (int e = threadIdx.x; e < a.d; e += kCombineThreads) {
        float v = 0.0f;
#pragma unroll
        for (int w = 0; w < kCombineThreads / 32; ++w) v += s_acc[w][e];
        v = total == 0.0f ? 0.0f : v / total;
        if constexpr (BF16) reinterpret_cast<__nv_bfloat16*>(a.O)[row * a.d + e] = __float2bfloat16_rn(v);
        else reinterpret_cast<__half*>(a.O)[row * a.d + e] = __float2half_rn(v);
    }
}

}  // namespace

int launch_kv_combine(sentry_ctx* ctx, const KvAttendArgs& a, const float* part, const float2* ml, int n_splits, cudaStream_t st) {
    const size_t rows = (size_t)a.B * a.k_h * a.Tq;
    LaunchScope ls(ctx, KS_KV_COMBINE, st);
    auto k = a.dtype == SENTRY_BF16 ? kv_combine_kernel<true> : kv_combine_kernel<false>;
    SENTRY_CUDA_TRY(launch_chained(k, dim3((unsigned)rows), dim3(kCombineThreads), 0, st, a, part, ml, n_splits));
    return SENTRY_OK;
}
