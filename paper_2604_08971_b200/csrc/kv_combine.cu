// Joins the parts of attention whose axis of keys was split over blocks.
#include "kv_attend.cuh"

namespace {

// Joins the parts of a split axis: a warp per row.
template <bool BF16>
__global__ void __launch_bounds__(128) kv_combine_kernel(const KvAttendArgs a, const float* __restrict__ part, const float2* __restrict__ ml, int n_splits) {
    const int lane = threadIdx.x & 31;
    const size_t rows = (size_t)a.B * a.k_h * a.Tq, row = (size_t)blockIdx.x * 4 + (threadIdx.x >> 5);
    grid_dependency_wait();
    if (row >= rows) return;
    const int j = (int)(row / a.Tq % a.k_h), b = (int)(row / a.Tq / a.k_h);
    if (kv_head(a, b, j) < 0) return;         // (its zero rows are written)
    float top = -INFINITY;
    for (int s = lane; s < n_splits; s += 32) top = fmaxf(top, ml[s * rows + row].x);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    const float ref = top == -INFINITY ? 0.0f : top;
    float acc[4] = {}, sum = 0.0f;
    const int cols = a.d / 32 ? a.d / 32 : 1, c0 = lane * cols;
    for (int s = 0; s < n_splits; ++s) {
        const float2 x = ml[s * rows + row];
        const float f = exp2_fast(x.x - ref);
        sum += x.y * f;
        if (x.x == -INFINITY && x.y == 0.0f) continue;    // (nothing seen there)
        if (c0 < a.d)
            for (int c = 0; c < cols; ++c) acc[c] += part[(s * rows + row) * a.d + c0 + c] * f;
    }
    if (c0 < a.d)
        for (int c = 0; c < cols; ++c) {
            const float v = sum == 0.0f ? 0.0f : acc[c] / sum;
            if constexpr (BF16) reinterpret_cast<__nv_bfloat16*>(a.O)[row * a.d + c0 + c] = __float2bfloat16_rn(v);
            else reinterpret_cast<__half*>(a.O)[row * a.d + c0 + c] = __float2half_rn(v);
        }
}

}  // namespace

int launch_kv_combine(sentry_ctx* ctx, const KvAttendArgs& a, const float* part, const float2* ml, int n_splits, cudaStream_t st) {
    const size_t rows = (size_t)a.B * a.k_h * a.Tq;
    LaunchScope ls(ctx, KS_KV_COMBINE, st);
    auto k = a.dtype == SENTRY_BF16 ? kv_combine_kernel<true> : kv_combine_kernel<false>;
    SENTRY_CUDA_TRY(launch_chained(k, dim3((unsigned)((rows + 3) / 4)), dim3(128), 0, st, a, part, ml, n_splits));
    return SENTRY_OK;
}
