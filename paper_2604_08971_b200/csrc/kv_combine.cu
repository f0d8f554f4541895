// Joins the parts of attention of many rows whose axis of keys was split over blocks.
#include "kv_attend.cuh"

namespace {

constexpr int kCombineThreads = 256, kAhead = 8;

// A thread takes four columns of a row and every G-th of its parts, kAhead of them on the way at once; G threads meet in shared memory.
// (G 1 up to kAhead parts: a block per row 15 us for 8192 rows of two parts.  8 beyond: a thread after part 37 us for 16 rows of 128.)
template <bool BF16>
__global__ void __launch_bounds__(kCombineThreads) kv_combine_kernel(const KvAttendArgs a, const float* __restrict__ part, const float2* __restrict__ ml, int n, int G) {
    __shared__ float4 s_acc[kCombineThreads];
    __shared__ float2 s_ml[kCombineThreads];
    const int cols = a.d / 4, c = threadIdx.x % cols * 4, gi = threadIdx.x / cols % G, per_block = kCombineThreads / (cols * G);
    const size_t each = (size_t)a.k_h * a.Tq, rows = (size_t)a.B * each;      // rows of a sample, of all
    const size_t row = (size_t)blockIdx.x * per_block + threadIdx.x / (cols * G);
    grid_dependency_wait();
    const int b = (int)(min(row, rows - 1) / each);
    const size_t in = row - (size_t)b * each;
    // (the rows of what is no head are written)
    const bool here = row < rows && kv_head(a, b, (int)(in / a.Tq)) >= 0;
    const size_t first = (size_t)b * n * each + in;
    float top = -INFINITY, total = 0.0f;
    float4 acc = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    for (int s0 = gi; here && s0 < n; s0 += kAhead * G) {
        float2 x[kAhead];
        float4 p[kAhead];
        float now = top;
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int s = s0 + i * G;
            x[i] = s < n ? ml[first + s * each] : make_float2(-INFINITY, 0.0f);
            p[i] = s < n ? *reinterpret_cast<const float4*>(part + (first + s * each) * a.d + c) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            now = fmaxf(now, x[i].x);
        }
        const float ref = now == -INFINITY ? 0.0f : now, keep = top == now ? 1.0f : exp2_fast(top - ref);
        top = now;
        total *= keep;
        acc.x *= keep; acc.y *= keep; acc.z *= keep; acc.w *= keep;
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            if (x[i].x == -INFINITY && x[i].y == 0.0f) continue;       // (a part that saw nothing has not been written)
            const float f = exp2_fast(x[i].x - ref);
            total += x[i].y * f;
            acc.x += p[i].x * f; acc.y += p[i].y * f; acc.z += p[i].z * f; acc.w += p[i].w * f;
        }
    }
    if (G > 1) {
        s_acc[threadIdx.x] = acc;
        s_ml[threadIdx.x] = make_float2(top, total);
        __syncthreads();
        if (gi != 0) return;
        for (int i = 1; i < G; ++i) {
            const float2 x = s_ml[threadIdx.x + i * cols];
            const float4 p = s_acc[threadIdx.x + i * cols];
            const float now = fmaxf(top, x.x), ref = now == -INFINITY ? 0.0f : now, keep = top == now ? 1.0f : exp2_fast(top - ref), f = exp2_fast(x.x - ref);
            top = now;
            total = total * keep + x.y * f;
            acc.x = acc.x * keep + p.x * f; acc.y = acc.y * keep + p.y * f; acc.z = acc.z * keep + p.z * f; acc.w = acc.w * keep + p.w * f;
        }
    }
    if (!here) return;
    const float inv = total == 0.0f ? 0.0f : 1.0f / total;
    *reinterpret_cast<uint2*>((uint16_t*)a.O + row * a.d + c) =
        total == 0.0f ? make_uint2(0u, 0u) : make_uint2(pack2<BF16>(acc.x * inv, acc.y * inv), pack2<BF16>(acc.z * inv, acc.w * inv));
}

}  // namespace

int launch_kv_combine(sentry_ctx* ctx, const KvAttendArgs& a, const float* part, const float2* ml, int n_splits, cudaStream_t st) {
    const size_t rows = (size_t)a.B * a.k_h * a.Tq;
    const int G = n_splits <= kAhead ? 1 : 8, per_block = kCombineThreads / (a.d / 4 * G);
    LaunchScope ls(ctx, KS_KV_COMBINE, st);
    auto k = a.dtype == SENTRY_BF16 ? kv_combine_kernel<true> : kv_combine_kernel<false>;
    SENTRY_CUDA_TRY(launch_chained(k, dim3((unsigned)((rows + per_block - 1) / per_block)), dim3(kCombineThreads), 0, st, a, part, ml, n_splits, G));
    return SENTRY_OK;
}
