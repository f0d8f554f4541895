// Serving attention for fp32 rows, on the plain ALUs: dense fp32 keys and values, or the 8-bit cache's.
//
// A block takes 16 rows of one kept head of a sample, four to a warp, and walks the keys 32 at a time through shared memory.  Scores: a lane
// is a key (rows of d + 1 floats, so that 32 lanes read 32 banks); values: a lane is a column.  fp32 is the type people validate
// with: the accuracy of expf and of fp32 sums counts here, and the rate does not.
#include "kv_attend.cuh"

namespace {

constexpr int kGRows = 16, kGKeys = 32;

// FORMAT: 0 dense fp32, 1 e4m3, 2 i8
template <int FORMAT, int D>
__global__ void __launch_bounds__(128) kv_generic_kernel(const KvAttendArgs a, int row_blocks) {
    __shared__ float sk[kGKeys][D + 1], sv[kGKeys][D];
    __shared__ __align__(16) float sq[kGRows][D];
    __shared__ unsigned s_vis;
    constexpr int COLS = D < 32 ? 1 : D / 32;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int rb = blockIdx.x % row_blocks, bj = blockIdx.x / row_blocks, b = bj / a.k_h, j = bj % a.k_h;
    grid_dependency_wait();
    const int h = kv_head(a, b, j);
    const int i0 = rb * kGRows, rows = min(kGRows, a.Tq - i0);
    float* out = (float*)a.O + ((size_t)bj * a.Tq + i0) * D;
    if (h < 0) {
        if (threadIdx.x == 0) atomicOr(a.status, SENTRY_STATUS_BIT_BAD_INDEX);
        for (int e = threadIdx.x; e < rows * D; e += 128) out[e] = 0.0f;
        return;
    }
    const int g = h / (a.Hq / a.Hk);
    const float scale = rsqrtf((float)D);
    const float* q = (const float*)a.Q + b * a.qs[0] + h * a.qs[1] + i0 * a.qs[2];
    for (int e = threadIdx.x; e < kGRows * D; e += 128) sq[e / D][e % D] = e / D < rows ? q[(e / D) * a.qs[2] + e % D] * scale : 0.0f;
    const int len = kv_length(a, b);
    const uint32_t mask = a.masks ? a.masks[b] : 0u;
    float m[4], l[4], o[4][COLS];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        m[r] = -INFINITY; l[r] = 0.0f;
#pragma unroll
        for (int c = 0; c < COLS; ++c) o[r][c] = 0.0f;
    }
    for (int n0 = 0; n0 < len; n0 += kGKeys) {
        __syncthreads();                    // the last tile has been read
        if (warp == 0) {
            const int n = n0 + lane;
            bool ok = n < len;
            if constexpr (FORMAT == 0) {
                if (ok && a.ids != nullptr) ok = kv_present(a.ids[n], mask);
            } else if (ok) {
                const int id = a.table[(size_t)b * a.max_pages + n / a.page];
                ok = id >= 0 && id < a.n_pages;
                if (!ok) atomicOr(a.status, SENTRY_STATUS_BIT_BAD_INDEX);
            }
            const unsigned vis = __ballot_sync(0xffffffffu, ok);
            if (lane == 0) s_vis = vis;
        }
        __syncthreads();
        const unsigned vis = s_vis;
        if (vis == 0) continue;
        for (int e = threadIdx.x; e < kGKeys * D; e += 128) {
            const int n = e / D, c = e % D;
            float k = 0.0f, v = 0.0f;
            if ((vis >> n) & 1u) {
                if constexpr (FORMAT == 0) {
                    k = ((const float*)a.K)[b * a.ks[0] + g * a.ks[1] + (n0 + n) * a.ks[2] + c];
                    v = ((const float*)a.V)[b * a.vs[0] + g * a.vs[1] + (n0 + n) * a.vs[2] + c];
                } else {
                    const int id = a.table[(size_t)b * a.max_pages + (n0 + n) / a.page];
                    const size_t ph = (size_t)id * a.Hk + g, at = (ph * a.page + (n0 + n) % a.page) * D + c;
                    k = code_value<FORMAT == 2>(((const uint8_t*)a.K)[at]) * a.k_scales[ph];
                    v = code_value<FORMAT == 2>(((const uint8_t*)a.V)[at]) * a.v_scales[ph];
                }
            }
            sk[n][c] = k;
            sv[n][c] = v;
        }
        __syncthreads();
        float s[4] = {};
#pragma unroll 4
        for (int c = 0; c < D; c += 4) {
            const float k0 = sk[lane][c], k1 = sk[lane][c + 1], k2 = sk[lane][c + 2], k3 = sk[lane][c + 3];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const float4 x = *reinterpret_cast<const float4*>(&sq[warp * 4 + r][c]);
                s[r] = fmaf(x.w, k3, fmaf(x.z, k2, fmaf(x.y, k1, fmaf(x.x, k0, s[r]))));
            }
        }
        float p[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            bool ok = (vis >> lane) & 1u;
            if (FORMAT != 0 && a.causal) ok = ok && n0 + lane <= len - a.Tq + i0 + warp * 4 + r;
            const float x = ok ? s[r] : -INFINITY;
            // (a score that is not a number stays one: fmaxf would drop it, the exponential below does not)
            float top = x;
#pragma unroll
            for (int w = 16; w > 0; w >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, w));
            top = fmaxf(top, m[r]);
            const float ref = top == -INFINITY ? 0.0f : top;
            const float keep = expf(m[r] - ref);
            p[r] = ok ? expf(x - ref) : 0.0f;
            l[r] = l[r] * keep + p[r];
#pragma unroll
            for (int c = 0; c < COLS; ++c) o[r][c] *= keep;
            m[r] = top;
        }
        for (int n = 0; n < kGKeys; ++n) {
            if (!((vis >> n) & 1u)) continue;
            float v[COLS];
#pragma unroll
            for (int c = 0; c < COLS; ++c) v[c] = lane + c * 32 < D ? sv[n][lane + c * 32] : 0.0f;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const float w = __shfl_sync(0xffffffffu, p[r], n);
                const bool sees = FORMAT == 0 || !a.causal || n0 + n <= len - a.Tq + i0 + warp * 4 + r;
#pragma unroll
                for (int c = 0; c < COLS; ++c) o[r][c] = sees ? fmaf(w, v[c], o[r][c]) : o[r][c];
            }
        }
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        float sum = l[r];
#pragma unroll
        for (int w = 16; w > 0; w >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, w);
        if (warp * 4 + r >= rows) continue;
#pragma unroll
        for (int c = 0; c < COLS; ++c)
            if (lane + c * 32 < D) out[(size_t)(warp * 4 + r) * D + lane + c * 32] = sum == 0.0f ? 0.0f : o[r][c] / sum;
    }
}

template <int FORMAT>
int launch_generic(sentry_ctx* ctx, const KvAttendArgs& a, cudaStream_t st) {
    const long long rb = (a.Tq + kGRows - 1) / kGRows;
    if (rb * a.B * a.k_h > 0x7fffffffLL) return SENTRY_ERR_UNSUPPORTED;
    auto k = a.d == 16 ? kv_generic_kernel<FORMAT, 16> : a.d == 32 ? kv_generic_kernel<FORMAT, 32> : a.d == 64 ? kv_generic_kernel<FORMAT, 64>
                                                                                                               : kv_generic_kernel<FORMAT, 128>;
    LaunchScope ls(ctx, KS_KV_ATTEND, st);
    SENTRY_CUDA_TRY(launch_chained(k, dim3((unsigned)(rb * a.B * a.k_h)), dim3(128), 0, st, a, (int)rb));
    return SENTRY_OK;
}

}  // namespace

int launch_kv_generic(sentry_ctx* ctx, const KvAttendArgs& a, cudaStream_t st) {
    return a.format == 0 ? launch_generic<0>(ctx, a, st) : a.format == SENTRY_FP8_E4M3 ? launch_generic<1>(ctx, a, st) : launch_generic<2>(ctx, a, st);
}
