// Serving attention for fp32 rows, on the plain ALUs: dense fp32 keys and values, or the 8-bit cache's.
//
// A block takes 16 rows of one kept head of a sample, two to a warp, and walks the keys 64 at a time through shared memory, the next
// tile's loads on the way in registers while it works on one.  Scores: a lane is two keys (rows of d + 4 floats, so that eight lanes' 16 bytes
// meet all banks); values: a lane is a column.  fp32 is the type people validate with: the accuracy of expf and of fp32 sums counts here,
// and the rate does not; small calls are bound by the latency of a tile.  (32 keys and four rows a warp, without loads ahead: 2 x 129
// rows of four heads on 333 keys 46 us; now 13.)
#include "kv_attend.cuh"

namespace {

constexpr int kGRows = 16, kGKeys = 64, kGThreads = 256;

// FORMAT: 0 dense fp32, 1 e4m3, 2 i8
template <int FORMAT, int D>
__global__ void __launch_bounds__(kGThreads) kv_generic_kernel(const KvAttendArgs a, int row_blocks) {
    constexpr int LD = D + 4, COLS = D < 32 ? 1 : D / 32, N4 = kGKeys * D / 4 / kGThreads;   // groups of four values a thread loads of K
    extern __shared__ __align__(16) float g_smem[];
    float *sk = g_smem, *sv = sk + kGKeys * LD, *sq = sv + kGKeys * LD, *sp = sq + kGRows * D;   // sp [kGRows][kGKeys]
    __shared__ unsigned s_vis[2];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int rb = blockIdx.x % row_blocks, bj = blockIdx.x / row_blocks, b = bj / a.k_h, j = bj % a.k_h;
    grid_dependency_wait();
    const int h = kv_head(a, b, j);
    const int i0 = rb * kGRows, rows = min(kGRows, a.Tq - i0);
    float* out = (float*)a.O + ((size_t)bj * a.Tq + i0) * D;
    if (h < 0) {
        if (threadIdx.x == 0) atomicOr(a.status, SENTRY_STATUS_BIT_BAD_INDEX);
        for (int e = threadIdx.x; e < rows * D; e += kGThreads) out[e] = 0.0f;
        return;
    }
    const int g = h / (a.Hq / a.Hk);
    const float scale = rsqrtf((float)D);
    const float* q = (const float*)a.Q + b * a.qs[0] + h * a.qs[1] + i0 * a.qs[2];
    for (int e = threadIdx.x; e < kGRows * D; e += kGThreads) sq[e] = e / D < rows ? q[(e / D) * a.qs[2] + e % D] * scale : 0.0f;
    const int len = kv_length(a, b);
    const uint32_t mask = a.masks ? a.masks[b] : 0u;
    const float *kd = (const float*)a.K + b * a.ks[0] + g * a.ks[1], *vd = (const float*)a.V + b * a.vs[0] + g * a.vs[1];

    // one tile's values in registers, and which of this warp's keys are present (warps 0 and 1)
    float4 rk[N4], rv[N4];
    bool here = false;
    auto fetch = [&](int n0) {
        if (warp < 2) {
            const int n = n0 + warp * 32 + lane;
            here = n < len;
            if constexpr (FORMAT == 0) {
                if (here && a.ids != nullptr) here = kv_present(a.ids[n], mask);
            } else if (here) {
                const int id = a.table[(size_t)b * a.max_pages + n / a.page];
                here = id >= 0 && id < a.n_pages;
                if (!here) atomicOr(a.status, SENTRY_STATUS_BIT_BAD_INDEX);
            }
        }
#pragma unroll
        for (int x = 0; x < N4; ++x) {
            const int e = x * kGThreads + threadIdx.x, n = n0 + e / (D / 4), c = e % (D / 4) * 4;
            rk[x] = rv[x] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            if (n >= len) continue;
            if constexpr (FORMAT == 0) {
                rk[x] = *reinterpret_cast<const float4*>(kd + n * a.ks[2] + c);
                rv[x] = *reinterpret_cast<const float4*>(vd + n * a.vs[2] + c);
            } else {
                const int id = a.table[(size_t)b * a.max_pages + n / a.page];
                if (id < 0 || id >= a.n_pages) continue;
                const size_t ph = (size_t)id * a.Hk + g, at = (ph * a.page + n % a.page) * D + c;
                const uint32_t kw = *reinterpret_cast<const uint32_t*>((const uint8_t*)a.K + at), vw = *reinterpret_cast<const uint32_t*>((const uint8_t*)a.V + at);
                const float ks = a.k_scales[ph], vs = a.v_scales[ph];
                float f[8];
#pragma unroll
                for (int y = 0; y < 4; ++y) {
                    f[y] = code_value<FORMAT == 2>((uint8_t)(kw >> (8 * y))) * ks;
                    f[4 + y] = code_value<FORMAT == 2>((uint8_t)(vw >> (8 * y))) * vs;
                }
                rk[x] = make_float4(f[0], f[1], f[2], f[3]);
                rv[x] = make_float4(f[4], f[5], f[6], f[7]);
            }
        }
    };
    float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.0f, 0.0f}, o[2][COLS];
#pragma unroll
    for (int r = 0; r < 2; ++r)
#pragma unroll
        for (int c = 0; c < COLS; ++c) o[r][c] = 0.0f;
    if (len > 0) fetch(0);
    for (int n0 = 0; n0 < len; n0 += kGKeys) {
        __syncthreads();                    // the last tile has been read
        if (warp < 2) {
            const unsigned vis = __ballot_sync(0xffffffffu, here);
            if (lane == 0) s_vis[warp] = vis;
        }
#pragma unroll
        for (int x = 0; x < N4; ++x) {
            const int e = x * kGThreads + threadIdx.x, n = e / (D / 4), c = e % (D / 4) * 4;
            *reinterpret_cast<float4*>(sk + n * LD + c) = rk[x];
            *reinterpret_cast<float4*>(sv + n * LD + c) = rv[x];
        }
        __syncthreads();
        if (n0 + kGKeys < len) fetch(n0 + kGKeys);
        const unsigned vis[2] = {s_vis[0], s_vis[1]};
        if ((vis[0] | vis[1]) == 0) continue;
        const float* qr = sq + warp * 2 * D;
        float s[2][2] = {};                 // [row][key lane, key lane + 32]
#pragma unroll 4
        for (int c = 0; c < D; c += 4) {
            const float4 k0 = *reinterpret_cast<const float4*>(sk + lane * LD + c), k1 = *reinterpret_cast<const float4*>(sk + (lane + 32) * LD + c);
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                const float4 x = *reinterpret_cast<const float4*>(qr + r * D + c);
                s[r][0] = fmaf(x.w, k0.w, fmaf(x.z, k0.z, fmaf(x.y, k0.y, fmaf(x.x, k0.x, s[r][0]))));
                s[r][1] = fmaf(x.w, k1.w, fmaf(x.z, k1.z, fmaf(x.y, k1.y, fmaf(x.x, k1.x, s[r][1]))));
            }
        }
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            bool ok[2];
#pragma unroll
            for (int y = 0; y < 2; ++y) {
                ok[y] = (vis[y] >> lane) & 1u;
                if (FORMAT != 0 && a.causal) ok[y] = ok[y] && n0 + y * 32 + lane <= len - a.Tq + i0 + warp * 2 + r;
                if (!ok[y]) s[r][y] = -INFINITY;
            }
            // (a score that is not a number stays one: fmaxf would drop it, the exponential below does not)
            float top = fmaxf(s[r][0], s[r][1]);
#pragma unroll
            for (int w = 16; w > 0; w >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, w));
            top = fmaxf(top, m[r]);
            const float ref = top == -INFINITY ? 0.0f : top, keep = expf(m[r] - ref);
            l[r] *= keep;
#pragma unroll
            for (int y = 0; y < 2; ++y) {
                const float p = ok[y] ? expf(s[r][y] - ref) : 0.0f;
                l[r] += p;
                sp[(warp * 2 + r) * kGKeys + y * 32 + lane] = p;
            }
#pragma unroll
            for (int c = 0; c < COLS; ++c) o[r][c] *= keep;
            m[r] = top;
        }
        __syncwarp();
        const float* pr = sp + warp * 2 * kGKeys;
        if ((vis[0] & vis[1]) == 0xffffffffu && !(FORMAT != 0 && a.causal)) {
#pragma unroll 4
            for (int n = 0; n < kGKeys; n += 4) {
                const float4 p0 = *reinterpret_cast<const float4*>(pr + n), p1 = *reinterpret_cast<const float4*>(pr + kGKeys + n);
#pragma unroll
                for (int c = 0; c < COLS; ++c) {
                    const float* v = sv + n * LD + (lane + c * 32) % D;
                    const float v0 = v[0], v1 = v[LD], v2 = v[2 * LD], v3 = v[3 * LD];
                    o[0][c] = fmaf(p0.w, v3, fmaf(p0.z, v2, fmaf(p0.y, v1, fmaf(p0.x, v0, o[0][c]))));
                    o[1][c] = fmaf(p1.w, v3, fmaf(p1.z, v2, fmaf(p1.y, v1, fmaf(p1.x, v0, o[1][c]))));
                }
            }
        } else {
            // what absent keys hold meets nothing
            for (int n = 0; n < kGKeys; ++n) {
                if (!((vis[n >> 5] >> (n & 31)) & 1u)) continue;
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    if (FORMAT != 0 && a.causal && n0 + n > len - a.Tq + i0 + warp * 2 + r) continue;
#pragma unroll
                    for (int c = 0; c < COLS; ++c) o[r][c] = fmaf(pr[r * kGKeys + n], sv[n * LD + (lane + c * 32) % D], o[r][c]);
                }
            }
        }
    }
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        float sum = l[r];
#pragma unroll
        for (int w = 16; w > 0; w >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, w);
        if (warp * 2 + r >= rows) continue;
#pragma unroll
        for (int c = 0; c < COLS; ++c)
            if (lane + c * 32 < D) out[(size_t)(warp * 2 + r) * D + lane + c * 32] = sum == 0.0f ? 0.0f : o[r][c] / sum;
    }
}

template <int FORMAT>
int launch_generic(sentry_ctx* ctx, const KvAttendArgs& a, cudaStream_t st) {
    const long long rb = (a.Tq + kGRows - 1) / kGRows;
    if (rb * a.B * a.k_h > 0x7fffffffLL) return SENTRY_ERR_UNSUPPORTED;
    auto k = a.d == 16 ? kv_generic_kernel<FORMAT, 16> : a.d == 32 ? kv_generic_kernel<FORMAT, 32> : a.d == 64 ? kv_generic_kernel<FORMAT, 64>
                                                                                                               : kv_generic_kernel<FORMAT, 128>;
    const int smem = (2 * kGKeys * (a.d + 4) + kGRows * (a.d + kGKeys)) * (int)sizeof(float);
    static std::atomic<unsigned long long> allowed[4];
    SENTRY_CUDA_TRY(allow_smem(k, smem, ctx->device, allowed[a.d == 16 ? 0 : a.d == 32 ? 1 : a.d == 64 ? 2 : 3]));
    LaunchScope ls(ctx, KS_KV_ATTEND, st);
    SENTRY_CUDA_TRY(launch_chained(k, dim3((unsigned)(rb * a.B * a.k_h)), dim3(kGThreads), (size_t)smem, st, a, (int)rb));
    return SENTRY_OK;
}

}  // namespace

int launch_kv_generic(sentry_ctx* ctx, const KvAttendArgs& a, cudaStream_t st) {
    return a.format == 0 ? launch_generic<0>(ctx, a, st) : a.format == SENTRY_FP8_E4M3 ? launch_generic<1>(ctx, a, st) : launch_generic<2>(ctx, a, st);
}
