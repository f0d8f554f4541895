// Linear layer in 8-bit integers: rows quantised per token, weights per output channel, exact 32-bit sums.
//
//   quantize_rows_kernel    s = max |x| / 127, c = nearest(x / s): a row is read once and stays in registers between the two
//   linear_i8_few_kernel    up to 64 tokens: warp MMA (s8 x s8 -> s32), bound by the weights' bytes and by latency
//   linear_i8_tc_kernel     tcgen05 kind::i8, operands by TMA, accumulators in tensor memory
#include <cuda.h>

#include "serving.cuh"
#include "tc_common.cuh"

namespace {

// ------------------------------------------------------------------------------------------------ quantise rows
// WARPS warps share a row (1: eight rows a block; 8: one row a block).  Up to HELD pieces of 16 bytes a lane stay in registers; what a
// longer row has beyond them is read a second time.
constexpr int kHeld = 8;

template <typename T, int WARPS>
__global__ void __launch_bounds__(256) quantize_rows_kernel(const T* __restrict__ X, int8_t* __restrict__ codes, float* __restrict__ scales,
                                                            int M, int K) {
    constexpr int N = Vec16<T>::N, LANES = 32 * WARPS;
    __shared__ float s_top[8];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const long long row = WARPS == 1 ? (long long)blockIdx.x * 8 + warp : blockIdx.x;
    const int at = WARPS == 1 ? lane : (int)threadIdx.x;
    grid_dependents_start_if_small();
    grid_dependency_wait();
    if (row >= M) return;                 // (whole warps, and no block-wide step follows where WARPS is 1)
    const uint4* src = reinterpret_cast<const uint4*>(X + row * K);
    const int pieces = K / N;
    uint4 held[kHeld];
    float top = 0.0f;
    bool bad = false;
    auto look = [&](const uint4& v) {
        float f[N];
        Vec16<T>::get(v, f);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float a = fabsf(f[i]);
            bad = bad || !(a <= 3.4028234e38f);
            top = fmaxf(top, a);
        }
    };
#pragma unroll
    for (int i = 0; i < kHeld; ++i) {
        const int p = at + i * LANES;
        held[i] = p < pieces ? src[p] : make_uint4(0, 0, 0, 0);
    }
#pragma unroll
    for (int i = 0; i < kHeld; ++i) look(held[i]);
    for (int p = at + kHeld * LANES; p < pieces; p += LANES) look(src[p]);
    if (bad) top = __int_as_float(0x7fc00000);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        const float other = __shfl_xor_sync(0xffffffffu, top, o);
        top = (isnan(top) || isnan(other)) ? __int_as_float(0x7fc00000) : fmaxf(top, other);
    }
    if (WARPS > 1) {
        if (lane == 0) s_top[warp] = top;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < WARPS; ++w) top = (isnan(top) || isnan(s_top[w])) ? __int_as_float(0x7fc00000) : fmaxf(top, s_top[w]);
    }
    const bool nan = isnan(top);
    const float s = nan ? top : scale_i8(top);
    const float inv = s > 0.0f ? __fdiv_rn(1.0f, s) : 0.0f;
    if (at == 0) scales[row] = s;
    int8_t* dst = codes + row * K;
    auto put = [&](const uint4& v, int p) {
        float f[N];
        Vec16<T>::get(v, f);
        uint32_t w[N / 4];
#pragma unroll
        for (int i = 0; i < N / 4; ++i) {
            int c[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) c[j] = s > 0.0f ? round_quotient_i8(f[4 * i + j], s, inv) : 0;
            w[i] = pack_i8x4(c[0], c[1], c[2], c[3]);
        }
        if constexpr (N == 8) *reinterpret_cast<uint2*>(dst + (size_t)p * 8) = make_uint2(w[0], w[1]);
        else *reinterpret_cast<uint32_t*>(dst + (size_t)p * 4) = w[0];
    };
#pragma unroll
    for (int i = 0; i < kHeld; ++i) {
        const int p = at + i * LANES;
        if (p < pieces) put(held[i], p);
    }
    for (int p = at + kHeld * LANES; p < pieces; p += LANES) put(src[p], p);
}

template <typename T>
int launch_quantize(sentry_ctx* ctx, int M, int K, const void* X, int8_t* codes, float* scales, cudaStream_t st) {
    LaunchScope ls(ctx, KS_QUANTIZE, st);
    // a warp per row where that fills the GPU and the row fits its registers
    const bool one = (long long)M >= 8LL * ctx->sm_count && K / Vec16<T>::N <= 32 * kHeld;
    if (one) SENTRY_CUDA_TRY(launch_chained(quantize_rows_kernel<T, 1>, dim3((unsigned)((M + 7) / 8)), dim3(256), 0, st, (const T*)X, codes, scales, M, K));
    else SENTRY_CUDA_TRY(launch_chained(quantize_rows_kernel<T, 8>, dim3((unsigned)M), dim3(256), 0, st, (const T*)X, codes, scales, M, K));
    return SENTRY_OK;
}

// ------------------------------------------------------------------------------------------------ few tokens
__device__ __forceinline__ void mma_i8(int32_t (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+r"(d[0]), "+r"(d[1]), "+r"(d[2]), "+r"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// A block: 16 output channels (the MMA's rows) and 8 TILES tokens (its columns); its eight warps split K in pieces of 64.  Inside a
// piece the order of k is free as long as both operands have the same, so a lane takes 16 consecutive bytes of its row for two MMAs:
// weights go from memory to the MMA without shared memory.
template <typename T, int TILES>
__global__ void __launch_bounds__(256) linear_i8_few_kernel(const int8_t* __restrict__ X, const int8_t* __restrict__ W, const float* __restrict__ xs,
                                                            const float* __restrict__ ws, const float* __restrict__ bias, T* __restrict__ Y,
                                                            int M, int K, int N) {
    __shared__ int32_t part[8][TILES][128];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
    const int n0 = blockIdx.x * 16;
    const uint4 zero = make_uint4(0, 0, 0, 0);
    int32_t acc[TILES][4] = {};
    grid_dependents_start_if_small();
    grid_dependency_wait();
    const bool r0 = n0 + g < N, r1 = n0 + g + 8 < N;
    const int8_t *w0 = W + (size_t)(n0 + g) * K, *w1 = w0 + (size_t)8 * K;
#pragma unroll 2
    for (int k0 = warp * 64; k0 < K; k0 += 512) {
        const int k = k0 + t * 16;
        const bool in = k < K;
        const uint4 a = in && r0 ? *reinterpret_cast<const uint4*>(w0 + k) : zero;
        const uint4 b = in && r1 ? *reinterpret_cast<const uint4*>(w1 + k) : zero;
        uint4 x[TILES];
#pragma unroll
        for (int i = 0; i < TILES; ++i) x[i] = in && i * 8 + g < M ? *reinterpret_cast<const uint4*>(X + (size_t)(i * 8 + g) * K + k) : zero;
#pragma unroll
        for (int i = 0; i < TILES; ++i) {
            mma_i8(acc[i], a.x, b.x, a.y, b.y, x[i].x, x[i].y);
            mma_i8(acc[i], a.z, b.z, a.w, b.w, x[i].z, x[i].w);
        }
    }
#pragma unroll
    for (int i = 0; i < TILES; ++i) {
        // element (channel, token) of the tile at token * 16 + channel
        part[warp][i][(2 * t) * 16 + g] = acc[i][0];
        part[warp][i][(2 * t + 1) * 16 + g] = acc[i][1];
        part[warp][i][(2 * t) * 16 + g + 8] = acc[i][2];
        part[warp][i][(2 * t + 1) * 16 + g + 8] = acc[i][3];
    }
    __syncthreads();
    for (int e = threadIdx.x; e < TILES * 128; e += 256) {
        const int i = e >> 7, in = e & 127, n = n0 + (in & 15), m = i * 8 + (in >> 4);
        if (n >= N || m >= M) continue;
        int32_t sum = 0;
#pragma unroll
        for (int w = 0; w < 8; ++w) sum += part[w][i][in];
        float y = (float)sum * xs[m] * ws[n];
        if (bias != nullptr) y += bias[n];
        Y[(size_t)m * N + n] = from_f32<T>(y);
    }
}

template <typename T>
int launch_few(sentry_ctx* ctx, const LinearArgs& a, cudaStream_t st) {
    const int M = a.d.M, tiles = (M + 7) / 8;
    auto k = tiles <= 1 ? linear_i8_few_kernel<T, 1> : tiles <= 2 ? linear_i8_few_kernel<T, 2> : tiles <= 4 ? linear_i8_few_kernel<T, 4>
                                                                                                             : linear_i8_few_kernel<T, 8>;
    LaunchScope ls(ctx, KS_LINEAR, st);
    SENTRY_CUDA_TRY(launch_chained(k, dim3((unsigned)((a.d.N + 15) / 16)), dim3(256), 0, st, a.X, a.W, a.xs, a.ws, a.bias, (T*)a.Y, M, a.d.K, a.d.N));
    return SENTRY_OK;
}

// ------------------------------------------------------------------------------------------------ tcgen05
// D[tmem] (+)= A[smem] * B[smem], s8 x s8 -> s32, 32 bytes of K a step; issued by one thread.
__device__ __forceinline__ void umma_i8(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::i8 [%0], %1, %2, %3, p;\n\t}"
        :
        : "r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate)
        : "memory");
}
// accumulator s32 (2), both operands s8 (1), K-major
__host__ __device__ constexpr uint32_t umma_idesc_i8(int M, int N) {
    return (2u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24);
}

constexpr int kLinBM = 128, kLinBN = 256, kLinStages = 4, kLinThreads = 256;
constexpr int kLinStageBytes = (kLinBM + kLinBN) * 128;
constexpr int kLinStore = 4 * 32 * 128;   // an epilogue warp's 32 rows of 128 bytes
constexpr int kLinSmem = kLinStages * kLinStageBytes + kLinStore + 1024 + 1024;

struct LinMisc {
    uint64_t full[kLinStages], empty[kLinStages], acc_full[2], acc_empty[2];
    uint32_t tmem_base;
    int abort_flag;
};

// i8 [rows, K] row-major -> boxes of box_rows x 128 bytes, 128-byte swizzle; what lies outside reads as 0
bool make_map_i8(CUtensorMap* tm, const void* ptr, uint64_t rows, uint64_t K, uint32_t box_rows) {
    EncodeTiledFn fn = get_encode_fn();
    if (fn == nullptr) return false;
    cuuint64_t dims[2] = {K, rows};
    cuuint64_t strides[1] = {K};
    cuuint32_t box[2] = {128, box_rows};
    cuuint32_t estr[2] = {1, 1};
    return fn(tm, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(ptr), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <typename T>
__global__ void __launch_bounds__(kLinThreads, 1)
linear_i8_tc_kernel(const __grid_constant__ CUtensorMap tm_x, const __grid_constant__ CUtensorMap tm_w, const float* __restrict__ xs,
                    const float* __restrict__ ws, const float* __restrict__ bias, T* __restrict__ Y, int M, int K, int N, unsigned int* status) {
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw_addr = ptx::smem_u32(smem_raw);
    const uint32_t base = (raw_addr + 1023u) & ~1023u;
    LinMisc* misc = reinterpret_cast<LinMisc*>(smem_raw + (base - raw_addr) + kLinStages * kLinStageBytes + kLinStore);
    volatile int* abort_flag = &misc->abort_flag;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int s = 0; s < kLinStages; ++s) {
            ptx::mbar_init(ptx::smem_u32(&misc->full[s]), 1);
            ptx::mbar_init(ptx::smem_u32(&misc->empty[s]), 1);
        }
        for (int s = 0; s < 2; ++s) {
            ptx::mbar_init(ptx::smem_u32(&misc->acc_full[s]), 1);
            ptx::mbar_init(ptx::smem_u32(&misc->acc_empty[s]), 4);
        }
        misc->abort_flag = 0;
        ptx::fence_barrier_init();
        ptx::prefetch_tensormap(&tm_x);
        ptx::prefetch_tensormap(&tm_w);
    }
    if (warp == 0) {
        ptx::tmem_alloc(ptx::smem_u32(&misc->tmem_base), 512);
        ptx::tmem_relinquish();
    }
    ptx::tc_fence_before_sync();
    __syncthreads();
    ptx::tc_fence_after_sync();
    const uint32_t tmem = misc->tmem_base;
    grid_dependency_wait();
    const int n_tiles = (N + kLinBN - 1) / kLinBN, m_tiles = (M + kLinBM - 1) / kLinBM;
    const long long tiles = (long long)n_tiles * m_tiles;
    const int KB = (K + 127) / 128;

    if (warp == 0) {
        bool ok = true;
        uint32_t it = 0;
        for (long long tile = blockIdx.x; tile < tiles && ok; tile += gridDim.x) {
            const int m0 = (int)(tile / n_tiles) * kLinBM, n0 = (int)(tile % n_tiles) * kLinBN;
            for (int kb = 0; kb < KB && ok; ++kb, ++it) {
                const uint32_t s = it % kLinStages, use = it / kLinStages;
                ok = warp_wait(&misc->empty[s], (use & 1) ^ 1, abort_flag);
                if (!ok) break;
                if (elect_one()) {
                    const uint32_t bar = ptx::smem_u32(&misc->full[s]), dst = base + s * kLinStageBytes;
                    ptx::mbar_arrive_expect_tx(bar, kLinStageBytes);
                    ptx::tma_load_2d(dst, &tm_x, kb * 128, m0, bar);
                    ptx::tma_load_2d(dst + kLinBM * 128, &tm_w, kb * 128, n0, bar);
                }
                __syncwarp();
            }
        }
    } else if (warp == 1) {
        const uint32_t idesc = umma_idesc_i8(kLinBM, kLinBN);
        bool ok = true;
        uint32_t it = 0, n = 0;
        for (long long tile = blockIdx.x; tile < tiles && ok; tile += gridDim.x, ++n) {
            const uint32_t buf = n & 1, acc = tmem + buf * kLinBN;
            ok = warp_wait(&misc->acc_empty[buf], ((n >> 1) & 1) ^ 1, abort_flag);
            ptx::tc_fence_after_sync();
            for (int kb = 0; kb < KB && ok; ++kb, ++it) {
                const uint32_t s = it % kLinStages, use = it / kLinStages;
                ok = warp_wait(&misc->full[s], use & 1, abort_flag);
                if (!ok) break;
                ptx::tc_fence_after_sync();
                if (elect_one()) {
                    const uint32_t a = base + s * kLinStageBytes, b = a + kLinBM * 128;
#pragma unroll
                    for (int ks = 0; ks < 4; ++ks)
                        umma_i8(acc, ptx::umma_smem_desc_sw128(a + ks * 32), ptx::umma_smem_desc_sw128(b + ks * 32), idesc, (kb > 0 || ks > 0) ? 1u : 0u);
                    ptx::umma_commit(ptx::smem_u32(&misc->empty[s]));
                    if (kb == KB - 1) ptx::umma_commit(ptx::smem_u32(&misc->acc_full[buf]));
                }
                __syncwarp();
            }
        }
    } else if (warp >= 4) {
        // rows of this warp's quarter; 128 bytes of every row at a time through shared memory, so that stores write whole lines
        constexpr int COLS = 128 / (int)sizeof(T);    // 64 or 32 columns
        const int quarter = warp & 3;
        const uint32_t stg = base + kLinStages * kLinStageBytes + quarter * 4096;
        bool ok = true;
        uint32_t n = 0;
        const bool whole = N % (16 / (int)sizeof(T)) == 0;    // rows of Y start on 16 bytes
        for (long long tile = blockIdx.x; tile < tiles && ok; tile += gridDim.x, ++n) {
            const uint32_t buf = n & 1, acc = tmem + buf * kLinBN + ((uint32_t)(quarter * 32) << 16);
            const int m0 = (int)(tile / n_tiles) * kLinBM + quarter * 32, n0 = (int)(tile % n_tiles) * kLinBN;
            const float sx = m0 + lane < M ? xs[m0 + lane] : 0.0f;
            ok = warp_wait(&misc->acc_full[buf], (n >> 1) & 1, abort_flag);
            if (!ok) break;
            ptx::tc_fence_after_sync();
            for (int c0 = 0; c0 < kLinBN && n0 + c0 < N; c0 += COLS) {
                uint32_t w[32];
#pragma unroll
                for (int h = 0; h < COLS / 32; ++h) {
                    uint32_t r[32];
                    ptx::tmem_ld_32x32(acc + c0 + h * 32, r);
                    ptx::tmem_ld_wait();
#pragma unroll
                    for (int i = 0; i < 32; ++i) {
                        const int col = n0 + c0 + h * 32 + i;
                        const bool in = col < N;
                        float y = (float)(int32_t)r[i] * sx * (in ? __ldg(ws + col) : 0.0f);
                        if (bias != nullptr && in) y += __ldg(bias + col);
                        if constexpr (sizeof(T) == 4) w[i] = __float_as_uint(y);
                        else {
                            const T v = from_f32<T>(y);
                            const uint32_t bits = *reinterpret_cast<const unsigned short*>(&v);
                            if (i & 1) w[h * 16 + i / 2] |= bits << 16;
                            else w[h * 16 + i / 2] = bits;
                        }
                    }
                }
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(stg + lane * 128 + ((i ^ (lane & 7)) << 4)), "r"(w[4 * i]),
                                 "r"(w[4 * i + 1]), "r"(w[4 * i + 2]), "r"(w[4 * i + 3])
                                 : "memory");
                __syncwarp();
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int row = i * 4 + (lane >> 3), ch = lane & 7, col = n0 + c0 + ch * (16 / (int)sizeof(T));
                    uint4 v;
                    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(stg + row * 128 + ((ch ^ (row & 7)) << 4)));
                    if (m0 + row >= M) continue;
                    T* dst = Y + (size_t)(m0 + row) * N + col;
                    if (whole) {
                        if (col < N) *reinterpret_cast<uint4*>(dst) = v;
                    } else {
                        const T* e = reinterpret_cast<const T*>(&v);
#pragma unroll
                        for (int j = 0; j < 16 / (int)sizeof(T); ++j)
                            if (col + j < N) dst[j] = e[j];
                    }
                }
                __syncwarp();
            }
            ptx::tc_fence_before_sync();
            warp_arrive(&misc->acc_empty[buf]);
        }
    }
    tc_cta_teardown(abort_flag, status, tmem, 512);
}

template <typename T>
int launch_tc(sentry_ctx* ctx, const LinearArgs& a, cudaStream_t st) {
    CUtensorMap mx, mw;
    if (!make_map_i8(&mx, a.X, a.d.M, a.d.K, kLinBM) || !make_map_i8(&mw, a.W, a.d.N, a.d.K, kLinBN)) return SENTRY_ERR_CUDA;
    const long long tiles = (long long)((a.d.M + kLinBM - 1) / kLinBM) * ((a.d.N + kLinBN - 1) / kLinBN);
    auto k = linear_i8_tc_kernel<T>;
    SENTRY_CUDA_TRY(cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, kLinSmem));
    LaunchScope ls(ctx, KS_LINEAR, st);
    SENTRY_CUDA_TRY(launch_chained(k, dim3((unsigned)(tiles < ctx->sm_count ? tiles : ctx->sm_count)), dim3(kLinThreads), kLinSmem, st, mx, mw, a.xs, a.ws,
                                   a.bias, (T*)a.Y, a.d.M, a.d.K, a.d.N, a.status));
    return SENTRY_OK;
}

template <typename T>
int launch_linear(sentry_ctx* ctx, const LinearArgs& a, cudaStream_t st) {
    return a.d.M <= 64 ? launch_few<T>(ctx, a, st) : launch_tc<T>(ctx, a, st);
}

}  // namespace

int launch_quantize_rows_i8(sentry_ctx* ctx, int M, int K, int dtype, const void* X, int8_t* codes, float* scales, cudaStream_t st) {
    switch (dtype) {
        case SENTRY_F32: return launch_quantize<float>(ctx, M, K, X, codes, scales, st);
        case SENTRY_BF16: return launch_quantize<__nv_bfloat16>(ctx, M, K, X, codes, scales, st);
        default: return launch_quantize<__half>(ctx, M, K, X, codes, scales, st);
    }
}
int launch_linear_i8(sentry_ctx* ctx, const LinearArgs& a, cudaStream_t st) {
    switch (a.d.dtype) {
        case SENTRY_F32: return launch_linear<float>(ctx, a, st);
        case SENTRY_BF16: return launch_linear<__nv_bfloat16>(ctx, a, st);
        default: return launch_linear<__half>(ctx, a, st);
    }
}
