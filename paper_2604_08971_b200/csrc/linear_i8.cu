// Linear layer in 8-bit integers: rows quantised per token, weights per output channel, exact 32-bit sums.
//
//   quantize_rows_kernel    s = max |x| / 127, c = nearest(x / s): a row is read once and stays in registers between the two
//   linear_i8_few_kernel    up to 64 tokens: warp MMA (s8 x s8 -> s32), bound by the weights' bytes and by latency
//   linear_i8_tc_kernel     tcgen05 kind::i8, operands by TMA, accumulators in tensor memory
#include <cuda.h>

#include <type_traits>

#include "linear_tiles.cuh"
#include "serving.cuh"
#include "tc_common.cuh"

namespace {

// ------------------------------------------------------------------------------------------------ quantise rows
// WARPS warps share a row (1: eight rows a block; 8: one row a block).  Up to HELD pieces of 16 bytes a lane stay in registers between the
// two steps; what a longer row has beyond them is read a second time.  Bound by the bytes, as long as a value costs few instructions:
// the maximum runs on pairs of magnitude bits, and the quotient is rounded by an addition, two at a time (codes_i8): 65536 x 1024 bf16
// in 31.5 us, 6.4 TB/s, what a copy reaches.
template <typename T, int WARPS, int HELD>
__global__ void __launch_bounds__(256) quantize_rows_kernel(const T* __restrict__ X, int8_t* __restrict__ codes, float* __restrict__ scales,
                                                            int M, int K) {
    constexpr int N = Vec16<T>::N, LANES = 32 * WARPS;
    __shared__ uint32_t s_top[8];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const long long row = WARPS == 1 ? (long long)blockIdx.x * 8 + warp : blockIdx.x;
    const int at = WARPS == 1 ? lane : (int)threadIdx.x;
    grid_dependents_start_if_small();
    grid_dependency_wait();
    if (row >= M) return;                 // (whole warps, and no block-wide step follows where WARPS is 1)
    const uint4* src = reinterpret_cast<const uint4*>(X + row * K);
    const int pieces = K / N;
    uint4 held[HELD];
    AbsMax<T> top;
#pragma unroll
    for (int i = 0; i < HELD; ++i) {
        const int p = at + i * LANES;
        held[i] = p < pieces ? src[p] : make_uint4(0, 0, 0, 0);
    }
#pragma unroll
    for (int i = 0; i < HELD; ++i) top.add(held[i]);
    for (int p = at + HELD * LANES; p < pieces; p += LANES) top.add(src[p]);
    uint32_t bits = __reduce_max_sync(0xffffffffu, top.bits());
    if (WARPS > 1) {
        if (lane == 0) s_top[warp] = bits;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < WARPS; ++w) bits = max(bits, s_top[w]);
    }
    const float most = magnitude<T>(bits);
    const float s = isnan(most) ? most : scale_i8(most);
    const float inv = s > 0.0f ? reciprocal_i8(s, most) : 0.0f;
    if (at == 0) scales[row] = s;
    int8_t* dst = codes + row * K;
    auto put_all = [&](auto check) {
        auto put = [&](const uint4& v, int p) {
            float f[N];
            uint32_t w[N / 4] = {};
            Vec16<T>::get(v, f);
            if (s > 0.0f) codes_i8<decltype(check)::value, N>(f, s, inv, w);
            if constexpr (N == 8) *reinterpret_cast<uint2*>(dst + (size_t)p * 8) = make_uint2(w[0], w[1]);
            else *reinterpret_cast<uint32_t*>(dst + (size_t)p * 4) = w[0];
        };
#pragma unroll
        for (int i = 0; i < HELD; ++i) {
            const int p = at + i * LANES;
            if (p < pieces) put(held[i], p);
        }
        for (int p = at + HELD * LANES; p < pieces; p += LANES) put(src[p], p);
    };
    if (sure_i8<T>(s, most)) put_all(std::false_type());
    else put_all(std::true_type());
}

template <typename T>
int launch_quantize(sentry_ctx* ctx, int M, int K, const void* X, int8_t* codes, float* scales, cudaStream_t st) {
    LaunchScope ls(ctx, KS_QUANTIZE, st);
    const int pieces = K / Vec16<T>::N;
    // a warp per row where that fills the GPU and the row fits its registers
    const bool one = (long long)M >= 8LL * ctx->sm_count && pieces <= 32 * 8;
    auto k = one ? (pieces <= 64 ? quantize_rows_kernel<T, 1, 2> : pieces <= 128 ? quantize_rows_kernel<T, 1, 4> : quantize_rows_kernel<T, 1, 8>)
                 : (pieces <= 256 ? quantize_rows_kernel<T, 8, 1> : quantize_rows_kernel<T, 8, 8>);
    SENTRY_CUDA_TRY(launch_chained(k, dim3((unsigned)(one ? linear_tiles(M, 8) : M)), dim3(256), 0, st, (const T*)X, codes, scales, M, K));
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
    SENTRY_CUDA_TRY(launch_chained(k, dim3((unsigned)linear_tiles(a.d.N, 16)), dim3(256), 0, st, a.X, a.W, a.xs, a.ws, a.bias, (T*)a.Y, M, a.d.K, a.d.N));
    return SENTRY_OK;
}

// ------------------------------------------------------------------------------------------------ tcgen05
// D[tmem] (+)= A[smem] * B[smem], s8 x s8 -> s32, 32 bytes of K a step; issued by one thread.  P: 2 for a pair of CTAs.
template <int P>
__device__ __forceinline__ void umma_i8(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
    if constexpr (P == 2)
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::2.kind::i8 [%0], %1, %2, %3, p;\n\t}" ::"r"(d_tmem), "l"(a_desc),
                     "l"(b_desc), "r"(idesc), "r"(accumulate)
                     : "memory");
    else
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::i8 [%0], %1, %2, %3, p;\n\t}" ::"r"(d_tmem), "l"(a_desc),
                     "l"(b_desc), "r"(idesc), "r"(accumulate)
                     : "memory");
}
// accumulator s32 (2), both operands s8 (1), K-major
__host__ __device__ constexpr uint32_t umma_idesc_i8(int M, int N) {
    return (2u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24);
}

// A tile: 128 P tokens x BN channels, K in steps of 128 bytes; a pair's CTAs have 128 tokens and half of the channels' weights each, so that
// a tile costs the L2 and shared memory two thirds of what two single CTAs' would.  Two accumulators in tensor memory: the eight
// epilogue warps scale one and store it, by TMA, while the other is summed.  Bound by the tensor pipe (74 % of its cycles) and the 268 MB
// of results beside it: 2.5 PFLOP/s of 8-bit products.
// Tried without gain at 65536 x 1024 x 2048 (108 us): the accumulator handed over before it is scaled (115), sixteen epilogue warps
// (114), six stages and stores of 32 bytes a row (125), a pair's weights kept in shared memory with three stages of X (141).
constexpr int kLinThreads = 384, kLinEpiWarp0 = 4, kLinEpiWarps = 8;

template <int P, int BN>
struct LinCfg {
    static constexpr int B_ROWS = BN / P;
    static constexpr int STAGE = (128 + B_ROWS) * 128;
    static constexpr int STAGES = 163840 / STAGE > 8 ? 8 : 163840 / STAGE;
    static constexpr int TMEM = BN <= 64 ? 128 : BN <= 128 ? 256 : 512;
    static constexpr int EPI = 4096, SCALES = (BN < 128 ? 128 : BN) * 4;   // a warp's 32 rows of 128 bytes; scales and biases of its columns
    static constexpr int SMEM = STAGES * STAGE + kLinEpiWarps * (EPI + SCALES) + 1024;
};
struct LinMisc {
    uint64_t full[8], empty[8], acc_full[2], acc_empty[2];
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

// Y [M, N] row-major -> boxes of 32 rows x 128 bytes, 128-byte swizzle; what lies outside is not written
template <typename T>
bool make_map_out(CUtensorMap* tm, const void* ptr, uint64_t M, uint64_t N) {
    EncodeTiledFn fn = get_encode_fn();
    if (fn == nullptr) return false;
    cuuint64_t dims[2] = {N, M};
    cuuint64_t strides[1] = {N * sizeof(T)};
    cuuint32_t box[2] = {128 / (cuuint32_t)sizeof(T), 32};
    cuuint32_t estr[2] = {1, 1};
    return fn(tm, sizeof(T) == 4 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : std::is_same_v<T, __half> ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2,
              const_cast<void*>(ptr), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_NONE,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
__device__ __forceinline__ void tma_store_2d(const void* tmap, int x, int y, uint32_t smem) {
    asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.tile.bulk_group [%0, {%1, %2}], [%3];" ::"l"(reinterpret_cast<uint64_t>(tmap)), "r"(x), "r"(y), "r"(smem)
                 : "memory");
    asm volatile("cp.async.bulk.commit_group;" ::: "memory");
}

template <typename T, int P, int BN>
__global__ void __launch_bounds__(kLinThreads, 1)
linear_i8_tc_kernel(const __grid_constant__ CUtensorMap tm_x, const __grid_constant__ CUtensorMap tm_w, const __grid_constant__ CUtensorMap tm_y, const float* __restrict__ xs,
                    const float* __restrict__ ws, const float* __restrict__ bias, T* __restrict__ Y, int M, int K, int N, unsigned int* status) {
    using C = LinCfg<P, BN>;
    extern __shared__ uint8_t smem_raw[];
    __shared__ LinMisc misc_s;
    LinMisc* misc = &misc_s;
    const uint32_t raw_addr = ptx::smem_u32(smem_raw), base = (raw_addr + 1023u) & ~1023u;
    volatile int* abort_flag = &misc->abort_flag;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = P == 2 ? (int)ptx::cluster_rank() : 0;      // CTA 0 of a pair issues the UMMAs of both
    if (threadIdx.x == 0) {
        for (int s = 0; s < C::STAGES; ++s) {
            ptx::mbar_init(ptx::smem_u32(&misc->full[s]), 1);
            ptx::mbar_init(ptx::smem_u32(&misc->empty[s]), 1);
        }
        for (int s = 0; s < 2; ++s) {
            ptx::mbar_init(ptx::smem_u32(&misc->acc_full[s]), 1);
            ptx::mbar_init(ptx::smem_u32(&misc->acc_empty[s]), P * kLinEpiWarps);
        }
        misc->abort_flag = 0;
        ptx::fence_barrier_init();
        ptx::prefetch_tensormap(&tm_x);
        ptx::prefetch_tensormap(&tm_w);
    }
    if (warp == 0) {
        if constexpr (P == 2) { ptx::tmem_alloc_pair(ptx::smem_u32(&misc->tmem_base), C::TMEM); ptx::tmem_relinquish_pair(); }
        else { ptx::tmem_alloc(ptx::smem_u32(&misc->tmem_base), C::TMEM); ptx::tmem_relinquish(); }
    }
    ptx::tc_fence_before_sync();
    __syncthreads();
    if constexpr (P == 2) ptx::cluster_sync();                   // the other CTA's barriers are initialised
    ptx::tc_fence_after_sync();
    const uint32_t tmem = misc->tmem_base;
    grid_dependency_wait();
    const int n_tiles = (int)linear_tiles(N, BN);
    const long long tiles = n_tiles * linear_tiles(M, 128 * P);
    const long long tile0 = blockIdx.x / P, tile_step = gridDim.x / P;
    const int KB = (K + 127) / 128;

    if (warp == 0) {
        bool ok = true;
        uint32_t it = 0;
        for (long long tile = tile0; tile < tiles && ok; tile += tile_step) {
            const int m0 = (int)(tile / n_tiles) * 128 * P + rank * 128, n0 = (int)(tile % n_tiles) * BN + rank * C::B_ROWS;
            for (int kb = 0; kb < KB && ok; ++kb, ++it) {
                const uint32_t s = it % C::STAGES, use = it / C::STAGES;
                ok = warp_wait(&misc->empty[s], (use & 1) ^ 1, abort_flag);
                if (!ok) break;
                if (elect_one()) {
                    const uint32_t bar = ptx::smem_u32(&misc->full[s]), dst = base + s * C::STAGE;
                    if (rank == 0) ptx::mbar_arrive_expect_tx(bar, P * C::STAGE);
                    if constexpr (P == 2) {
                        const uint32_t bar0 = ptx::cluster_addr(bar, 0);
                        ptx::tma_load_2d_pair(dst, &tm_x, kb * 128, m0, bar0);
                        ptx::tma_load_2d_pair(dst + 128 * 128, &tm_w, kb * 128, n0, bar0);
                    } else {
                        ptx::tma_load_2d(dst, &tm_x, kb * 128, m0, bar);
                        ptx::tma_load_2d(dst + 128 * 128, &tm_w, kb * 128, n0, bar);
                    }
                }
                __syncwarp();
            }
        }
    } else if (warp == 1 && rank == 0) {
        constexpr uint32_t idesc = umma_idesc_i8(128 * P, BN);
        // (in a pair, the other CTA's copies and threads arrive on these barriers too)
        auto wait = [&](uint64_t* bar, uint32_t parity) {
            const bool got = warp_wait(bar, parity, abort_flag);
            if constexpr (P == 2) { if (got) (void)ptx::mbar_try_wait_cluster(ptx::smem_u32(bar), parity); }   // acquired at cluster scope too
            return got;
        };
        bool ok = true;
        uint32_t it = 0, n = 0;
        for (long long tile = tile0; tile < tiles && ok; tile += tile_step, ++n) {
            const uint32_t buf = n & 1, acc = tmem + buf * BN;
            ok = wait(&misc->acc_empty[buf], ((n >> 1) & 1) ^ 1);
            if (!ok) break;
            ptx::tc_fence_after_sync();
            for (int kb = 0; kb < KB && ok; ++kb, ++it) {
                const uint32_t s = it % C::STAGES, use = it / C::STAGES;
                ok = wait(&misc->full[s], use & 1);
                if (!ok) break;
                ptx::tc_fence_after_sync();
                if (elect_one()) {
                    const uint32_t a = base + s * C::STAGE, b = a + 128 * 128;
#pragma unroll
                    for (int ks = 0; ks < 4; ++ks)
                        umma_i8<P>(acc, ptx::umma_smem_desc_sw128(a + ks * 32), ptx::umma_smem_desc_sw128(b + ks * 32), idesc, (kb > 0 || ks > 0) ? 1u : 0u);
                    if constexpr (P == 2) ptx::umma_commit_pair(ptx::smem_u32(&misc->empty[s]));
                    else ptx::umma_commit(ptx::smem_u32(&misc->empty[s]));
                    if (kb == KB - 1) {
                        if constexpr (P == 2) ptx::umma_commit_pair(ptx::smem_u32(&misc->acc_full[buf]));
                        else ptx::umma_commit(ptx::smem_u32(&misc->acc_full[buf]));
                    }
                }
                __syncwarp();
            }
        }
    } else if (warp >= kLinEpiWarp0) {
        // Rows of this warp's quarter and every other 128 bytes of columns, through shared memory, so that stores write whole lines.
        constexpr int COLS = 128 / (int)sizeof(T), STEPS = BN / (2 * COLS) > 0 ? BN / (2 * COLS) : 1, PER = 16 / (int)sizeof(T);
        const int quarter = warp & 3, half = (warp - kLinEpiWarp0) >> 2;
        const uint32_t own = C::STAGES * C::STAGE + (base - raw_addr) + (warp - kLinEpiWarp0) * C::EPI;
        const uint32_t stg = raw_addr + own;
        float* s_scale = reinterpret_cast<float*>(smem_raw + C::STAGES * C::STAGE + (base - raw_addr) + kLinEpiWarps * C::EPI + (warp - kLinEpiWarp0) * C::SCALES);
        // ([STEPS * COLS] scales, then biases)
        float* s_bias = s_scale + STEPS * COLS;
        bool ok = true;
        uint32_t n = 0;
        const bool whole = N % PER == 0;                                      // rows of Y start on 16 bytes
        // scales and biases of the next tile, asked for while this one is worked on
        constexpr int AHEAD = STEPS * COLS / 32;
        float next_scale[AHEAD], next_bias[AHEAD], next_sx = 0.0f;
        auto ask = [&](long long tile) {
            const int m = (int)(tile / n_tiles) * 128 * P + rank * 128 + quarter * 32 + lane, n0 = (int)(tile % n_tiles) * BN;
            next_sx = tile < tiles && m < M ? xs[m] : 0.0f;
#pragma unroll
            for (int x = 0; x < AHEAD; ++x) {
                const int e = x * 32 + lane, col = n0 + (e / COLS * 2 + half) * COLS + e % COLS;
                const bool in = tile < tiles && col < N;
                next_scale[x] = in ? ws[col] : 0.0f;
                next_bias[x] = in && bias != nullptr ? bias[col] : 0.0f;
            }
        };
        ask(tile0);
        for (long long tile = tile0; tile < tiles && ok; tile += tile_step, ++n) {
            const uint32_t buf = n & 1, acc = tmem + buf * BN + ((uint32_t)(quarter * 32) << 16);
            const int m0 = (int)(tile / n_tiles) * 128 * P + rank * 128 + quarter * 32, n0 = (int)(tile % n_tiles) * BN;
            const float sx = next_sx;
#pragma unroll
            for (int x = 0; x < AHEAD; ++x) {
                s_scale[x * 32 + lane] = next_scale[x];
                s_bias[x * 32 + lane] = next_bias[x];
            }
            __syncwarp();
            ask(tile + tile_step);
            ok = warp_wait(&misc->acc_full[buf], (n >> 1) & 1, abort_flag);
            if (!ok) break;
            ptx::tc_fence_after_sync();
#pragma unroll 1
            for (int step = 0; step < STEPS; ++step) {
                const int c0 = (step * 2 + half) * COLS;
                if (c0 >= BN || n0 + c0 >= N) break;
                uint32_t r[COLS / 32][32];
#pragma unroll
                for (int h = 0; h < COLS / 32; ++h) ptx::tmem_ld_32x32(acc + c0 + h * 32, r[h]);
                ptx::tmem_ld_wait();
                if (whole) {                       // the copy of the last 128 bytes has read them
                    asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
                    __syncwarp();
                }
                const float4* sc4 = reinterpret_cast<const float4*>(s_scale + step * COLS);
                const float4* bi4 = reinterpret_cast<const float4*>(s_bias + step * COLS);
                const uint64_t sx2 = pair_f32(sx, sx);
#pragma unroll
                for (int i = 0; i < COLS; i += PER) {
                    float y[PER];
#pragma unroll
                    for (int x = 0; x < PER; x += 4) {
                        const float4 f = sc4[(i + x) / 4], c = bi4[(i + x) / 4];
                        const uint32_t* q = &r[(i + x) / 32][(i + x) % 32];
                        const uint64_t lo = mul_pair(pair_f32((float)(int32_t)q[0], (float)(int32_t)q[1]), sx2);
                        const uint64_t hi = mul_pair(pair_f32((float)(int32_t)q[2], (float)(int32_t)q[3]), sx2);
                        const float2 u = pair_of(fma_pair(lo, pair_f32(f.x, f.y), pair_f32(c.x, c.y))), v = pair_of(fma_pair(hi, pair_f32(f.z, f.w), pair_f32(c.z, c.w)));
                        y[x] = u.x;
                        y[x + 1] = u.y;
                        y[x + 2] = v.x;
                        y[x + 3] = v.y;
                    }
                    uint32_t w[4];
                    if constexpr (sizeof(T) == 4) {
#pragma unroll
                        for (int x = 0; x < 4; ++x) w[x] = __float_as_uint(y[x]);
                    } else {
#pragma unroll
                        for (int x = 0; x < 4; ++x) {
                            if constexpr (std::is_same_v<T, __half>) asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(w[x]) : "f"(y[2 * x + 1]), "f"(y[2 * x]));
                            else asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w[x]) : "f"(y[2 * x + 1]), "f"(y[2 * x]));
                        }
                    }
                    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(stg + lane * 128 + (((i / PER) ^ (lane & 7)) << 4)), "r"(w[0]), "r"(w[1]), "r"(w[2]),
                                 "r"(w[3])
                                 : "memory");
                }
                if (whole) ptx::fence_proxy_async_smem();
                __syncwarp();
                if (whole) {
                    if (m0 < M && elect_one()) tma_store_2d(&tm_y, n0 + c0, m0, stg);
                } else {
                    // rows that start anywhere: neighbouring lanes store neighbouring elements
                    const T* line = reinterpret_cast<const T*>(smem_raw + own);
#pragma unroll 4
                    for (int row = 0; row < 32 && m0 + row < M; ++row) {
#pragma unroll
                        for (int h = 0; h < COLS / 32; ++h) {
                            const int e = h * 32 + lane, col = n0 + c0 + e;
                            const T v = line[row * COLS + ((e / PER) ^ (row & 7)) * PER + e % PER];
                            if (col < N) Y[(size_t)(m0 + row) * N + col] = v;
                        }
                    }
                }
                __syncwarp();
            }
            ptx::tc_fence_before_sync();
            __syncwarp();
            if (lane == 0) {
                const uint32_t bar = ptx::smem_u32(&misc->acc_empty[buf]);
                if constexpr (P == 2) ptx::mbar_arrive_cluster(ptx::cluster_addr(bar, 0));
                else ptx::mbar_arrive(bar);
            }
        }
    }
    asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");      // this thread's stores to Y
    if constexpr (P == 2) {
        __syncwarp();
        ptx::cluster_sync();                    // the pair's UMMAs read both CTAs' shared memory, its barriers hear from both
    }
    tc_cta_teardown<P>(abort_flag, status, tmem, C::TMEM);
}

template <typename T, int P, int BN>
int launch_tc(sentry_ctx* ctx, const LinearArgs& a, cudaStream_t st) {
    using C = LinCfg<P, BN>;
    CUtensorMap mx, mw, my = {};
    if (!make_map_i8(&mx, a.X, a.d.M, a.d.K, 128) || !make_map_i8(&mw, a.W, a.d.N, a.d.K, C::B_ROWS)) return SENTRY_ERR_CUDA;
    if (a.d.N % (16 / (int)sizeof(T)) == 0 && !make_map_out<T>(&my, a.Y, a.d.M, a.d.N)) return SENTRY_ERR_CUDA;
    const long long tiles = linear_tiles(a.d.M, 128 * P) * linear_tiles(a.d.N, BN), most = ctx->sm_count / P;
    auto k = linear_i8_tc_kernel<T, P, BN>;
    static std::atomic<unsigned long long> allowed{0};
    SENTRY_CUDA_TRY(allow_smem(k, C::SMEM, ctx->device, allowed));
    LaunchScope ls(ctx, KS_LINEAR, st);
    SENTRY_CUDA_TRY(launch_chained_clusters(P, k, dim3((unsigned)((tiles < most ? tiles : most) * P)), dim3(kLinThreads), C::SMEM, st, mx, mw, my, a.xs, a.ws, a.bias,
                                            (T*)a.Y, a.d.M, a.d.K, a.d.N, a.status));
    return SENTRY_OK;
}

template <typename T>
int launch_linear(sentry_ctx* ctx, const LinearArgs& a, cudaStream_t st) {
    if (a.d.M <= 64) return launch_few<T>(ctx, a, st);
    // pairs where their tiles fill the GPU; else narrower tiles, so that more SMs have one
    auto tiles = [&](int m, int n) { return linear_tiles(a.d.M, m) * linear_tiles(a.d.N, n); };
    if (2 * tiles(256, 256) >= ctx->sm_count) return launch_tc<T, 2, 256>(ctx, a, st);
    return 2 * tiles(128, 128) >= ctx->sm_count ? launch_tc<T, 1, 128>(ctx, a, st) : launch_tc<T, 1, 64>(ctx, a, st);
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
