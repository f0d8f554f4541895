// Attention of many rows on the 5th-generation tensor cores (16-bit rows; dense 16-bit keys, or the 8-bit cache).
//
// The rows of a KV group (kept heads x Tq) are packed; a CTA takes two tiles of 128 of them and walks the present keys, KN at a time:
//   S_t = Q_t K^T        tcgen05, both operands in shared memory (128-byte rows, swizzled), S in tensor memory
//   P_t = 2^(S c - m c)  a thread is a row: it reads its scores, keeps its running maximum and sum, and writes the weights in 16 bits over
//                        the scores that it has read
//   O_t += P_t V         tcgen05, P from tensor memory, V as it lies in memory (MN-major)
// Two tiles, so that the tensor core works for one while the other's rows are exponentiated.  The accumulator follows the running maximum
// only where it grew by more than 2^8 (bf16 weights) or 2^4 (fp16): until then weights are that much larger than 1, for which there is
// range, and almost no iteration touches O.
//
// Bound by the exponentials (16 a clock and SM) up to d 64, by those and the products together at d 128.  Up to d 64 a step is of 64 keys and
// an SM holds two CTAs, four tiles that wait for one another's latencies (4 x 4096 rows on 8192 keys, 16 heads on 4, d 64, bf16: 830 us, against
// 910 with one CTA and 128 keys; 32 samples of 211 rows on 648 keys, 7 of 12 heads on 4: 28 us against 32); at d 128 tensor memory has room for
// one, whose steps are of 128 keys (the same rows at d 128: 917 us in a burst, 1.2 PFLOP/s; 1050 under the power limit).  On dense keys registers hold all
// but the last 32 scores of a step from the maximum to the weights: those are read twice (none of them at d 128: 945 us, with spills).
// Dense K and V come by TMA where the present keys of a step follow one another, and row by row (16-byte asynchronous copies, zeros for what is not there)
// where they do not: the last tile of a sample, and tiles across the border of a missing modality.
// A cache's codes are made fp16 by the loading warps, exactly; Q and the weights meet them as fp16.  A page's key scale multiplies its scores, and the
// logarithm of its value scale is added to them, so that the weights carry it and O needs no unit of its own; the sum takes it out again.
// (A step of two tiles of 128 rows on 128 codes, d 128: some 6000 cycles, against 3900 on dense keys: the loading warps' conversions and the softmax's, which at 13
// warps has 128 registers a thread, keeps no scores and runs 32 of them at a time through one loop.  2048 rows of 8 groups on 8192 tokens: 142 us; with the loop
// unrolled and 64 scores kept 148; before that, three loading warps and 168 registers 183, five 159, seven 160, four whose rows lie a multiple of 16 apart 148.)
// Every wait is bounded; on expiry the CTA raises SENTRY_STATUS_BIT_TIMEOUT and unwinds.
#include "kv_attend.cuh"
#include "kv_maps.cuh"

namespace {

constexpr int kTM = 128;                     // rows of a tile
constexpr float kTcLog2e = 1.4426950408889634f;
constexpr int kTcListed = 4096;              // keys whose list of present ones a CTA makes for itself

__device__ __forceinline__ float max3_nan(float a, float b, float c) {     // not a number if one of them is none
    float r;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}

template <int D, bool CODES>
struct TcCfg {
    static constexpr int KN = D <= 64 ? 64 : 128;            // keys of a step
    static constexpr int CTAS = KN == 64 ? 2 : 1;            // of an SM
    // after the four softmax warps of each tile; then one issuer.  (Who makes 16 bits of codes has more to do than who waits for copies.)
    static constexpr int LOAD_WARPS = CODES ? (KN == 64 ? 2 : 4) : KN == 64 ? 1 : 3;
    static constexpr int LOAD_WARP0 = 8, ISSUE_WARP = LOAD_WARP0 + LOAD_WARPS, THREADS = (ISSUE_WARP + 1) * 32;
    static constexpr int TMEM = 512 / CTAS, O_COL = 2 * KN;  // tensor memory: S of both tiles, then O of both
    static constexpr int RB = D >= 64 ? 128 : D * 2;         // bytes of a shared-memory row (64 elements at most)
    static constexpr int SLABS = D * 2 / RB;                 // column slabs of a tile
    static constexpr int SLAB = kTM * RB, TILE = SLABS * SLAB;         // of Q: 128 rows of D elements
    static constexpr int KSLAB = KN * RB, KTILE = SLABS * KSLAB;       // of K and V
    static constexpr int STAGES = D == 128 ? 2 : 4;          // of K, and of V
    static constexpr int HELD = CODES ? 0 : KN == 64 ? 1 : 3;   // blocks of 32 scores that a thread keeps from the maximum to the weights
    static constexpr int META = 2 * STAGES;                  // steps whose pages' scales are kept: what a reader of one needs lies at most STAGES ahead
    static constexpr int SMEM = 2 * TILE + 2 * STAGES * KTILE + 1024;
    static_assert(O_COL + 2 * D <= TMEM && (KN == 128 || SLABS == 1), "tensor memory, and slabs of 128 rows");
};
struct TcMisc {
    uint64_t k_full[4], k_empty[4], v_full[4], v_empty[4];
    uint64_t s_full[2], p_full[2], o_full[2], meta_full[8];
    uint32_t tmem_base;
    int abort_flag;
    int n_heads;
    short head[kServeMaxHeads], pos[kServeMaxHeads];
    int red[66];
    union {
        uint16_t list[kTcListed];
        struct {                            // of a cache
            float4 meta[8][8];              // of every 16 keys of a step: key scale, log2 of the value scale in units of vref, its inverse, -
            unsigned holes[8];              // which of them are not there
            float q_scale[2 * kTM];
            unsigned top[16];
        } c;
    };
};

// 16-byte piece c of row r in a tile of rows of RB bytes, swizzled in that row width's mode
template <int RB>
__device__ __forceinline__ uint32_t tile_offset(int r, int c) {
    constexpr int PER = RB / 16;                   // pieces of a row
    const int f = RB == 128 ? r & 7 : RB == 64 ? (r >> 1) & 3 : (r >> 2) & 1;
    return (uint32_t)((c / PER) * (128 * RB) + r * RB + (((c % PER) ^ f) << 4));
}

template <int D, bool BF16, int FMT>
__global__ void __launch_bounds__(TcCfg<D, FMT != 0>::THREADS, TcCfg<D, FMT != 0>::CTAS)
kv_tc_kernel(const __grid_constant__ KvMaps maps, const KvAttendArgs a, const int32_t* __restrict__ list, const int32_t* __restrict__ counts,
             float* __restrict__ part, float2* __restrict__ ml, int n_splits) {
    constexpr bool CODES = FMT != 0, I8 = FMT == SENTRY_I8;
    using C = TcCfg<D, CODES>;
    constexpr int KN = C::KN;
    constexpr bool OP_BF16 = BF16 && !CODES;          // operands of the products: codes are fp16 exactly, and Q and the weights meet them as fp16
    extern __shared__ uint8_t smem_raw[];
    __shared__ TcMisc misc_s;
    TcMisc* misc = &misc_s;
    volatile int* abort_flag = &misc->abort_flag;
    const uint32_t q_smem = (ptx::smem_u32(smem_raw) + 1023u) & ~1023u;
    const uint32_t k_smem = q_smem + 2 * C::TILE, v_smem = k_smem + C::STAGES * C::KTILE;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int split = blockIdx.x % n_splits, bg = blockIdx.x / n_splits, b = bg / a.Hk, g = bg % a.Hk;
    if (threadIdx.x == 0) {
        for (int s = 0; s < C::STAGES; ++s) {
            ptx::mbar_init(ptx::smem_u32(&misc->k_full[s]), C::LOAD_WARPS);
            ptx::mbar_init(ptx::smem_u32(&misc->k_empty[s]), 1);
            ptx::mbar_init(ptx::smem_u32(&misc->v_full[s]), C::LOAD_WARPS);
            ptx::mbar_init(ptx::smem_u32(&misc->v_empty[s]), 1);
        }
        for (int t = 0; t < 2; ++t) {
            ptx::mbar_init(ptx::smem_u32(&misc->s_full[t]), 1);
            ptx::mbar_init(ptx::smem_u32(&misc->p_full[t]), 4);
            ptx::mbar_init(ptx::smem_u32(&misc->o_full[t]), 1);
        }
        if (CODES)
            for (int m = 0; m < C::META; ++m) ptx::mbar_init(ptx::smem_u32(&misc->meta_full[m]), 1);
        misc->abort_flag = 0;
        ptx::fence_barrier_init();
        if (!CODES) {
            ptx::prefetch_tensormap(&maps.k);
            ptx::prefetch_tensormap(&maps.v);
        }
    }
    grid_dependency_wait();
    if (warp == 0) {
        const int n = kv_group_heads(a, b, g, g == 0 && split == 0 && blockIdx.y == 0, misc->head, misc->pos);
        if (lane == 0) misc->n_heads = n;
    }
    __syncthreads();
    const int rows = misc->n_heads * a.Tq;
    if ((int)blockIdx.y * 2 * kTM >= rows) return;
    if (warp == C::ISSUE_WARP) {
        ptx::tmem_alloc(ptx::smem_u32(&misc->tmem_base), C::TMEM);
        ptx::tmem_relinquish();
    }
    ptx::tc_fence_before_sync();
    __syncthreads();
    ptx::tc_fence_after_sync();
    const uint32_t tmem = misc->tmem_base;

    // Q of a row block, by all threads
    auto load_q = [&](int row0) {
        const int halves = rows - row0 > kTM ? 2 : 1;
        if constexpr (CODES && BF16) {
            // as fp16, a row to a warp, four on the way at once: scaled by a power of two so that the largest value lies in [1,2)
            constexpr int W = (D + 63) / 64, STEP = C::THREADS / 32;
            for (int r0 = warp; r0 < halves * kTM; r0 += 4 * STEP) {
                uint32_t w[4][W];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int row = row0 + r0 + i * STEP;
                    const bool in = row < rows && r0 + i * STEP < halves * kTM;
                    const uint32_t* src = in ? (const uint32_t*)((const uint16_t*)a.Q + b * a.qs[0] + misc->head[row / a.Tq] * a.qs[1] + row % a.Tq * a.qs[2]) : nullptr;
#pragma unroll
                    for (int x = 0; x < W; ++x) w[i][x] = in && x * 32 + lane < D / 2 ? src[x * 32 + lane] : 0u;
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int r = r0 + i * STEP;
                    if (r >= halves * kTM) break;
                    uint32_t top = 0u;
#pragma unroll
                    for (int x = 0; x < W; ++x) top = max(top, max(w[i][x] & 0x7fffu, w[i][x] >> 16 & 0x7fffu));
                    top = __reduce_max_sync(0xffffffffu, top);
                    const int e = min(max((int)(top >> 7) - 127, -120), 120);       // (what is no number stays none)
                    const float down = __uint_as_float((uint32_t)(127 - e) << 23);
#pragma unroll
                    for (int x = 0; x < W; ++x) {
                        const int at = x * 32 + lane;
                        if (at < D / 2)
                            asm volatile("st.shared.b32 [%0], %1;" ::"r"(q_smem + (r >> 7) * C::TILE + tile_offset<C::RB>(r & 127, at >> 2) + (at & 3) * 4),
                                         "r"(pack2<false>(__uint_as_float(w[i][x] << 16) * down, __uint_as_float(w[i][x] & 0xffff0000u) * down))
                                         : "memory");
                    }
                    if (lane == 0) misc->c.q_scale[r] = __uint_as_float((uint32_t)(127 + e) << 23);
                }
            }
        } else {
        for (int e = threadIdx.x; e < halves * kTM * (D / 8); e += C::THREADS) {
            const int r = e / (D / 8), c = e % (D / 8), row = row0 + r;
            const uint32_t dst = q_smem + (r >> 7) * C::TILE + tile_offset<C::RB>(r & 127, c);
            if (row < rows) {
                const long long src = b * a.qs[0] + misc->head[row / a.Tq] * a.qs[1] + row % a.Tq * a.qs[2] + c * 8;
                ptx::cp_async_16(dst, (const uint16_t*)a.Q + src);
            } else {
                asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(dst), "r"(0) : "memory");
            }
        }
        ptx::cp_async_commit();
        }
    };
    load_q(blockIdx.y * 2 * kTM);                 // (on its way while the list is made)
    // present keys of the sample, in order: the first `count`, those of this CTA's list, or of one that was made before
    const bool own = a.ids != nullptr && a.Tk <= kTcListed;
    int count;
    if (own) count = block_build_valid(a.ids, kv_length(a, b), a.masks[b], misc->list, misc->red);
    else count = list ? counts[b] : kv_length(a, b);
    const int32_t* far = list ? list + (size_t)b * a.Tk : nullptr;
    auto key_at = [&](int p) { return own ? (int)misc->list[p] : far ? far[p] : p; };
    const int tiles = (count + KN - 1) / KN, per_split = (tiles + n_splits - 1) / n_splits;
    const int t0 = min(split * per_split, tiles), t1 = min(t0 + per_split, tiles);
    // A page's value scale goes into its keys' exponents, so that O needs no unit that follows the pages: in units of the largest one of this
    // CTA's pages (vref).  (2^-100 of it and less leaves zeros of the page's values.)
    float vref = 1.0f;
    const int page_shift = CODES ? 31 - __clz(a.page) : 0;
    if constexpr (CODES) {
        uint32_t top = 0u;
        const int32_t* pages = a.table + (size_t)b * a.max_pages;
#pragma unroll 4
        for (int p = (t0 * KN >> page_shift) + (int)threadIdx.x; p < a.max_pages && p << page_shift < min(t1 * KN, count); p += C::THREADS) {
            const int id = pages[p];
            if ((unsigned)id >= (unsigned)a.n_pages) continue;
            const uint32_t v = __float_as_uint(a.v_scales[(size_t)id * a.Hk + g]) & 0x7fffffffu;
            if (v < 0x7f800000u) top = max(top, v);
        }
        top = __reduce_max_sync(0xffffffffu, top);
        if (lane == 0) misc->c.top[warp] = top;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < C::THREADS / 32; ++w) top = max(top, misc->c.top[w]);
        vref = top == 0u ? 1.0f : fmaxf(__uint_as_float(top), 7.5231638e-37f);     // (2^-120)
    }
    uint32_t done = 0;                            // steps of the row blocks before
    int steps = 0;

    for (int rb = blockIdx.y; rb * 2 * kTM < rows; rb += gridDim.y, done += (uint32_t)steps) {
        const int row0 = rb * 2 * kTM;
        const int halves = rows - row0 > kTM ? 2 : 1;
        steps = t1 - t0;
        if (CODES && a.causal) {                  // no row of these sees more
            const int end = min(row0 + 2 * kTM, rows) - 1, i = end / a.Tq != row0 / a.Tq ? a.Tq - 1 : end % a.Tq, seen = max(count - a.Tq + i + 1, 0);
            steps = max(min(t1, (seen + KN - 1) / KN) - t0, 0);
        }
        if (rb != (int)blockIdx.y) load_q(row0);
        ptx::cp_async_wait_all();
        ptx::fence_proxy_async_smem();
        __syncthreads();
        if (warp >= C::LOAD_WARP0 && warp < C::LOAD_WARP0 + C::LOAD_WARPS) {
            // ---------------------------------------------------------------- K and V
            const int lw = warp - C::LOAD_WARP0;
            const int kb = a.ks[0] ? b : 0, kg = a.ks[1] ? g : 0, vb = a.vs[0] ? b : 0, vg = a.vs[1] ? g : 0;
            bool ok = true;
            if constexpr (CODES) {
                // 16 codes a lane at a time, as fp16; zeros for keys that are not there.  K's and V's codes of the next step are on their way to
                // registers while this one's are converted, and its pages' numbers a step before those.
                // A lane's rows lie a multiple of 16 apart, so that their places in a page, in the tile and in its swizzle differ by constants.
                constexpr int PER = D / 16, ROWS = C::LOAD_WARPS * 32 / PER, IT = (KN + ROWS - 1) / ROWS;
                static_assert(ROWS % 16 == 0 && ROWS <= KN, "rows of a lane");
                const int first = (lw * 32 + lane) / PER, c = (lw * 32 + lane) % PER;          // this lane's rows: first + i ROWS
                const uint32_t to0 = tile_offset<C::RB>(first, 2 * c), to1 = tile_offset<C::RB>(first, 2 * c + 1);
                const uint32_t lane_at = (first & 15) * D + c * 16;
                const int32_t* pages = a.table + (size_t)b * a.max_pages;
                const float inv_vref = 1.0f / vref;
                auto page_of = [&](int j) {                 // of 16 keys of a step, a lane each
                    const int p = (t0 + j) * KN + lane * 16;
                    const int id = j < steps && lane < KN / 16 && p < count ? pages[p >> page_shift] : -1;
                    if (id != -1 && (unsigned)id >= (unsigned)a.n_pages) return -2;      // (an entry that is needed, and no page; -1 counts below)
                    return id;
                };
                struct Step { int id; float ks, vs; };
                auto of_page = [&](int id) {
                    Step x = {id, 0.0f, 0.0f};
                    if (id >= 0) { x.ks = a.k_scales[(size_t)id * a.Hk + g]; x.vs = a.v_scales[(size_t)id * a.Hk + g]; }
                    return x;
                };
                auto fetch = [&](uint4 (&v)[IT], const void* codes, int j, int id) {
                    const int p0 = (t0 + j) * KN;
                    // (rows of the pool: below 2^31)
                    const int row = id < 0 ? -1 : (id * a.Hk + g) * a.page + ((p0 + lane * 16) & (a.page - 1));
#pragma unroll
                    for (int i = 0; i < IT; ++i) {
                        const int r = first + i * ROWS, at = __shfl_sync(0xffffffffu, row, r >> 4);
                        v[i] = at >= 0 && p0 + r < count ? *reinterpret_cast<const uint4*>((const uint8_t*)codes + (size_t)at * D + lane_at) : make_uint4(0, 0, 0, 0);
                    }
                };
                // sign: of the values of 16 keys, a lane each; -1: all are zero
                auto convert = [&](const uint4 (&v)[IT], uint32_t dst, int sign) {
                    const bool signs = __any_sync(0xffffffffu, sign != 0);
#pragma unroll
                    for (int i = 0; i < IT; ++i) {
                        const uint32_t w[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
                        uint32_t f[8];
#pragma unroll
                        for (int x = 0; x < 4; ++x) codes_to_f16<I8>(w[x], f[2 * x], f[2 * x + 1]);
                        if (signs) {
                            const int how = __shfl_sync(0xffffffffu, sign, (first + i * ROWS) >> 4);
#pragma unroll
                            for (int x = 0; x < 8; ++x) f[x] = how < 0 ? 0u : f[x] ^ (how > 0 ? 0x80008000u : 0u);
                        }
                        const uint32_t at = dst + i * ROWS * C::RB;
                        // (two lanes of eight write to the second slab: in the other order, which keeps their banks apart)
                        const bool turned = C::SLABS == 2 && c >= PER / 2;
#pragma unroll
                        for (int x = 0; x < 2; ++x) {
                            const bool hi = (x == 1) != turned;
                            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at + (hi ? to1 : to0)), "r"(hi ? f[4] : f[0]), "r"(hi ? f[5] : f[1]), "r"(hi ? f[6] : f[2]),
                                         "r"(hi ? f[7] : f[3])
                                         : "memory");
                        }
                    }
                    ptx::fence_proxy_async_smem();
                };
                uint4 kv[IT], vv[IT];
                Step now = of_page(page_of(0));
                int next = page_of(1);
                fetch(kv, a.K, 0, now.id);
                fetch(vv, a.V, 0, now.id);
                for (int j = 0; j < steps && ok; ++j) {
                    const uint32_t n = done + j, s = n % C::STAGES, use = n / C::STAGES, slot = n % C::META;
                    const int p = (t0 + j) * KN + lane * 16;
                    if (lw == 0 && lane < KN / 16 && p < count && now.id < 0) atomicOr(a.status, SENTRY_STATUS_BIT_BAD_INDEX);
                    const unsigned holes = __ballot_sync(0xffffffffu, now.id < 0);
                    const Step then = of_page(next);
                    next = page_of(j + 2);
                    ok = warp_wait(&misc->k_empty[s], (use & 1) ^ 1, abort_flag);
                    if (!ok) break;
                    if (lw == 0) {
                        if (lane < KN / 16) {
                            const float ratio = fabsf(now.vs) <= 3.4028234e38f ? fmaxf(fabsf(now.vs) * inv_vref, 7.8886091e-31f) : __int_as_float(0x7fc00000);    // (2^-100)
                            misc->c.meta[slot][lane] = make_float4(now.ks, log2f(ratio), 1.0f / ratio, 0.0f);
                        }
                        if (lane == 0) misc->c.holes[slot] = holes;
                        warp_arrive(&misc->meta_full[slot]);
                    }
                    convert(kv, k_smem + s * C::KTILE, 0);
                    warp_arrive(&misc->k_full[s]);
                    fetch(kv, a.K, j + 1, then.id);
                    ok = warp_wait(&misc->v_empty[s], (use & 1) ^ 1, abort_flag);
                    if (!ok) break;
                    convert(vv, v_smem + s * C::KTILE, now.id < 0 ? 0 : fabsf(now.vs) * inv_vref <= 7.8886091e-31f ? -1 : now.vs < 0.0f);
                    warp_arrive(&misc->v_full[s]);
                    fetch(vv, a.V, j + 1, then.id);
                    now = then;
                }
            } else {
            // A tile that is gathered counts as here STAGES tiles (of K and V in turn) later, so that as many are on their way; what
            // the tiles' users wait for meanwhile lies before those.
            uint32_t gathered = 0;
            auto arrive = [&](int i) {                      // (i: tiles of K and V in turn)
                const uint32_t n = done + (i >> 1), s = n % C::STAGES;
                ptx::fence_proxy_async_smem();
                warp_arrive(i & 1 ? &misc->v_full[s] : &misc->k_full[s]);
            };
            for (int j = 0; j < steps && ok; ++j) {
                const uint32_t n = done + j, s = n % C::STAGES, use = n / C::STAGES;
                const int p0 = (t0 + j) * KN;
                const bool full = p0 + KN <= count;
                const int first = key_at(p0);
                const bool together = full && key_at(p0 + KN - 1) - first == KN - 1;
#pragma unroll 1
                for (int is_v = 0; is_v < 2 && ok; ++is_v) {
                    uint64_t* full_bar = is_v ? &misc->v_full[s] : &misc->k_full[s];
                    ok = warp_wait(is_v ? &misc->v_empty[s] : &misc->k_empty[s], (use & 1) ^ 1, abort_flag);
                    if (!ok) break;
                    const uint32_t dst = (is_v ? v_smem : k_smem) + s * C::KTILE;
                    if (together) {
                        if (lw == 0) {
                            if (elect_one()) {
                                const uint32_t bar = ptx::smem_u32(full_bar);
                                ptx::mbar_arrive_expect_tx(bar, C::KTILE);
#pragma unroll
                                for (int c = 0; c < C::SLABS; ++c)
                                    tma_load_4d(dst + c * C::KSLAB, is_v ? &maps.v : &maps.k, c * 64, first, is_v ? vg : kg, is_v ? vb : kb, bar);
                            }
                            __syncwarp();
                        } else {
                            warp_arrive(full_bar);
                        }
                    } else {
                        const long long* st = is_v ? a.vs : a.ks;
                        const uint16_t* src = (const uint16_t*)(is_v ? a.V : a.K) + b * st[0] + g * st[1];
                        for (int e = lw * 32 + lane; e < KN * (D / 8); e += C::LOAD_WARPS * 32) {
                            const int r = e / (D / 8), c = e % (D / 8);
                            const uint32_t to = dst + tile_offset<C::RB>(r, c);
                            if (p0 + r < count) ptx::cp_async_16(to, src + key_at(p0 + r) * st[2] + c * 8);
                            else asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(to), "r"(0) : "memory");
                        }
                    }
                    ptx::cp_async_commit();
                    gathered = gathered << 1 | !together;
                    if (gathered >> C::STAGES & 1u) {
                        ptx::cp_async_wait_group<C::STAGES>();
                        arrive(2 * j + is_v - C::STAGES);
                    }
                }
            }
            ptx::cp_async_wait_all();
            if (ok)
                for (int back = C::STAGES - 1; back >= 0; --back)
                    if (gathered >> back & 1u) arrive(2 * steps - 1 - back);
            }
        } else if (warp == C::ISSUE_WARP) {
            // ---------------------------------------------------------------- UMMAs
            constexpr uint32_t qk = OP_BF16 ? ptx::umma_idesc_bf16(kTM, KN) : ptx::umma_idesc_f16(kTM, KN);
            constexpr uint32_t pv = OP_BF16 ? ptx::umma_idesc_bf16_major(kTM, D, false, true) : ptx::umma_idesc_f16_major(kTM, D, false, true);
            bool ok = true;
            auto scores = [&](int t, uint32_t s) {
#pragma unroll
                for (int k = 0; k < D / 16; ++k) {
                    const uint32_t slab = k * 32 / C::RB, off = k * 32 % C::RB;
                    ptx::umma_bf16(tmem + t * KN, ptx::umma_smem_desc_rows(q_smem + t * C::TILE + slab * C::SLAB + off, C::RB),
                                   ptx::umma_smem_desc_rows(k_smem + s * C::KTILE + slab * C::KSLAB + off, C::RB), qk, k > 0 ? 1u : 0u);
                }
                ptx::umma_commit(ptx::smem_u32(&misc->s_full[t]));
            };
            if (steps > 0) {
                const uint32_t s = done % C::STAGES, use = done / C::STAGES;
                ok = warp_wait(&misc->k_full[s], use & 1, abort_flag);
                if (ok) {
                    ptx::tc_fence_after_sync();
                    if (elect_one()) {
                        for (int t = 0; t < halves; ++t) scores(t, s);
                        ptx::umma_commit(ptx::smem_u32(&misc->k_empty[s]));
                    }
                    __syncwarp();
                }
            }
            for (int j = 0; j < steps && ok; ++j) {
                const uint32_t n = done + j, s = n % C::STAGES, use = n / C::STAGES;
                const uint32_t s2 = (n + 1) % C::STAGES, use2 = (n + 1) / C::STAGES;
                const bool more = j + 1 < steps;
                ok = warp_wait(&misc->v_full[s], use & 1, abort_flag);
                for (int t = 0; t < halves && ok; ++t) {
                    ok = warp_wait(&misc->p_full[t], n & 1, abort_flag);
                    if (ok && more && t == 0) ok = warp_wait(&misc->k_full[s2], use2 & 1, abort_flag);
                    if (!ok) break;
                    ptx::tc_fence_after_sync();
                    if (elect_one()) {
#pragma unroll
                        for (int k = 0; k < KN / 16; ++k)
                            ptx::umma_bf16_tmem_a(tmem + C::O_COL + t * D, tmem + t * KN + k * 8,
                                                  ptx::umma_smem_desc_rows(v_smem + s * C::KTILE + k * 16 * C::RB, C::RB, C::KSLAB), pv, (j > 0 || k > 0) ? 1u : 0u);
                        ptx::umma_commit(ptx::smem_u32(&misc->o_full[t]));
                        if (t == halves - 1) ptx::umma_commit(ptx::smem_u32(&misc->v_empty[s]));
                        if (more) {
                            scores(t, s2);
                            if (t == halves - 1) ptx::umma_commit(ptx::smem_u32(&misc->k_empty[s2]));
                        }
                    }
                    __syncwarp();
                }
            }
        } else if (warp < C::LOAD_WARP0) {
            // ---------------------------------------------------------------- softmax: a thread is a row
            const int t = warp >> 2;
            const int row = row0 + t * kTM + (warp & 3) * 32 + lane;
            const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
            const uint32_t sc = tmem + t * KN + lanes, oc = tmem + C::O_COL + t * D + lanes;
            const float c = rsqrtf((float)D) * kTcLog2e;
            // what a score is multiplied by on its way to log2; those of a cache have been, with their page's scale and Q's
            const float cm = CODES ? 1.0f : c;
            float cq = c;
            int last = count;                                  // keys that this row sees end here
            if constexpr (CODES) {
                if (BF16) cq *= misc->c.q_scale[t * kTM + (warp & 3) * 32 + lane];
                if (a.causal) last = min(count, count - a.Tq + row % a.Tq + 1);
            }
            // The maximum is followed where a score exceeds it by 2^kLag.  fp16 weights are taken 2^kShift times as large (2^15 at most): its range is
            // what small ones run out of, below 2^-25 of the largest (times its value scale), from where they round to multiples of 2^-35 of that.
            constexpr float kLag = OP_BF16 ? 8.0f : 4.0f, kShift = OP_BF16 ? 0.0f : 11.0f, kUnshift = OP_BF16 ? 1.0f : 1.0f / 2048.0f;
            float m = -INFINITY, l = 0.0f;
            bool ok = true;
            for (int j = 0; j < steps && ok && t < halves; ++j) {
                const uint32_t n = done + j;
                ok = warp_wait(&misc->s_full[t], n & 1, abort_flag);
                if (!ok) break;
                ptx::tc_fence_after_sync();
                const int valid = last - (t0 + j) * KN;
                const uint32_t slot = n % C::META;
                unsigned holes = 0u;
                if constexpr (CODES) {
                    ok = warp_wait(&misc->meta_full[slot], n / C::META & 1, abort_flag);
                    if (!ok) break;
                    holes = misc->c.holes[slot];
                }
                uint32_t s[CODES ? 1 : KN / 32][32];
                auto settle = [&](int z, float add) {              // (add: to what a cache's scores become; dense ones stay as they are)
                    const int at = CODES ? 0 : z;
                    if constexpr (CODES) {
#pragma unroll
                        for (int x = 0; x < 2; ++x) {
                            const float4 page = misc->c.meta[slot][z * 2 + x];
                            const uint64_t f = pair_f32(cq * page.x, cq * page.x), e = pair_f32(page.y + add, page.y + add);
#pragma unroll
                            for (int y = x * 16; y < x * 16 + 16; y += 2) {
                                const float2 u = pair_of(fma_pair(pair_f32(__uint_as_float(s[at][y]), __uint_as_float(s[at][y + 1])), f, e));
                                s[at][y] = __float_as_uint(u.x);
                                s[at][y + 1] = __float_as_uint(u.y);
                            }
                        }
                        if (holes >> (z * 2) & 3u) {
#pragma unroll
                            for (int y = 0; y < 32; ++y)
                                if (holes >> (z * 2 + (y >> 4)) & 1u) s[at][y] = 0xff800000u;
                        }
                    }
                    if (valid < KN) {
#pragma unroll
                        for (int y = 0; y < 32; ++y)
                            if (z * 32 + y >= valid) s[at][y] = 0xff800000u;
                    }
                };
                // (a score that is not a number makes the maximum one, and with it the whole row)
                float top[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
                auto look = [&](int z) {
                    const int at = CODES ? 0 : z;
                    settle(z, 0.0f);
#pragma unroll
                    for (int y = 0; y < 32; y += 2) top[(y >> 1) & 3] = max3_nan(top[(y >> 1) & 3], __uint_as_float(s[at][y]), __uint_as_float(s[at][y + 1]));
                };
                if constexpr (CODES) {              // (one block of scores in registers at a time)
#pragma unroll 1
                    for (int z = 0; z < KN / 32; ++z) {
                        ptx::tmem_ld_32x32(sc + z * 32, s[0]);
                        ptx::tmem_ld_wait();
                        look(z);
                    }
                } else {
#pragma unroll
                    for (int z = 0; z < KN / 32; ++z) ptx::tmem_ld_32x32(sc + z * 32, s[z]);
                    ptx::tmem_ld_wait();
#pragma unroll
                    for (int z = 0; z < KN / 32; ++z) look(z);
                }
                const float now = max3_nan(max3_nan(m, top[0], top[1]), top[2], top[3]);
                if (j == 0) m = now;
                else {
                    const bool grew = !((now - m) * cm <= kLag);
                    if (__any_sync(0xffffffffu, grew)) {
                        // O follows the maximum; the last product into it has to be complete
                        ok = warp_wait(&misc->o_full[t], (n - 1) & 1, abort_flag);
                        if (!ok) break;
                        ptx::tc_fence_after_sync();
                        // (each row for itself: what its neighbours hold changes no bit of it)
                        const float keep = grew && m != now ? exp2_fast((m - now) * cm) : 1.0f;
                        if (grew) m = now;
                        l *= keep;
#pragma unroll
                        for (int z = 0; z < D; z += 16) {
                            uint32_t o[16];
                            ptx::tmem_ld_32x16(oc + z, o);
                            ptx::tmem_ld_wait();
#pragma unroll
                            for (int y = 0; y < 16; ++y) o[y] = __float_as_uint(__uint_as_float(o[y]) * keep);
                            ptx::tmem_st_32x16(oc + z, o);
                        }
                    }
                }
                const float mc = (m == -INFINITY ? 0.0f : m * cm) - kShift;
                const uint64_t cc = pair_f32(cm, cm), mcc = pair_f32(-mc, -mc), one = pair_f32(1.0f, 1.0f);
                uint64_t sum[2] = {pair_f32(0.0f, 0.0f), pair_f32(0.0f, 0.0f)};
#pragma unroll(CODES ? 1 : KN / 32)
                for (int z = 0; z < KN / 32; ++z) {
                    const int at = CODES ? 0 : z;
                    uint32_t w[16];
                    if (z >= C::HELD) {                // (read again: the registers do not hold them all)
                        ptx::tmem_ld_32x32(sc + z * 32, s[at]);
                        ptx::tmem_ld_wait();
                        settle(z, -mc);
                    }
#pragma unroll
                    for (int y = 0; y < 16; ++y) {
                        if constexpr (CODES) {         // a weight counts in the sum without its page's value scale
                            if (y % 8 == 0) sum[0] = sum[1] = pair_f32(0.0f, 0.0f);
                        }
                        uint64_t u2 = pair_f32(__uint_as_float(s[at][2 * y]), __uint_as_float(s[at][2 * y + 1]));
                        if (!CODES) u2 = fma_pair(u2, cc, mcc);
                        const float2 u = pair_of(u2);
                        const float p0 = exp2_fast(u.x), p1 = exp2_fast(u.y);
                        sum[y & 1] = fma_pair(pair_f32(p0, p1), one, sum[y & 1]);
                        w[y] = pack2<OP_BF16>(p0, p1);
                        if constexpr (CODES) {
                            if (y % 8 == 7) {
                                const float2 x0 = pair_of(sum[0]), x1 = pair_of(sum[1]);
                                const float group = (x0.x + x0.y) + (x1.x + x1.y);
                                // (keys that this row does not see add nothing, whatever their page's scale is)
                                l += group != 0.0f ? group * misc->c.meta[slot][z * 2 + (y >> 3)].z : 0.0f;
                            }
                        }
                    }
                    ptx::tmem_st_32x16(sc + z * 16, w);
                }
                const float2 sums[2] = {pair_of(sum[0]), pair_of(sum[1])};
                if (!CODES) l += (sums[0].x + sums[0].y) + (sums[1].x + sums[1].y);
                ptx::tmem_st_wait();
                ptx::tc_fence_before_sync();
                warp_arrive(&misc->p_full[t]);
            }
            // ---------------------------------------------------------------- results
            if (t < halves && steps > 0 && ok) ok = warp_wait(&misc->o_full[t], (done + steps - 1) & 1, abort_flag);
            ptx::tc_fence_after_sync();
            if (t < halves && ok) {
                const bool in = row < rows;
                const size_t each = (size_t)a.k_h * a.Tq, within = in ? (size_t)misc->pos[row / a.Tq] * a.Tq + row % a.Tq : 0;
                const size_t out = b * each + within, pat = ((size_t)b * n_splits + split) * each + within;
                const float inv = l == 0.0f ? 0.0f : vref / l;
                if (n_splits > 1 && in) ml[pat] = steps > 0 ? make_float2(m * cm, l * kUnshift) : make_float2(-INFINITY, 0.0f);
#pragma unroll
                for (int z = 0; z < D; z += 16) {
                    uint32_t o[16];
                    if (steps > 0) {
                        ptx::tmem_ld_32x16(oc + z, o);
                        ptx::tmem_ld_wait();
                    } else {
#pragma unroll
                        for (int y = 0; y < 16; ++y) o[y] = 0u;
                    }
                    if (!in) continue;
                    if (n_splits == 1) {
                        uint32_t w[8];
#pragma unroll
                        for (int y = 0; y < 8; ++y) w[y] = l == 0.0f ? 0u : pack2<BF16>(__uint_as_float(o[2 * y]) * inv, __uint_as_float(o[2 * y + 1]) * inv);
                        uint4* dst = reinterpret_cast<uint4*>((uint16_t*)a.O + out * D + z);
                        dst[0] = make_uint4(w[0], w[1], w[2], w[3]);
                        dst[1] = make_uint4(w[4], w[5], w[6], w[7]);
                    } else if (steps > 0) {
                        uint4* dst = reinterpret_cast<uint4*>(part + pat * D + z);
#pragma unroll
                        for (int y = 0; y < 16; ++y) o[y] = __float_as_uint(__uint_as_float(o[y]) * kUnshift * vref);     // (large values have room)
#pragma unroll
                        for (int y = 0; y < 4; ++y) dst[y] = make_uint4(o[4 * y], o[4 * y + 1], o[4 * y + 2], o[4 * y + 3]);
                    }
                }
            }
            ptx::tc_fence_before_sync();
        }
        __syncthreads();                      // Q and O may be taken over
        ptx::tc_fence_after_sync();
    }
    ptx::tc_fence_before_sync();
    __syncthreads();
    if (*abort_flag) {
        if (threadIdx.x == 0) atomicOr(a.status, SENTRY_STATUS_BIT_TIMEOUT);
        const long long start = clock64();
        while (clock64() - start < 2000000LL) __nanosleep(1000);
        __syncthreads();
    }
    if (warp == C::ISSUE_WARP) {
        ptx::tc_fence_after_sync();
        ptx::tmem_dealloc(tmem, C::TMEM);
    }
}

// The present keys of every sample, in order: a block per sample.
__global__ void __launch_bounds__(1024) kv_plan_kernel(const KvAttendArgs a, int32_t* __restrict__ list, int32_t* __restrict__ counts) {
    __shared__ int s_warp[32];
    const int b = blockIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    grid_dependents_start_if_small();
    grid_dependency_wait();
    const int len = kv_length(a, b);
    const uint32_t mask = a.masks[b];
    int base = 0;
    for (int n0 = 0; n0 < len; n0 += 1024) {
        const int n = n0 + threadIdx.x;
        const bool ok = n < len && kv_present(a.ids[n], mask);
        const unsigned here = __ballot_sync(0xffffffffu, ok);
        __syncthreads();
        if (lane == 0) s_warp[warp] = __popc(here);
        __syncthreads();
        int before = base, all = 0;
        for (int w = 0; w < 32; ++w) { if (w < warp) before += s_warp[w]; all += s_warp[w]; }
        if (ok) list[(size_t)b * a.Tk + before + __popc(here & ((1u << lane) - 1u))] = n;
        base += all;
    }
    if (threadIdx.x == 0) counts[b] = base;
}

int group_rows(const KvAttendArgs& a) {
    const int per = a.Hq / a.Hk, heads = per < a.k_h ? per : a.k_h;
    const long long r = (long long)heads * a.Tq;
    return r > 0x7fffffffLL ? 0x7fffffff : (int)r;
}
long long row_blocks(const KvAttendArgs& a) {
    const long long n = ((long long)group_rows(a) + 2 * kTM - 1) / (2 * kTM);
    return n > 65535 ? 65535 : n;
}
int tc_keys(int d) { return d <= 64 ? TcCfg<64, false>::KN : TcCfg<128, false>::KN; }
int tc_ctas(int d) { return d <= 64 ? TcCfg<64, false>::CTAS : TcCfg<128, false>::CTAS; }
// Blocks along the keys: where the row blocks alone leave SMs idle, each with two steps at least.
int tc_splits(const KvAttendArgs& a) {
    const long long units = (long long)a.B * a.Hk * row_blocks(a);
    const long long tiles = ((long long)a.Tk + tc_keys(a.d) - 1) / tc_keys(a.d);
    if (units == 0) return 1;
    long long n = (long long)tc_ctas(a.d) * kSmCount / units;
    if (n > tiles / 2) n = tiles / 2;
    return n < 1 ? 1 : n > 64 ? 64 : (int)n;
}
bool tc_planned(const KvAttendArgs& a) { return a.ids != nullptr && a.Tk > kTcListed; }

template <int D, bool BF16, int FMT>
int launch_tc(sentry_ctx* ctx, const KvAttendArgs& a, WsAlloc& ws, cudaStream_t st) {
    using C = TcCfg<D, FMT != 0>;
    KvMaps maps = {};
    if (FMT == 0 && (!make_map_dense(&maps.k, a.K, a, a.ks, C::KN) || !make_map_dense(&maps.v, a.V, a, a.vs, C::KN))) return SENTRY_ERR_CUDA;
    const int n_splits = tc_splits(a);
    const size_t rows = (size_t)a.B * a.k_h * a.Tq;
    float* part = nullptr;
    float2* ml = nullptr;
    int32_t *list = nullptr, *counts = nullptr;
    if (n_splits > 1) {
        part = ws.take<float>(n_splits * rows * D);
        ml = ws.take<float2>(n_splits * rows);
    }
    if (tc_planned(a)) {
        list = ws.take<int32_t>((size_t)a.B * a.Tk);
        counts = ws.take<int32_t>(a.B);
    }
    if (!ws.ok) return SENTRY_ERR_WORKSPACE;
    if (tc_planned(a)) {
        LaunchScope ls(ctx, KS_KV_PLAN, st);
        SENTRY_CUDA_TRY(launch_chained(kv_plan_kernel, dim3((unsigned)a.B), dim3(1024), 0, st, a, list, counts));
    }
    auto k = kv_tc_kernel<D, BF16, FMT>;
    static std::atomic<unsigned long long> allowed{0};
    SENTRY_CUDA_TRY(allow_smem(k, C::SMEM, ctx->device, allowed));
    {
        LaunchScope ls(ctx, KS_KV_ATTEND, st);
        SENTRY_CUDA_TRY(launch_chained(k, dim3((unsigned)((long long)a.B * a.Hk * n_splits), (unsigned)row_blocks(a)), dim3(C::THREADS), C::SMEM, st, maps, a, (const int32_t*)list,
                                       (const int32_t*)counts, part, ml, n_splits));
    }
    return n_splits > 1 ? launch_kv_combine(ctx, a, part, ml, n_splits, st) : SENTRY_OK;
}

template <bool BF16, int FMT>
int launch_tc_d(sentry_ctx* ctx, const KvAttendArgs& a, WsAlloc& ws, cudaStream_t st) {
    switch (a.d) {
        case 16: return launch_tc<16, BF16, FMT>(ctx, a, ws, st);
        case 32: return launch_tc<32, BF16, FMT>(ctx, a, ws, st);
        case 64: return launch_tc<64, BF16, FMT>(ctx, a, ws, st);
        default: return launch_tc<128, BF16, FMT>(ctx, a, ws, st);
    }
}

}  // namespace

// Which of the two 16-bit forms: kv_rows_kernel's work is its row tiles of 16 times their keys, 128 at a time, in a wave or two of small blocks; a CTA here has a
// setup of several microseconds and takes 256 rows at once.
// Dense keys, bf16 (here against there): 2 x 40 rows of 4 groups on 77 keys, d 64 (24 units) 8.2 against 6.2 us; 64 x 4 rows of 16 groups on 256 (512) 13.3
// against 9.5; 20 x 3 of 64 on 300 (768) 12.5 against 10.4; 17 x 4 of 64 on 512 (1280) 10.8 against 12.3; 512 x 4 of 2 on 512 (1024) 13.6 against 19.6.  At d 128
// only the smallest lose: 40 x 4 of 2 on 256 (40) 11.5 against 15.7.
// A cache, i8: 75 x 2 of 6 on 128 (60) 16.7 against 7.5; 128 x 4 of 8 on 512 (1024) 32.5 against 19.0; 17 x 4 of 64 on 512 (1280) 17.6 against 15.8; 16 x 4 of 64
// on 2048 (4096) 46 against 49; 24 x 4 of 16 on 8192 (6144) 37 against 52; 512 x 4 of 8 on 8192 (65536) 142 against 619; but 128 x 4 of 32 on 128 (1024 tiles, more than
// a wave) 19.2 against 24.2.
bool kv_tc_takes(const KvAttendArgs& a) {
    if (a.dtype == SENTRY_F32 || a.Tk == 0 || group_rows(a) <= (a.format == 0 ? 32 : 64)) return false;
    const long long row_tiles = (long long)a.B * a.Hk * ((group_rows(a) + 15) / 16), work = row_tiles * (((long long)a.Tk + 127) / 128);
    if (a.format == 0) return a.d > 64 || work > 768;
    return work > 2048 || row_tiles > 4 * kSmCount;
}
size_t kv_tc_ws_bytes(const KvAttendArgs& a) {
    const int n = tc_splits(a);
    const size_t rows = (size_t)a.B * a.k_h * a.Tq;
    size_t bytes = 0;
    if (n > 1) bytes += align_up(n * rows * a.d * sizeof(float), 256) + align_up(n * rows * sizeof(float2), 256);
    if (a.format != 0 || a.Tk <= kTcListed) return bytes + 512;        // (a cache has no modality ids)
    // (whether a dense call has some is not in the descriptor)
    return bytes + align_up((size_t)a.B * a.Tk * sizeof(int32_t), 256) + align_up((size_t)a.B * sizeof(int32_t), 256) + 512;
}
int launch_kv_tc(sentry_ctx* ctx, const KvAttendArgs& a, WsAlloc& ws, cudaStream_t st) {
    const bool bf16 = a.dtype == SENTRY_BF16;
    if (a.format == 0) return bf16 ? launch_tc_d<true, 0>(ctx, a, ws, st) : launch_tc_d<false, 0>(ctx, a, ws, st);
    if (a.format == SENTRY_FP8_E4M3) return bf16 ? launch_tc_d<true, SENTRY_FP8_E4M3>(ctx, a, ws, st) : launch_tc_d<false, SENTRY_FP8_E4M3>(ctx, a, ws, st);
    return bf16 ? launch_tc_d<true, SENTRY_I8>(ctx, a, ws, st) : launch_tc_d<false, SENTRY_I8>(ctx, a, ws, st);
}
