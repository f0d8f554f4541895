// Serving attention for few rows: a decoder's single tokens and short blocks, over dense 16-bit keys and values or the 8-bit cache.
//
// The rows of one KV group (kept heads x Tq) share its keys, so they are packed into tiles of 8 or 16 rows, and a block takes a tile and a
// stretch of the keys.  One warp brings tiles of 32 keys into a ring by TMA, which also swizzles them against bank conflicts; four others
// take them in turn, each with a running maximum and sum of its own (log2 domain) and both products on the warp MMA: no barrier between
// them until the four partial results meet.  Long axes are shared out over blocks; the last to finish joins the parts.
// The keys are the MMA's 16 rows and the queries its 8 columns (S^T = K Q^T, O^T = V^T P^T): a decoder's few rows fill it, where queries as
// rows left half of it and half of the exponentials empty.
// What bounds it: the bytes of K and V, read once from memory, and the instructions that turn codes into operands.  They go from
// shared memory through registers straight into the MMA: the order of the inner index is free as long as both operands share it, so that
// a lane's 16 consecutive bytes of a key are its operand for K's product; and for V's, where pairs run along the keys, two keys'
// words are interleaved byte by byte.  The weights get from the first product's layout to the second's by a transposition of 8 x 8
// matrices among registers.  8-bit codes become fp16 exactly; a page's key scale multiplies the scores, the logarithm of its value scale is
// added to them.  The maximum is followed only where a score exceeds it by 2^4 (fp16 weights) or 2^8 (bf16).
// (Value scales that multiplied the weights, without the weights' 2^11, cost 0.6 us less here and lost small weights beside a large one.)
// One token of 32 samples of up to 4096 e4m3 tokens (16 heads on 4, d 128, 87 MB): 25 us, 3.5 TB/s over all; a block's first keys arrive 3.5 us
// after its start (lengths, page, keys: three loads that depend on one another), between that and the last tile the loads run at 5 to 5.7 TB/s,
// and the parts meet in 3.  i8 of d 64 (2 x 131072 tokens, 67 MB): 29 us, issue slots 48 % and memory 36 % busy: some 640 instructions a warp for 32 keys, which wait
// for one another at 16 working warps an SM.
// Every wait is bounded; on expiry the block raises SENTRY_STATUS_BIT_TIMEOUT and unwinds.
#include "kv_attend.cuh"
#include "kv_maps.cuh"
#include "kv_rows_ring.cuh"

namespace {

constexpr int kWarps = kRowsWarps, kKeys = kRowsKeys, kRowsThreads = (kWarps + 1) * 32;
constexpr float kLog2e = 1.4426950408889634f;

enum { KV_BF16 = 0, KV_F16 = 1, KV_E4M3 = 2, KV_I8 = 3 };

template <int KV, int D>
struct RowsCfg {
    static constexpr int ESIZE = KV <= KV_F16 ? 2 : 1;
    static constexpr int ROW = D * ESIZE;                    // bytes of a key
    static constexpr int RB = ROW < 128 ? ROW : 128;         // of a row in shared memory; wider keys lie in slabs
    static constexpr int TILE = kKeys * ROW < 1024 ? 1024 : kKeys * ROW;   // of K or V, on the swizzle's boundary
    // tiles of the ring, and blocks on an SM
    static constexpr int STAGES = rows_stages(TILE);
    static_assert(STAGES % kWarps == 0, "a slot is one warp's");
    static constexpr int BLOCKS = TILE > 4096 ? 2 : TILE > 2048 ? 3 : 4;
    static constexpr int RING = STAGES * 2 * TILE;
    static constexpr int MERGE = kWarps * 16 * D * 4;
    static constexpr int SMEM = (RING > MERGE ? RING : MERGE) + 1024;
};

// 16-byte piece c of key r lies at piece c ^ piece_shift(r) of its row of RB bytes (the copies' swizzle).
template <int RB>
__device__ __forceinline__ int piece_shift(int r) {
    return RB == 128 ? r & 7 : RB == 64 ? (r >> 1) & 3 : RB == 32 ? (r >> 2) & 1 : 0;
}
template <int BYTES>
__device__ __forceinline__ void lds(uint32_t addr, uint32_t* r) {
    if constexpr (BYTES == 16) asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr));
    else if constexpr (BYTES == 8) asm volatile("ld.shared.v2.b32 {%0,%1}, [%2];" : "=r"(r[0]), "=r"(r[1]) : "r"(addr));
    else if constexpr (BYTES == 4) asm volatile("ld.shared.b32 %0, [%1];" : "=r"(r[0]) : "r"(addr));
    else {
        unsigned short v;
        asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(addr));
        r[0] = v;
    }
}
template <bool BF16>
__device__ __forceinline__ void mma16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    if constexpr (BF16)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
template <bool BF16>
__device__ __forceinline__ float2 unpack2(uint32_t w) {
    if constexpr (BF16) return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
    else return __half22float2(*reinterpret_cast<const __half2*>(&w));
}
// 8 x 8 matrix of 16-bit values spread over a warp (a row's pairs over four lanes), transposed
__device__ __forceinline__ uint32_t transposed(uint32_t x) {
    uint32_t r;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
    return r;
}

// Which stretch of which sample's keys a block takes.  The samples' lengths differ and only the device knows them, so that every block works
// out the same shares: as many blocks to a sample as it has stretches of `chunk` tiles (one at least), so that all fit one wave.
struct RowsShare { int b, split, n, first, len; };   // first: number of the sample's first part among all samples' parts; len: its keys
__device__ __forceinline__ RowsShare rows_share(const KvAttendArgs& a, int unit, int room) {
    const int lane = threadIdx.x & 31;
    if (a.lengths == nullptr) {             // all alike: no search
        const int each = min((room + a.B) / a.B, max(1, (a.Tk + kKeys - 1) / kKeys / kWarps)), b = unit / each;
        return RowsShare{b < a.B ? b : -1, unit % each, each, b * each, a.Tk};
    }
    auto length_of = [&](int b) { return b < a.B ? kv_length(a, b) : 0; };
    auto tiles = [](int len) { return (len + kKeys - 1) / kKeys; };
    const int mine = length_of(lane);
    int sum = tiles(mine);
#pragma unroll 4
    for (int b0 = 32; b0 < a.B; b0 += 32) sum += tiles(length_of(b0 + lane));
    const long long total = (long long)__reduce_add_sync(0xffffffffu, sum >> 8) * 256 + __reduce_add_sync(0xffffffffu, sum & 255);
    int chunk = max((int)((total + room - 1) / room), kWarps);
    if (a.B <= 32) {
        // the smallest stretch with which all fit; the one above leaves out that few samples are a whole number of stretches
        int low = max((int)(total / (room + a.B)), kWarps);
        for (int step = 0; step < 6 && low < chunk; ++step) {
            const int mid = (low + chunk) / 2;
            const int n = __reduce_add_sync(0xffffffffu, lane < a.B ? max(1, (tiles(mine) + mid - 1) / mid) : 0);
            if (n <= room + a.B) chunk = mid;
            else low = mid + 1;
        }
    }
    RowsShare r = {-1, 0, 0, 0, 0};
    int base = 0;
    for (int b0 = 0; b0 < a.B; b0 += 32) {
        const int b = b0 + lane, len = b0 ? length_of(b) : mine, n = b < a.B ? max(1, (tiles(len) + chunk - 1) / chunk) : 0;
        int incl = n;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int v = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o) incl += v;
        }
        const unsigned hit = __ballot_sync(0xffffffffu, unit >= base + incl - n && unit < base + incl);
        if (hit) {
            const int who = __ffs(hit) - 1;
            r.b = b0 + who;
            r.first = base + __shfl_sync(0xffffffffu, incl - n, who);
            r.n = __shfl_sync(0xffffffffu, n, who);
            r.len = __shfl_sync(0xffffffffu, len, who);
            r.split = unit - r.first;
            break;
        }
        base += __shfl_sync(0xffffffffu, incl, 31);
    }
    return r;
}

// Where the parts of split axes meet.  part: [parts][k_h][Tq][D] sums, ml: [parts][k_h][Tq] (maximum, total).  The last block of every
// kJoin neighbouring parts of a group's row tile joins those into one of `part2`, the last of these joins the results; kJoin parts at most
// go straight to the second step.  (A launch of its own for it costs 6 us behind the blocks' end, and one block alone is slow with a hundred parts.)
// counters: one of every group's row tile, then one of every kJoin parts of it; left at zero.
constexpr int kJoin = 16;
struct RowsJoin {
    float *part, *part2;
    float2 *ml, *ml2;
    unsigned int* counters;
    int room;                  // parts beside the first of every sample; 0: no axis is split, a block per group and row tile takes all keys
};

// Four columns of n parts of a row, `each` rows apart, and their (maximum, total).  Not inlined: what it holds of kJoin / 2 parts at a time
// would cost the loop over the keys its registers.
template <int D>
__device__ __noinline__ float4 join_parts(const float* part, const float2* ml, size_t each, int n, float2& out) {
    constexpr int S = kJoin / 2;
    float top = -INFINITY, sum = 0.0f;
    float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    for (int s0 = 0; s0 < n; s0 += S, part += S * each * D, ml += S * each) {
        float2 x[S];
        float4 p[S];
        float now = top;
#pragma unroll
        for (int s = 0; s < S; ++s) {
            const bool in = s0 + s < n;
            x[s] = in ? __ldcg(ml + s * each) : make_float2(-INFINITY, 0.0f);
            p[s] = in ? __ldcg(reinterpret_cast<const float4*>(part + s * each * D)) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        }
#pragma unroll
        for (int s = 0; s < S; ++s) now = fmaxf(now, x[s].x);
        const float ref = now == -INFINITY ? 0.0f : now, keep = top == now ? 1.0f : exp2_fast(top - ref);
        top = now;
        sum *= keep;
        v.x *= keep; v.y *= keep; v.z *= keep; v.w *= keep;
#pragma unroll
        for (int s = 0; s < S; ++s) {
            const float f = exp2_fast(x[s].x - ref);
            sum += x[s].y * f;
            v.x += p[s].x * f; v.y += p[s].y * f; v.z += p[s].z * f; v.w += p[s].w * f;
        }
    }
    out = make_float2(top, sum);
    return v;
}

template <int KV, int D, bool BF16, int NT>
__global__ void __launch_bounds__(kRowsThreads, RowsCfg<KV, D>::BLOCKS - (NT > 1 && RowsCfg<KV, D>::BLOCKS > 2))
kv_rows_kernel(const __grid_constant__ KvMaps maps, const KvAttendArgs a, const RowsJoin meet) {
    using C = RowsCfg<KV, D>;
    constexpr bool DENSE = KV <= KV_F16, I8 = KV == KV_I8;
    constexpr bool MMA_BF16 = KV == KV_BF16;
    constexpr bool SPLIT_P = DENSE || !BF16;                 // weights as a head and a remainder
    // The maximum is followed where a score exceeds it by 2^kLag.  fp16 weights are taken 2^kShift times as large (2^15 at most): its range is what
    // small ones run out of, below 2^-25 of the largest weight (times its value scale), from where they round to multiples of 2^-35 of that.
    // bf16 has fp32's range.
    constexpr float kLag = MMA_BF16 ? 8.0f : 4.0f, kShift = MMA_BF16 ? 0.0f : 11.0f, kUnshift = MMA_BF16 ? 1.0f : 1.0f / 2048.0f;
    constexpr int KSTEPS = D / 16, DT = D / 16, ROWS = 8 * NT, RB = C::RB;
    extern __shared__ uint8_t smem_raw[];
    __shared__ unsigned s_vis[C::STAGES];                   // keys of the slot's tile that are there
    __shared__ uint64_t s_kfull[C::STAGES], s_vfull[C::STAGES], s_kempty[C::STAGES], s_vempty[C::STAGES];
    __shared__ short s_head[kServeMaxHeads], s_pos[kServeMaxHeads];
    __shared__ int s_heads, s_abort;
    __shared__ float s_m[kWarps][ROWS], s_l[kWarps][ROWS];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, gq = lane >> 2, t4 = lane & 3;
    const int g = blockIdx.x % a.Hk;
    const uint32_t raw_addr = ptx::smem_u32(smem_raw), ring = (raw_addr + 1023u) & ~1023u;
    volatile int* abort_flag = &s_abort;
    if (threadIdx.x == 0) {
        for (int s = 0; s < C::STAGES; ++s) {
            ptx::mbar_init(ptx::smem_u32(&s_kfull[s]), 1);
            ptx::mbar_init(ptx::smem_u32(&s_vfull[s]), 1);
            ptx::mbar_init(ptx::smem_u32(&s_kempty[s]), 1);
            ptx::mbar_init(ptx::smem_u32(&s_vempty[s]), 1);
        }
        s_abort = 0;
        ptx::fence_barrier_init();
    }
    grid_dependents_start_if_small();
    grid_dependency_wait();
    RowsShare share = {(int)blockIdx.x / a.Hk, 0, 1, 0, 0};
    if (meet.room > 0) share = rows_share(a, blockIdx.x / a.Hk, meet.room);       // (every warp for itself)
    else share.len = kv_length(a, share.b);
    if (share.b < 0) return;
    const int b = share.b;
    if (warp == 0) {
        const int n = kv_group_heads(a, b, g, g == 0 && share.split == 0 && blockIdx.y == 0, s_head, s_pos);
        if (lane == 0) s_heads = n;
    }
    const int len = share.len;
    const int tiles = (len + kKeys - 1) / kKeys;
    const int t0 = (int)((long long)tiles * share.split / share.n), t1 = (int)((long long)tiles * (share.split + 1) / share.n);
    // the copying warp: of 32 tiles at a time, a lane each, the pages of the first 16 keys and of the others (-1: none)
    const int page_shift = DENSE ? 0 : 31 - __clz(a.page);
    int id0 = -1, id1 = -1;
    auto ask_pages = [&](int tile) {
        const int32_t* pages = a.table + (size_t)b * a.max_pages;
        const int n = (tile + lane) * kKeys;
        const bool in = tile + lane < t1, second = in && n + 16 < len;
        id0 = in ? pages[n >> page_shift] : -1;
        id1 = page_shift > 4 ? id0 : second ? pages[(n >> 4) + 1] : -1;
        const bool bad0 = in && (unsigned)id0 >= (unsigned)a.n_pages, bad1 = second && (unsigned)id1 >= (unsigned)a.n_pages;
        if (bad0 || bad1) atomicOr(a.status, SENTRY_STATUS_BIT_BAD_INDEX);
        if ((unsigned)id0 >= (unsigned)a.n_pages) id0 = -1;
        if ((unsigned)id1 >= (unsigned)a.n_pages) id1 = -1;
    };
    if constexpr (!DENSE)
        if (warp == kWarps) ask_pages(t0);                  // (while another warp reads the list of heads)
    __syncthreads();
    const int rows = s_heads * a.Tq;
    uint32_t done = 0;                                      // tiles of the row tiles before

    for (int row0 = blockIdx.y * ROWS; row0 < rows; row0 += gridDim.y * ROWS, done += (uint32_t)(t1 - t0)) {
        bool ok = true;
        if (warp == kWarps) {
            // ---------------------------------------------------------------- copies
            const uint32_t mask = a.masks ? a.masks[b] : 0u;
            const int kb = a.ks[0] ? b : 0, kg = a.ks[1] ? g : 0, vb = a.vs[0] ? b : 0, vg = a.vs[1] ? g : 0;
            int ahead = DENSE && a.ids != nullptr && t0 * kKeys + lane < len ? a.ids[t0 * kKeys + lane] : 0;
            uint32_t s = done % C::STAGES, use = done / C::STAGES;
            for (int tile = t0; tile < t1 && ok; ++tile) {
                const int n0 = tile * kKeys;
                unsigned vis;
                int at0 = 0, at1 = 0;
                if constexpr (DENSE) {
                    bool here = n0 + lane < len;
                    if (a.ids != nullptr) {
                        here = here && kv_present(ahead, mask);
                        ahead = n0 + kKeys + lane < len ? a.ids[n0 + kKeys + lane] : 0;
                    }
                    vis = __ballot_sync(0xffffffffu, here);
                } else {
                    const int turn = (tile - t0) & 31;
                    if (turn == 0 && (tile > t0 || (t1 - t0 > 32 && done > 0))) ask_pages(tile);
                    at0 = __shfl_sync(0xffffffffu, id0, turn);
                    at1 = __shfl_sync(0xffffffffu, id1, turn);
                    vis = len - n0 >= 32 ? 0xffffffffu : (1u << (len - n0)) - 1u;
                    if (at0 < 0) vis &= 0xffff0000u;
                    if (at1 < 0) vis &= 0x0000ffffu;
                }
                ok = warp_wait(&s_kempty[s], (use & 1) ^ 1, abort_flag);
                if (ok) {
                    // (whoever reads the slot's bits does so before it gives K's half back)
                    if (lane == 0) s_vis[s] = vis;
                    __syncwarp();
                    if (elect_one()) {
#pragma unroll
                        for (int is_v = 0; is_v < 2; ++is_v) {
                            const CUtensorMap* map = is_v ? &maps.v : &maps.k;
                            const uint32_t bar = ptx::smem_u32(is_v ? &s_vfull[s] : &s_kfull[s]), dst = ring + s * 2 * C::TILE + is_v * C::TILE;
                            if (is_v && !ptx::mbar_wait(ptx::smem_u32(&s_vempty[s]), (use & 1) ^ 1, abort_flag)) break;
                            if (vis == 0) { ptx::mbar_arrive(bar); continue; }
                            if constexpr (DENSE) {
                                ptx::mbar_arrive_expect_tx(bar, kKeys * C::ROW);
#pragma unroll
                                for (int c = 0; c < C::ROW / RB; ++c) tma_load_4d(dst + c * kKeys * RB, map, c * 64, n0, is_v ? vg : kg, is_v ? vb : kb, bar);
                            } else if (page_shift > 4) {
                                ptx::mbar_arrive_expect_tx(bar, kKeys * C::ROW);
                                ptx::tma_load_2d(dst, map, 0, (at0 * a.Hk + g) * a.page + (n0 & (a.page - 1)), bar);
                            } else {
                                ptx::mbar_arrive_expect_tx(bar, ((at0 >= 0) + (at1 >= 0)) * 16 * C::ROW);
                                if (at0 >= 0) ptx::tma_load_2d(dst, map, 0, (at0 * a.Hk + g) * 16, bar);
                                if (at1 >= 0) ptx::tma_load_2d(dst + 16 * C::ROW, map, 0, (at1 * a.Hk + g) * 16, bar);
                            }
                        }
                    }
                    __syncwarp();
                    ok = __all_sync(0xffffffffu, *abort_flag == 0);
                }
                if (++s == C::STAGES) { s = 0; ++use; }
            }
        }
        float o[DT][NT][4], m[NT][2], l[NT][2], vref = 1.0f;        // O is in units of vref (8-bit values; see below)
        if (warp < kWarps) {
        uint32_t qf[NT][KSTEPS][2];
        float scale[NT][2];                                     // of rows 2 t4 and 2 t4 + 1, whose scores this lane will hold
        int last[NT][2];                                        // keys that they see end here
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const int r = row0 + nt * 8 + gq;
            const bool in = r < rows;
            const char* q = (const char*)a.Q + (b * a.qs[0] + (in ? s_head[r / a.Tq] : 0) * a.qs[1] + (in ? r % a.Tq : 0) * a.qs[2]) * 2;
            // elements of a chunk that one lane has: 16 bytes of a key, or a quarter of a shorter one
            constexpr int E = (C::ROW / 4 < 16 ? C::ROW / 4 : 16) / C::ESIZE;
#pragma unroll
            for (int s = 0; s < KSTEPS; ++s) {
                const int e = (s / (E / 4)) * 4 * E + t4 * E + (s % (E / 4)) * 4;
                const uint2 x = in ? *reinterpret_cast<const uint2*>(q + e * 2) : make_uint2(0, 0);
                qf[nt][s][0] = x.x;
                qf[nt][s][1] = x.y;
            }
            float rs = rsqrtf((float)D) * kLog2e;
            if constexpr (!DENSE && BF16) {
                // bf16 rows as fp16: scaled by a power of two so that the largest value lies in [1,2)
                float top = 0.0f;
#pragma unroll
                for (int s = 0; s < KSTEPS; ++s)
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        const float2 f = unpack2<true>(qf[nt][s][x]);
                        top = fmaxf(top, fmaxf(fabsf(f.x), fabsf(f.y)));
                    }
                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
                int e = (int)(__float_as_uint(top) >> 23) - 127;      // (infinities: 128, and the row is not a number in any case)
                e = min(max(e, -120), 120);
                const float down = __uint_as_float((uint32_t)(127 - e) << 23);
                rs *= __uint_as_float((uint32_t)(127 + e) << 23);
#pragma unroll
                for (int s = 0; s < KSTEPS; ++s)
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        const float2 f = unpack2<true>(qf[nt][s][x]);
                        qf[nt][s][x] = pack2<false>(f.x * down, f.y * down);
                    }
            }
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                scale[nt][x] = __shfl_sync(0xffffffffu, rs, (2 * t4 + x) * 4);
                const int i = (row0 + nt * 8 + 2 * t4 + x) % a.Tq;
                last[nt][x] = !DENSE && a.causal ? min(len, len - a.Tq + i + 1) : len;
            }
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            m[nt][0] = m[nt][1] = -INFINITY;
            l[nt][0] = l[nt][1] = 0.0f;
#pragma unroll
            for (int j = 0; j < DT; ++j)
#pragma unroll
                for (int x = 0; x < 4; ++x) o[j][nt][x] = 0.0f;
        }
        // where this lane reads: K's pieces of key gq of every eight, V's pieces of keys 2 t4 and 2 t4 + 1 of every eight
        constexpr int VB = D / 8 * C::ESIZE;                        // bytes of a key of V that a lane takes
        constexpr int PIECE = VB < 16 ? VB : 16, PIECES = VB / PIECE, WORDS = VB < 4 ? 1 : VB / 4;
        constexpr int KB = C::ROW / 4 < 16 ? C::ROW / 4 : 16;       // of a key of K, at a time
        const int k_at = gq * RB + ((((t4 * KB) >> 4) ^ piece_shift<RB>(gq)) << 4) + ((t4 * KB) & 15);
        int v_at[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int at = gq * VB;
            v_at[u] = at / RB * (kKeys * RB) + (2 * t4 + u) * RB + (((at % RB >> 4) ^ piece_shift<RB>(2 * t4 + u)) << 4) + (at & 15);
        }
        // keys below this are seen by every row of the warp
        int all_see = len;
        if (!DENSE && a.causal) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) all_see = min(all_see, min(last[nt][0], last[nt][1]));
            all_see = __reduce_min_sync(0xffffffffu, all_see);
        }
        // A page's value scale goes into its keys' exponents, in units of the largest one of this warp's pages (vref): the maximum is then that of
        // weight times scale, and no weight is lost whose values count.  The sum takes it out again.
        // Key scales of this warp's next 32 tiles, a lane each (of the first 16 keys and of the others), logarithms and signs of the value scales.
        // (A scale of 2^-100 of vref and less leaves zeros of its values; one that is no number makes them none.)
        constexpr float kNoneLog = -99.99f;
        float ks0 = 0.0f, ks1 = 0.0f, lg0 = 0.0f, lg1 = 0.0f;
        unsigned odd0 = 0u, odd1 = 0u;                          // tiles with a scale below zero, or as good as zero
        int turn = 0;
        auto pages_of = [&](int tile, int& id0, int& id1) {
            const int32_t* pages = a.table + (size_t)b * a.max_pages;
            const int mine = tile + lane * kWarps, n = mine * kKeys, shift = 31 - __clz(a.page);
            id0 = id1 = mine < t1 ? pages[n >> shift] : -1;
            if (shift == 4) id1 = mine < t1 && n + 16 < len ? pages[(n >> 4) + 1] : -1;
            if ((unsigned)id0 >= (unsigned)a.n_pages) id0 = -1;
            if ((unsigned)id1 >= (unsigned)a.n_pages) id1 = -1;
        };
        auto scale_of = [&](const float* scales, int id, float none) { return id >= 0 ? scales[(size_t)id * a.Hk + g] : none; };
        auto size_of = [&](float vs) {                          // (as bits, which order sizes; what is no number counts as nothing)
            const uint32_t v = __float_as_uint(vs) & 0x7fffffffu;
            return v < 0x7f800000u ? v : 0u;
        };
        auto log_of = [&](float vs) { return fabsf(vs) <= 3.4028234e38f ? log2f(fmaxf(fabsf(vs) * (1.0f / vref), 7.8886091e-31f)) : __int_as_float(0x7fc00000); };
        auto take = [&](int id0, int id1, float vs0, float vs1) {
            ks0 = scale_of(a.k_scales, id0, 0.0f);
            ks1 = scale_of(a.k_scales, id1, 0.0f);
            lg0 = log_of(vs0);
            lg1 = log_of(vs1);
            odd0 = __ballot_sync(0xffffffffu, vs0 < 0.0f || lg0 <= kNoneLog);
            odd1 = __ballot_sync(0xffffffffu, vs1 < 0.0f || lg1 <= kNoneLog);
        };
        if constexpr (!DENSE) {
            int id0, id1;
            pages_of(t0 + warp, id0, id1);
            const float vs0 = scale_of(a.v_scales, id0, 0.0f), vs1 = scale_of(a.v_scales, id1, 0.0f);
            uint32_t top = max(size_of(vs0), size_of(vs1));
#pragma unroll 1
            for (int tile = t0 + warp + 32 * kWarps; tile < t1; tile += 32 * kWarps) {
                int far0, far1;
                pages_of(tile, far0, far1);
                top = max(top, max(size_of(scale_of(a.v_scales, far0, 0.0f)), size_of(scale_of(a.v_scales, far1, 0.0f))));
            }
            top = __reduce_max_sync(0xffffffffu, top);
            vref = top == 0u ? 1.0f : fmaxf(__uint_as_float(top), 7.5231638e-37f);     // (2^-120)
            take(id0, id1, vs0, vs1);
        }

        // -------------------------------------------------------------------- tiles of 32 keys
        for (int tile = t0 + warp; tile < t1; tile += kWarps) {
            const uint32_t n = done + (uint32_t)(tile - t0), slot = n % C::STAGES, parity = n / C::STAGES & 1;
            if constexpr (!DENSE) {
                if (turn == 0 && tile >= t0 + kWarps) {
                    int id0, id1;
                    pages_of(tile, id0, id1);
                    take(id0, id1, scale_of(a.v_scales, id0, 0.0f), scale_of(a.v_scales, id1, 0.0f));
                }
            }
            if (!warp_wait(&s_kfull[slot], parity, abort_flag)) break;
            const int n0 = tile * kKeys;
            const uint32_t kt = ring + slot * 2 * C::TILE, vt = kt + C::TILE;
            const unsigned vis = s_vis[slot];
            float kscale[2] = {1.0f, 1.0f}, vlog[2] = {0.0f, 0.0f};
            const int now = turn;
            if constexpr (!DENSE) {
                kscale[0] = __shfl_sync(0xffffffffu, ks0, now); kscale[1] = __shfl_sync(0xffffffffu, ks1, now);
                vlog[0] = __shfl_sync(0xffffffffu, lg0, now); vlog[1] = __shfl_sync(0xffffffffu, lg1, now);
                turn = (turn + 1) & 31;
            }
            const bool any = __any_sync(0xffffffffu, vis != 0), full = __all_sync(0xffffffffu, vis == 0xffffffffu && n0 + kKeys <= all_see);
            float s[2][NT][4];
            if (any) {
                // ------ scores: element (key mt * 16 + gq + 8 * (x >> 1), row nt * 8 + 2 t4 + (x & 1))
#pragma unroll
                for (int mt = 0; mt < 2; ++mt) {
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int x = 0; x < 4; ++x) s[mt][nt][x] = 0.0f;
#pragma unroll
                    for (int c = 0; c < (C::ROW + 63) / 64; ++c) {
                        uint32_t w0[4], w1[4];                      // keys gq and gq + 8
                        const uint32_t at = kt + c / (RB / 64 > 0 ? RB / 64 : 1) * (kKeys * RB) + (k_at ^ (c % (RB / 64 > 0 ? RB / 64 : 1) * 64)) + mt * 16 * RB;
                        lds<KB>(at, w0);
                        lds<KB>(at + 8 * RB, w1);
#pragma unroll
                        for (int x = 0; x < KB / (DENSE ? 8 : 4); ++x) {
                            uint32_t f[4];
                            if constexpr (DENSE) { f[0] = w0[2 * x]; f[1] = w1[2 * x]; f[2] = w0[2 * x + 1]; f[3] = w1[2 * x + 1]; }
                            else {
                                codes_to_f16<I8>(w0[x], f[0], f[2]);
                                codes_to_f16<I8>(w1[x], f[1], f[3]);
                            }
                            constexpr int PER = KB / (DENSE ? 8 : 4);
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt) mma16<MMA_BF16>(s[mt][nt], f, qf[nt][c * PER + x][0], qf[nt][c * PER + x][1]);
                        }
                    }
                }
#pragma unroll
                for (int mt = 0; mt < 2; ++mt) {
                    const float ks = kscale[mt];
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        const float c0 = scale[nt][0] * ks, c1 = scale[nt][1] * ks;
#pragma unroll
                        for (int x = 0; x < 4; ++x) s[mt][nt][x] = DENSE ? s[mt][nt][x] * (x & 1 ? c1 : c0) : fmaf(s[mt][nt][x], x & 1 ? c1 : c0, vlog[mt]);
                    }
                }
            }
            warp_arrive(&s_kempty[slot]);
            if (any) {
                if (!full) {
#pragma unroll
                    for (int mt = 0; mt < 2; ++mt)
#pragma unroll
                        for (int x = 0; x < 4; ++x) {
                            const int n = mt * 16 + gq + (x >> 1) * 8;
                            const bool here = (vis >> n) & 1u;
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt)
                                if (!here || n0 + n >= last[nt][x & 1]) s[mt][nt][x] = -INFINITY;
                        }
                }
                // ------ softmax
                bool over = false;
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        const float top = fmaxf(fmaxf(s[0][nt][x], s[0][nt][x + 2]), fmaxf(s[1][nt][x], s[1][nt][x + 2]));
                        over = over || top - m[nt][x] > kLag;
                    }
                if (__any_sync(0xffffffffu, over)) {
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        float keep[2];
#pragma unroll
                        for (int x = 0; x < 2; ++x) {
                            float top = fmaxf(fmaxf(s[0][nt][x], s[0][nt][x + 2]), fmaxf(s[1][nt][x], s[1][nt][x + 2]));
#pragma unroll
                            for (int y = 4; y < 32; y <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, y));
                            // (each row for itself: what its neighbours hold changes no bit of it)
                            const bool grew = top - m[nt][x] > kLag;
                            keep[x] = grew ? exp2_fast(m[nt][x] - top) : 1.0f;
                            m[nt][x] = grew ? top : m[nt][x];
                            l[nt][x] *= keep[x];
                        }
#pragma unroll
                        for (int j = 0; j < DT; ++j)
#pragma unroll
                            for (int x = 0; x < 4; ++x) o[j][nt][x] *= keep[x & 1];
                    }
                }
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    const float ref[2] = {(m[nt][0] == -INFINITY ? 0.0f : m[nt][0]) - kShift, (m[nt][1] == -INFINITY ? 0.0f : m[nt][1]) - kShift};
#pragma unroll
                    for (int mt = 0; mt < 2; ++mt) {
#pragma unroll
                        for (int x = 0; x < 4; ++x) s[mt][nt][x] = exp2_fast(s[mt][nt][x] - ref[x & 1]);
#pragma unroll
                        for (int x = 0; x < 2; ++x) {
                            const float sum = s[mt][nt][x] + s[mt][nt][x + 2];
                            if constexpr (DENSE) l[nt][x] += sum;
                            else {
                                // a weight counts in the sum without its page's value scale (which may be no number, where a row sees nothing of the page)
                                const float out = exp2_fast(-vlog[mt]);
                                l[nt][x] = full || sum != 0.0f ? fmaf(sum, out, l[nt][x]) : l[nt][x];
                            }
                        }
                    }
                }
                if (!warp_wait(&s_vfull[slot], parity, abort_flag)) break;
                // ------ values, 16 keys at a time: column gq * (D / 8) + 2 j is row gq of the MMA's tile j, the next column its row gq + 8
#pragma unroll
                for (int kk = 0; kk < 2; ++kk) {
                    if constexpr (!DENSE) {
                        if (!full && ((vis >> (kk * 16)) & 0xffffu) == 0) continue;
                        if ((kk ? odd1 : odd0) >> now & 1u) {
                            const float f = __shfl_sync(0xffffffffu, kk ? lg1 : lg0, now) <= kNoneLog ? 0.0f : -1.0f;
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                                for (int x = 0; x < 4; ++x) s[kk][nt][x] *= f;
                        }
                    }
                    uint32_t p[NT][2], q[NT][2];
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int y = 0; y < 2; ++y) {
                            const float x0 = s[kk][nt][2 * y], x1 = s[kk][nt][2 * y + 1];
                            const uint32_t w = pack2<MMA_BF16>(x0, x1);
                            p[nt][y] = transposed(w);
                            if constexpr (SPLIT_P) {
                                const float2 f = unpack2<MMA_BF16>(w);
                                q[nt][y] = transposed(pack2<MMA_BF16>(x0 - f.x, x1 - f.y));
                            }
                        }
                    uint32_t v[4][WORDS];
#pragma unroll
                    for (int x = 0; x < 4; ++x)
#pragma unroll
                        for (int y = 0; y < PIECES; ++y) lds<PIECE>(vt + (v_at[x & 1] ^ (y * 16)) + (kk * 16 + (x >> 1) * 8) * RB, &v[x][y * 4]);
                    if (!full) {
                        // what absent keys hold may not be a number, which a weight of zero does not make one
#pragma unroll
                        for (int x = 0; x < 4; ++x)
                            if (!((vis >> (kk * 16 + 2 * t4 + (x & 1) + (x >> 1) * 8)) & 1u)) {
#pragma unroll
                                for (int y = 0; y < WORDS; ++y) v[x][y] = 0u;
                            }
                    }
                    auto product = [&](int j, const uint32_t (&f)[4]) {
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) {
                            mma16<MMA_BF16>(o[j][nt], f, p[nt][0], p[nt][1]);
                            if constexpr (SPLIT_P) mma16<MMA_BF16>(o[j][nt], f, q[nt][0], q[nt][1]);
                        }
                    };
                    if constexpr (DENSE) {
#pragma unroll
                        for (int j = 0; j < DT; ++j) {
                            const uint32_t f[4] = {__byte_perm(v[0][j], v[1][j], 0x5410), __byte_perm(v[0][j], v[1][j], 0x7632), __byte_perm(v[2][j], v[3][j], 0x5410),
                                                   __byte_perm(v[2][j], v[3][j], 0x7632)};
                            product(j, f);
                        }
                    } else {
#pragma unroll
                        for (int jw = 0; jw < WORDS; ++jw) {
                            uint32_t f[2][4];
#pragma unroll
                            for (int y = 0; y < 2; ++y) {
                                uint32_t w0 = v[2 * y][jw], w1 = v[2 * y + 1][jw];
                                if constexpr (I8) { w0 ^= 0x80808080u; w1 ^= 0x80808080u; }
                                const uint32_t lo = __byte_perm(w0, w1, 0x5140), hi = __byte_perm(w0, w1, 0x7362);   // (a0 b0 a1 b1), (a2 b2 a3 b3)
                                if constexpr (I8) {
                                    f[0][2 * y] = biased_to_f16x2(__byte_perm(lo, 0x64646464u, 0x4140));
                                    f[0][2 * y + 1] = biased_to_f16x2(__byte_perm(lo, 0x64646464u, 0x4342));
                                    f[1][2 * y] = biased_to_f16x2(__byte_perm(hi, 0x64646464u, 0x4140));
                                    f[1][2 * y + 1] = biased_to_f16x2(__byte_perm(hi, 0x64646464u, 0x4342));
                                } else {
                                    f[0][2 * y] = e4m3x2_to_f16x2(lo);
                                    f[0][2 * y + 1] = e4m3x2_hi_to_f16x2(lo);
                                    f[1][2 * y] = e4m3x2_to_f16x2(hi);
                                    f[1][2 * y + 1] = e4m3x2_hi_to_f16x2(hi);
                                }
                            }
                            product(jw * 2, f[0]);
                            if (jw * 2 + 1 < DT) product(jw * 2 + 1, f[1]);
                        }
                    }
                }
            }
            if (!any && !warp_wait(&s_vfull[slot], parity, abort_flag)) break;
            warp_arrive(&s_vempty[slot]);
        }
        }
        // -------------------------------------------------------------------- the four warps' parts
        __syncthreads();                       // every tile has been read
        float* so = reinterpret_cast<float*>(smem_raw + (ring - raw_addr));
        if (warp < kWarps) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const int r = nt * 8 + 2 * t4 + x;
#pragma unroll
                for (int y = 4; y < 32; y <<= 1) l[nt][x] += __shfl_xor_sync(0xffffffffu, l[nt][x], y);
                if (gq == 0) { s_m[warp][r] = m[nt][x]; s_l[warp][r] = l[nt][x] * kUnshift; }
#pragma unroll
                for (int j = 0; j < DT; ++j) {
                    // (first one, then the other: large values have room, and vref may be as small as numbers get)
                    *reinterpret_cast<float2*>(so + (warp * ROWS + r) * D + gq * (D / 8) + 2 * j) = make_float2(o[j][nt][x] * kUnshift * vref, o[j][nt][x + 2] * kUnshift * vref);
                }
            }
        }
        __syncthreads();
        for (int e = threadIdx.x; e < ROWS * D / 2; e += kRowsThreads) {
            const int r = e / (D / 2), c = e % (D / 2) * 2, row = row0 + r;
            if (row >= rows) break;
            float top = -INFINITY;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) top = fmaxf(top, s_m[w][r]);
            const float ref = top == -INFINITY ? 0.0f : top;
            float sum = 0.0f, x = 0.0f, y = 0.0f;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) {
                const float f = exp2_fast(s_m[w][r] - ref);
                const float2 v = *reinterpret_cast<const float2*>(so + (w * ROWS + r) * D + c);
                sum += s_l[w][r] * f;
                x += v.x * f;
                y += v.y * f;
            }
            const size_t in = (size_t)s_pos[row / a.Tq] * a.Tq + row % a.Tq, out = (size_t)b * a.k_h * a.Tq + in;
            if (share.n == 1) {
                const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
                reinterpret_cast<uint32_t*>(a.O)[(out * D + c) / 2] = pack2<BF16>(sum == 0.0f ? 0.0f : x * inv, sum == 0.0f ? 0.0f : y * inv);
            } else {
                const size_t at = (size_t)(share.first + share.split) * a.k_h * a.Tq + in;
                *reinterpret_cast<float2*>(meet.part + at * D + c) = make_float2(x, y);
                if (c == 0) meet.ml[at] = make_float2(top, sum);
            }
        }
        ptx::fence_proxy_async_smem();          // the next rows' copies come where these parts lay
        __syncthreads();
        if (*abort_flag) break;
    }
    if (share.n > 1) {
        const size_t each = (size_t)a.k_h * a.Tq;
        auto is_last = [&](unsigned int* counter, int of) {
            __threadfence();
            __syncthreads();
            if (threadIdx.x == 0) s_heads = atomicAdd(counter, 1u) == (unsigned)of - 1u;
            __syncthreads();
            if (!s_heads) return false;
            __threadfence();
            if (threadIdx.x == 0) *counter = 0u;
            return true;
        };
        // n parts from part `first` on, into part `to` of the second step, or (to < 0) into the result
        auto join = [&](const float* part, const float2* ml, size_t first, int n, long long to) {
            for (int row0 = blockIdx.y * ROWS; row0 < rows; row0 += gridDim.y * ROWS)
                for (int e = threadIdx.x; e < min(ROWS, rows - row0) * (D / 4); e += kRowsThreads) {
                    const int row = row0 + e / (D / 4), c = e % (D / 4) * 4;
                    const size_t in = (size_t)s_pos[row / a.Tq] * a.Tq + row % a.Tq, from = first * each + in;
                    float2 x;
                    const float4 v = join_parts<D>(part + from * D + c, ml + from, each, n, x);
                    if (to >= 0) {
                        const size_t at = (size_t)to * each + in;
                        *reinterpret_cast<float4*>(meet.part2 + at * D + c) = v;
                        if (c == 0) meet.ml2[at] = x;
                    } else {
                        const float inv = x.y == 0.0f ? 0.0f : 1.0f / x.y;
                        *reinterpret_cast<uint2*>((uint16_t*)a.O + ((size_t)b * each + in) * D + c) =
                            x.y == 0.0f ? make_uint2(0u, 0u) : make_uint2(pack2<BF16>(v.x * inv, v.y * inv), pack2<BF16>(v.z * inv, v.w * inv));
                    }
                }
        };
        unsigned int* own = meet.counters + ((size_t)b * a.Hk + g) * gridDim.y + blockIdx.y;
        if (share.n <= kJoin) {
            if (is_last(own, share.n)) join(meet.part, meet.ml, share.first, share.n, -1);
        } else {
            // (a sample's results of the first step lie behind those of the samples before: that many are enough for all)
            const int sets = (share.n + kJoin - 1) / kJoin, set = share.split / kJoin, to = share.first / kJoin + b;
            unsigned int* counter = meet.counters + ((size_t)(a.B + to + set) * a.Hk + g) * gridDim.y + blockIdx.y;
            const int n = min(kJoin, share.n - set * kJoin);
            if (is_last(counter, n)) {
                join(meet.part, meet.ml, share.first + set * kJoin, n, to + set);
                if (is_last(own, sets)) join(meet.part2, meet.ml2, to, sets, -1);
            }
        }
    }
    if (*abort_flag) {
        if (threadIdx.x == 0) atomicOr(a.status, SENTRY_STATUS_BIT_TIMEOUT);
        const long long start = clock64();      // copies that are still on their way land before the shared memory goes
        while (clock64() - start < 2000000LL) __nanosleep(1000);
    }
}

// Tiles of rows: 8 where a group has no more, else 16.
int rows_tile(const KvAttendArgs& a) {
    const int per = a.Hq / a.Hk, heads = per < a.k_h ? per : a.k_h;
    return (long long)heads * a.Tq <= 8 ? 8 : 16;
}
long long rows_tiles(const KvAttendArgs& a) {
    const int per = a.Hq / a.Hk, heads = per < a.k_h ? per : a.k_h, tile = rows_tile(a);
    const long long n = ((long long)heads * a.Tq + tile - 1) / tile;
    return n < 64 ? n : 64;
}
// Blocks that one wave holds for every row tile (RowsCfg::BLOCKS an SM); 0: the groups alone fill it, and no axis is split.
int rows_wave(const KvAttendArgs& a) {
    const int tile = kKeys * a.d * (a.format == 0 ? 2 : 1);
    const int blocks = tile > 4096 ? 2 : (tile > 2048 ? 3 : 4) - (rows_tile(a) > 8);
    const long long slots = blocks * kSmCount, wave = rows_tiles(a) > 0 ? slots / rows_tiles(a) : 0;
    return a.B < wave / a.Hk && a.Tk > kWarps * kKeys ? (int)wave : 0;
}

// Parts of the second step of the joining: those of all samples, a last one with fewer than kJoin for each.
// (2 B + parts / kJoin counters of every group's row tile, and B of those are less than a wave's blocks.)
static_assert(2 * 4 * kSmCount + 4 * kSmCount / kJoin <= kCounters, "counters");
size_t rows_parts2(const KvAttendArgs& a, int wave) { return (size_t)(wave / a.Hk / kJoin + a.B); }

template <int KV, int D, bool BF16, int NT>
int launch_rows(sentry_ctx* ctx, const KvAttendArgs& a, WsAlloc& ws, cudaStream_t st) {
    using C = RowsCfg<KV, D>;
    const int wave = rows_wave(a);
    RowsJoin meet = {};
    if (wave > 0) {
        const size_t rows = (size_t)a.k_h * a.Tq;
        meet.part = ws.take<float>(wave / a.Hk * rows * D);
        meet.ml = ws.take<float2>(wave / a.Hk * rows);
        meet.part2 = ws.take<float>(rows_parts2(a, wave) * rows * D);
        meet.ml2 = ws.take<float2>(rows_parts2(a, wave) * rows);
        meet.counters = ctx->d_counters;
        meet.room = wave / a.Hk - a.B;
        if (!ws.ok) return SENTRY_ERR_WORKSPACE;
    }
    KvMaps maps = {};
    if (KV <= KV_F16 ? a.Tk > 0 && (!make_map_dense(&maps.k, a.K, a, a.ks, kKeys) || !make_map_dense(&maps.v, a.V, a, a.vs, kKeys))
                     : a.n_pages > 0 && (!make_map_codes(&maps.k, a.K, a, a.page < kKeys ? a.page : kKeys) || !make_map_codes(&maps.v, a.V, a, a.page < kKeys ? a.page : kKeys)))
        return SENTRY_ERR_CUDA;
    auto k = kv_rows_kernel<KV, D, BF16, NT>;
    static std::atomic<unsigned long long> allowed{0};
    SENTRY_CUDA_TRY(allow_smem(k, C::SMEM, ctx->device, allowed));
    {
        LaunchScope ls(ctx, KS_KV_ATTEND, st);
        SENTRY_CUDA_TRY(launch_chained(k, dim3((unsigned)(wave > 0 ? wave / a.Hk * a.Hk : a.B * a.Hk), (unsigned)rows_tiles(a)), dim3(kRowsThreads), C::SMEM, st, maps, a, meet));
    }
    return SENTRY_OK;
}

template <int KV, int D, bool BF16>
int launch_nt(sentry_ctx* ctx, const KvAttendArgs& a, WsAlloc& ws, cudaStream_t st) {
    return rows_tile(a) == 8 ? launch_rows<KV, D, BF16, 1>(ctx, a, ws, st) : launch_rows<KV, D, BF16, 2>(ctx, a, ws, st);
}

template <int KV, bool BF16>
int launch_d(sentry_ctx* ctx, const KvAttendArgs& a, WsAlloc& ws, cudaStream_t st) {
    switch (a.d) {
        case 16: return launch_nt<KV, 16, BF16>(ctx, a, ws, st);
        case 32: return launch_nt<KV, 32, BF16>(ctx, a, ws, st);
        case 64: return launch_nt<KV, 64, BF16>(ctx, a, ws, st);
        default: return launch_nt<KV, 128, BF16>(ctx, a, ws, st);
    }
}

}  // namespace

size_t kv_rows_ws_bytes(const KvAttendArgs& a) {
    const int wave = rows_wave(a);
    if (wave == 0) return 0;
    const size_t rows = (size_t)a.k_h * a.Tq;
    size_t bytes = 512;
    for (const size_t parts : {(size_t)(wave / a.Hk), rows_parts2(a, wave)})
        bytes += align_up(parts * rows * a.d * sizeof(float), 256) + align_up(parts * rows * sizeof(float2), 256);
    return bytes;
}

int launch_kv_rows(sentry_ctx* ctx, const KvAttendArgs& a, WsAlloc& ws, cudaStream_t st) {
    const bool bf16 = a.dtype == SENTRY_BF16;
    if (a.format == 0) return bf16 ? launch_d<KV_BF16, true>(ctx, a, ws, st) : launch_d<KV_F16, false>(ctx, a, ws, st);
    if (a.format == SENTRY_FP8_E4M3) return bf16 ? launch_d<KV_E4M3, true>(ctx, a, ws, st) : launch_d<KV_E4M3, false>(ctx, a, ws, st);
    return bf16 ? launch_d<KV_I8, true>(ctx, a, ws, st) : launch_d<KV_I8, false>(ctx, a, ws, st);
}
