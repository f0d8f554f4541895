// Serving attention for few rows: a decoder's single tokens and short blocks, over dense 16-bit keys and values or the 8-bit cache.
//
// The rows of one KV group (kept heads x Tq) share its keys, so they are packed into tiles of 8 or 16 rows, and a block takes a tile and a
// stretch of the keys.  Each of its four warps walks tiles of 32 keys by itself, with a ring of asynchronous copies of its own, a running
// maximum and sum of its own (log2 domain), and both products on the warp MMA: no barrier until the four partial results meet.
// Long axes are split over blocks; kv_combine_kernel joins the parts.
// The keys are the MMA's 16 rows and the queries its 8 columns (S^T = K Q^T, O^T = V^T P^T): a decoder's few rows fill it, where queries as
// rows left half of it and half of the exponentials empty (two hours of cached tokens 31 us so, with 840 instructions a tile of 4 KB).
// What bounds it: the bytes of K and V, read once from memory.  For that the codes go through registers straight into MMA operands:
// the order of the inner index is free as long as both operands share it, so that a lane's 16 consecutive bytes of a key are its operand
// for K's product; and for V's, where pairs run along the keys, two keys' words are interleaved byte by byte.  The weights get from the
// first product's layout to the second's by a transposition of 8 x 8 matrices among registers.  8-bit codes become fp16 exactly; a
// page's key scale multiplies the scores, its value scale the weights.  The maximum is followed only where a score exceeds it by 2^8.
#include "kv_attend.cuh"
#include "ptx/sm100.cuh"

namespace {

constexpr int kWarps = 4, kKeys = 32;
constexpr float kLog2e = 1.4426950408889634f;

enum { KV_BF16 = 0, KV_F16 = 1, KV_E4M3 = 2, KV_I8 = 3 };

template <int KV, int D>
struct RowsCfg {
    static constexpr int ESIZE = KV <= KV_F16 ? 2 : 1;
    static constexpr int ROW = D * ESIZE;                    // bytes of a key
    static constexpr int CHUNKS = ROW / 16;
    static constexpr int STAGE = 2 * kKeys * ROW;            // K and V of a tile
    // Two tiles of copies on the way for every warp at least, and as many blocks on an SM as that leaves room for.
    static constexpr int FIT = 49152 / (kWarps * STAGE);
    static constexpr int STAGES = FIT < 2 ? (STAGE > 8192 ? 3 : 2) : FIT > 4 ? 4 : FIT;
    static constexpr int BLOCKS = STAGE > 8192 ? 1 : FIT < 2 ? 3 : 4;
    static constexpr int RING = kWarps * STAGES * STAGE;
    static constexpr int MERGE = kWarps * 16 * D * 4;
    static constexpr int SMEM = RING > MERGE ? RING : MERGE;
};

// Piece c of key r lies at piece c ^ bank_shift(r) of its row: lanes that read one piece number of eight keys, or several of one, meet
// different banks.  (Linear over XOR in the bits of r, so that constant parts of r shift by constants.)
template <int CHUNKS>
__host__ __device__ __forceinline__ constexpr int bank_shift(int r) {
    return ((((r >> 1) & 3) * 2) ^ ((r & 1) * 4)) & (CHUNKS - 1);
}
__device__ __forceinline__ void cp_async_16_full(uint32_t dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async_16_or_zero(uint32_t dst, const void* src, bool yes) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(yes ? 16 : 0) : "memory");
}
__device__ __forceinline__ void cp_async_4(uint32_t dst, const void* src) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
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
// two codes in the low 16 bits of w -> fp16 pair
__device__ __forceinline__ uint32_t e4m3x2_to_f16x2(uint32_t w) {
    uint32_t r;
    asm("{\n\t.reg .b16 lo, hi;\n\tmov.b32 {lo, hi}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, lo;\n\t}" : "=r"(r) : "r"(w));
    return r;
}
__device__ __forceinline__ uint32_t e4m3x2_hi_to_f16x2(uint32_t w) {
    uint32_t r;
    asm("{\n\t.reg .b16 lo, hi;\n\tmov.b32 {lo, hi}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, hi;\n\t}" : "=r"(r) : "r"(w));
    return r;
}
// bytes (already + 128) -> fp16: 0x6400 | u is 1024 + u, exactly
__device__ __forceinline__ uint32_t biased_to_f16x2(uint32_t pair) {
    const uint32_t bias = 0x64806480u;   // 1152
    uint32_t r;
    asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(pair), "r"(bias));
    return r;
}
// four codes of a word, in order, as two fp16 pairs
template <bool I8>
__device__ __forceinline__ void codes_to_f16(uint32_t w, uint32_t& p01, uint32_t& p23) {
    if constexpr (I8) {
        const uint32_t u = w ^ 0x80808080u;
        p01 = biased_to_f16x2(__byte_perm(u, 0x64646464u, 0x4140));
        p23 = biased_to_f16x2(__byte_perm(u, 0x64646464u, 0x4342));
    } else {
        p01 = e4m3x2_to_f16x2(w);
        p23 = e4m3x2_hi_to_f16x2(w);
    }
}

// 8 x 8 matrix of 16-bit values spread over a warp (a row's pairs over four lanes), transposed
__device__ __forceinline__ uint32_t transposed(uint32_t x) {
    uint32_t r;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
    return r;
}

struct RowsMeta { float ks[2], vs[2]; unsigned vis; };

// Which stretch of which sample's keys a block takes.  The samples' lengths differ and only the device knows them, so that every block works
// out the same shares: stretches of `chunk` tiles, as many blocks to a sample as it has of them (one at least), so that all fit one wave.
struct RowsShare { int b, split, n, first; };   // first: number of the sample's first part among all samples' parts
__device__ __forceinline__ RowsShare rows_share(const KvAttendArgs& a, int unit, int room, int& chunk) {
    const int lane = threadIdx.x & 31;
    auto tiles_of = [&](int b) { return b < a.B ? (kv_length(a, b) + kKeys - 1) / kKeys : 0; };
    int sum = 0;
#pragma unroll 4
    for (int b0 = 0; b0 < a.B; b0 += 32) sum += tiles_of(b0 + lane);
    const long long total = (long long)__reduce_add_sync(0xffffffffu, sum >> 8) * 256 + __reduce_add_sync(0xffffffffu, sum & 255);
    chunk = (int)((total + room - 1) / room);
    chunk = max((chunk + kWarps - 1) / kWarps * kWarps, kWarps);
    RowsShare r = {-1, 0, 0, 0};
    int base = 0;
    for (int b0 = 0; b0 < a.B; b0 += 32) {
        const int b = b0 + lane, n = b < a.B ? max(1, (tiles_of(b) + chunk - 1) / chunk) : 0;
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
            r.split = unit - r.first;
            break;
        }
        base += __shfl_sync(0xffffffffu, incl, 31);
    }
    return r;
}

// KV: type of the keys and values; BF16: type of Q and O; NT: tiles of 8 rows a block takes at a time.
// room: 0: a block per group and row tile takes all of its keys.  Otherwise the keys are shared out (rows_share), part: [parts][k_h][Tq][D] sums,
// ml: [parts][k_h][Tq] (maximum, total), and plan: [B] (first part, parts) for those who join them.
template <int KV, int D, bool BF16, int NT>
__global__ void __launch_bounds__(kWarps * 32, NT == 1 ? RowsCfg<KV, D>::BLOCKS : RowsCfg<KV, D>::BLOCKS < 3 ? 1 : 3)
kv_rows_kernel(const KvAttendArgs a, float* __restrict__ part, float2* __restrict__ ml, int2* __restrict__ plan, int room) {
    using C = RowsCfg<KV, D>;
    constexpr bool DENSE = KV <= KV_F16, I8 = KV == KV_I8;
    constexpr bool MMA_BF16 = KV == KV_BF16;
    constexpr bool SPLIT_P = DENSE || !BF16;                 // weights as a head and a remainder
    constexpr int KSTEPS = D / 16, DT = D / 16, ROWS = 8 * NT;
    extern __shared__ __align__(16) uint8_t smem[];
    __shared__ RowsMeta s_meta[kWarps][C::STAGES];
    __shared__ short s_head[kServeMaxHeads], s_pos[kServeMaxHeads];
    __shared__ int s_heads;
    __shared__ float s_m[kWarps][ROWS], s_l[kWarps][ROWS];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, gq = lane >> 2, t4 = lane & 3;
    const int g = blockIdx.x % a.Hk;
    grid_dependents_start_if_small();
    grid_dependency_wait();
    RowsShare share = {(int)blockIdx.x / a.Hk, 0, 1, 0};
    int chunk = 0x7fffffff / kKeys;
    if (room > 0) share = rows_share(a, blockIdx.x / a.Hk, room, chunk);   // (every warp for itself)
    if (share.b < 0) return;
    const int b = share.b;
    if (warp == 0) {
        const int n = kv_group_heads(a, b, g, g == 0 && share.split == 0 && blockIdx.y == 0, s_head, s_pos);
        if (lane == 0) s_heads = n;
        if (room > 0 && lane == 0 && share.split == 0 && g == 0 && blockIdx.y == 0) plan[b] = make_int2(share.first, share.n);
    }
    const int len = kv_length(a, b);
    const uint32_t mask = a.masks ? a.masks[b] : 0u;
    __syncthreads();
    const int rows = s_heads * a.Tq;
    const int tiles = (len + kKeys - 1) / kKeys;
    const int t0 = min(share.split * chunk, tiles), t1 = min(t0 + chunk, tiles);
    const uint32_t ring = ptx::smem_u32(smem) + warp * C::STAGES * C::STAGE;
    RowsMeta* meta = s_meta[warp];
    const char *kbase, *vbase;
    if constexpr (DENSE) {
        kbase = (const char*)a.K + (b * a.ks[0] + g * a.ks[1]) * 2;
        vbase = (const char*)a.V + (b * a.vs[0] + g * a.vs[1]) * 2;
    } else {
        kbase = (const char*)a.K;
        vbase = (const char*)a.V;
    }
    const int page_shift = DENSE ? 0 : 31 - __clz(a.page);
    const int32_t* pages = DENSE ? nullptr : a.table + (size_t)b * a.max_pages;

    for (int row0 = blockIdx.y * ROWS; row0 < rows; row0 += gridDim.y * ROWS) {
        // -------------------------------------------------------------------- copies
        // `ahead`: the modality id, or the page, of this lane's key of the tile that is issued next
        auto look_ahead = [&](int tile) -> int {
            const int n = tile * kKeys + lane;
            if (tile >= t1 || n >= len) return -1;
            if constexpr (DENSE) return a.ids ? a.ids[n] : 0;
            else return pages[n >> page_shift];
        };
        // where this lane's first piece of a tile goes, and the distance between its pieces (32 lanes x 16 bytes: 32 / CHUNKS keys)
        constexpr int RPI = 32 / C::CHUNKS;
        const int my_row = lane / C::CHUNKS, my_chunk = lane % C::CHUNKS;
        const int my_dst = my_row * C::ROW + ((my_chunk ^ bank_shift<C::CHUNKS>(my_row)) << 4);
        // K's and V's copies of a tile are two groups: the slot of K is free, and filled again, half a tile before that of V
        int next = t0 + warp, next_slot = 0, ahead = look_ahead(next);
        unsigned next_vis = 0;
        // this lane's first piece of the tile: of a dense tensor, or of a page and group (the pieces of a page's tile follow one another)
        const char *k_first = kbase, *v_first = vbase;
        long long k_step = 0, v_step = 0;
        unsigned id[2] = {0, 0}, in_page = 0;                         // pages of the tile's first 16 keys and of the others; bytes into the first
        if constexpr (DENSE) {
            k_step = a.ks[2] * 2; v_step = a.vs[2] * 2;
            k_first += my_row * k_step + my_chunk * 16;
            v_first += my_row * v_step + my_chunk * 16;
        } else {
            k_first += (long long)(g << page_shift) * D + (C::CHUNKS > 1 ? lane : lane & 15) * 16;
            v_first += (long long)(g << page_shift) * D + (C::CHUNKS > 1 ? lane : lane & 15) * 16;
        }
        const unsigned page_bytes = DENSE ? 0u : (unsigned)(a.Hk << page_shift) * D;    // of all groups: below 2^32
        auto issue = [&](bool is_v) {
            if (next < t1) {
                const uint32_t dst = ring + next_slot * C::STAGE + (is_v ? kKeys * C::ROW : 0);
                const int n0 = next * kKeys;
                if (!is_v) {
                    RowsMeta* mt = meta + next_slot;
                    bool ok = n0 + lane < len;
                    if constexpr (DENSE) ok = ok && (a.ids == nullptr || kv_present(ahead, mask));
                    else {
                        const bool good = (unsigned)ahead < (unsigned)a.n_pages;
                        if (ok && !good) atomicOr(a.status, SENTRY_STATUS_BIT_BAD_INDEX);
                        ok = ok && good;
                    }
                    next_vis = __ballot_sync(0xffffffffu, ok);
                    if (lane == 0) mt->vis = next_vis;
                    if constexpr (!DENSE) {
                        if ((lane & 15) == 0 && ok) {
                            const size_t ph = (size_t)(unsigned)ahead * (unsigned)a.Hk + g;
                            cp_async_4(ptx::smem_u32(&mt->ks[lane >> 4]), a.k_scales + ph);
                            cp_async_4(ptx::smem_u32(&mt->vs[lane >> 4]), a.v_scales + ph);
                        }
                        id[0] = __shfl_sync(0xffffffffu, ahead, 0);
                        id[1] = __shfl_sync(0xffffffffu, ahead, 16);
                        in_page = (unsigned)(n0 & (a.page - 1)) * D;
                    }
                }
                if (next_vis != 0) {
                    const char* base = is_v ? vbase : kbase;
                    const char* first = is_v ? v_first : k_first;
                    const long long step = is_v ? v_step : k_step;
                    const char *lo = first, *hi = first;
                    if constexpr (DENSE) lo += n0 * step;
                    else {
                        lo += (unsigned long long)id[0] * page_bytes + in_page;
                        hi = a.page == 16 ? first + (unsigned long long)id[1] * page_bytes : lo + 16 * D;
                    }
                    auto piece = [&](int i, const char*& src) {
                        if constexpr (DENSE) src = lo + i * RPI * step;
                        else if constexpr (C::CHUNKS == 1) src = lane < 16 ? lo : hi;
                        else src = i < C::CHUNKS / 2 ? lo + i * 512 : hi + (i - C::CHUNKS / 2) * 512;
                        return dst + (my_dst ^ (bank_shift<C::CHUNKS>(i * RPI) << 4)) + i * 512;
                    };
                    const char* src;
                    if (next_vis == 0xffffffffu) {
#pragma unroll
                        for (int i = 0; i < C::CHUNKS; ++i) {
                            const uint32_t at = piece(i, src);
                            cp_async_16_full(at, src);
                        }
                    } else {
#pragma unroll 1
                        for (int i = 0; i < C::CHUNKS; ++i) {
                            const uint32_t at = piece(i, src);
                            const bool yes = (next_vis >> (i * RPI + my_row)) & 1u;
                            cp_async_16_or_zero(at, yes ? src : base, yes);
                        }
                    }
                }
                if (is_v) {
                    next += kWarps;
                    next_slot = next_slot + 1 == C::STAGES ? 0 : next_slot + 1;
                    ahead = look_ahead(next);
                }
            }
            ptx::cp_async_commit();
        };
#pragma unroll 1
        for (int s = 0; s < C::STAGES; ++s) { issue(false); issue(true); }

        // -------------------------------------------------------------------- rows of Q as MMA operands: lane (gq, t4) has row gq of every eight
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
        float o[DT][NT][4], m[NT][2], l[NT][2];
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
        const int k_at = gq * C::ROW + ((((t4 * KB) >> 4) ^ bank_shift<C::CHUNKS>(gq)) << 4) + ((t4 * KB) & 15);
        int v_at[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) v_at[u] = (2 * t4 + u) * C::ROW + ((((gq * VB) >> 4) ^ bank_shift<C::CHUNKS>(2 * t4 + u)) << 4) + ((gq * VB) & 15);
        // keys below this are seen by every row of the warp
        int all_see = len;
        if (!DENSE && a.causal) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) all_see = min(all_see, min(last[nt][0], last[nt][1]));
            all_see = __reduce_min_sync(0xffffffffu, all_see);
        }
        float vref = 0.0f, inv_vref = 0.0f;                         // O is in units of vref (8-bit values; see below)

        // -------------------------------------------------------------------- tiles of 32 keys
        int slot = 0;
        for (int tile = t0 + warp; tile < t1; tile += kWarps) {
            ptx::cp_async_wait_group<2 * C::STAGES - 1>();
            __syncwarp();
            const int n0 = tile * kKeys;
            const uint32_t kt = ring + slot * C::STAGE, vt = kt + kKeys * C::ROW;
            const unsigned vis = meta[slot].vis;
            const float vscale[2] = {DENSE ? 1.0f : meta[slot].vs[0], DENSE ? 1.0f : meta[slot].vs[1]};
            const bool full = vis == 0xffffffffu && n0 + kKeys <= all_see;
            float s[2][NT][4];
            if (vis != 0) {
                // ------ scores: element (key mt * 16 + gq + 8 * (x >> 1), row nt * 8 + 2 t4 + (x & 1))
#pragma unroll
                for (int mt = 0; mt < 2; ++mt) {
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int x = 0; x < 4; ++x) s[mt][nt][x] = 0.0f;
#pragma unroll
                    for (int c = 0; c < (C::CHUNKS + 3) / 4; ++c) {
                        uint32_t w0[4], w1[4];                      // keys gq and gq + 8
                        lds<KB>(kt + (k_at ^ (c * 64)) + mt * 16 * C::ROW, w0);
                        lds<KB>(kt + (k_at ^ (c * 64)) + (mt * 16 + 8) * C::ROW, w1);
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
                    const float ks = DENSE ? 1.0f : meta[slot].ks[mt];
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        const float c0 = scale[nt][0] * ks, c1 = scale[nt][1] * ks;
#pragma unroll
                        for (int x = 0; x < 4; ++x) s[mt][nt][x] *= x & 1 ? c1 : c0;
                    }
                }
            }
            __syncwarp();
            issue(false);
            if (vis != 0) {
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
                        over = over || top - m[nt][x] > 8.0f;
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
                            top = fmaxf(top, m[nt][x]);
                            keep[x] = top == m[nt][x] ? 1.0f : exp2_fast(m[nt][x] - top);
                            m[nt][x] = top;
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
                    const float ref[2] = {m[nt][0] == -INFINITY ? 0.0f : m[nt][0], m[nt][1] == -INFINITY ? 0.0f : m[nt][1]};
#pragma unroll
                    for (int mt = 0; mt < 2; ++mt)
#pragma unroll
                        for (int x = 0; x < 4; ++x) {
                            s[mt][nt][x] = exp2_fast(s[mt][nt][x] - ref[x & 1]);
                            l[nt][x & 1] += s[mt][nt][x];
                        }
                }
                ptx::cp_async_wait_group<2 * C::STAGES - 1>();
                __syncwarp();
                // ------ values, 16 keys at a time: column gq * (D / 8) + 2 j is row gq of the MMA's tile j, the next column its row gq + 8
#pragma unroll
                for (int kk = 0; kk < 2; ++kk) {
                    if constexpr (!DENSE) {
                        // The page's scale multiplies the weights, as a ratio to vref; where it is far from that, O changes its unit.
                        // (A page 2^64 times smaller leaves it: its values are nothing beside what O may hold.)
                        if (((vis >> (kk * 16)) & 0xffffu) == 0) continue;
                        const float vs = vscale[kk];
                        float ratio = vs * inv_vref;
                        if (!(fabsf(ratio) >= 0.0625f && fabsf(ratio) <= 16.0f)) {
                            if (!(fabsf(vs) <= 3.4028234e38f)) ratio = __int_as_float(0x7fc00000);
                            else if (fabsf(vs) >= fmaxf(1.17549435e-38f, fabsf(vref) * 5.42101086e-20f)) {
                                const float f = vref / vs;
#pragma unroll
                                for (int j = 0; j < DT; ++j)
#pragma unroll
                                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                                        for (int x = 0; x < 4; ++x) o[j][nt][x] *= f;
                                vref = vs;
                                inv_vref = 1.0f / vs;
                                ratio = 1.0f;
                            }
                        }
                        if (full) {
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                                for (int x = 0; x < 4; ++x) s[kk][nt][x] *= ratio;
                        } else {
                            // (a row that sees nothing of the page takes nothing of its scale, which may not be a number)
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                                for (int x = 0; x < 4; ++x) s[kk][nt][x] = s[kk][nt][x] != 0.0f ? s[kk][nt][x] * ratio : 0.0f;
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
                        for (int y = 0; y < PIECES; ++y) lds<PIECE>(vt + (v_at[x & 1] ^ (y * 16)) + (kk * 16 + (x >> 1) * 8) * C::ROW, &v[x][y * 4]);
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
            __syncwarp();
            issue(true);
            slot = slot + 1 == C::STAGES ? 0 : slot + 1;
        }
        ptx::cp_async_wait_all();
        // -------------------------------------------------------------------- the four warps' parts
        __syncthreads();                       // every ring has been read
        float* so = reinterpret_cast<float*>(smem);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const int r = nt * 8 + 2 * t4 + x;
#pragma unroll
                for (int y = 4; y < 32; y <<= 1) l[nt][x] += __shfl_xor_sync(0xffffffffu, l[nt][x], y);
                if (gq == 0) { s_m[warp][r] = m[nt][x]; s_l[warp][r] = l[nt][x]; }
#pragma unroll
                for (int j = 0; j < DT; ++j) {
                    const float f = DENSE ? 1.0f : vref;
                    *reinterpret_cast<float2*>(so + (warp * ROWS + r) * D + gq * (D / 8) + 2 * j) = make_float2(o[j][nt][x] * f, o[j][nt][x + 2] * f);
                }
            }
        __syncthreads();
        for (int e = threadIdx.x; e < ROWS * D / 2; e += kWarps * 32) {
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
                *reinterpret_cast<float2*>(part + at * D + c) = make_float2(x, y);
                if (c == 0) ml[at] = make_float2(top, sum);
            }
        }
        __syncthreads();
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
    const int stage = 2 * kKeys * a.d * (a.format == 0 ? 2 : 1);
    const long long slots = (stage > 8192 ? 1 : stage > 6144 || rows_tile(a) > 8 ? 3 : 4) * kSmCount, wave = rows_tiles(a) > 0 ? slots / rows_tiles(a) : 0;
    return a.B < wave / a.Hk && a.Tk > kWarps * kKeys ? (int)wave : 0;
}

template <int KV, int D, bool BF16, int NT>
int launch_rows(sentry_ctx* ctx, const KvAttendArgs& a, WsAlloc& ws, cudaStream_t st) {
    using C = RowsCfg<KV, D>;
    const int wave = rows_wave(a), room = wave / a.Hk - a.B;      // parts beside the first of every sample
    const size_t rows = (size_t)a.k_h * a.Tq;
    float* part = nullptr;
    float2* ml = nullptr;
    int2* plan = nullptr;
    if (wave > 0) {
        part = ws.take<float>(wave / a.Hk * rows * D);
        ml = ws.take<float2>(wave / a.Hk * rows);
        plan = ws.take<int2>(a.B);
        if (!ws.ok) return SENTRY_ERR_WORKSPACE;
    }
    auto k = kv_rows_kernel<KV, D, BF16, NT>;
    static std::atomic<unsigned long long> allowed{0};
    SENTRY_CUDA_TRY(allow_smem(k, C::SMEM, ctx->device, allowed));
    {
        LaunchScope ls(ctx, KS_KV_ATTEND, st);
        SENTRY_CUDA_TRY(launch_chained(k, dim3((unsigned)(wave > 0 ? wave / a.Hk * a.Hk : a.B * a.Hk), (unsigned)rows_tiles(a)), dim3(kWarps * 32), C::SMEM, st, a, part, ml,
                                       plan, wave > 0 ? room : 0));
    }
    return wave > 0 ? launch_kv_combine(ctx, a, part, ml, plan, 0, st) : SENTRY_OK;
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
    const size_t parts = wave / a.Hk, rows = (size_t)a.k_h * a.Tq;
    return align_up(parts * rows * a.d * sizeof(float), 256) + align_up(parts * rows * sizeof(float2), 256) + a.B * sizeof(int2) + 512;
}

int launch_kv_rows(sentry_ctx* ctx, const KvAttendArgs& a, WsAlloc& ws, cudaStream_t st) {
    const bool bf16 = a.dtype == SENTRY_BF16;
    if (a.format == 0) return bf16 ? launch_d<KV_BF16, true>(ctx, a, ws, st) : launch_d<KV_F16, false>(ctx, a, ws, st);
    if (a.format == SENTRY_FP8_E4M3) return bf16 ? launch_d<KV_E4M3, true>(ctx, a, ws, st) : launch_d<KV_E4M3, false>(ctx, a, ws, st);
    return bf16 ? launch_d<KV_I8, true>(ctx, a, ws, st) : launch_d<KV_I8, false>(ctx, a, ws, st);
}
