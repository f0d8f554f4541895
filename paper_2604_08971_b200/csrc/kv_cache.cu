// Storing keys and values in an 8-bit paged cache: codes with one scale per page (a block of tokens) and KV head.
//
// A block takes a few pages of one sample (all heads): it finds the present tokens that land there, and its warps, one or a few together, take
// K or V of one head of one page at a time: the largest magnitude, the page's scale, the codes.  Bound by the bytes of K and V: a warp has all loads of its
// rows on the way at once (up to kHold pieces of 16 bytes a lane).  32 x 2048 tokens of four heads, d 128, with absent modalities, bf16 -> i8
// (67 MB read, 34 written): 26.6 us, 3.8 TB/s, half of the issue slots; one new token of 32 samples: 3.3 us.
#include <cuda_fp8.h>

#include <type_traits>

#include "append_team.cuh"
#include "serving.cuh"

namespace {

constexpr int kAppPages = 4;      // of a block, at most

__device__ __forceinline__ float nan_f32() { return __int_as_float(0x7fc00000); }

// The scale under which `top` is coded: see sentry_cache_append.
template <bool I8>
__device__ __forceinline__ float page_scale(float top) {
    if (isnan(top)) return top;
    if constexpr (I8) return scale_i8(top);
    if (!(top > 0.0f)) return 0.0f;
    int e;
    const float m = frexpf(top, &e);     // top = m 2^e, 1/2 <= m < 1; 448 = 7/8 2^9
    return ldexpf(1.0f, max(e - (m > 0.875f ? 8 : 9), -126));
}
__device__ __forceinline__ uint32_t e4m3x2(float lo, float hi) {
    return (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(lo, hi), __NV_SATFINITE, __NV_E4M3);
}
// The e4m3 code nearest to q, where a rounding to fp32 on the way could decide a tie.
__device__ __noinline__ uint32_t e4m3_of(double q) {
    int e;
    frexp(q, &e);
    const double step = ldexp(1.0, max(e, -5) - 4);
    return (uint32_t)__nv_cvt_float_to_fp8((float)(rint(q / step) * step), __NV_SATFINITE, __NV_E4M3);
}
// N values under scale s (0 or not a number: zero codes).  This library's e4m3 scales are powers of two, so that x / s = x * inv is
// exact but for results below e4m3's smallest step, which round to 0 or to it either way; a scale of somebody else's need not be one.
template <bool I8, bool CHECK, int N>
__device__ __forceinline__ void codes_of(const float (&x)[N], float s, float inv, uint32_t (&w)[N / 4]) {
#pragma unroll
    for (int i = 0; i < N / 4; ++i) w[i] = 0u;
    if (!(s >= 1.17549435e-38f)) return;
    if constexpr (I8) codes_i8<CHECK, N>(x, s, inv, w);
    else if (__float_as_uint(s) & 0x7fffffu) {
#pragma unroll
        for (int i = 0; i < N; ++i) w[i / 4] |= e4m3_of((double)x[i] / (double)s) << (8 * (i & 3));
    } else {
#pragma unroll
        for (int i = 0; i < N / 4; ++i) w[i] = e4m3x2(x[4 * i] * inv, x[4 * i + 1] * inv) | (e4m3x2(x[4 * i + 2] * inv, x[4 * i + 3] * inv) << 16);
    }
}
// A stored code under a larger scale: code * old / now to the nearest code.  (Doubles hold the product exactly, and the quotient to
// more places than a tie can differ by; rare, so its cost does not matter.)
template <bool I8>
__device__ uint8_t again(uint8_t c, float old, float now) {
    if (!(now > 0.0f)) return 0;
    if constexpr (I8) {
        const double q = rint((double)(int8_t)c * (double)old / (double)now);
        return (uint8_t)(int8_t)(int)fmin(fmax(q, -127.0), 127.0);
    } else {
        const __half_raw h = __nv_cvt_fp8_to_halfraw(c, __NV_E4M3);
        return (uint8_t)e4m3_of((double)__half2float(__half(h)) * (double)old / (double)now);
    }
}

template <typename T, bool I8>
__global__ void __launch_bounds__(kAppThreads, 3) cache_append_kernel(const AppendArgs a, int page_blocks, int pages) {
    constexpr int N = Vec16<T>::N;
    __shared__ int s_token[kAppPages * 128], s_id[kAppPages];
    __shared__ uint32_t s_top[kAppThreads / 32];
    __shared__ int s_count[kAppThreads / 32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int b = blockIdx.x / page_blocks, pb = blockIdx.x % page_blocks;
    const int page = a.c.page, T_ = a.d.T, Hk = a.c.Hk, d = a.c.d;
    grid_dependents_start_if_small();
    grid_dependency_wait();
    const int cap = a.c.max_pages * page;
    const int given = a.lengths[b];
    const bool sane = given >= 0 && given <= cap;
    const int len = min(max(given, 0), cap);
    const int most = a.token_lengths ? min(max(a.token_lengths[b], 0), T_) : T_;
    // this block's pages: from `at0` on, `pages` of them; the present tokens of ranks from start - len on lie there
    const int at0 = len / page + pb * pages;
    const int start = max(at0 * page, len), window = pages * page;
    int total = most;                                      // present tokens of the sample
    if (a.ids != nullptr) {
        // a warp counts a stretch of the tokens, then notes those of its own that these pages take
        const uint32_t mask = a.masks[b];
        const int per = ((most + kAppThreads - 1) / kAppThreads) * 32;
        const int w0 = min(warp * per, most), w1 = min(w0 + per, most);
        auto here = [&](int t) {
            const int m = t < w1 ? a.ids[t] : -1;
            return __ballot_sync(0xffffffffu, (unsigned)m < 32u && ((mask >> (m & 31)) & 1u));
        };
        int mine = 0;
#pragma unroll 4
        for (int t = w0; t < w1; t += 32) mine += __popc(here(t + lane));
        if (lane == 0) s_count[warp] = mine;
        __syncthreads();
        int r = 0;
        total = 0;
#pragma unroll
        for (int w = 0; w < kAppThreads / 32; ++w) { if (w < warp) r += s_count[w]; total += s_count[w]; }
        const int r0 = start - len;
        if (r < r0 + window && r + mine > r0)
            for (int t = w0; t < w1 && r < r0 + window; t += 32) {
                const unsigned bits = here(t + lane);
                const int at_rank = r + __popc(bits & ((1u << lane) - 1u)) - r0;
                if (((bits >> lane) & 1u) && at_rank >= 0 && at_rank < window) s_token[at_rank] = t + lane;
                r += __popc(bits);
            }
    }
    const int room = sane ? cap - len : 0, put = min(total, room);
    if (pb == 0 && threadIdx.x == 0) {
        a.new_lengths[b] = len + put;
        if (put < total || !sane) atomicOr(a.status, SENTRY_STATUS_BIT_BAD_INDEX);
    }
    const int all = min(len + put, (at0 + pages) * page) - start;    // new tokens of these pages
    if (all <= 0) return;
    if (a.ids == nullptr)
        for (int t = threadIdx.x; t < all; t += kAppThreads) s_token[t] = start - len + t;
    if ((int)threadIdx.x < pages) {
        const int at = at0 + threadIdx.x;
        int id = -1;
        if (at * page < len + put) {
            id = a.c.page_table[(size_t)b * a.c.max_pages + at];
            if (id < 0 || id >= a.c.n_pages) {
                id = -1;
                atomicOr(a.status, SENTRY_STATUS_BIT_BAD_INDEX);
            }
        }
        s_id[threadIdx.x] = id;
    }
    __syncthreads();
    // (K or V, head) of a page: a team of warps
    const int shift = 31 - __clz(d / N), per_row = 1 << shift;       // pieces of a row
    const int team = append_team(page, T_, shift), team_shift = 31 - __clz(team), lanes = 32 << team_shift, me = append_place(warp, lane, team);
    const int units = pages * 2 * Hk, at_a_time = (kAppThreads / 32) >> team_shift;
    for (int u0 = 0; u0 < units; u0 += at_a_time) {                  // (the same number of rounds for every warp)
        const int u = u0 + (warp >> team_shift), pi = u / (2 * Hk), unit = u - pi * 2 * Hk;
        const int id = u < units ? s_id[pi] : -1;
        const bool is_v = unit >= Hk;
        const int h = is_v ? unit - Hk : unit;
        const int lo = max((at0 + pi) * page, len), n = id < 0 ? 0 : min(len + put, (at0 + pi + 1) * page) - lo, slot0 = lo - (at0 + pi) * page;
        const int* token = s_token + (lo - start);
        const int pieces = n << shift;
        const long long step = is_v ? a.vs[2] : a.ks[2];
        const T* src = is_v ? (const T*)a.V + b * a.vs[0] + h * a.vs[1] : (const T*)a.K + b * a.ks[0] + h * a.ks[1];
        uint8_t* codes = (uint8_t*)(is_v ? a.c.v : a.c.k) + ((size_t)max(id, 0) * Hk + h) * page * d;
        float* scale = (is_v ? a.c.v_scales : a.c.k_scales) + (size_t)max(id, 0) * Hk + h;
        const float old = n > 0 && slot0 > 0 ? *scale : 0.0f;
        auto piece = [&](int p) { return *reinterpret_cast<const uint4*>(src + token[p >> shift] * step + (p & (per_row - 1)) * N); };
        uint4 held[kHold];
        AbsMax<T> top;
        if (n > 0 && token[n - 1] - token[0] == n - 1) {              // tokens that follow one another
            const T* first = src + (token[0] + (me >> shift)) * step + (me & (per_row - 1)) * N;
            const long long stride = (lanes >> shift) * step;          // (a row is no wider than a warp)
#pragma unroll
            for (int i = 0; i < kHold; ++i) {
                held[i] = i * lanes + me < pieces ? *reinterpret_cast<const uint4*>(first) : make_uint4(0, 0, 0, 0);
                first += stride;
            }
        } else {
#pragma unroll
            for (int i = 0; i < kHold; ++i) held[i] = i * lanes + me < pieces ? piece(i * lanes + me) : make_uint4(0, 0, 0, 0);
        }
#pragma unroll
        for (int i = 0; i < kHold; ++i) top.add(held[i]);
        for (int p = kHold * lanes + me; p < pieces; p += lanes) top.add(piece(p));
        uint32_t bits = __reduce_max_sync(0xffffffffu, top.bits());
        if (team > 1) {
            __syncthreads();
            if (lane == 0) s_top[warp] = bits;
            __syncthreads();
            for (int w = 0; w < team; ++w) bits = max(bits, s_top[(warp & ~(team - 1)) + w]);
        }
        if (n <= 0) continue;
        const float most = magnitude<T>(bits);
        const float now = isnan(most) || isnan(old) ? nan_f32() : fmaxf(page_scale<I8>(most), old);
        const float inv = !(now > 0.0f) ? 0.0f : I8 && now != old ? reciprocal_i8(now, most) : __fdiv_rn(1.0f, now);
        // older codes of the page under its new scale
        if (slot0 > 0 && !(now == old))
            for (int i = me; i < slot0 * d; i += lanes) codes[i] = again<I8>(codes[i], old, now);
        uint8_t* dst = codes + (size_t)slot0 * d;
        auto store_all = [&](auto check) {
            auto store = [&](const uint4& v, int p) {
                float f[N];
                uint32_t w[N / 4];
                Vec16<T>::get(v, f);
                codes_of<I8, decltype(check)::value, N>(f, now, inv, w);
                if constexpr (N == 8) *reinterpret_cast<uint2*>(dst + p * 8) = make_uint2(w[0], w[1]);
                else *reinterpret_cast<uint32_t*>(dst + p * 4) = w[0];
            };
#pragma unroll
            for (int i = 0; i < kHold; ++i)
                if (i * lanes + me < pieces) store(held[i], i * lanes + me);
            for (int p = kHold * lanes + me; p < pieces; p += lanes) store(piece(p), p);
        };
        if (I8 && now != old && sure_i8<T>(now, most)) store_all(std::false_type());
        else store_all(std::true_type());
        if (me == 0 && !(now == old && slot0 > 0)) *scale = now;
    }
}

}  // namespace

int launch_cache_append(sentry_ctx* ctx, const AppendArgs& a, cudaStream_t st) {
    // pages that T tokens can touch, wherever they start
    const long long blocks = a.d.T > 0 ? ((long long)a.d.T + a.c.page - 2) / a.c.page + 1 : 1;
    // pages of a block: one while that fills the GPU no more than a few times, else several, which share the search for their tokens
    const long long few = blocks * a.d.B / (4 * ctx->sm_count);
    const int pages = few < 1 ? 1 : few > kAppPages ? kAppPages : (int)few;
    if (blocks * a.d.B > 0x7fffffffLL) return SENTRY_ERR_UNSUPPORTED;
    const bool i8 = a.c.format == SENTRY_I8;
    auto k = a.d.dtype == SENTRY_F32    ? (i8 ? cache_append_kernel<float, true> : cache_append_kernel<float, false>)
             : a.d.dtype == SENTRY_BF16 ? (i8 ? cache_append_kernel<__nv_bfloat16, true> : cache_append_kernel<__nv_bfloat16, false>)
                                        : (i8 ? cache_append_kernel<__half, true> : cache_append_kernel<__half, false>);
    LaunchScope ls(ctx, KS_CACHE_APPEND, st);
    SENTRY_CUDA_TRY(launch_chained(k, dim3((unsigned)((blocks + pages - 1) / pages * a.d.B)), dim3(kAppThreads), 0, st, a, (int)((blocks + pages - 1) / pages), pages));
    return SENTRY_OK;
}
