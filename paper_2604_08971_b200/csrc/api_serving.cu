// C ABI of the serving operators (8-bit linear layer, cross attention, 8-bit cache): argument checks and dispatch.
#include "serving.cuh"

namespace {

inline bool aligned(const void* p, size_t a) { return ((uintptr_t)p % a) == 0; }
inline bool dense_type(int t) { return t == SENTRY_F32 || t == SENTRY_BF16 || t == SENTRY_F16; }
inline bool head_dim(int d) { return d == 16 || d == 32 || d == 64 || d == 128; }
constexpr long long kMaxRows = 1 << 24;

// Strides of a [B,H,T,d] view in elements: as given, or contiguous where all are 0.
int strides_of(const int64_t given[3], int H, int T, int d, int dtype, long long out[3]) {
    if (given[0] == 0 && given[1] == 0 && given[2] == 0) {
        out[0] = (long long)H * T * d; out[1] = (long long)T * d; out[2] = d;
        return SENTRY_OK;
    }
    const int unit = dtype == SENTRY_F32 ? 4 : 8;
    for (int i = 0; i < 3; ++i) {
        if (given[i] < 0) return SENTRY_ERR_BAD_SHAPE;
        if (given[i] % unit != 0 || given[i] > (1LL << 38)) return SENTRY_ERR_UNSUPPORTED;
        out[i] = given[i];
    }
    return SENTRY_OK;
}

int check_heads(int B, int Tq, int Hq, int Hk, int d, int k_h) {
    if (B < 0 || Tq < 0 || Hq < 1 || Hk < 1 || k_h < 1 || Hq % Hk != 0 || k_h > Hq) return SENTRY_ERR_BAD_SHAPE;
    if (!head_dim(d) || Hq > kServeMaxHeads || Tq >= kMaxRows || (long long)B * Hq >= kMaxRows) return SENTRY_ERR_UNSUPPORTED;
    if ((long long)k_h * Tq >= 1LL << 30) return SENTRY_ERR_UNSUPPORTED;      // a sample's rows are counted in 32 bits, a block's ahead
    return SENTRY_OK;
}

int cross_args(const sentry_cross_desc* d, KvAttendArgs& a) {
    if (d == nullptr || !dense_type(d->dtype)) return SENTRY_ERR_INVALID_ARG;
    int rc = check_heads(d->B, d->Tq, d->Hq, d->Hk, d->d, d->k_h);
    if (rc != SENTRY_OK) return rc;
    if (d->Tk < 0) return SENTRY_ERR_BAD_SHAPE;
    if (d->Tk >= kMaxRows) return SENTRY_ERR_UNSUPPORTED;
    a = KvAttendArgs{};
    a.B = d->B; a.Tq = d->Tq; a.Tk = d->Tk; a.Hq = d->Hq; a.Hk = d->Hk; a.d = d->d; a.k_h = d->k_h; a.dtype = d->dtype;
    if ((rc = strides_of(d->q_stride, d->Hq, d->Tq, d->d, d->dtype, a.qs)) != SENTRY_OK) return rc;
    if ((rc = strides_of(d->k_stride, d->Hk, d->Tk, d->d, d->dtype, a.ks)) != SENTRY_OK) return rc;
    if ((rc = strides_of(d->v_stride, d->Hk, d->Tk, d->d, d->dtype, a.vs)) != SENTRY_OK) return rc;
    if (d->Tk > 1 && (a.ks[2] == 0 || a.vs[2] == 0)) return SENTRY_ERR_UNSUPPORTED;   // one key for all of them
    return SENTRY_OK;
}

int check_cache(const sentry_kv_cache* c) {
    if (c == nullptr) return SENTRY_ERR_INVALID_ARG;
    if (c->format != SENTRY_FP8_E4M3 && c->format != SENTRY_I8) return SENTRY_ERR_INVALID_ARG;
    if (c->Hk < 1 || c->n_pages < 0 || c->max_pages < 0) return SENTRY_ERR_BAD_SHAPE;
    if (!head_dim(c->d) || c->Hk > kServeMaxHeads) return SENTRY_ERR_UNSUPPORTED;
    if (c->page != 16 && c->page != 32 && c->page != 64 && c->page != 128) return SENTRY_ERR_UNSUPPORTED;
    if ((long long)c->max_pages * c->page > 0x7fffffffLL - 4096) return SENTRY_ERR_UNSUPPORTED;
    if ((long long)c->n_pages * c->Hk > 0x7fffffffLL / c->page) return SENTRY_ERR_UNSUPPORTED;   // rows of the pool are counted in 32 bits
    return SENTRY_OK;
}
int check_cache_pointers(const sentry_kv_cache* c) {
    // (an empty pool and an empty table have no address)
    if (c->n_pages > 0 && (c->k == nullptr || c->v == nullptr || c->k_scales == nullptr || c->v_scales == nullptr)) return SENTRY_ERR_INVALID_ARG;
    if (c->max_pages > 0 && c->page_table == nullptr) return SENTRY_ERR_INVALID_ARG;
    if (!aligned(c->k, 16) || !aligned(c->v, 16) || !aligned(c->k_scales, 4) || !aligned(c->v_scales, 4) || !aligned(c->page_table, 4))
        return SENTRY_ERR_INVALID_ARG;
    return SENTRY_OK;
}

int cache_args(const sentry_kv_cache* c, const sentry_cache_attend_desc* d, KvAttendArgs& a) {
    int rc = check_cache(c);
    if (rc != SENTRY_OK) return rc;
    if (d == nullptr || !dense_type(d->dtype)) return SENTRY_ERR_INVALID_ARG;
    if ((rc = check_heads(d->B, d->Tq, d->Hq, c->Hk, c->d, d->k_h)) != SENTRY_OK) return rc;
    a = KvAttendArgs{};
    a.B = d->B; a.Tq = d->Tq; a.Tk = c->max_pages * c->page; a.Hq = d->Hq; a.Hk = c->Hk; a.d = c->d; a.k_h = d->k_h; a.dtype = d->dtype;
    a.format = c->format; a.page = c->page; a.n_pages = c->n_pages; a.max_pages = c->max_pages; a.causal = d->causal != 0;
    a.K = c->k; a.V = c->v; a.k_scales = c->k_scales; a.v_scales = c->v_scales; a.table = c->page_table;
    return strides_of(d->q_stride, d->Hq, d->Tq, c->d, d->dtype, a.qs);
}

size_t kv_ws_bytes(const KvAttendArgs& a) { return a.dtype == SENTRY_F32 ? 0 : kv_tc_takes(a) ? kv_tc_ws_bytes(a) : kv_rows_ws_bytes(a); }

int run_attend(sentry_ctx* ctx, KvAttendArgs& a, cudaStream_t st) {
    ctx->last_launches = 0;
    if (a.B == 0 || a.Tq == 0) return SENTRY_OK;
    a.status = ctx->d_status;
    a.sm_count = ctx->sm_count;
    SENTRY_ON_DEVICE(ctx->device);
    if (a.dtype == SENTRY_F32) return launch_kv_generic(ctx, a, st);
    WsAlloc ws(ctx->workspace, ctx->workspace_bytes);
    return kv_tc_takes(a) ? launch_kv_tc(ctx, a, ws, st) : launch_kv_rows(ctx, a, ws, st);
}

}  // namespace

extern "C" {

int sentry_quantize_rows_i8(sentry_ctx* ctx, int M, int K, int dtype, const void* X, int8_t* codes, float* scales, void* stream) {
    if (ctx == nullptr || !dense_type(dtype)) return SENTRY_ERR_INVALID_ARG;
    if (M < 0 || K < 1) return SENTRY_ERR_BAD_SHAPE;
    if (K % 16 != 0 || K > 65536) return SENTRY_ERR_UNSUPPORTED;
    ctx->last_launches = 0;
    if (M == 0) return SENTRY_OK;
    if (X == nullptr || codes == nullptr || scales == nullptr) return SENTRY_ERR_INVALID_ARG;
    if (!aligned(X, 16) || !aligned(codes, 16) || !aligned(scales, 4)) return SENTRY_ERR_INVALID_ARG;
    SENTRY_ON_DEVICE(ctx->device);
    return launch_quantize_rows_i8(ctx, M, K, dtype, X, codes, scales, (cudaStream_t)stream);
}

int sentry_linear_i8(sentry_ctx* ctx, const sentry_linear_desc* desc, const int8_t* codes, const float* x_scales, const int8_t* W,
                     const float* w_scales, const float* bias, void* Y, void* stream) {
    if (ctx == nullptr || desc == nullptr || !dense_type(desc->dtype)) return SENTRY_ERR_INVALID_ARG;
    if (desc->M < 0 || desc->N < 0 || desc->K < 1) return SENTRY_ERR_BAD_SHAPE;
    if (desc->K % 16 != 0 || desc->K > 65536) return SENTRY_ERR_UNSUPPORTED;
    ctx->last_launches = 0;
    if (desc->M == 0 || desc->N == 0) return SENTRY_OK;
    if (codes == nullptr || x_scales == nullptr || W == nullptr || w_scales == nullptr || Y == nullptr) return SENTRY_ERR_INVALID_ARG;
    if (!aligned(codes, 16) || !aligned(W, 16) || !aligned(Y, 16) || !aligned(x_scales, 4) || !aligned(w_scales, 4) || !aligned(bias, 4))
        return SENTRY_ERR_INVALID_ARG;
    SENTRY_ON_DEVICE(ctx->device);
    LinearArgs a;
    a.d = *desc;
    a.X = codes; a.W = W; a.xs = x_scales; a.ws = w_scales; a.bias = bias; a.Y = Y;
    a.status = ctx->d_status;
    return launch_linear_i8(ctx, a, (cudaStream_t)stream);
}

size_t sentry_cross_workspace_bytes(const sentry_cross_desc* desc) {
    KvAttendArgs a;
    return cross_args(desc, a) == SENTRY_OK ? align_up(kv_ws_bytes(a), 256) : 0;
}

int sentry_cross_attend_fwd(sentry_ctx* ctx, const sentry_cross_desc* desc, const void* Q, const void* K, const void* V,
                            const int32_t* kept_heads, const int32_t* key_modality_ids, const uint32_t* masks,
                            const int32_t* key_lengths, void* O, void* stream) {
    if (ctx == nullptr) return SENTRY_ERR_INVALID_ARG;
    KvAttendArgs a;
    const int rc = cross_args(desc, a);
    if (rc != SENTRY_OK) return rc;
    if (kept_heads == nullptr && desc->k_h != desc->Hq) return SENTRY_ERR_BAD_SHAPE;
    if ((key_modality_ids == nullptr) != (masks == nullptr)) return SENTRY_ERR_INVALID_ARG;
    if (a.B > 0 && a.Tq > 0) {
        if (Q == nullptr || O == nullptr || (a.Tk > 0 && (K == nullptr || V == nullptr))) return SENTRY_ERR_INVALID_ARG;
        if (!aligned(Q, 16) || !aligned(K, 16) || !aligned(V, 16) || !aligned(O, 16) || !aligned(kept_heads, 4) ||
            !aligned(key_modality_ids, 4) || !aligned(masks, 4) || !aligned(key_lengths, 4))
            return SENTRY_ERR_INVALID_ARG;
    }
    a.Q = Q; a.K = K; a.V = V; a.O = O;
    a.kept = kept_heads; a.ids = key_modality_ids; a.masks = masks; a.lengths = key_lengths;
    return run_attend(ctx, a, (cudaStream_t)stream);
}

int sentry_cache_append(sentry_ctx* ctx, const sentry_kv_cache* cache, const sentry_append_desc* desc, const void* K, const void* V,
                        const int32_t* token_modality_ids, const uint32_t* masks, const int32_t* token_lengths,
                        const int32_t* lengths, int32_t* new_lengths, void* stream) {
    if (ctx == nullptr) return SENTRY_ERR_INVALID_ARG;
    int rc = check_cache(cache);
    if (rc != SENTRY_OK) return rc;
    if (desc == nullptr || !dense_type(desc->dtype)) return SENTRY_ERR_INVALID_ARG;
    if (desc->B < 0 || desc->T < 0) return SENTRY_ERR_BAD_SHAPE;
    if (desc->T >= kMaxRows || (long long)desc->B * cache->Hk >= kMaxRows) return SENTRY_ERR_UNSUPPORTED;
    AppendArgs a;
    a.c = *cache; a.d = *desc;
    if ((rc = strides_of(desc->k_stride, cache->Hk, desc->T, cache->d, desc->dtype, a.ks)) != SENTRY_OK) return rc;
    if ((rc = strides_of(desc->v_stride, cache->Hk, desc->T, cache->d, desc->dtype, a.vs)) != SENTRY_OK) return rc;
    if ((token_modality_ids == nullptr) != (masks == nullptr)) return SENTRY_ERR_INVALID_ARG;
    ctx->last_launches = 0;
    if (desc->B == 0) return SENTRY_OK;
    if ((rc = check_cache_pointers(cache)) != SENTRY_OK) return rc;
    if (lengths == nullptr || new_lengths == nullptr || (desc->T > 0 && (K == nullptr || V == nullptr))) return SENTRY_ERR_INVALID_ARG;
    if (!aligned(K, 16) || !aligned(V, 16) || !aligned(lengths, 4) || !aligned(new_lengths, 4) || !aligned(token_modality_ids, 4) ||
        !aligned(masks, 4) || !aligned(token_lengths, 4))
        return SENTRY_ERR_INVALID_ARG;
    // every CTA of a sample reads its length while one writes the new one
    if (new_lengths < lengths + desc->B && lengths < new_lengths + desc->B) return SENTRY_ERR_INVALID_ARG;
    a.K = K; a.V = V; a.ids = token_modality_ids; a.masks = masks; a.token_lengths = token_lengths;
    a.lengths = lengths; a.new_lengths = new_lengths;
    a.status = ctx->d_status;
    SENTRY_ON_DEVICE(ctx->device);
    return launch_cache_append(ctx, a, (cudaStream_t)stream);
}

size_t sentry_cache_workspace_bytes(const sentry_kv_cache* cache, const sentry_cache_attend_desc* desc) {
    KvAttendArgs a;
    return cache_args(cache, desc, a) == SENTRY_OK ? align_up(kv_ws_bytes(a), 256) : 0;
}

int sentry_cache_attend_fwd(sentry_ctx* ctx, const sentry_kv_cache* cache, const sentry_cache_attend_desc* desc, const void* Q,
                            const int32_t* kept_heads, const int32_t* lengths, void* O, void* stream) {
    if (ctx == nullptr) return SENTRY_ERR_INVALID_ARG;
    KvAttendArgs a;
    int rc = cache_args(cache, desc, a);
    if (rc != SENTRY_OK) return rc;
    if (kept_heads == nullptr && desc->k_h != desc->Hq) return SENTRY_ERR_BAD_SHAPE;
    if (a.B > 0 && a.Tq > 0) {
        if ((rc = check_cache_pointers(cache)) != SENTRY_OK) return rc;
        if (Q == nullptr || O == nullptr || lengths == nullptr) return SENTRY_ERR_INVALID_ARG;
        if (!aligned(Q, 16) || !aligned(O, 16) || !aligned(kept_heads, 4) || !aligned(lengths, 4)) return SENTRY_ERR_INVALID_ARG;
    }
    a.Q = Q; a.O = O; a.kept = kept_heads; a.lengths = lengths;
    return run_attend(ctx, a, (cudaStream_t)stream);
}

}  // extern "C"
