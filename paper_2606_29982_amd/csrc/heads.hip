// Attention with grouped heads over a paged cache: checks, workspace and
// launches of caee_head_attention.
#include <math.h>

#include <algorithm>

#include "heads.h"

namespace caee {
namespace {

size_t up256(size_t n) { return (n + 255) & ~(size_t)255; }

// Units and pieces are counted in 32 bits.
bool few_fits(const caee_head_desc_t& d) {
    const double tiles = (double)d.kv_heads * (((long long)d.max_new * (d.heads / d.kv_heads) + kFewRows - 1) / kFewRows);
    return (double)(d.max_kv / kFewTokens + d.B) * tiles <= kHeadMaxUnits;
}

// Which kernel: that of few rows or of many.
constexpr int kHeadFewRows = 64;
bool head_few(const caee_head_desc_t& d) {
    return d.form != CAEE_HEAD_WHOLE && (long long)d.max_new * (d.heads / d.kv_heads) <= kHeadFewRows && few_fits(d);
}
// Whether row tiles stay whole.
bool head_whole(const caee_head_desc_t& d) {
    if (d.form != CAEE_HEAD_AUTO) return d.form == CAEE_HEAD_WHOLE;
    if (head_few(d)) return false;
    const long long before = d.max_kv > d.T ? d.max_kv - d.T : 0;
    return (long long)d.T * d.heads >= kTilePieces * kTileRows || before + d.max_new <= 24 * kTileTokens;
}

HeadWs head_ws(const caee_head_desc_t& d) {
    HeadWs L{};
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t here = at;
        at += up256(bytes);
        return here;
    };
    L.meta = take((size_t)(d.B + 2) * 4);
    // One size for whatever the split form takes, and for AUTO: smaller calls need no more.
    const size_t part_rows = d.form == CAEE_HEAD_WHOLE ? 0 : (size_t)std::max(2 * kFewGroups * kFewRows, kTilePieces * kTileRows);
    L.part = take(part_rows * d.dim * 4);
    L.part_ml = take(part_rows * 2 * 4);
    L.total = at;
    return L;
}

caee_status_t check_heads(const caee_head_desc_t* d, HeadCache* c) {
    if (!d) return fail(CAEE_ERR_INVALID_ARG, "desc is NULL");
    if (d->T < 0 || d->B < 0) return fail(CAEE_ERR_INVALID_ARG, "T=%d and B=%d must be >= 0", d->T, d->B);
    if (d->heads < 1 || d->kv_heads < 1 || d->heads % d->kv_heads)
        return fail(CAEE_ERR_INVALID_ARG, "heads=%d must be a positive multiple of kv_heads=%d", d->heads, d->kv_heads);
    if (d->max_blocks < 1) return fail(CAEE_ERR_INVALID_ARG, "max_blocks=%d must be >= 1", d->max_blocks);
    if (d->max_new < 0 || d->max_kv < 0)
        return fail(CAEE_ERR_INVALID_ARG, "max_new=%d and max_kv=%lld must be >= 0", d->max_new, (long long)d->max_kv);
    if (d->causal != 0 && d->causal != 1) return fail(CAEE_ERR_INVALID_ARG, "causal=%d must be 0 or 1", d->causal);
    if (d->tree_words < 0 || (d->tree_words > 0 && !d->causal))
        return fail(CAEE_ERR_INVALID_ARG, "tree_words=%d must be >= 0, and causal 1 with a tree", d->tree_words);
    if (d->form != CAEE_HEAD_AUTO && d->form != CAEE_HEAD_SPLIT && d->form != CAEE_HEAD_WHOLE)
        return fail(CAEE_ERR_INVALID_ARG, "unknown form=%d", d->form);
    if (d->y_dtype != CAEE_F32 && d->y_dtype != CAEE_BF16)
        return fail(CAEE_ERR_INVALID_ARG, "y_dtype=%d must be CAEE_F32 or CAEE_BF16", d->y_dtype);
    if (!(isfinite(d->scale) && d->scale > 0.0f)) return fail(CAEE_ERR_INVALID_ARG, "scale must be finite and > 0");
    // Limits of this build.
    if (d->dim != 64 && d->dim != 128) return fail(CAEE_ERR_UNSUPPORTED, "dim=%d must be 64 or 128", d->dim);
    if (d->q_stride % 8 || d->q_stride < (int64_t)d->heads * d->dim)
        return fail(CAEE_ERR_INVALID_ARG, "q_stride=%lld must be a multiple of 8 and hold heads * dim values",
                    (long long)d->q_stride);
    if (d->heads > 1024 || d->B > 65536 || d->T > (1 << 20) || d->q_stride > (1ll << 40))
        return fail(CAEE_ERR_UNSUPPORTED, "heads=%d, B=%d, T=%d or q_stride exceeds 1024, 65536, %d or 2^40", d->heads, d->B,
                    d->T, 1 << 20);
    if (d->tree_words > 32)
        return fail(CAEE_ERR_UNSUPPORTED, "tree_words=%d exceeds 32 (1024 new tokens of a request)", d->tree_words);
    CAEE_TRY(head_cache(d->kv_heads, d->dim, d->block_size, d->n_blocks, d->page_stride, d->row_stride, d->head_stride, c));
    if (d->max_kv > (1 << 30))
        return fail(CAEE_ERR_UNSUPPORTED, "%lld tokens in all exceed 2^30", (long long)d->max_kv);
    return CAEE_OK;
}

}  // namespace
}  // namespace caee

using namespace caee;

extern "C" {

caee_status_t caee_head_workspace_size(const caee_head_desc_t* desc, size_t* bytes) {
    clear_last_error();
    if (!bytes) return fail(CAEE_ERR_INVALID_ARG, "bytes is NULL");
    HeadCache c;
    CAEE_TRY(check_heads(desc, &c));
    *bytes = head_ws(*desc).total;
    return CAEE_OK;
}

caee_status_t caee_head_attention(const caee_head_desc_t* desc, const void* q, const void* k_cache, const void* v_cache,
                                  const int32_t* block_table, const int32_t* cu_new, const int32_t* seq_len,
                                  const uint32_t* tree, void* y, float* lse, void* ws, size_t ws_bytes, void* stream) {
    clear_last_error();
    HeadCache c;
    CAEE_TRY(check_heads(desc, &c));
    const caee_head_desc_t& d = *desc;
    const bool any = d.T > 0;
    CAEE_TRY(check_ptr(q, "q", any));
    CAEE_TRY(check_ptr(k_cache, "k_cache", any));
    CAEE_TRY(check_ptr(v_cache, "v_cache", any));
    CAEE_TRY(check_ptr(block_table, "block_table", any && d.B > 0));
    CAEE_TRY(check_ptr(cu_new, "cu_new", any));
    CAEE_TRY(check_ptr(seq_len, "seq_len", any && d.B > 0));
    CAEE_TRY(check_ptr(tree, "tree", any && d.tree_words > 0));
    CAEE_TRY(check_ptr(y, "y", any));
    CAEE_TRY(check_ptr(lse, "lse", false));
    if (!any) return CAEE_OK;
    const HeadWs L = head_ws(d);
    if (!ws) return fail(CAEE_ERR_WORKSPACE, "workspace is NULL");
    if (((uintptr_t)ws & 255u) != 0) return fail(CAEE_ERR_WORKSPACE, "workspace is not 256-byte aligned");
    if (ws_bytes < L.total) return fail(CAEE_ERR_WORKSPACE, "workspace has %zu bytes, %zu needed", ws_bytes, L.total);
    char* w = (char*)ws;
    HeadParams p{};
    p.T = d.T;
    p.B = d.B;
    p.H = d.heads;
    p.G = d.kv_heads;
    p.ratio = d.heads / d.kv_heads;
    p.dim = d.dim;
    p.max_blocks = d.max_blocks;
    p.max_new = d.max_new;
    p.causal = d.causal;
    p.y_bf16 = d.y_dtype == CAEE_BF16;
    p.words = d.tree_words;
    p.c = c;
    p.max_kv = d.max_kv;
    p.q_stride = d.q_stride;
    p.scale_log2 = d.scale * 1.4426950408889634f;
    p.q = (const uint16_t*)q;
    p.k = (const uint16_t*)k_cache;
    p.v = (const uint16_t*)v_cache;
    p.table = block_table;
    p.cu_new = cu_new;
    p.seq_len = seq_len;
    p.tree = d.tree_words > 0 ? tree : nullptr;
    p.y = y;
    p.lse = lse;
    p.meta = (int32_t*)(w + L.meta);
    p.part = head_whole(d) ? nullptr : (float*)(w + L.part);
    p.part_ml = (float*)(w + L.part_ml);
    hipStream_t s = (hipStream_t)stream;
    return timed_launch(CAEE_KERNEL_ATTENTION, s, "head attention", [&] {
        return head_few(d) ? launch_head_few(p, s) : launch_head_many(p, s);
    });
}

}  // extern "C"
