// Host side of caee_latent_attention: checks, workspace, the two forms'
// launches.
#include <math.h>

#include "latent.h"

namespace caee {
namespace {

size_t up256(size_t n) { return (n + 255) & ~(size_t)255; }

constexpr long long kExpandMaxKv = 65534ll * 256;      // tokens in all of the expanded form: one launch's rows of tiles

bool expanded_fits(const caee_latent_desc_t& d) { return d.max_kv <= kExpandMaxKv; }

// Shares of the absorbed form are counted in 32 bits.
bool absorbed_fits(const caee_latent_desc_t& d) {
    const long long tiles = ((long long)d.max_new * d.heads + kAbsTileRows - 1) / kAbsTileRows;
    return (d.max_kv / 64 + d.B) * tiles <= INT32_MAX / 2;
}

LatentWs latent_ws(const caee_latent_desc_t& d, bool expanded) {
    LatentWs L{};
    L.expanded = expanded;
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t here = at;
        at += up256(bytes);
        return here;
    };
    L.meta = take((size_t)(d.B + 1) * 4);
    if (L.expanded) {
        L.kv = take((size_t)d.max_kv * d.heads * (d.nope + d.v) * 2);
        L.kr = take((size_t)d.max_kv * kRopeDim * 2);
    } else {
        const size_t th = (size_t)d.T * d.heads;
        const size_t part_rows = (size_t)2 * kAbsGroups * kAbsTileRows;
        L.q = take(th * (d.latent + kRopeDim) * 2);
        L.o = take(th * d.latent * 4);
        L.part = take(part_rows * d.latent * 4);
        L.part_ml = take(part_rows * 2 * 4);
    }
    L.total = at;
    return L;
}

// The expanded form pays for every cached token once, the absorbed one 3.4
// times as much per pair of tokens, so the new tokens per request decide.
// Absorbed and expanded, us, 128 heads: 8 requests behind 8000 tokens with 64
// new ones each 1598 and 3744, with 128 3304 and 3804, with 256 6988 and 3949;
// behind 1000 with 64 391 and 524, with 128 780 and 568; one request behind 8000
// with 128 409 and 522, with 256 816 and 549.  16 heads, behind 1000: with 64 76
// and 89, with 128 98 and 92.  Without a cached prefix they meet at about 12 new
// ones: 8 requests with 8 41 and 53, 12 53 and 53, 16 65 and 54, 32 119 and 57;
// 16 heads with 8 25.3 and 25.6, 16 26.5 and 25.9, 64 requests of 15 54.4 and
// 54.3.
// The expanded form's keys and values may be far more than anything else the
// call needs (8 requests of 128 new tokens behind a million, 128 heads: 61 GiB,
// the absorbed form 0.45): where they pass CAEE_LATENT_EXPAND_BYTES the
// absorbed form, if it needs less, goes on to twice the limit (2 requests
// behind 130000 tokens, 128 heads, with 200 new ones each 13.6 and 15.1 ms, with
// 400 27.4 and 18.8).
bool latent_expanded(const caee_latent_desc_t& d) {
    if (d.form != CAEE_LATENT_AUTO) return d.form == CAEE_LATENT_EXPANDED;
    if (!expanded_fits(d) || !absorbed_fits(d)) return expanded_fits(d);       // the one that takes the call
    const long long B = d.B > 0 ? d.B : 1;
    if (d.T < CAEE_LATENT_EXPAND_NEW * B && (d.T < CAEE_LATENT_EXPAND_FRESH * B || d.max_kv > 2ll * d.T)) return false;
    if (d.T >= 2 * CAEE_LATENT_EXPAND_NEW * B) return true;
    const size_t keys = latent_ws(d, true).total;
    return keys <= (size_t)CAEE_LATENT_EXPAND_BYTES || latent_ws(d, false).total >= keys;
}

LatentWs latent_ws(const caee_latent_desc_t& d) { return latent_ws(d, latent_expanded(d)); }

caee_status_t check_latent(const caee_latent_desc_t* d) {
    if (!d) return fail(CAEE_ERR_INVALID_ARG, "desc is NULL");
    if (d->T < 0 || d->B < 0) return fail(CAEE_ERR_INVALID_ARG, "T=%d and B=%d must be >= 0", d->T, d->B);
    if (d->heads < 1) return fail(CAEE_ERR_INVALID_ARG, "heads=%d must be >= 1", d->heads);
    if (d->nope < 1 || d->rope < 1 || d->latent < 1 || d->v < 1)
        return fail(CAEE_ERR_INVALID_ARG, "nope=%d, rope=%d, latent=%d and v=%d must be >= 1", d->nope, d->rope,
                    d->latent, d->v);
    if (d->block_size < 1 || d->block_size > 65536)
        return fail(CAEE_ERR_INVALID_ARG, "block_size=%d must be in [1, 65536]", d->block_size);
    if (d->n_blocks < 1 || d->max_blocks < 1)
        return fail(CAEE_ERR_INVALID_ARG, "n_blocks=%d and max_blocks=%d must be >= 1", d->n_blocks, d->max_blocks);
    if (d->max_new < 0 || d->max_kv < 0)
        return fail(CAEE_ERR_INVALID_ARG, "max_new=%d and max_kv=%lld must be >= 0", d->max_new, (long long)d->max_kv);
    if (d->causal != 0 && d->causal != 1) return fail(CAEE_ERR_INVALID_ARG, "causal=%d must be 0 or 1", d->causal);
    if (d->form != CAEE_LATENT_AUTO && d->form != CAEE_LATENT_ABSORBED && d->form != CAEE_LATENT_EXPANDED)
        return fail(CAEE_ERR_INVALID_ARG, "unknown form=%d", d->form);
    if (d->y_dtype != CAEE_F32 && d->y_dtype != CAEE_BF16)
        return fail(CAEE_ERR_INVALID_ARG, "y_dtype=%d must be CAEE_F32 or CAEE_BF16", d->y_dtype);
    if (!(isfinite(d->scale) && d->scale > 0.0f)) return fail(CAEE_ERR_INVALID_ARG, "scale must be finite and > 0");
    if (d->q_stride % 8 || d->q_stride < (int64_t)d->heads * (d->nope + d->rope))
        return fail(CAEE_ERR_INVALID_ARG, "q_stride=%lld must be a multiple of 8 and hold heads * (nope + rope) values",
                    (long long)d->q_stride);
    // Limits of this build.
    if ((d->nope != 64 && d->nope != 128) || d->rope != kRopeDim || (d->v != 64 && d->v != 128) ||
        (d->latent != 128 && d->latent != 256 && d->latent != 512))
        return fail(CAEE_ERR_UNSUPPORTED, "head parts nope=%d rope=%d latent=%d v=%d: nope and v must be 64 or 128, "
                    "rope %d, latent 128, 256 or 512", d->nope, d->rope, d->latent, d->v, kRopeDim);
    if (d->heads > 1024 || d->B > 65536 || d->T > (1 << 20))
        return fail(CAEE_ERR_UNSUPPORTED, "heads=%d, B=%d or T=%d exceeds 1024, 65536 or %d", d->heads, d->B, d->T,
                    1 << 20);
    if ((long long)d->n_blocks * d->block_size > INT32_MAX || d->max_kv > (1 << 30))
        return fail(CAEE_ERR_UNSUPPORTED, "a cache of %lld rows exceeds 2^31 - 1, or %lld tokens in all 2^30",
                    (long long)d->n_blocks * d->block_size, (long long)d->max_kv);
    const bool expanded = latent_expanded(*d);
    if (expanded && !expanded_fits(*d))
        return fail(CAEE_ERR_UNSUPPORTED, "the expanded form takes at most %lld tokens in all, not max_kv=%lld",
                    kExpandMaxKv, (long long)d->max_kv);
    if (!expanded && !absorbed_fits(*d))
        return fail(CAEE_ERR_UNSUPPORTED, "max_new=%d new tokens over max_kv=%lld: too many pairs for the absorbed form",
                    d->max_new, (long long)d->max_kv);
    return CAEE_OK;
}

}  // namespace
}  // namespace caee

using namespace caee;

extern "C" {

caee_status_t caee_latent_workspace_size(const caee_latent_desc_t* desc, size_t* bytes) {
    clear_last_error();
    if (!bytes) return fail(CAEE_ERR_INVALID_ARG, "bytes is NULL");
    CAEE_TRY(check_latent(desc));
    *bytes = latent_ws(*desc).total;
    return CAEE_OK;
}

caee_status_t caee_latent_attention(const caee_latent_desc_t* desc, const void* q, const caee_latent_weights_t* weights,
                                    const void* cache, const int32_t* block_table, const int32_t* cu_new,
                                    const int32_t* cu_kv, const int32_t* seq_len, void* y, float* lse, void* ws,
                                    size_t ws_bytes, void* stream) {
    clear_last_error();
    CAEE_TRY(check_latent(desc));
    const caee_latent_desc_t& d = *desc;
    const LatentWs L = latent_ws(d);
    if (!weights) return fail(CAEE_ERR_INVALID_ARG, "weights is NULL");
    const bool any = d.T > 0;
    CAEE_TRY(check_ptr(q, "q", any));
    CAEE_TRY(check_ptr(weights->w_uk, "weights->w_uk", any && L.expanded));
    CAEE_TRY(check_ptr(weights->w_uk_t, "weights->w_uk_t", any && !L.expanded));
    CAEE_TRY(check_ptr(weights->w_uv, "weights->w_uv", any));
    CAEE_TRY(check_ptr(cache, "cache", any));
    CAEE_TRY(check_ptr(block_table, "block_table", any && d.B > 0));
    CAEE_TRY(check_ptr(cu_new, "cu_new", any));
    CAEE_TRY(check_ptr(cu_kv, "cu_kv", any && L.expanded));
    CAEE_TRY(check_ptr(seq_len, "seq_len", any && d.B > 0));
    CAEE_TRY(check_ptr(y, "y", any));
    CAEE_TRY(check_ptr(lse, "lse", false));
    if (!any) return CAEE_OK;
    if (!ws) return fail(CAEE_ERR_WORKSPACE, "workspace is NULL");
    if (((uintptr_t)ws & 255u) != 0) return fail(CAEE_ERR_WORKSPACE, "workspace is not 256-byte aligned");
    if (ws_bytes < L.total) return fail(CAEE_ERR_WORKSPACE, "workspace has %zu bytes, %zu needed", ws_bytes, L.total);
    char* w = (char*)ws;
    LatentParams p{};
    p.T = d.T;
    p.B = d.B;
    p.H = d.heads;
    p.nope = d.nope;
    p.latent = d.latent;
    p.v = d.v;
    p.block = d.block_size;
    p.n_blocks = d.n_blocks;
    p.max_blocks = d.max_blocks;
    p.max_new = d.max_new;
    p.causal = d.causal;
    p.y_bf16 = d.y_dtype == CAEE_BF16;
    p.max_kv = d.max_kv;
    p.q_stride = d.q_stride;
    p.scale = d.scale;
    p.scale_log2 = d.scale * 1.4426950408889634f;
    p.q = (const uint16_t*)q;
    p.w_uk = (const uint16_t*)weights->w_uk;
    p.w_uk_t = (const uint16_t*)weights->w_uk_t;
    p.w_uv = (const uint16_t*)weights->w_uv;
    p.cache = (const uint16_t*)cache;
    p.table = block_table;
    p.cu_new = cu_new;
    p.cu_kv = cu_kv;
    p.seq_len = seq_len;
    p.y = y;
    p.lse = lse;
    p.meta = (int32_t*)(w + L.meta);
    p.qw = (uint16_t*)(w + L.q);
    p.o = (float*)(w + L.o);
    p.part = (float*)(w + L.part);
    p.part_ml = (float*)(w + L.part_ml);
    p.kv = (uint16_t*)(w + L.kv);
    p.kr = (uint16_t*)(w + L.kr);
    hipStream_t s = (hipStream_t)stream;
    return timed_launch(CAEE_KERNEL_ATTENTION, s, "latent attention", [&] {
        return L.expanded ? launch_latent_expanded(p, s) : launch_latent_absorbed(p, s);
    });
}

}  // extern "C"
