// Attention with grouped heads over a paged cache: checks, workspace and
// launches of caee_head_attention.
#include <math.h>

#include <algorithm>

#include "heads.h"

namespace caee {
namespace {

constexpr float kLog2E = 1.4426950408889634f;

size_t up256(size_t n) { return (n + 255) & ~(size_t)255; }

// Units that a list's start and end count as, by the rows' size, where there are
// more units than shares.  us for 0, 1, 2 and 3 of them: decode of 64 users, 64
// heads, 8 groups, lengths at random up to 4100, heads of 128 127, 107, 107 and 106, of
// 64 89, 66, 64 and 63; 256 users up to 2000, 32 heads 234, 199, 197 and 200, up to 500 87,
// 73, 70 and 71; of one length nothing changes (64 of 2048 100).  With fewer units than
// shares they are only more partial results (13 drafts behind 2000 16.6 and 17.1).
constexpr int kFewStarts = 128;

// What the device will find by the host's bounds: the longest request's tokens
// (padded rows count as new ones), the row tiles of a request and the units of
// all requests of the kernel of few rows.
struct HeadBounds {
    long long longest, few_tiles;
    double few_units, few_limit;       // as the device will find; no more than these, whatever rows are padded
};
HeadBounds head_bounds(const caee_head_desc_t& d) {
    HeadBounds b;
    const long long kv = d.max_kv, before = std::max(kv - d.T, 0ll);
    b.longest = std::min(std::min(kv, (long long)d.max_blocks * d.block_size), before + d.max_new);
    b.few_tiles = ((long long)d.max_new * (d.heads / d.kv_heads) + kFewRows - 1) / kFewRows;
    const long long per = (b.longest + kFewTokens - 1) / kFewTokens;
    b.few_units = (double)std::min(d.B * per, kv / kFewTokens + d.B) * (double)b.few_tiles * d.kv_heads;
    b.few_limit = (double)(kv / kFewTokens + (1 + kFewStarts / d.dim) * (long long)d.B) * (double)b.few_tiles * d.kv_heads;
    return b;
}

// Which kernel: of few rows, of many, of many whose row tiles stay whole.  The
// kernel of few rows reads its tokens once for each 32 rows, that of many once
// for 128 and with more to do before and after.  us, few and many: 1 request of
// 4000 tokens, 8 groups of 8 heads, with 1 new token (256 units) 14.7 and 16.9,
// 13 (1024) 21.5 and 26.0, 32 (2048) 27.9 and 29.4, 61 (4096) 39.6 and 33.7; of
// 30000 with 8 (3760) 54.6 and 34.9; 16 requests of 4000, 1 group, with 32 (4096)
// 37.4 and 38.8, 61 (8192) 53.0 and 41.2.  One row tile a request and group, in
// which neither reads a token twice: 16 requests of 4000, 8 groups 54.0 and 53.3.
// Up to kHeadShort tokens cutting row tiles gains nothing over leaving them whole
// (61 requests of 200, 1 group, with 61 new tokens: few 39.5, many 29.4, whole 17.0),
// which takes 7 us and 1.2 a step, however many requests there are, up to a
// round of workgroups.  Few rows take 12 and more with their units.  Few and whole, 8
// groups of 4 heads: 1 request with 13 new tokens of 213 (32 units) 14.1 and 11.4, of
// 463 (64) 16.2 and 16.2, of 813 (112) 16.8 and 21.8, of 1413 (192) 17.1 and 34.0; 4 of
// 463 (256) 18.6 and 16.4, of 813 (448) 20.1 and 22.1, of 1413 (768) 22.1 and 34.4; 4 with
// 30 of 830 (896) 25.9 and 22.2, of 1430 (1536) 32.0 and 34.3; 16 with 30 of 1430 (6144)
// 38.6 and 36.2.  One row tile: 16 requests up to 200 14.7 and 11.4, up to 500 15.1 and
// 16.3, 1000 18.3 and 26.3, 1400 18.6 and 33.2; 64 23.0 and 14.6, 26.4 and 23.0, 33.7 and
// 35.3, 45.3 and 44.5; 256 up to 1000 108 and 133.
// Where there are kTilePieces row tiles or more none is cut.
constexpr long long kHeadShort = 24 * kTileTokens, kHeadShorter = 8 * kTileTokens;
constexpr double kHeadFewUnits = 2048;
enum class HeadWay { few, many, whole };
HeadWay head_way(const caee_head_desc_t& d) {
    if (d.form == CAEE_HEAD_WHOLE) return HeadWay::whole;
    const HeadBounds b = head_bounds(d);
    const bool once = b.few_tiles <= 1 && b.few_limit <= kHeadMaxUnits;        // (units are counted in 32 bits)
    if (d.form == CAEE_HEAD_AUTO && b.longest <= kHeadShort)
        return b.few_units <= (double)b.longest - 400.0 || (once && b.longest > kHeadShorter) ? HeadWay::few : HeadWay::whole;
    if (b.few_units <= kHeadFewUnits || once) return HeadWay::few;
    return d.form == CAEE_HEAD_AUTO && (long long)d.T * d.heads >= kTilePieces * kTileRows ? HeadWay::whole : HeadWay::many;
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
    L.part_sum = take(part_rows * 4);
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
    if (!(isfinite(d->scale * kLog2E) && d->scale > 0.0f))
        return fail(CAEE_ERR_INVALID_ARG, "scale must be > 0 and finite, times log2(e) too");
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
    p.by_ratio = head_by(p.ratio);
    p.by_block = head_by(c.block);
    p.max_kv = std::min((long long)d.max_kv, (long long)d.max_blocks * d.block_size);
    p.q_stride = d.q_stride;
    p.scale_log2 = d.scale * kLog2E;
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
    const HeadWay way = head_way(d);
    p.few_start = head_bounds(d).few_units > kFewGroups ? kFewStarts / d.dim : 0;
    p.part = way == HeadWay::whole ? nullptr : (float*)(w + L.part);
    p.part_ml = (float*)(w + L.part_ml);
    p.part_sum = way == HeadWay::many && p.y_bf16 && lse ? (float*)(w + L.part_sum) : nullptr;
    hipStream_t s = (hipStream_t)stream;
    return timed_launch(CAEE_KERNEL_ATTENTION, s, "head attention", [&] {
        return way == HeadWay::few ? launch_head_few(p, s) : launch_head_many(p, s);
    });
}

}  // extern "C"
