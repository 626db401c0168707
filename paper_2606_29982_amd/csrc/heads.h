// Shared by the kernels of attention with grouped heads over a paged cache of
// keys and values: parameter block, workspace layout and device helpers.
#pragma once

#include "latent.h"

namespace caee {

// Where a head's keys (and values, in an array of the same strides) of a page lie.
struct HeadCache {
    int block, n_blocks;
    long long page_stride, row_stride, head_stride;    // elements; 0 where there is one page, row or head
};
// Checks the cache fields that both entry points have; *c gets the strides that the kernels use.
caee_status_t head_cache(int kv_heads, int dim, int block_size, int n_blocks, long long page_stride,
                         long long row_stride, long long head_stride, HeadCache* c);

struct HeadParams {
    int T, B, H, G, ratio, dim, max_blocks, max_new, causal, y_bf16, words;
    HeadCache c;
    long long max_kv, q_stride;
    float scale_log2;     // scale * log2(e): softmax in powers of two
    const uint16_t* q;
    const uint16_t* k;
    const uint16_t* v;
    const int32_t* table;
    const int32_t* cu_new;
    const int32_t* seq_len;
    const uint32_t* tree;
    void* y;
    float* lse;
};

// New tokens and length of request b as the kernels use them: 0 <= new <=
// max_new, rows within [0, T), 0 <= seq <= max_kv, and the tokens before its
// new ones, by the lengths as they are.
__device__ inline LatentReq head_req(const HeadParams& p, int b) {
    LatentReq r;
    const int a = p.cu_new[b], e = p.cu_new[b + 1];
    r.t0 = min(max(a, 0), p.T);
    r.add = min(max(min(e, p.T) - r.t0, 0), p.max_new);
    const int len = max(p.seq_len[b], 0);
    r.seq = min(len, (int)p.max_kv);
    r.before = len - (e - a);
    return r;
}
// Tokens up to which new token i of the request may see some; with a tree not all of them.
__device__ inline int head_sees(const HeadParams& p, const LatentReq& r, int i) {
    return p.causal && !p.tree ? min(max(r.before + i + 1, 0), r.seq) : r.seq;
}

hipError_t launch_head_attention(const HeadParams& p, hipStream_t s);

}  // namespace caee
