// Attention with grouped heads over a paged cache.
#include "heads.h"

namespace caee {
namespace {

// One wave per (token, head): 64 tokens at a time, a lane each for the scores,
// D / 64 values a lane for the sums.
template <int D>
__global__ __launch_bounds__(256) void k_head_plain(HeadParams p) {
    const int lane = threadIdx.x & 63;
    const long long at = (long long)lat_workgroup() * 4 + (threadIdx.x >> 6);
    const int t = (int)(at / p.H), h = (int)(at - (long long)t * p.H), g = h / p.ratio;
    if (t >= p.T) return;
    constexpr int V = D / 64;
    float m = kNoScore, l = 0.0f, o[V] = {};
    const int end = p.B > 0 ? p.cu_new[p.B] : 0;
    if (t < end) {
        const int b = lat_find_wave(p.cu_new, p.B, t);
        const LatentReq rq = head_req(p, b);
        const int i = t - rq.t0, limit = i < rq.add ? head_sees(p, rq, i) : 0;
        const uint16_t* q = p.q + (long long)t * p.q_stride + (long long)h * D;
        for (int s = 0; s < limit; s += 64) {
            const int pos = s + lane;
            bool seen = pos < limit;
            const int bit = pos - rq.before;
            if (p.tree && bit >= 0) seen = seen && bit < 32 * p.words && (p.tree[(size_t)t * p.words + (bit >> 5)] >> (bit & 31) & 1);
            const unsigned j = (unsigned)min(pos, limit - 1) / (unsigned)p.c.block;
            const int entry = p.table[(size_t)b * p.max_blocks + min(j, (unsigned)p.max_blocks - 1u)];
            const long long row = (long long)min(max(entry, 0), p.c.n_blocks - 1) * p.c.page_stride +
                                  (long long)(min(pos, limit - 1) - (int)(j * p.c.block)) * p.c.row_stride + g * p.c.head_stride;
            float sc = 0.0f;
            for (int d = 0; d < D; d += 2) {
                const uint32_t a = *(const uint32_t*)(q + d), k = *(const uint32_t*)(p.k + row + d);
                sc += __uint_as_float(a << 16) * __uint_as_float(k << 16);
                sc += __uint_as_float(a & 0xFFFF0000u) * __uint_as_float(k & 0xFFFF0000u);
            }
            sc = seen ? sc : -INFINITY;
            float mt = sc * p.scale_log2;
            for (int d = 32; d >= 1; d >>= 1) mt = fmaxf(mt, __shfl_xor(mt, d));
            const float mn = fmaxf(m, mt), f = __builtin_amdgcn_exp2f(m - mn);
            m = mn;
            const float w = lat_weight(sc, p.scale_log2, m);
            l *= f;
            for (int v = 0; v < V; ++v) o[v] *= f;
            for (int e = 0; e < 64; ++e) {
                const float we = __shfl(w, e);
                const long long re = __shfl(row, e);
                const bool see = __shfl((int)seen, e);
                l += we;
                for (int v = 0; v < V; ++v)
                    if (see) o[v] += we * __uint_as_float((uint32_t)p.v[re + V * lane + v] << 16);
            }
        }
    }
    const float inv = lat_inverse(l);
    for (int v = 0; v < V; ++v) {
        if (p.y_bf16) ((__bf16*)p.y)[at * D + V * lane + v] = (__bf16)(o[v] * inv);
        else ((float*)p.y)[at * D + V * lane + v] = o[v] * inv;
    }
    if (p.lse && lane == 0) p.lse[at] = lat_lse(m, l);
}

}  // namespace

hipError_t launch_head_attention(const HeadParams& p, hipStream_t s) {
    const unsigned n = (unsigned)(((long long)p.T * p.H + 3) / 4);
    if (p.dim == 128) hipLaunchKernelGGL(k_head_plain<128>, lat_grid(n), dim3(256), 0, s, p);
    else hipLaunchKernelGGL(k_head_plain<64>, lat_grid(n), dim3(256), 0, s, p);
    return hipGetLastError();
}

}  // namespace caee
