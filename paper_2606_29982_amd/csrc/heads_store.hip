// Heads' keys and values into a paged cache, queries beside them: norm of each
// head, rotation by position, rounding to bf16 (caee_head_store).
#include <math.h>

#include <utility>

#include "heads.h"

namespace caee {

caee_status_t head_cache(int kv_heads, int dim, int block_size, int n_blocks, long long page_stride,
                         long long row_stride, long long head_stride, HeadCache* c) {
    if (block_size < 1 || block_size > 65536)
        return fail(CAEE_ERR_INVALID_ARG, "block_size=%d must be in [1, 65536]", block_size);
    if (n_blocks < 1) return fail(CAEE_ERR_INVALID_ARG, "n_blocks=%d must be >= 1", n_blocks);
    *c = {block_size, n_blocks, n_blocks > 1 ? page_stride : 0, block_size > 1 ? row_stride : 0,
          kv_heads > 1 ? head_stride : 0};
    if (c->page_stride % 8 || c->row_stride % 8 || c->head_stride % 8)
        return fail(CAEE_ERR_INVALID_ARG, "cache strides %lld, %lld, %lld must be multiples of 8", page_stride, row_stride,
                    head_stride);
    // Heads and rows of a page one inside the other, pages outside: no two values share a place.
    constexpr long long kMax = 1ll << 40;
    if (c->page_stride > kMax || c->row_stride > kMax || c->head_stride > kMax)
        return fail(CAEE_ERR_UNSUPPORTED, "cache strides %lld, %lld, %lld exceed 2^40", page_stride, row_stride, head_stride);
    struct {
        long long n, stride;
    } in = {kv_heads, c->head_stride}, out = {block_size, c->row_stride};
    if (in.n > 1 && out.n > 1 && in.stride > out.stride) {
        const auto t = in;
        in = out;
        out = t;
    }
    long long extent = dim;
    for (const auto& d : {in, out}) {
        if (d.n > 1 && d.stride < extent)
            return fail(CAEE_ERR_INVALID_ARG, "cache rows %lld and heads %lld elements apart overlap", row_stride, head_stride);
        extent += (d.n - 1) * d.stride;
    }
    if (n_blocks > 1 && c->page_stride < extent)
        return fail(CAEE_ERR_INVALID_ARG, "cache pages %lld elements apart overlap (a page takes %lld)", page_stride, extent);
    if (extent >= (1ll << 30))
        return fail(CAEE_ERR_UNSUPPORTED, "a cache page of %lld elements exceeds 2^30", extent);
    if ((long long)n_blocks * block_size > INT32_MAX)
        return fail(CAEE_ERR_UNSUPPORTED, "a cache of %lld rows exceeds 2^31 - 1", (long long)n_blocks * block_size);
    if ((double)n_blocks * (double)c->page_stride > 1e17)
        return fail(CAEE_ERR_UNSUPPORTED, "%d cache pages %lld elements apart exceed the address space", n_blocks, page_stride);
    return CAEE_OK;
}

namespace {

// Whether heads of two caches of the same strides, `apart` elements from one another, share a
// place: some pages, rows and heads on, the other's head begins within one.  What lies inside
// a page (row, head) takes no more than the stride, so two numbers of each come into question.
bool caches_meet(const HeadCache& c, int kv_heads, int dim, long long apart) {
    struct Level {
        long long n, stride;
    } levels[3] = {{c.n_blocks, c.page_stride}, {c.block, c.row_stride}, {kv_heads, c.head_stride}};
    if (c.head_stride > c.row_stride && c.block > 1) std::swap(levels[1], levels[2]);
    auto meet = [&](auto&& self, int i, long long left) -> bool {
        if (i == 3) return left < dim && left > -dim;
        if (levels[i].n == 1) return self(self, i + 1, left);
        const long long n = levels[i].n, k = left / levels[i].stride - (left < 0);
        for (long long at : {k, k + 1})
            if (at < n && at > -n && self(self, i + 1, left - at * levels[i].stride)) return true;
        return false;
    };
    return meet(meet, 0, apart);
}

constexpr int kStoreThreads = 256;
constexpr int kStoreSpread = 2048;     // workgroups up to which a token's passes are spread

struct HeadStoreParams {
    int T, H, G, rope, steps;          // steps: passes of a workgroup over its token's heads
    long long q_stride, k_stride, v_stride, y_stride, n_slots;
    HeadCache c;
    float eps;
    const void* q;
    const void* k;
    const void* v;
    const float* q_norm;
    const float* k_norm;
    const double* freq;
    const int32_t* position;
    const int64_t* slots;
    uint16_t* y;
    uint16_t* k_cache;
    uint16_t* v_cache;
};

template <int C>
__device__ inline float dpp_add(float v) {
    return v + __uint_as_float((uint32_t)__builtin_amdgcn_mov_dpp((int)__float_as_uint(v), C, 0xF, 0xF, true));
}
// Sum over the D / 8 lanes of a head (16, or 8).
template <int D>
__device__ inline float head_sum(float v) {
    v = dpp_add<0xB1>(v);                          // neighbours, pairs, quads, halves of 16 lanes
    v = dpp_add<0x4E>(v);
    v = dpp_add<0x141>(v);
    if constexpr (D == 128) v = dpp_add<0x140>(v);
    return v;
}

// A workgroup has one token and kStoreThreads / (D / 8) heads in a pass (of its
// queries, keys and values, in that order), D / 8 lanes a head, 16 bytes of
// bf16 a lane.  The token's angles are made once for all heads: position * freq in
// 64 bits, whose whole turns are taken off before the sine and cosine of 32 bits.
// The norm is in 32 bits; q, k and v are rounded once, at the end, to the type the
// attention reads.
// Memory bounds it: 16381 tokens of 32 + 2 x 8 heads of 128, 403 MB read and
// written in 87 us (4.6 TB/s; a large copy 5.0).  The next head's load issued before
// this one's work gained nothing (99 to 107 us), as six to eight workgroups a CU hide it.
// 32 tokens take 3.9 us, a launch and a chain of three loads.
template <bool kF32, int D, bool kAdjacent>
__global__ __launch_bounds__(kStoreThreads) void k_head_store(HeadStoreParams p) {
    constexpr int kLanes = D / 8, kHeads = kStoreThreads / kLanes;
    __shared__ float2 turn[D / 2];                 // cosine, sine
    const int t = blockIdx.x, tid = threadIdx.x, l = tid % kLanes;
    const int rows = p.H + 2 * p.G, half = p.rope >> 1;
    if (tid < half) {
        const double a = (double)p.position[t] * p.freq[tid] * 0.15915494309189535;   // turns: / 2 pi
        const double r = a - rint(a);
        float sn, cs;
        sincospif((float)(r + r), &sn, &cs);
        turn[tid] = make_float2(cs, sn);
    }
    const long long slot = p.slots[t];
    const bool there = slot >= 0 && slot < p.n_slots;
    const unsigned page = there ? (unsigned)slot / (unsigned)p.c.block : 0u;
    const long long at = (long long)page * p.c.page_stride + (slot - (long long)page * p.c.block) * p.c.row_stride;
    __syncthreads();
    const bool rotated = 8 * l < p.rope;
    // Halves: value i < rope / 2 is a pair's first, its partner i + rope / 2.
    const bool first = 8 * l < half;
    const int partner = (tid & (kWave - 1)) + (first ? half / 8 : -(half / 8));
    for (int i = 0; i < p.steps; ++i) {
        const int r = ((int)blockIdx.y * p.steps + i) * kHeads + tid / kLanes;
        if (r >= rows) return;         // the lanes of a head leave together, and no other head's are read
        const int kind = r < p.H ? 0 : r < p.H + p.G ? 1 : 2, h = kind == 0 ? r : kind == 1 ? r - p.H : r - p.H - p.G;
        const void* base = kind == 0 ? p.q : kind == 1 ? p.k : p.v;
        const long long src = (long long)t * (kind == 0 ? p.q_stride : kind == 1 ? p.k_stride : p.v_stride) + h * D + 8 * l;
        float x[8];
        if constexpr (kF32) {
            const float4 a = *(const float4*)((const float*)base + src), b = *(const float4*)((const float*)base + src + 4);
            x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
        } else {
            const lat_u32x4 a = *(const lat_u32x4*)((const uint16_t*)base + src);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                x[2 * e] = __uint_as_float(a[e] << 16);
                x[2 * e + 1] = __uint_as_float(a[e] & 0xFFFF0000u);
            }
        }
        if (kind < 2) {
            const float* w = kind == 0 ? p.q_norm : p.k_norm;
            if (w) {
                float s = 0.0f;
#pragma unroll
                for (int e = 0; e < 8; ++e) s += x[e] * x[e];
                const float f = 1.0f / sqrtf(head_sum<D>(s) * (1.0f / D) + p.eps);
                const float4 a = *(const float4*)(w + 8 * l), b = *(const float4*)(w + 8 * l + 4);
                x[0] *= f * a.x, x[1] *= f * a.y, x[2] *= f * a.z, x[3] *= f * a.w;
                x[4] *= f * b.x, x[5] *= f * b.y, x[6] *= f * b.z, x[7] *= f * b.w;
            }
            if (p.rope > 0) {
                if constexpr (kAdjacent) {
                    if (rotated) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const float2 c = turn[4 * l + e];
                            const float a = x[2 * e], b = x[2 * e + 1];
                            x[2 * e] = a * c.x - b * c.y;
                            x[2 * e + 1] = a * c.y + b * c.x;
                        }
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float o = __shfl(x[e], partner);
                        if (rotated) {
                            const float2 c = turn[(first ? 8 * l : 8 * l - half) + e];
                            x[e] = first ? x[e] * c.x - o * c.y : o * c.y + x[e] * c.x;
                        }
                    }
                }
            }
        }
        const lat_u32x4 out = {lat_pack(x[0], x[1]), lat_pack(x[2], x[3]), lat_pack(x[4], x[5]), lat_pack(x[6], x[7])};
        if (kind == 0) *(lat_u32x4*)(p.y + (long long)t * p.y_stride + h * D + 8 * l) = out;
        else if (there) *(lat_u32x4*)((kind == 1 ? p.k_cache : p.v_cache) + at + h * p.c.head_stride + 8 * l) = out;
    }
}

}  // namespace
}  // namespace caee

using namespace caee;

extern "C" caee_status_t caee_head_store(const caee_head_store_desc_t* desc, const void* q, const void* k, const void* v,
                                         const float* q_norm, const float* k_norm, const double* freq,
                                         const int32_t* position, const int64_t* slots, void* q_out, void* k_cache,
                                         void* v_cache, void* stream) {
    clear_last_error();
    if (!desc) return fail(CAEE_ERR_INVALID_ARG, "desc is NULL");
    const caee_head_store_desc_t& d = *desc;
    if (d.T < 0) return fail(CAEE_ERR_INVALID_ARG, "T=%d must be >= 0", d.T);
    if (d.heads < 1 || d.kv_heads < 1)
        return fail(CAEE_ERR_INVALID_ARG, "heads=%d and kv_heads=%d must be >= 1", d.heads, d.kv_heads);
    if (d.dim != 64 && d.dim != 128) return fail(CAEE_ERR_UNSUPPORTED, "dim=%d must be 64 or 128", d.dim);
    if (d.rope < 0 || d.rope > d.dim || d.rope % 16)
        return fail(CAEE_ERR_INVALID_ARG, "rope=%d must be a multiple of 16 of at most dim=%d", d.rope, d.dim);
    if (d.adjacent != 0 && d.adjacent != 1) return fail(CAEE_ERR_INVALID_ARG, "adjacent=%d must be 0 or 1", d.adjacent);
    if (d.x_dtype != CAEE_F32 && d.x_dtype != CAEE_BF16)
        return fail(CAEE_ERR_INVALID_ARG, "x_dtype=%d must be CAEE_F32 or CAEE_BF16", d.x_dtype);
    if (!(isfinite(d.eps) && d.eps >= 0.0f)) return fail(CAEE_ERR_INVALID_ARG, "eps must be finite and >= 0");
    if (d.heads > 1024 || d.kv_heads > 1024 || d.T > (1 << 20))
        return fail(CAEE_ERR_UNSUPPORTED, "heads=%d, kv_heads=%d or T=%d exceeds 1024, 1024 or %d", d.heads, d.kv_heads, d.T,
                    1 << 20);
    const int unit = d.x_dtype == CAEE_BF16 ? 8 : 4;   // elements of 16 bytes
    const int64_t wide = (int64_t)d.heads * d.dim, narrow = (int64_t)d.kv_heads * d.dim;
    if (d.q_stride < wide || d.q_stride % unit || d.k_stride < narrow || d.k_stride % unit || d.v_stride < narrow ||
        d.v_stride % unit)
        return fail(CAEE_ERR_INVALID_ARG, "token strides %lld, %lld, %lld must hold the heads and keep them 16-byte aligned",
                    (long long)d.q_stride, (long long)d.k_stride, (long long)d.v_stride);
    if (d.q_out_stride < wide || d.q_out_stride % 8)
        return fail(CAEE_ERR_INVALID_ARG, "q_out_stride=%lld must be a multiple of 8 and hold the heads",
                    (long long)d.q_out_stride);
    constexpr int64_t kMaxStride = 1ll << 40;
    if (d.q_stride > kMaxStride || d.k_stride > kMaxStride || d.v_stride > kMaxStride || d.q_out_stride > kMaxStride)
        return fail(CAEE_ERR_UNSUPPORTED, "a token stride exceeds 2^40");
    HeadCache c;
    CAEE_TRY(head_cache(d.kv_heads, d.dim, d.block_size, d.n_blocks, d.page_stride, d.row_stride, d.head_stride, &c));
    const bool any = d.T > 0;
    CAEE_TRY(check_ptr(q, "q", any));
    CAEE_TRY(check_ptr(k, "k", any));
    CAEE_TRY(check_ptr(v, "v", any));
    CAEE_TRY(check_ptr(q_norm, "q_norm", false));
    CAEE_TRY(check_ptr(k_norm, "k_norm", false));
    CAEE_TRY(check_ptr(freq, "freq", any && d.rope > 0));
    CAEE_TRY(check_ptr(position, "position", any && d.rope > 0));
    CAEE_TRY(check_ptr(slots, "slots", any));
    CAEE_TRY(check_ptr(q_out, "q_out", any));
    CAEE_TRY(check_ptr(k_cache, "k_cache", any));
    CAEE_TRY(check_ptr(v_cache, "v_cache", any));
    if (!any) return CAEE_OK;
    if (caches_meet(c, d.kv_heads, d.dim, ((intptr_t)v_cache - (intptr_t)k_cache) / 2))
        return fail(CAEE_ERR_INVALID_ARG, "k_cache and v_cache overlap");
    // Queries may be written over themselves; other tokens' rows that a
    // workgroup may still have to read may not be.
    if (q_out == q ? d.x_dtype != CAEE_BF16 || (d.T > 1 && d.q_out_stride != d.q_stride) : false)
        return fail(CAEE_ERR_INVALID_ARG, "q_out may be q itself for bf16 of the same token stride only");
    const int xb = d.x_dtype == CAEE_BF16 ? 2 : 4;
    struct Rows {
        const char* name;
        uintptr_t at;
        int64_t stride, width;      // bytes
    };
    const Rows out = {"q_out", (uintptr_t)q_out, 2 * d.q_out_stride, 2 * wide};
    for (const Rows& in : {Rows{"q", (uintptr_t)q, xb * d.q_stride, xb * wide}, Rows{"k", (uintptr_t)k, xb * d.k_stride, xb * narrow},
                           Rows{"v", (uintptr_t)v, xb * d.v_stride, xb * narrow}}) {
        if (in.at == (uintptr_t)q_out && in.name[0] == 'q') continue;
        const bool apart = in.at < out.at ? out.at - in.at >= (uintptr_t)((d.T - 1) * in.stride + in.width)
                                          : in.at - out.at >= (uintptr_t)((d.T - 1) * out.stride + out.width);
        if (apart) continue;
        // Slices of one wider array: rows of one stride that lie beside each other.
        int64_t ahead = (int64_t)(in.at - out.at) % out.stride;
        if (ahead < 0) ahead += out.stride;
        if (in.stride == out.stride && ahead >= out.width && ahead + in.width <= out.stride) continue;
        return fail(CAEE_ERR_INVALID_ARG, "q_out overlaps %s", in.name);
    }
    HeadStoreParams p{d.T,     d.heads, d.kv_heads, d.rope,  1,     d.q_stride, d.k_stride, d.v_stride, d.q_out_stride,
                      (int64_t)d.n_blocks * d.block_size, c, d.eps, q, k, v, q_norm, k_norm, freq, position, slots,
                      (uint16_t*)q_out, (uint16_t*)k_cache, (uint16_t*)v_cache};
    const int per = kStoreThreads / (d.dim / 8), passes = (d.heads + 2 * d.kv_heads + per - 1) / per;
    // Passes one after the other make the angles once; of a few tokens each has a
    // workgroup of its own (32 tokens, 5 passes: 5.8 and 4.3 us on the GPU).
    p.steps = (long long)d.T * passes <= kStoreSpread ? 1 : passes;
    const dim3 grid(d.T, (passes + p.steps - 1) / p.steps);
    hipStream_t s = (hipStream_t)stream;
    return timed_launch(CAEE_KERNEL_PLAN, s, "head store", [&] {
        auto run = [&](auto f32, auto dim, auto adjacent) {
            constexpr bool kF32 = decltype(f32)::value != 0, kAdj = decltype(adjacent)::value != 0;
            constexpr int D = decltype(dim)::value;
            hipLaunchKernelGGL((k_head_store<kF32, D, kAdj>), grid, dim3(kStoreThreads), 0, s, p);
        };
        auto pairs = [&](auto f32, auto dim) {
            if (d.adjacent) run(f32, dim, LatInt<1>{});
            else run(f32, dim, LatInt<0>{});
        };
        auto width = [&](auto f32) {
            if (d.dim == 128) pairs(f32, LatInt<128>{});
            else pairs(f32, LatInt<64>{});
        };
        if (d.x_dtype == CAEE_F32) width(LatInt<1>{});
        else width(LatInt<0>{});
        return hipGetLastError();
    });
}
