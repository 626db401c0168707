// The paged latent cache: pages, block tables and slots from request lengths
// (caee_paged_plan), and the new tokens' rows into their slots
// (caee_latent_store).
#include "latent.h"

namespace caee {
namespace {

constexpr int kPlanThreads = 1024;
constexpr int kMaxRequests = 65536;
// Tokens of the step per workgroup of the plan (one each for its threads).
constexpr int kPlanTokens = kPlanThreads;
constexpr int kPlanMaxGroups = 256;

struct PlanParams {
    int B, T, block, max_blocks, n_free, chunk;
    const int32_t* ctx_len;
    const int32_t* new_len;
    int32_t* table;
    const int32_t* free_list;
    const int32_t* free_head;
    caee_paged_plan_out_t o;
};

struct PlanLen {
    int ctx, add, have, want;   // tokens held and new; pages held and to take
};

__device__ inline PlanLen plan_len(const PlanParams& p, int b) {
    PlanLen r;
    r.ctx = max(p.ctx_len[b], 0);
    r.add = max(p.new_len[b], 0);
    r.have = (int)(((unsigned)r.ctx + (unsigned)p.block - 1u) / (unsigned)p.block);
    r.want = (int)(((unsigned)(r.ctx + r.add) + (unsigned)p.block - 1u) / (unsigned)p.block) - r.have;
    return r;
}

// Inclusive scans of N values per thread over the workgroup.
template <int N>
__device__ inline void scan_inclusive(int (&v)[N], int (*part)[kPlanThreads / kWave], int tid) {
    constexpr int kWaves = kPlanThreads / kWave;
    const int lane = tid & (kWave - 1), wave = tid / kWave;
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1)
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int u = __shfl_up(v[i], d);
            if (lane >= d) v[i] += u;
        }
    if (lane == kWave - 1) {
#pragma unroll
        for (int i = 0; i < N; ++i) part[i][wave] = v[i];
    }
    __syncthreads();
    // Every wave adds up the waves before it.
#pragma unroll
    for (int i = 0; i < N; ++i) {
        int u = lane < wave ? part[i][lane & (kWaves - 1)] : 0;
#pragma unroll
        for (int d = kWaves / 2; d >= 1; d >>= 1) u += __shfl_xor(u, d);
        v[i] += __builtin_amdgcn_readfirstlane(u);
    }
}

// Three prefix sums over the requests (new tokens, pages to take, cached
// tokens) and everything that follows from them, in one launch: latency is
// what bounds it, so every workgroup scans all requests for itself (a few
// thousand integers from L2) instead of waiting for another's scan, then
// takes its share of the tokens and of the requests' table rows.  Thread i
// scans requests [i chunk, (i + 1) chunk); a token finds its request by
// bisection over those 1024 ranges in LDS and a walk within one (a single
// request up to B = 1024).  A token's page comes from the lengths, not from
// the table entry another workgroup may be writing, so the workgroups share
// nothing.
__global__ __launch_bounds__(kPlanThreads) void k_paged_plan(PlanParams p) {
    __shared__ int s_new[kPlanThreads + 1], s_take[kPlanThreads + 1];
    __shared__ int part[3][kPlanThreads / kWave], part_over[1][kPlanThreads / kWave];
    const int tid = threadIdx.x;
    const int b0 = min(tid * p.chunk, p.B), b1 = min(b0 + p.chunk, p.B);
    const int head = max(p.free_head[0], 0);
    const int left = max(p.n_free - head, 0);
    int n_new = 0, n_take = 0, n_kv = 0;
    for (int b = b0; b < b1; ++b) {
        const PlanLen l = plan_len(p, b);
        n_new += l.add;
        n_take += l.want;
        n_kv += l.ctx + l.add;
    }
    int scan[3] = {n_new, n_take, n_kv};
    scan_inclusive(scan, part, tid);
    const int i_new = scan[0], i_take = scan[1], i_kv = scan[2];
    s_new[tid + 1] = i_new;
    s_take[tid + 1] = i_take;
    if (tid == 0) s_new[0] = s_take[0] = 0;
    if (blockIdx.x == 0) {
        int a = i_new - n_new, kv = i_kv - n_kv, over = 0, take = i_take - n_take;
        for (int b = b0; b < b1; ++b) {
            const PlanLen l = plan_len(p, b);
            p.o.cu_new[b] = a;
            p.o.cu_kv[b] = kv;
            p.o.seq_len[b] = l.ctx + l.add;
            a += l.add;
            kv += l.ctx + l.add;
            // pages that the list gives and the table has no entry for
            const int from = max(l.have, p.max_blocks), to = l.have + min(l.want, max(left - take, 0));
            over += max(to - from, 0);
            take += l.want;
        }
        int sum[1] = {over};
        scan_inclusive(sum, part_over, tid);
        const int i_over = sum[0];
        if (tid == kPlanThreads - 1) {
            p.o.cu_new[p.B] = i_new;
            p.o.cu_kv[p.B] = i_kv;
            p.o.free_head[0] = head + min(i_take, left);
            p.o.lacking[0] = max(i_take - left, 0) + i_over;
        }
    }
    __syncthreads();

    // Table rows: one wave per range of requests, lanes over the new pages (1000
    // requests that take a page each, one token: 45 us, none of them 11).
    const int lane = tid & (kWave - 1), wave = tid / kWave;
    const int n_waves = gridDim.x * (kPlanThreads / kWave), ranges = (p.B + p.chunk - 1) / p.chunk;
    for (int i = blockIdx.x * (kPlanThreads / kWave) + wave; i < ranges; i += n_waves) {
        int at = s_take[i];
        if (s_take[i + 1] == at) continue;
        const int e1 = min((i + 1) * p.chunk, p.B);
        for (int b = i * p.chunk; b < e1; ++b) {
            const PlanLen l = plan_len(p, b);
            int32_t* row = p.table + (size_t)b * p.max_blocks;
            for (int j = lane; j < l.want && l.have + j < p.max_blocks; j += kWave)
                row[l.have + j] = at + j < left ? p.free_list[head + at + j] : -1;
            at += l.want;
        }
    }

    const int total = s_new[kPlanThreads];
    for (int t = blockIdx.x * kPlanTokens + tid; t < p.T; t += gridDim.x * kPlanTokens) {
        long long slot = -1;
        int pos = -1, b = -1;
        if (t < total) {
            int lo = 0, hi = ranges;                // s_new[lo] <= t < s_new[hi]
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (s_new[mid] <= t) lo = mid;
                else hi = mid;
            }
            int first = s_new[lo], at = s_take[lo];
            b = lo * p.chunk;
            PlanLen l = plan_len(p, b);
            while (t >= first + l.add) {
                first += l.add;
                at += l.want;
                l = plan_len(p, ++b);
            }
            pos = l.ctx + (t - first);
            const int j = pos / p.block;
            if (j < p.max_blocks) {
                int page;
                if (j < l.have) page = p.table[(size_t)b * p.max_blocks + j];
                else page = at + (j - l.have) < left ? p.free_list[head + at + (j - l.have)] : -1;
                if (page >= 0) slot = (long long)page * p.block + (pos - j * p.block);
            }
        }
        p.o.slots[t] = slot;
        if (p.o.position) p.o.position[t] = pos;
        if (p.o.request) p.o.request[t] = b;
    }
}

struct StoreParams {
    int T, latent, rope, row_pieces, latent_pieces;
    const void* c;
    const void* r;
    long long c_stride, r_stride;
    const int64_t* slots;
    uint16_t* cache;
    long long n_slots;
};

// One thread moves 8 values (16 bytes of the cache row): consecutive lanes
// write consecutive pieces of a row, whole lines except at a row's ends.
// Bandwidth bounds it: 4 bytes moved per value.
template <bool kF32>
__global__ __launch_bounds__(256) void k_latent_store(StoreParams p) {
    const long long n = (long long)p.T * p.row_pieces;
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < n; i += (long long)gridDim.x * 256) {
        const int t = (int)(i / p.row_pieces), q = (int)(i - (long long)t * p.row_pieces);
        const long long slot = p.slots[t];
        if (slot < 0 || slot >= p.n_slots) continue;
        const bool lat = q < p.latent_pieces;
        const long long o = lat ? (long long)t * p.c_stride + 8 * q : (long long)t * p.r_stride + 8 * (q - p.latent_pieces);
        const void* base = lat ? p.c : p.r;
        uint4 v;
        if constexpr (kF32) {
            const float4 a = *(const float4*)((const float*)base + o), b = *(const float4*)((const float*)base + o + 4);
            v.x = lat_pack(a.x, a.y);
            v.y = lat_pack(a.z, a.w);
            v.z = lat_pack(b.x, b.y);
            v.w = lat_pack(b.z, b.w);
        } else {
            v = *(const uint4*)((const uint16_t*)base + o);
        }
        *(uint4*)(p.cache + slot * (p.latent + p.rope) + 8 * q) = v;
    }
}

// Workgroups read lengths, pages and the head while others write, in any
// order: an array that the plan writes may share no byte with another one.
caee_status_t check_plan_apart(const PlanParams& p) {
    struct Span {
        const char* name;
        const void* at;
        size_t bytes;
    };
    const size_t b = (size_t)p.B * 4, t = (size_t)p.T;
    const Span written[] = {{"block_table", p.table, b * (size_t)p.max_blocks}, {"out->cu_new", p.o.cu_new, b + 4},
                            {"out->cu_kv", p.o.cu_kv, b + 4},   {"out->seq_len", p.o.seq_len, b},
                            {"out->slots", p.o.slots, 8 * t},   {"out->position", p.o.position, 4 * t},
                            {"out->request", p.o.request, 4 * t}, {"out->free_head", p.o.free_head, 4},
                            {"out->lacking", p.o.lacking, 4}};
    const Span read[] = {{"ctx_len", p.ctx_len, b}, {"new_len", p.new_len, b},
                         {"free_list", p.free_list, (size_t)p.n_free * 4}, {"free_head", p.free_head, 4}};
    auto check = [](const Span& u, const Span& v) {
        const uintptr_t a = (uintptr_t)u.at, c = (uintptr_t)v.at;
        if (!u.at || !v.at || !u.bytes || !v.bytes || (a < c ? c - a >= u.bytes : a - c >= v.bytes)) return CAEE_OK;
        return fail(CAEE_ERR_INVALID_ARG, "%s overlaps %s", u.name, v.name);
    };
    for (const Span& w : written) {
        for (const Span& r : read) CAEE_TRY(check(w, r));
        for (const Span* other = written; other != &w; ++other) CAEE_TRY(check(w, *other));
    }
    return CAEE_OK;
}

}  // namespace
}  // namespace caee

using namespace caee;

extern "C" {

caee_status_t caee_paged_plan(int32_t B, int32_t T, int32_t block_size, int32_t max_blocks, const int32_t* ctx_len,
                              const int32_t* new_len, int32_t* block_table, const int32_t* free_list, int32_t n_free,
                              const int32_t* free_head, const caee_paged_plan_out_t* out, void* stream) {
    clear_last_error();
    if (B < 0 || T < 0) return fail(CAEE_ERR_INVALID_ARG, "B=%d and T=%d must be >= 0", B, T);
    if (block_size < 1 || block_size > 65536)
        return fail(CAEE_ERR_INVALID_ARG, "block_size=%d must be in [1, 65536]", block_size);
    if (max_blocks < 1) return fail(CAEE_ERR_INVALID_ARG, "max_blocks=%d must be >= 1", max_blocks);
    if (n_free < 0) return fail(CAEE_ERR_INVALID_ARG, "n_free=%d must be >= 0", n_free);
    if (!out) return fail(CAEE_ERR_INVALID_ARG, "out is NULL");
    CAEE_TRY(check_ptr(ctx_len, "ctx_len", B > 0));
    CAEE_TRY(check_ptr(new_len, "new_len", B > 0));
    CAEE_TRY(check_ptr(block_table, "block_table", B > 0));
    CAEE_TRY(check_ptr(free_list, "free_list", n_free > 0));
    CAEE_TRY(check_ptr(free_head, "free_head", true));
    CAEE_TRY(check_ptr(out->cu_new, "out->cu_new", true));
    CAEE_TRY(check_ptr(out->cu_kv, "out->cu_kv", true));
    CAEE_TRY(check_ptr(out->seq_len, "out->seq_len", B > 0));
    CAEE_TRY(check_ptr(out->slots, "out->slots", T > 0));
    CAEE_TRY(check_ptr(out->position, "out->position", false));
    CAEE_TRY(check_ptr(out->request, "out->request", false));
    CAEE_TRY(check_ptr(out->free_head, "out->free_head", true));
    CAEE_TRY(check_ptr(out->lacking, "out->lacking", true));
    if (B > kMaxRequests) return fail(CAEE_ERR_UNSUPPORTED, "B=%d exceeds %d", B, kMaxRequests);
    PlanParams p{B, T, block_size, max_blocks, n_free, (B + kPlanThreads - 1) / kPlanThreads, ctx_len, new_len,
                 block_table, free_list, free_head, *out};
    if (p.chunk < 1) p.chunk = 1;
    CAEE_TRY(check_plan_apart(p));
    int groups = (T + kPlanTokens - 1) / kPlanTokens;
    groups = groups < 1 ? 1 : groups > kPlanMaxGroups ? kPlanMaxGroups : groups;
    hipStream_t s = (hipStream_t)stream;
    return timed_launch(CAEE_KERNEL_PLAN, s, "paged plan", [&] {
        hipLaunchKernelGGL(k_paged_plan, dim3(groups), dim3(kPlanThreads), 0, s, p);
        return hipGetLastError();
    });
}

caee_status_t caee_latent_store(int32_t T, int32_t latent, int32_t rope, int32_t x_dtype, const void* c,
                                int64_t c_stride, const void* r, int64_t r_stride, const int64_t* slots, void* cache,
                                int64_t n_slots, void* stream) {
    clear_last_error();
    if (T < 0) return fail(CAEE_ERR_INVALID_ARG, "T=%d must be >= 0", T);
    if (latent < 8 || latent % 8 || rope < 8 || rope % 8 || latent > 65536 || rope > 65536)
        return fail(CAEE_ERR_INVALID_ARG, "latent=%d and rope=%d must be multiples of 8 in [8, 65536]", latent, rope);
    if (x_dtype != CAEE_BF16 && x_dtype != CAEE_F32)
        return fail(CAEE_ERR_INVALID_ARG, "x_dtype=%d must be CAEE_BF16 or CAEE_F32", x_dtype);
    const int unit = x_dtype == CAEE_BF16 ? 8 : 4;   // elements of 16 bytes
    if (c_stride < latent || c_stride % unit || r_stride < rope || r_stride % unit)
        return fail(CAEE_ERR_INVALID_ARG, "row strides %lld, %lld must hold the rows and keep them 16-byte aligned",
                    (long long)c_stride, (long long)r_stride);
    if (n_slots < 0) return fail(CAEE_ERR_INVALID_ARG, "n_slots=%lld must be >= 0", (long long)n_slots);
    if (T == 0) return CAEE_OK;
    CAEE_TRY(check_ptr(c, "c", true));
    CAEE_TRY(check_ptr(r, "r", true));
    CAEE_TRY(check_ptr(slots, "slots", true));
    CAEE_TRY(check_ptr(cache, "cache", true));
    StoreParams p{T, latent, rope, (latent + rope) / 8, latent / 8, c, r, c_stride, r_stride, slots, (uint16_t*)cache,
                  n_slots};
    const long long n = (long long)T * p.row_pieces;
    const long long groups = (n + 255) / 256;
    const dim3 grid((unsigned)(groups < 65536 ? groups : 65536));
    hipStream_t s = (hipStream_t)stream;
    return timed_launch(CAEE_KERNEL_PLAN, s, "latent store", [&] {
        if (x_dtype == CAEE_F32) hipLaunchKernelGGL(k_latent_store<true>, grid, dim3(256), 0, s, p);
        else hipLaunchKernelGGL(k_latent_store<false>, grid, dim3(256), 0, s, p);
        return hipGetLastError();
    });
}

}  // extern "C"
