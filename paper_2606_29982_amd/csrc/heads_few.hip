// Attention with grouped heads, split form of few rows: decode steps and small
// trees, up to 32 query rows a tile.
//
//   k_head_meta   prefix sums, where there are more than 64 requests
//   k_head_few    a share of all requests' tokens a workgroup
//   k_head_join   partial results of rows whose tokens several shares have
#include <algorithm>

#include "heads.h"

namespace caee {
namespace {

constexpr int kFewThreads = 256;
constexpr int kWaveTokens = 32;

// First unit of each request (meta[b]; meta[B] the total); or first piece, of one
// group, and the steps of a piece (meta[B + 1]): row tiles are cut where all of
// them would leave CUs idle.  One workgroup, a few requests a lane, scans over
// them: a chain of loads and barriers (launch included 5 us for 300 requests, which
// is why up to 64 requests the workgroups sum by themselves).
__global__ __launch_bounds__(kFewThreads) void k_head_meta(HeadParams p, int few) {
    __shared__ int part[kFewThreads];
    __shared__ float work[kFewThreads];
    const int tid = threadIdx.x;
    const int chunk = (p.B + kFewThreads - 1) / kFewThreads;
    const int b0 = min(tid * chunk, p.B), b1 = min(b0 + chunk, p.B);
    int per = INT32_MAX / 2;
    if (!few && p.part) {
        int tiles = 0;
        float steps = 0.0f;
        for (int b = b0; b < b1; ++b) {
            const LatentReq r = head_req(p, b);
            const int t = head_tiles(p, r);
            tiles = head_add_units(tiles, t);
            steps += (float)t * (float)head_steps(r);
        }
        part[tid] = tiles;
        work[tid] = steps;
        __syncthreads();
        for (int d = kFewThreads / 2; d >= 1; d >>= 1) {
            if (tid < d) {
                part[tid] = head_add_units(part[tid], part[tid + d]);
                work[tid] += work[tid + d];
            }
            __syncthreads();
        }
        // (a row tile has fewer than steps / per + 1 pieces; what is rounded in `work` has room)
        if ((long long)part[0] * p.G < kTileSlots) per = max((int)ceilf(work[0] * (1.001f / kTileSlots) * (float)p.G), 1);
        __syncthreads();
    }
    auto number = [&](int b) {
        const LatentReq r = head_req(p, b);
        return few ? head_few_units(p, r) : head_tiles(p, r) * head_cut(head_steps(r), per);
    };
    int n = 0;
    for (int b = b0; b < b1; ++b) n = head_add_units(n, number(b));
    part[tid] = n;
    __syncthreads();
    for (int d = 1; d < kFewThreads; d <<= 1) {
        const int u = tid >= d ? part[tid - d] : 0;
        __syncthreads();
        part[tid] = head_add_units(part[tid], u);
        __syncthreads();
    }
    int at = tid > 0 ? part[tid - 1] : 0;
    for (int b = b0; b < b1; ++b) {
        p.meta[b] = at;
        at = head_add_units(at, number(b));
    }
    if (tid == kFewThreads - 1) {
        p.meta[p.B] = part[kFewThreads - 1];
        p.meta[p.B + 1] = per;
    }
}

// A list of units of one row tile, and where in it a share goes on.
struct FewList {
    int b, at;            // request, its first unit
    LatentReq rq;
    int n, tile, first;   // units of each of the request's lists; which list; the first unit of it
};
// Units of tokens before unit i of a list.
__device__ inline int few_before(const HeadParams& p, int i) { return max(i - p.few_start, 0); }
__device__ inline int few_tiles(const HeadParams& p, const FewList& x) { return (x.rq.add * p.ratio + kFewRows - 1) / kFewRows; }
__device__ inline FewList few_request(const HeadParams& p, const HeadLine& line, int b) {
    FewList x = {};
    x.b = b;
    x.rq = head_line_req(p, line, b, &x.at);
    x.n = head_few_list(p, x.rq);
    return x;
}
// The list that unit u is of.
__device__ inline FewList few_list(const HeadParams& p, const HeadLine& line, int u) {
    FewList x = few_request(p, line, head_line_find(p, line, u));
    x.tile = head_div(u - x.at, x.n);
    x.first = u - x.at - x.tile * x.n;
    return x;
}
// The list after x, which begins with unit u: mostly of the same request, or of the next one.
__device__ inline FewList few_after(const HeadParams& p, const HeadLine& line, const FewList& x, int u) {
    if (x.tile + 1 < p.G * few_tiles(p, x)) return {x.b, x.at, x.rq, x.n, x.tile + 1, 0};
    if (p.B > kWave && x.b + 1 < p.B && __builtin_amdgcn_readfirstlane(p.meta[x.b + 2]) > u) return few_request(p, line, x.b + 1);
    return few_request(p, line, head_line_find(p, line, u));
}

// Keys or values of 32 tokens for each wave: blocks of 8 rows x 128 bytes,
// swizzled, so that one direct-to-LDS load fills a block.
template <int D>
struct FewStage {
    lat_u32x4 v[4][kWaveTokens / 8][D / 64][kWave];
};

// A workgroup walks over its share, 32 tokens a wave and step.  A wave keeps its
// tokens' keys and values in a part of LDS of its own and its row statistics and
// sums in registers, so the waves meet only at a row tile's end.  Keys are the
// M side of the scores, so that a lane holds 16 scores of one row, whose
// weights are, in that order, a fragment of the second product; values are read
// transposed.  The next keys are fetched as soon as the scores are made, the
// next values after the sums; another workgroup of the CU fills the gaps.
// Weights are multiplied in two bf16 parts, so that they lose nothing beside
// the result's own rounding (matrix units are busy 10 to 13 % of the time: the
// second part is free; a result of 32 bits has three).
// Memory bounds it: 5 users of 120000 tokens, 8 groups 367 us for 2.34 GB (6.4
// TB/s, of the 6.95 that a large copy reads); 64 users of 2050 tokens on average
// 93 us for 503 MB (5.4), as a share begins and ends two lists, which the other
// workgroup of the CU hides in part; the next list's queries and pages are asked for
// while the last one's results leave (256 users of 1000 tokens 224 and 235).  Finer shares
// dealt out in turn gained nothing (2 and 4 times as many: 354 and 360 us beside 351
// for long lists, 104 and 109 beside 100 for short ones).  A user of 902 tokens
// takes 7.9, a chain of launch, lengths, pages, fetch, one step
// and the result's way out.  Pages by head are 6 % faster than by token (92 and 98 us
// for 64 users), as a wave's eight rows are one line after the other.
template <int D, bool kTree, bool kOnce, bool kLast>
__global__ __launch_bounds__(kFewThreads, 2) void k_head_few(HeadParams p) {
#if defined(__HIP_DEVICE_COMPILE__)   // the buffer-descriptor type exists for the GPU target only
    constexpr int kG = D / 64, kJ = D / 16, NC = D / 32, kLoads = kWaveTokens / 8 * kG;
    __shared__ FewStage<D> ks, vs;
    __shared__ lat_u32x4 qs[kFewRows / 8][kG][kWave];
    __shared__ float2 ml[4][kFewRows];
    __shared__ int row_at[2][kFewRows];    // of this list and the next
    const int lane = threadIdx.x & 63, n = lane & 31, hf = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    HeadLine line = head_line(p);
    head_line_sum(p, &line, head_few_units(p, line.mine));
    const int per = head_share(line.total), group = head_group(blockIdx.x);
    const int share0 = (int)min((long long)group * per, (long long)line.total), share1 = min(share0 + per, line.total);

    const int kp0 = (n >> 3) * (kG * kWave) + (n & 7) * 8 + (hf ^ lat_swz(n));
    const int vrow = 4 * hf + ((lane & 15) >> 2);
    int vpos[2][2];       // [column tile parity][eight of a 16-token step]
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int e = 0; e < 2; ++e)
            vpos[j][e] = 2 * (vrow * 8 + ((4 * j + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) ^ lat_swz(8 * e + vrow))) + (lane & 1);
    const uint32_t row_bytes = (uint32_t)p.c.row_stride * 2u;

    constexpr int kEights = kWaveTokens / 8, kLook = kHeadWindow / kEights;
    auto look_at = [&](const FewList& x, int s) __attribute__((always_inline)) {
        return head_look(p, x.b, x.rq.seq, (few_before(p, x.first) + s + lane / kEights) * kFewTokens + kWaveTokens * wave + 8 * (lane % kEights));
    };
    // Asks for a list's queries and its first pages.
    auto open = [&](const FewList& x, int parity) __attribute__((always_inline)) {
        const int tiles = few_tiles(p, x), g = head_div(x.tile, tiles), row0 = (x.tile - g * tiles) * kFewRows;
        const HeadLook soon = look_at(x, 0);
        const int r = 8 * wave + (lane >> 3), rr = min(row0 + r, x.rq.add * p.ratio - 1), i = head_over(rr, p.by_ratio);
        const uint16_t* src = p.q + (size_t)(x.rq.t0 + i) * p.q_stride + (size_t)(g * p.ratio + rr - i * p.ratio) * D +
                              8 * ((lane & 7) ^ lat_swz(r));
#pragma unroll
        for (int gg = 0; gg < kG; ++gg)
            __builtin_amdgcn_global_load_lds((lat_g_void*)(src + 64 * gg), (lat_lds_void*)&qs[wave][gg][0], 16, 0, 0);
        if ((lane & 7) == 0) row_at[parity][r] = (x.rq.t0 + i) * p.H + g * p.ratio + rr - i * p.ratio;
        return soon;
    };
    if (share0 >= share1) return;
    FewList list = few_list(p, line, share0);
    HeadLook soon = open(list, 0);     // of kLook tiles: the first ones, and then the next
    for (int u = share0, parity = 0;; parity ^= 1) {
        const int b = list.b, n_u = list.n, first = list.first;
        const LatentReq rq = list.rq;
        const int rows = rq.add * p.ratio, tiles = few_tiles(p, list);
        const int g = head_div(list.tile, tiles), rt = list.tile - g * tiles;
        const int last = min(n_u, first + (share1 - u));
        const bool whole = first == 0 && last == n_u, head = u == share0;
        u += last - first;

        const int row0 = rt * kFewRows, n_rows = min(kFewRows, rows - row0);
        const int row = row0 + min(n, n_rows - 1), tok = head_over(row, p.by_ratio);
        const int limit = head_sees(p, rq, tok);
        // Tokens from lim_min on some row does not see.
        const int lim_min = kTree ? min(max(rq.before, 0), rq.seq) : head_sees(p, rq, head_over(row0, p.by_ratio));
        const int end = min(few_before(p, last) * kFewTokens, head_sees(p, rq, head_over(row0 + n_rows - 1, p.by_ratio)));
        const int tok0 = few_before(p, first) * kFewTokens + kWaveTokens * wave;
        const int steps = end > tok0 ? (end - tok0 + kFewTokens - 1) / kFewTokens : 0;
        const uint32_t* mask = kTree ? p.tree + (size_t)(rq.t0 + tok) * p.words : nullptr;

        auto piece = [&](int i) __attribute__((always_inline)) { return 16u * ((lane & 7) ^ lat_swz(8 * (i & 1) + (lane >> 3))); };
        const char *const k_base = head_base(p, p.k, g), *const v_base = head_base(p, p.v, g);
        // A buffer of size 0 past the last tile: its loads cost no traffic, and their
        // number does not depend on a branch.
        auto fetch = [&](const char* cache, FewStage<D>& st, int s, const HeadWindow& w) __attribute__((always_inline)) {
            const bool there = s < steps;
            bool far = false;
#pragma unroll
            for (int i = 0; i < kEights; ++i) {
                const HeadEight e = head_eight(w, s % kLook * kEights + i);
                const __amdgpu_buffer_rsrc_t buf =
                    __builtin_amdgcn_make_buffer_rsrc((void*)(cache + e.off), 0, there && e.span >= 0 ? kLatBufBytes : 0, kLatBufWord3);
                const uint32_t at = (uint32_t)min(lane >> 3, e.span) * row_bytes + piece(i);
#pragma unroll
                for (int gg = 0; gg < kG; ++gg)
                    __builtin_amdgcn_raw_ptr_buffer_load_lds(buf, (lat_lds_void*)&st.v[wave][i][gg][0], 16, at, 128 * gg, 0, kOnce ? 2 : 0);
                far |= e.span < 0;
            }
            if (there && far) {
                // Rows in several pages, each by an address of its own, after the loads above, which touch nothing there.
                lat_wait_vm<0>();
#pragma unroll 1
                for (int i = 0; i < kEights; ++i) {
                    if (__builtin_amdgcn_readlane(w.span, s % kLook * kEights + i) >= 0) continue;
                    const int pos = min(tok0 + s * kFewTokens + 8 * i + (lane >> 3), rq.seq - 1);
                    const char* row = cache + head_row(p, b, pos) + piece(i);
#pragma unroll
                    for (int gg = 0; gg < kG; ++gg)
                        __builtin_amdgcn_global_load_lds((lat_g_void*)(row + 128 * gg), (lat_lds_void*)&st.v[wave][i][gg][0], 16, 0, 0);
                }
                lat_wait_vm<0>();
            }
        };

        HeadWindow win = head_window(p, soon);         // of kLook tiles
        lat_wait_vm<0>();
        __syncthreads();       // the queries are there, the list before is done with LDS
        fetch(k_base, ks, 0, win);
        fetch(v_base, vs, 0, win);
        lat_u32x4 qf[kJ];
#pragma unroll
        for (int j = 0; j < kJ; ++j) qf[j] = (&qs[0][0][0])[(kp0 ^ (2 * (j & 3))) + (j >> 2) * kWave];
        lat_f32x16 o[NC];
#pragma unroll
        for (int c = 0; c < NC; ++c) o[c] = lat_f32x16{};
        float m = kNoScore, l = 0.0f;
        bool odd = false;      // an infinity or NaN was taken out of the values

        for (int s = 0; s < steps; ++s) {
            const int tb = tok0 + s * kFewTokens;
            lat_wait_vm<kLoads>();             // the keys are there, the values may be on their way
            asm volatile("" ::: "memory");
            const lat_u32x4* keys = &ks.v[wave][0][0][0];
            lat_f32x16 sc = {};
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int j = 0; j < kJ; ++j) sc = lat_mma(keys[(kp0 ^ (2 * (j & 3))) + (j >> 2) * kWave], qf[j], sc);
            __builtin_amdgcn_s_waitcnt(15 | (7 << 4) | (0 << 8) | (3 << 14));
            __builtin_amdgcn_sched_barrier(0);
            // the window of tile s + 1 on, asked for half a window before
            if ((s + 1) % kLook == kLook / 2) soon = look_at(list, (s + 1) / kLook * kLook + kLook);
            if ((s + 1) % kLook == 0) win = head_window(p, soon);
            fetch(k_base, ks, s + 1, win);
            const bool masked = tb + kWaveTokens > lim_min;
            if (masked) {
                asm volatile("");       // a branch, not selects in every step
                const int left = limit - (tb + 4 * hf);
                const uint32_t bits = kTree ? head_tree_bits(mask, p.words, tb - rq.before) >> (4 * hf) : 0u;
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    constexpr auto at = [](int x) constexpr { return 8 * (x >> 2) + (x & 3); };
                    if (at(i) >= left || (kTree && !(bits >> at(i) & 1))) sc[i] = -INFINITY;
                }
            }
            // The weights by the running maximum; where it has to move they are made again.
            lat_u32x4 pf[2], pr[2], pl[2];
            float more = 0.0f;
            auto weights = [&](auto&& weight) __attribute__((always_inline)) {
#pragma unroll
                for (int k = 0; k < 2; ++k)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float a = weight(sc[8 * k + 2 * i], p.scale_log2, m);
                        const float e = weight(sc[8 * k + 2 * i + 1], p.scale_log2, m);
                        pf[k][i] = lat_pack(a, e);
                        const lat_f32x2 rest = lat_rest(pf[k][i], a, e);
                        pr[k][i] = lat_pack(rest[0], rest[1]);
                        if constexpr (kLast) {
                            const lat_f32x2 last = lat_rest(pr[k][i], rest[0], rest[1]);
                            pl[k][i] = lat_pack(last[0], last[1]);
                        }
                        more += a + e;
                    }
            };
            if (s > 0) weights(head_weight);
            if (s == 0 || __any(head_moves(more, m))) {
                float mt = sc[0];
#pragma unroll
                for (int i = 1; i < 16; ++i) mt = fmaxf(mt, sc[i]);
                mt = lat_max_pair(mt) * p.scale_log2;
                const float mn = fmaxf(m, mt), f = __builtin_amdgcn_exp2f(m - mn);
                l *= f;
                m = mn;
#pragma unroll
                for (int c = 0; c < NC; ++c) o[c] *= f;
                more = 0.0f;
                weights(lat_weight);
            }
            l += more;
            lat_wait_vm<kLoads>();             // the values are there
            asm volatile("" ::: "memory");
            if (masked) {
                // Tokens that some rows do not see may hold anything: infinities
                // and NaNs must not meet their zero weights.
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (tb + 8 * i + (lane >> 3) >= lim_min) {
#pragma unroll
                        for (int gg = 0; gg < kG; ++gg) {
                            const lat_u32x4 v = vs.v[wave][i][gg][lane];
                            lat_u32x4 w;
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                w[e] = lat_finite(v[e]);
                                odd |= w[e] != v[e];
                            }
                            vs.v[wave][i][gg][lane] = w;
                        }
                    }
                __builtin_amdgcn_s_waitcnt(15 | (7 << 4) | (0 << 8) | (3 << 14));
                asm volatile("" ::: "memory");
            }
            const lat_u32x2* base = (const lat_u32x2*)&vs.v[wave][0][0][0];
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int c = 0; c < NC; ++c) {
                    lat_u32x2 w[2];
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const lat_u32x2* at = base + ((2 * k + e) * kG + (c >> 1)) * (2 * kWave) + vpos[c & 1][e];
                        w[e] = __builtin_bit_cast(lat_u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lat_lds_s16x4*)at));
                    }
                    const lat_u32x4 vf = {w[0][0], w[0][1], w[1][0], w[1][1]};
                    o[c] = lat_mma(vf, pf[k], o[c]);
                    o[c] = lat_mma(vf, pr[k], o[c]);
                    if constexpr (kLast) o[c] = lat_mma(vf, pl[k], o[c]);
                }
            __builtin_amdgcn_s_waitcnt(15 | (7 << 4) | (0 << 8) | (3 << 14));
            __builtin_amdgcn_sched_barrier(0);
            fetch(v_base, vs, s + 1, win);
        }
        lat_wait_vm<0>();
        l = lat_sum_pair(l);
        odd |= head_odd(o, l);
        // The waves' results through LDS, 16 rows in the wave's keys and 16 in its
        // values, unit c (16 bytes) of a row at c ^ (row % units).
        constexpr int kUnits = D / 4;
        int ln = lane;         // addresses made here: the registers that they would take through the loop are not there
        asm volatile("" : "+v"(ln));
        if (hf == 0) ml[wave][n] = make_float2(m, l);
        auto place = [&](int w, int r, int c) __attribute__((always_inline)) {
            return (float4*)(r < 16 ? &ks.v[w][0][0][0] : &vs.v[w][0][0][0]) + (r & 15) * kUnits + (c ^ (r & 15));
        };
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                *place(wave, ln & 31, 8 * c + 2 * i + (ln >> 5)) = make_float4(o[c][4 * i], o[c][4 * i + 1], o[c][4 * i + 2], o[c][4 * i + 3]);
        if (__any(odd)) {
            auto sees = [&](int pos) { return pos < limit && (!kTree || (head_tree_bits(mask, p.words, pos - rq.before) & 1)); };
            head_put_odd<D>(p, b, g, tok0, kWaveTokens, kFewTokens, end, sees,
                            [&](int d, float v, bool again) {
                                float& at = ((float*)place(wave, n, d >> 2))[d & 3];
                                at = again ? at + v : v;
                            });
        }
        __syncthreads();
        const bool more = u < share1;
        if (more) {            // the next list's queries and pages are on their way while this one's results leave
            list = few_after(p, line, list, u);
            soon = open(list, parity ^ 1);
        }
        const size_t slot0 = ((size_t)blockIdx.x * 2 + (head ? 0 : 1)) * kFewRows;
        for (int x = threadIdx.x; x < n_rows * kUnits; x += kFewThreads) {
            const int r = x / kUnits, c = x % kUnits;
            float2 w[4];
            float mx = kNoScore, lx = 0.0f;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                w[i] = ml[i][r];
                mx = fmaxf(mx, w[i].x);
            }
            float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            auto sum = [&](auto odd) __attribute__((always_inline)) {
                constexpr bool kOdd = decltype(odd)::value != 0;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float f = __builtin_amdgcn_exp2f(w[i].x - mx);
                    const float4 t = *place(i, r, c);
                    if (!kOdd) lx += w[i].y * f;
                    v = make_float4(head_join<kOdd>(v.x, 1.0f, t.x, f), head_join<kOdd>(v.y, 1.0f, t.y, f), head_join<kOdd>(v.z, 1.0f, t.z, f),
                                    head_join<kOdd>(v.w, 1.0f, t.w, f));
                }
            };
            sum(LatInt<0>{});
            if (!head_finite(v)) {
                v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                sum(LatInt<1>{});
            }
            if (!whole) {
                *(float4*)(p.part + (slot0 + r) * D + 4 * c) = v;
                if (c == 0) *(float2*)(p.part_ml + 2 * (slot0 + r)) = make_float2(mx, lx);
                continue;
            }
            const float f = head_inverse(lx);
            const size_t at = (size_t)row_at[parity][r];
            if (p.y_bf16) *(lat_u32x2*)((uint16_t*)p.y + at * D + 4 * c) = lat_u32x2{lat_pack(v.x * f, v.y * f), lat_pack(v.z * f, v.w * f)};
            else *(float4*)((float*)p.y + at * D + 4 * c) = make_float4(v.x * f, v.y * f, v.z * f, v.w * f);
            if (p.lse && c == 0) p.lse[at] = lat_lse(mx, lx);
        }
        if (!more) return;
    }
#endif
}

// Rows whose tokens lie in one share (piece) are done; the others are the sum of
// their shares' partial results, D / 4 lanes a row and 16 bytes a lane; rows that see
// no token are zero.  A workgroup has a token's heads: few rows, which have many
// partial results, one pass of heads (64 / (D / 4)) whose shares go over the four
// waves in turn, their sums added in order; many rows four passes a wave.  Each
// partial result is read once (m and l of a row by all its lanes): 4.4 us for 64 users'
// 64 heads, 3.5 for 8 rows of a launch's latency; of many rows 50 MB in 13 us for 16
// trees of 61 tokens, 60 in 17 for 259 tokens of 2 prompts behind 30000.
constexpr int kJoinRows = 4096;        // (token, head) rows from which on they are many
template <int D, bool kMany, bool kSum>
__global__ __launch_bounds__(kFewThreads) void k_head_join(HeadParams p, int few) {
    constexpr int kLanes = D / 4, kHeads = kWave / kLanes, kPasses = kMany ? 4 : 1, kWaves = kFewThreads / kWave;
    __shared__ float4 red_v[kMany ? 1 : kWaves - 1][kWave];
    __shared__ float2 red_ml[kMany ? 1 : kWaves - 1][kWave];
    __shared__ float red_all[kMany || !kSum ? 1 : kWaves - 1][kWave];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int per_wg = kMany ? kHeads * kPasses * kWaves : kHeads, wgs = (p.H + per_wg - 1) / per_wg;
    const int wg = (int)lat_workgroup(), t = head_div(wg, wgs);
    if (t >= p.T) return;
    const int h0 = (wg - t * wgs) * per_wg + (kMany ? kHeads * kPasses * wave : 0) + lane / kLanes, c = lane % kLanes;
    HeadLine line = head_line(p);
    const int piece = few ? 1 : __builtin_amdgcn_readfirstlane(p.meta[p.B + 1]);
    head_line_sum(p, &line, few ? head_few_units(p, line.mine) : head_tiles(p, line.mine) * head_cut(head_steps(line.mine), piece));
    auto leave = [&](int h, const float4& v, float m, float l, float all) __attribute__((always_inline)) {
        const size_t at = (size_t)t * p.H + h;
        const float inv = head_inverse(l);
        if (p.lse && c == 0) p.lse[at] = lat_lse(m, all);
        if (p.y_bf16) *(lat_u32x2*)((uint16_t*)p.y + at * D + 4 * c) = lat_u32x2{lat_pack(v.x * inv, v.y * inv), lat_pack(v.z * inv, v.w * inv)};
        else *(float4*)((float*)p.y + at * D + 4 * c) = make_float4(v.x * inv, v.y * inv, v.z * inv, v.w * inv);
    };
    const float4 zero = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    // Units of a row tile; 0 where the row sees nothing.
    int b = 0, at_u = 0, n_u = 0;
    LatentReq rq = {};
    if (p.B > kWave) {
        if (t < p.cu_new[p.B]) {
            b = lat_find_wave(p.cu_new, p.B, t);
            rq = head_line_req(p, line, b, &at_u);
        }
    } else {
        // the last request whose tokens begin at or before t; rows past it have none
        const unsigned long long before = __ballot(lane < p.B && line.mine.t0 <= t);
        if (before) {
            b = 63 - __clzll(before);
            rq = head_line_req(p, line, b, &at_u);
        }
    }
    if (t >= rq.t0 && t - rq.t0 < rq.add) n_u = few ? head_few_list(p, rq) : head_steps(rq);
    if (n_u == 0) {
#pragma unroll
        for (int i = 0; i < kPasses; ++i)
            if (h0 + kHeads * i < p.H && (kMany || wave == 0)) leave(h0 + kHeads * i, zero, kNoScore, 0.0f, 0.0f);
        return;
    }
    const int tile_rows = few ? kFewRows : kTileRows;
    const int tiles = (rq.add * p.ratio + tile_rows - 1) / tile_rows;
    const int per = few ? head_share(line.total) : 1, cut = few ? 1 : __builtin_amdgcn_readfirstlane(head_cut(n_u, piece));
    if (!few && cut == 1) return;
    float4 sum[kPasses];
    float m[kPasses], l[kPasses], all[kPasses];      // all: the sum before the weights were rounded
    int g0[kPasses], g1[kPasses], a[kPasses], rr[kPasses], most = 0;
#pragma unroll
    for (int i = 0; i < kPasses; ++i) {
        const int h = min(h0 + kHeads * i, p.H - 1), kv = head_over(h, p.by_ratio), r = (t - rq.t0) * p.ratio + h - kv * p.ratio;
        rr[i] = r % tile_rows;
        if (few) {         // shares
            a[i] = at_u + (kv * tiles + r / kFewRows) * n_u;
            g0[i] = min((int)((unsigned)a[i] / (unsigned)per), kFewGroups - 1);
            g1[i] = min((int)((unsigned)(a[i] + n_u - 1) / (unsigned)per), kFewGroups - 1);
        } else {           // pieces
            g0[i] = kv * line.total + at_u + r / kTileRows * cut;
            g1[i] = g0[i] + cut - 1;
            a[i] = 0;
        }
        if (g0[i] < g1[i] && h0 + kHeads * i < p.H) most = max(most, g1[i] - g0[i] + 1);
    }
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) most = max(most, __shfl_xor(most, d));
    if (most == 0 && kMany) return;
    // Share k of each pass's row: its second slot when the row tile's line begins inside the share.
    auto add = [&](int k0, auto count, auto odd) __attribute__((always_inline)) {
        constexpr int U = decltype(count)::value;
        float2 w[U][kPasses];
        float4 x[U][kPasses];
        float wa[U][kPasses];
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int i = 0; i < kPasses; ++i) {
                const int g = min(g0[i] + k0 + (kMany ? u : kWaves * u), g1[i]);
                const size_t at = few ? (size_t)head_workgroup(g) * 2 + (g == g0[i] && a[i] > g0[i] * per ? 1 : 0) : (size_t)g;
                const size_t slot = at * tile_rows + rr[i];
                w[u][i] = ((const float2*)p.part_ml)[slot];
                x[u][i] = *(const float4*)(p.part + slot * D + 4 * c);
                if constexpr (kSum) wa[u][i] = p.part_sum[slot];
                else wa[u][i] = w[u][i].y;
            }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int i = 0; i < kPasses; ++i) {
                if (g0[i] + k0 + (kMany ? u : kWaves * u) > g1[i] || w[u][i].x == kNoPart) continue;
                head_merge<decltype(odd)::value != 0>(sum[i], m[i], l[i], all[i], x[u][i], w[u][i], wa[u][i]);
            }
    };
    // The shares of this wave, and those with sums that are no numbers once more.
    auto join = [&](auto count, auto odd) __attribute__((always_inline)) {
        constexpr int kStep = kMany ? 1 : kWaves, U = decltype(count)::value;
#pragma unroll
        for (int i = 0; i < kPasses; ++i) {
            sum[i] = zero;
            m[i] = kNoScore;
            l[i] = all[i] = 0.0f;
        }
        for (int k = kMany ? 0 : wave; k < most; k += U * kStep) add(k, count, odd);
    };
    join(LatInt<kMany ? 2 : 8>{}, LatInt<0>{});
    bool odd = false;
#pragma unroll
    for (int i = 0; i < kPasses; ++i) odd |= g0[i] < g1[i] && !head_finite(sum[i]);
    if (odd) join(LatInt<1>{}, LatInt<1>{});
    if constexpr (!kMany) {
        if (wave > 0) {
            red_v[wave - 1][lane] = sum[0];
            red_ml[wave - 1][lane] = make_float2(m[0], l[0]);
            if constexpr (kSum) red_all[wave - 1][lane] = all[0];
        }
        __syncthreads();
        if (wave > 0) return;
        const float4 sum0 = sum[0];
        const float m0 = m[0], l0 = l[0], all0 = all[0];
        auto waves = [&](auto odd) __attribute__((always_inline)) {
#pragma unroll
            for (int w = 0; w < kWaves - 1; ++w) {
                const float2 ml = red_ml[w][lane];
                head_merge<decltype(odd)::value != 0>(sum[0], m[0], l[0], all[0], red_v[w][lane], ml, kSum ? red_all[w][lane] : ml.y);
            }
        };
        waves(LatInt<0>{});
        if (g0[0] < g1[0] && !head_finite(sum[0])) {
            sum[0] = sum0, m[0] = m0, l[0] = l0, all[0] = all0;
            waves(LatInt<1>{});
        }
    }
#pragma unroll
    for (int i = 0; i < kPasses; ++i)
        if (h0 + kHeads * i < p.H && g0[i] < g1[i]) leave(h0 + kHeads * i, sum[i], m[i], l[i], all[i]);
}

}  // namespace

namespace {

void meta(const HeadParams& p, int few, hipStream_t s) {
    if (p.B > kWave) hipLaunchKernelGGL(k_head_meta, dim3(1), dim3(kFewThreads), 0, s, p, few);
}

void join(const HeadParams& p, int few, hipStream_t s) {
    auto run = [&](auto dim, auto many, auto sum) {
        constexpr int D = decltype(dim)::value, kPer = kWave / (D / 4) * (decltype(many)::value ? 16 : 1);
        hipLaunchKernelGGL((k_head_join<D, decltype(many)::value != 0, decltype(sum)::value != 0>),
                           lat_grid((unsigned)(p.T * ((p.H + kPer - 1) / kPer))), dim3(kFewThreads), 0, s, p, few);
    };
    auto sums = [&](auto dim, auto many) {
        if (p.part_sum) run(dim, many, LatInt<1>{});
        else run(dim, many, LatInt<0>{});
    };
    auto dims = [&](auto many) {
        if (p.dim == 128) sums(LatInt<128>{}, many);
        else sums(LatInt<64>{}, many);
    };
    if ((long long)p.T * p.H >= kJoinRows) dims(LatInt<1>{});
    else dims(LatInt<0>{});
}

}  // namespace

hipError_t launch_head_few(const HeadParams& p, hipStream_t s) {
    meta(p, 1, s);
    const bool once = (long long)p.max_new * p.ratio <= kFewRows;      // one row tile a request and group reads its tokens
    auto few = [&](auto dim, auto tree, auto reads) {
        constexpr int D = decltype(dim)::value;
        constexpr bool kTree = decltype(tree)::value != 0, kOnce = decltype(reads)::value != 0;
        if (p.y_bf16) hipLaunchKernelGGL((k_head_few<D, kTree, kOnce, false>), dim3(kFewGroups), dim3(kFewThreads), 0, s, p);
        else hipLaunchKernelGGL((k_head_few<D, kTree, kOnce, true>), dim3(kFewGroups), dim3(kFewThreads), 0, s, p);
    };
    auto trees = [&](auto dim, auto reads) {
        if (p.tree) few(dim, LatInt<1>{}, reads);
        else few(dim, LatInt<0>{}, reads);
    };
    auto dims = [&](auto reads) {
        if (p.dim == 128) trees(LatInt<128>{}, reads);
        else trees(LatInt<64>{}, reads);
    };
    if (once) dims(LatInt<1>{});
    else dims(LatInt<0>{});
    join(p, 1, s);
    return hipGetLastError();
}

hipError_t launch_head_many(const HeadParams& p, hipStream_t s) {
    meta(p, 0, s);
    // Row tiles of a group at most; pieces, where they are cut.
    long long tiles = std::max(p.B, 1) * (((long long)p.max_new * p.ratio + kTileRows - 1) / kTileRows);
    tiles = std::max(std::min(tiles, (long long)p.T * p.ratio / kTileRows + p.B), 1ll);
    if (p.part) tiles = std::max(tiles, (long long)(kTilePieces / p.G));
    // As many for each of the XCDs that share a group; blanks.
    long long grid = tiles * p.G;
    if (p.G % kXcds && kXcds % p.G == 0) grid = (tiles + kXcds / p.G - 1) / (kXcds / p.G) * kXcds;
    if (!p.part) grid += kHeadBlank;
    const hipError_t err = p.dim == 128 ? launch_head_tile_128(p, (unsigned)grid, (int)tiles, s)
                                        : launch_head_tile_64(p, (unsigned)grid, (int)tiles, s);
    if (err == hipSuccess && p.part) join(p, 0, s);
    return err == hipSuccess ? hipGetLastError() : err;
}

}  // namespace caee
