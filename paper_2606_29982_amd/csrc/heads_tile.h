// Attention with grouped heads, many rows: 256 query rows of a request and
// group (its new tokens' heads, head fastest) a workgroup, over all tokens that
// the rows see or a piece of them.
#pragma once

#include "heads.h"

namespace caee {
namespace {

constexpr int kTileThreads = 512;

// Steps of a piece at most.  A lane tries cutting the longest request's row tiles
// into lane + 1 pieces, others' as far as theirs are longer; what decides is
// the time that the CUs take for all pieces, with kStart steps for a piece's start
// and end and kJoin for the partial results.
__device__ inline int head_piece(const HeadParams& p, const HeadLine& line) {
    constexpr float kStart = 5.0f, kJoin = 8.0f;
    const int lane = threadIdx.x & (kWave - 1);
    const int tiles = lane < p.B ? head_tiles(p, line.mine) : 0, n = tiles > 0 ? head_steps(line.mine) : 0;
    int most = n, least = tiles > 0 ? n : INT32_MAX, all = tiles;
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) {
        most = max(most, __shfl_xor(most, d));
        least = min(least, __shfl_xor(least, d));
        all = head_add_units(all, __shfl_xor(all, d));
    }
    most = max(__builtin_amdgcn_readfirstlane(most), 1);
    all = __builtin_amdgcn_readfirstlane(all);
    if (!p.part || (long long)all * p.G > kTilePieces) return most;
    const int per = (most + lane) / (lane + 1);
    const float inverse = 1.0f / (float)per;
    int pieces = 0;
    float units = 0.0f;
    for (int b = 0; b < p.B; ++b) {
        const int t = __builtin_amdgcn_readlane(tiles, b), m = __builtin_amdgcn_readlane(n, b);
        int c = (int)((float)m * inverse);      // ceil(m / per), in two corrections
        c += c * per < m;
        c -= (c - 1) * per >= m;
        pieces += t * max(c, 1);
        units += (float)t * (float)m;
    }
    pieces *= p.G;
    const int rounds = (pieces + kHeadCus - 1) / kHeadCus;
    const float each = (float)per + kStart;
    const float mean = (units * (float)p.G + (float)pieces * kStart) * (1.0f / kHeadCus);
    // Pieces of one size run in rounds; others fill each other's gaps.
    float cost = __builtin_amdgcn_readfirstlane(least) == most ? (float)rounds * each : fmaxf(each, mean + 0.5f * (float)per);
    if (lane > 0) cost = pieces <= kTilePieces ? cost + kJoin : INFINITY;
    float best = cost;
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) best = fminf(best, __shfl_xor(best, d));
    return __builtin_amdgcn_readlane(per, __ffsll((unsigned long long)__ballot(cost == best)) - 1);
}

// Row tile q of all requests' by where it begins in its request, the last first:
// those see the most tokens, and what starts last should be short.  (Up to
// kOrdered requests; a lane tries a place, all 64 at a time.)
constexpr int kOrdered = 16;
struct HeadAt {
    int b, rt;
};
__device__ inline HeadAt head_order(const HeadParams& p, const HeadLine& line, int q) {
    const int lane = threadIdx.x & (kWave - 1);
    // Row tiles of a request that begin at token x or later.
    auto from = [&](int tiles, int before, int add, int x) {
        return tiles - min(tiles, (min(max(x - before, 0), add) * p.ratio + kTileRows - 1) / kTileRows);
    };
    const int tiles = line.n;
    int lo = 0, hi = 1;
    for (int b = 0; b < p.B; ++b) {
        const int before = __builtin_amdgcn_readlane(line.mine.before, b);
        lo = min(lo, before);
        hi = max(hi, before + __builtin_amdgcn_readlane(line.mine.add, b));
    }
    auto count = [&](int x) {
        int n = 0;
        for (int b = 0; b < p.B; ++b)
            n += from(__builtin_amdgcn_readlane(tiles, b), __builtin_amdgcn_readlane(line.mine.before, b),
                      __builtin_amdgcn_readlane(line.mine.add, b), x);
        return n;
    };
    while (hi - lo > 1) {          // count(lo) > q >= count(hi)
        const int step = (hi - lo + kWave - 1) / kWave, x = lo + (lane + 1) * step;
        const int n = count(x), k = __popcll(__ballot(x < hi && n > q));
        hi = min(hi, lo + (k + 1) * step);
        lo += k * step;
    }
    int left = q - __builtin_amdgcn_readfirstlane(count(lo + 1));
    const int here = from(tiles, line.mine.before, line.mine.add, lo), later = from(tiles, line.mine.before, line.mine.add, lo + 1);
    HeadAt at = {0, 0};
    for (int b = 0; b < p.B; ++b) {
        const int h = __builtin_amdgcn_readlane(here, b), n = h - __builtin_amdgcn_readlane(later, b);
        if (left >= 0 && left < n) at = {b, __builtin_amdgcn_readlane(tiles, b) - h + left};
        left -= n;
    }
    return at;
}

// Keys or values of 64 tokens, or the queries of two waves, 32 each: blocks of 8
// rows x 128 bytes, swizzled.
template <int G>
struct HeadTile {
    lat_u32x4 v[kTileTokens / 8][G][kWave];
};

template <int D, bool kTree, bool kRest>
__global__ __launch_bounds__(kTileThreads) void k_head_tile(HeadParams p, int tiles) {
#if defined(__HIP_DEVICE_COMPILE__)   // the buffer-descriptor type exists for the GPU target only
    constexpr int kG = D / 64, kJ = D / 16, NC = D / 32;
    constexpr int kAhead = 5;                  // fragments read from LDS ahead of their MFMAs
    constexpr int kLoads = 2 * kG;             // loads of a wave per tile: one block of 8 tokens
    using Stage = HeadTile<kG>;
    // An object per stage: the compiler can tell the reads of one from the
    // loads that fill another.
    __shared__ Stage kt0, kt1, kt2, vt0, vt1, vt2;
    __shared__ int odd_values;                 // an infinity or NaN was taken out of the values
    const int lane = threadIdx.x & 63, n = lane & 31, hf = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const bool second = wave >= 4;
    const int kp0 = (n >> 3) * (kG * kWave) + (n & 7) * 8 + (hf ^ lat_swz(n));
    const int vrow = 4 * hf + ((lane & 15) >> 2);
    const int vp0 = 2 * (vrow * 8 + ((2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) ^ lat_swz(vrow))) + (lane & 1);
    const uint32_t row_bytes = (uint32_t)p.c.row_stride * 2u;
    const uint32_t swz = 16u * ((lane & 7) ^ lat_swz(8 * wave + (lane >> 3)));

    // Workgroups go to the XCDs round robin.  The last ones blank the rows of no request.
    const unsigned wg = lat_workgroup();
    int g, q;
    if (p.G % kXcds == 0) {            // all row tiles of a group on one XCD, whose L2 holds its keys and values
        const int k = wg / kXcds;
        g = wg % kXcds + kXcds * (k / tiles);
        q = k % tiles;
    } else if (kXcds % p.G == 0) {     // or on some of them
        const int x = wg % kXcds, subs = kXcds / p.G;
        g = x % p.G;
        q = (int)(wg / kXcds) * subs + x / p.G;
        if (q >= (tiles + subs - 1) / subs * subs) g = p.G;
    } else {
        g = wg / tiles;
        q = wg % tiles;
    }
    if (g >= p.G) {
        const long long words = (long long)p.H * D * (p.y_bf16 ? 2 : 4) / 16;
        const int from = p.B > 0 ? min(max(p.cu_new[p.B], 0), p.T) : 0;
        const long long n_w = (p.T - from) * words, n_r = (long long)(p.T - from) * p.H;
        const long long first = ((long long)gridDim.x * gridDim.y - 1 - wg) * kTileThreads + threadIdx.x;
        constexpr long long kBy = (long long)kHeadBlank * kTileThreads;
        if (first >= kBy) return;
        for (long long i = first; i < n_w; i += kBy) ((lat_u32x4*)p.y)[from * words + i] = lat_u32x4{0, 0, 0, 0};
        if (p.lse)
            for (long long i = first; i < n_r; i += kBy) p.lse[(long long)from * p.H + i] = -INFINITY;
        return;
    }
    HeadLine line = head_line(p);
    const int per = p.B > kWave ? __builtin_amdgcn_readfirstlane(p.meta[p.B + 1]) : head_piece(p, line);
    if (p.B <= kWave && wg == 0 && threadIdx.x == 0) p.meta[p.B + 1] = per;       // for the join
    head_line_sum(p, &line, head_tiles(p, line.mine) * head_cut(head_steps(line.mine), per));
    if (q >= line.total) return;
    int b, rt, part = 0, parts = 1;
    const bool cut = p.B <= kWave && __any(line.n > head_tiles(p, line.mine));
    if (p.B > 1 && p.B <= kOrdered && !cut && line.total * p.G > kHeadCus) {
        const HeadAt at = head_order(p, line, q);
        b = at.b;
        rt = at.rt;
    } else {
        const int u = line.total - 1 - q;
        int at_u;
        b = head_line_find(p, line, u);
        const LatentReq r = head_line_req(p, line, b, &at_u);
        parts = __builtin_amdgcn_readfirstlane(head_cut(head_steps(r), per));
        rt = head_div(u - at_u, parts);
        part = u - at_u - rt * parts;
    }
    int at_b;
    const LatentReq rq = head_line_req(p, line, b, &at_b);
    {
        const int rows = rq.add * p.ratio, steps_all = head_steps(rq);
        const int first = head_div(steps_all * part, parts), last = head_div(steps_all * (part + 1), parts);
        const bool whole = parts == 1;
        const int row0 = rt * kTileRows, my0 = row0 + 32 * wave;
        auto sees = [&](int r) { return head_sees(p, rq, head_div(min(r, rows - 1), p.ratio)); };
        const int row = min(my0 + n, rows - 1), tok = row / p.ratio;
        const int limit = head_sees(p, rq, tok);
        // Tokens from lim_min (lim_wg) on some row of the wave (the workgroup) does not see.
        const int lim_tree = min(max(rq.before, 0), rq.seq);
        const int lim_min = kTree ? lim_tree : sees(my0), lim_wg = kTree ? lim_tree : sees(row0);
        const int end = min(last * kTileTokens, sees(row0 + kTileRows - 1));
        const int tok0 = first * kTileTokens;
        const int steps = end > tok0 ? (end - tok0 + kTileTokens - 1) / kTileTokens : 0;
        const int at_row = (rq.t0 + tok) * p.H + g * p.ratio + row - tok * p.ratio;      // of y and lse
        const uint32_t* mask = kTree ? p.tree + (size_t)(rq.t0 + tok) * p.words : nullptr;

        if (threadIdx.x == 0) odd_values = 0;
        // A wave's queries, as its results at the end, go through a part of LDS of
        // its own, eight lanes a 128-byte line.  The stages of tile 0, fetched
        // meanwhile, are left out.
        lat_u32x4* const own = &(wave < 2 ? kt1 : wave < 4 ? kt2 : wave < 6 ? vt1 : vt2).v[4 * (wave & 1)][0][0];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = 8 * i + (lane >> 3), rr = min(my0 + r, rows - 1), t = rr / p.ratio;
            const uint16_t* src = p.q + (size_t)(rq.t0 + t) * p.q_stride + (size_t)(g * p.ratio + rr - t * p.ratio) * D +
                                  8 * ((lane & 7) ^ lat_swz(r));
#pragma unroll
            for (int gg = 0; gg < kG; ++gg)
                __builtin_amdgcn_global_load_lds((lat_g_void*)(src + 64 * gg), (lat_lds_void*)(own + (kG * i + gg) * kWave), 16, 0, 0);
        }
        lat_u32x4 qf[kJ];
        lat_f32x16 o[NC];
#pragma unroll
        for (int c = 0; c < NC; ++c) o[c] = lat_f32x16{};
        float m = kNoScore, l = 0.0f;

        // A wave fetches 8 tokens of a tile; the pages of tiles are looked up a
        // step before their keys are.
        auto eight = [&](int s) __attribute__((always_inline)) { return head_eight(p, b, rq.seq, tok0 + min(s, steps - 1) * kTileTokens + 8 * wave); };
        const char *const k_base = head_base(p, p.k, g), *const v_base = head_base(p, p.v, g);
        auto load = [&](const char* cache, const HeadEight& e, int s, Stage& st) __attribute__((always_inline)) {
            const __amdgpu_buffer_rsrc_t buf = __builtin_amdgcn_make_buffer_rsrc(
                (void*)(cache + head_offset(p, e.page, e.at)), 0, e.one ? kLatBufBytes : 0, kLatBufWord3);
            const uint32_t at = (uint32_t)min(lane >> 3, e.span) * row_bytes + swz;
#pragma unroll
            for (int gg = 0; gg < kG; ++gg)
                __builtin_amdgcn_raw_ptr_buffer_load_lds(buf, (lat_lds_void*)&st.v[wave][gg][0], 16, at, 128 * gg, 0, 0);
            if (!e.one) {      // rows in several pages go one by one, after the loads above, which touch nothing
                lat_wait_vm<0>();
                const int p0 = tok0 + min(s, steps - 1) * kTileTokens + 8 * wave;
#pragma unroll 1
                for (int r = 0; r < 8; ++r) {
                    const __amdgpu_buffer_rsrc_t far = __builtin_amdgcn_make_buffer_rsrc(
                        (void*)(cache + head_row(p, b, min(p0 + r, rq.seq - 1))), 0, kLatBufBytes, kLatBufWord3);
                    if (lane >> 3 == r) {
#pragma unroll
                        for (int gg = 0; gg < kG; ++gg)
                            __builtin_amdgcn_raw_ptr_buffer_load_lds(far, (lat_lds_void*)&st.v[wave][gg][0], 16, swz, 128 * gg, 0, 0);
                    }
                }
                lat_wait_vm<0>();
            }
        };
        // Step s has two phases: X multiplies the keys of tile s and sums the
        // values of tile s - 1, Y makes the weights of tile s (exponentials) and
        // starts loads.  The two waves of a SIMD take turns: waves 4 .. 7 run one
        // barrier behind waves 0 .. 3, so that one is in X while the other is in Y.
        // Keys of tile s are read in phases 2 s (waves 0 .. 3) and 2 s + 1 (4 .. 7),
        // values in 2 s + 2 and 2 s + 3; so in Y(s) the first waves, in phase 2 s + 1,
        // may load the keys of tile s + 2 and the values of tile s + 1 into rings of
        // three, the others, in phase 2 s + 2, those of one tile more.  At the end of
        // the odd phases (Y of the first waves, X of the others) a wave waits for
        // all but its latest step's loads: what the next phase reads is then there.
        // Past the last tile the loads read it again, for nobody.
        auto clear = [&](int s, Stage& d) __attribute__((always_inline)) {
            // Tokens that some rows do not see may hold anything: infinities and NaNs
            // must not meet their zero weights, so a wave clears them from the
            // values that it loaded, before the barrier that publishes them.
            const int tb = tok0 + s * kTileTokens;
            if (s >= steps || tb + kTileTokens <= lim_wg) return;
            if (tb + 8 * wave + (lane >> 3) >= lim_wg) {
                bool odd = false;
#pragma unroll
                for (int gg = 0; gg < kG; ++gg) {
                    const lat_u32x4 v = d.v[wave][gg][lane];
                    lat_u32x4 w;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        w[e] = lat_finite(v[e]);
                        odd |= w[e] != v[e];
                    }
                    d.v[wave][gg][lane] = w;
                }
                if (odd) odd_values = 1;
            }
            __builtin_amdgcn_s_waitcnt(15 | (7 << 4) | (0 << 8) | (3 << 14));
        };
        auto odd_end = [&](int s, Stage& values) __attribute__((always_inline)) {
            lat_wait_vm<kLoads>();
            asm volatile("" ::: "memory");
            clear(s, values);
        };
        lat_u32x4 pf[4] = {}, pr[kRest ? 4 : 1] = {}, pl[kRest ? 4 : 1] = {};       // weights of the tile before, their remainders
        lat_f32x16 sc[2];
        // X's MFMAs, 2 kJ of the scores and 4 NC of the sums, evenly mixed (two
        // chains of sums alone would wait for each other), their fragments read
        // kAhead before they are used.
        constexpr int kOps = 2 * kJ + 4 * NC;
        auto sums_before = [](int i) constexpr { return i * (4 * NC) / kOps; };
        auto value = [&](const Stage& d, int i, int vp) __attribute__((always_inline)) {
            const lat_u32x2* base = (const lat_u32x2*)&d.v[0][0][0];
            const int ks = i / NC, c = i % NC;
            lat_u32x2 w[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const lat_u32x2* at = base + ((2 * ks + e) * kG + (c >> 1)) * (2 * kWave) + (vp ^ (8 * (c & 1) + 2 * e));
                w[e] = __builtin_bit_cast(lat_u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lat_lds_s16x4*)at));
            }
            return lat_u32x4{w[0][0], w[0][1], w[1][0], w[1][1]};
        };
        auto sum = [&](const lat_u32x4& v, int i) __attribute__((always_inline)) {
            o[i % NC] = lat_mma(v, pf[i / NC], o[i % NC]);
            if constexpr (kRest) {
                o[i % NC] = lat_mma(v, pr[i / NC], o[i % NC]);
                o[i % NC] = lat_mma(v, pl[i / NC], o[i % NC]);
            }
        };
        HeadEight e_k = {}, e_v = {}, e_next = {};      // of the keys and values that Y loads, and of the next keys
        const int more_k = second ? 3 : 2;
        // k, k2: the keys of tile s (their stage then takes those of tile s + 3)
        // and the stage for those of tile s + 2; v0, v1, v2: the values of tiles
        // s - 1 (their stage then takes those of tile s + 2) and s and the stage
        // for those of tile s + 1.
        auto step = [&](int s, Stage& k, Stage& k2, Stage& v0, Stage& v1, Stage& v2) __attribute__((always_inline)) {
            const int tb = tok0 + s * kTileTokens;
            const lat_u32x4* keys = &k.v[0][0][0];
            // made here: the registers that a stage's addresses would take through the loop are not there
            int kp = kp0, vp = vp0;
            asm volatile("" : "+v"(kp), "+v"(vp));
            auto fetch = [&](auto ic) __attribute__((always_inline)) {
                constexpr int i = decltype(ic)::value, v = sums_before(i);
                if constexpr (sums_before(i + 1) > v) {
                    return value(v0, v, vp);
                } else {
                    constexpr int j = (i - v) >> 1, e = (i - v) & 1;
                    return keys[(kp ^ (2 * (j % 4))) + (4 * e * kG + j / 4) * kWave];
                }
            };
            __builtin_amdgcn_sched_barrier(0);
            lat_u32x4 fr[kAhead];
            sc[0] = sc[1] = lat_f32x16{};
            lat_for<0, kAhead>([&](auto ic) __attribute__((always_inline)) { fr[decltype(ic)::value] = fetch(ic); });
            lat_for<0, kOps>([&](auto ic) __attribute__((always_inline)) {
                constexpr int i = decltype(ic)::value, v = sums_before(i), j = i - v;
                if constexpr (sums_before(i + 1) > v) sum(fr[i % kAhead], v);
                else sc[j & 1] = lat_mma(fr[i % kAhead], qf[j >> 1], sc[j & 1]);
                if constexpr (i + kAhead < kOps) fr[i % kAhead] = fetch(LatInt<i + kAhead>{});
                __builtin_amdgcn_sched_barrier(0);
            });
            if (second) odd_end(s, v1);
            lat_barrier();
            e_v = e_k;
            e_k = e_next;
            if (second) {
                load(k_base, e_k, s + more_k, k);
                load(v_base, e_v, s + more_k - 1, v0);
            } else {
                load(k_base, e_k, s + more_k, k2);
                load(v_base, e_v, s + more_k - 1, v2);
            }
            e_next = eight(s + more_k + 1);
            if (tb + kTileTokens > lim_min) {
                asm volatile("");       // a branch, not 32 selects in every step
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int left = limit - (tb + 32 * e + 4 * hf);
                    const uint32_t bits = kTree ? head_tree_bits(mask, p.words, tb + 32 * e - rq.before) >> (4 * hf) : 0u;
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        constexpr auto at = [](int x) constexpr { return 8 * (x >> 2) + (x & 3); };
                        if (at(i) >= left || (kTree && !(bits >> at(i) & 1))) sc[e][i] = -INFINITY;
                    }
                }
            }
            // The weights by the running maximum; where it has to move they are made again.
            float more = 0.0f;
            auto weights = [&](auto&& weight) __attribute__((always_inline)) {
#pragma unroll
                for (int k = 0; k < 4; ++k)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float a = weight(sc[k >> 1][8 * (k & 1) + 2 * i], p.scale_log2, m);
                        const float e = weight(sc[k >> 1][8 * (k & 1) + 2 * i + 1], p.scale_log2, m);
                        pf[k][i] = lat_pack(a, e);
                        if constexpr (kRest) {
                            const lat_f32x2 rest = lat_rest(pf[k][i], a, e);
                            pr[k][i] = lat_pack(rest[0], rest[1]);
                            const lat_f32x2 last = lat_rest(pr[k][i], rest[0], rest[1]);
                            pl[k][i] = lat_pack(last[0], last[1]);
                            more += a + e;
                        } else {
                            more = lat_sum2(pf[k][i], more);
                        }
                    }
            };
            weights(head_weight);
            if (__any(head_moves(more, m))) {
                float mt = fmaxf(sc[0][0], sc[1][0]);
#pragma unroll
                for (int i = 1; i < 16; ++i) mt = fmaxf(mt, fmaxf(sc[0][i], sc[1][i]));
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
            if (!second) odd_end(s, v1);
            lat_barrier();
        };
        if (steps > 0) {
            // Tile 0, the keys of tile 1 (and what the second waves' Y(-1) would
            // have loaded); the values of "tile -1" are zeros.
            const HeadEight e0 = eight(0), e1 = eight(1), e2 = eight(2);
            load(k_base, e0, 0, kt0);
            load(v_base, e0, 0, vt0);
            lat_wait_vm<kLoads>();
            asm volatile("" ::: "memory");
#pragma unroll
            for (int j = 0; j < kJ; ++j)
                qf[j] = own[(kp0 ^ (2 * (j & 3))) + (j >> 2) * kWave];
            __builtin_amdgcn_s_waitcnt(15 | (7 << 4) | (0 << 8) | (3 << 14));
            lat_barrier();             // the stages the queries came through are free
            load(k_base, e1, 1, kt1);
            if (second) {
                load(k_base, e2, 2, kt2);
                load(v_base, e1, 1, vt1);
                e_k = e2;
                e_next = eight(3);
            } else {
                e_k = e1;
                e_next = e2;
            }
#pragma unroll
            for (int gg = 0; gg < kG; ++gg) vt2.v[wave][gg][lane] = lat_u32x4{0, 0, 0, 0};
            // Tile 0 is there; the keys of tile 1 are waited for at the end of phase 1.
            if (second) lat_wait_vm<kG + kLoads>();
            else lat_wait_vm<kG>();
            asm volatile("" ::: "memory");
            clear(0, vt0);
            __builtin_amdgcn_s_waitcnt(15 | (7 << 4) | (0 << 8) | (3 << 14));
            lat_barrier();
            if (second) lat_barrier();
            for (int s = 0; s < steps; s += 3) {
                step(s, kt0, kt2, vt2, vt0, vt1);
                if (s + 1 < steps) step(s + 1, kt1, kt0, vt0, vt1, vt2);
                if (s + 2 < steps) step(s + 2, kt2, kt1, vt1, vt2, vt0);
            }
            if (!second) lat_barrier();
            lat_wait_vm<0>();          // the last tile's second readings have landed
            auto finish = [&](const Stage& d) __attribute__((always_inline)) {
#pragma unroll
                for (int i = 0; i < 4 * NC; ++i) sum(value(d, i, vp0), i);
            };
            const int at = (steps - 1) % 3;
            if (at == 0) finish(vt0);
            else if (at == 1) finish(vt1);
            else finish(vt2);
        }

        lat_wait_vm<0>();
        lat_barrier();             // nobody's loads are on their way into the stages any more
        l = lat_sum_pair(l);
        const bool odd = __builtin_amdgcn_readfirstlane(odd_values) || __any(head_odd(o, l));
        const size_t slot0 = ((size_t)g * line.total + at_b + rt * parts + part) * kTileRows;
        const float f = whole ? lat_inverse(l) : 1.0f;
        if (hf == 0 && my0 + n < rows) {
            if (!whole) *(float2*)(p.part_ml + 2 * (slot0 + 32 * wave + n)) = make_float2(m, l);
            else if (p.lse) p.lse[at_row] = lat_lse(m, l);
        }
        // 8 (dim 64: 4) KiB a wave: as much of a row at a time as a bf16 row has, unit
        // u (16 bytes) of it at u ^ (row % units).
        lat_u32x4* const out = &(wave < 2 ? kt0 : wave < 4 ? kt1 : wave < 6 ? kt2 : vt0).v[4 * (wave & 1)][0][0];
        constexpr int kUnits = D / 8;
        // (made here, as above)
        int ln = lane;
        asm volatile("" : "+v"(ln));
        const int nn = ln & 31, hh = ln >> 5;
        auto leave = [&](auto bytes_of, auto&& row_of) __attribute__((always_inline)) {
            constexpr int kSize = decltype(bytes_of)::value, kPasses = kSize / 2, kTiles = NC / kPasses;
#pragma unroll
            for (int pass = 0; pass < kPasses; ++pass) {
#pragma unroll
                for (int c = 0; c < kTiles; ++c)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const lat_f32x16& v = o[kTiles * pass + c];
                        const float v0 = v[4 * i] * f, v1 = v[4 * i + 1] * f, v2 = v[4 * i + 2] * f, v3 = v[4 * i + 3] * f;
                        const int unit = kSize == 2 ? 4 * c + i : 8 * c + 2 * i + hh;
                        lat_u32x4* const at = out + nn * kUnits + (unit ^ (nn & (kUnits - 1)));
                        if constexpr (kSize == 2) ((lat_u32x2*)at)[hh] = lat_u32x2{lat_pack(v0, v1), lat_pack(v2, v3)};
                        else *at = lat_u32x4{__float_as_uint(v0), __float_as_uint(v1), __float_as_uint(v2), __float_as_uint(v3)};
                    }
                __builtin_amdgcn_s_waitcnt(15 | (7 << 4) | (0 << 8) | (3 << 14));
                asm volatile("" ::: "memory");
#pragma unroll
                for (int i = 0; i < kUnits / 2; ++i) {
                    const int r = (64 * i + ln) / kUnits, un = (64 * i + ln) % kUnits;
                    const lat_u32x4 v = out[r * kUnits + (un ^ (r & (kUnits - 1)))];
                    if (my0 + r < rows) *(lat_u32x4*)((char*)row_of(r) + 16 * kUnits * pass + 16 * un) = v;
                }
                __builtin_amdgcn_s_waitcnt(15 | (7 << 4) | (0 << 8) | (3 << 14));
                asm volatile("" ::: "memory");
            }
        };
        if (!whole) {
            if (steps > 0) leave(LatInt<4>{}, [&](int r) { return p.part + (slot0 + 32 * wave + r) * D; });
        } else {
            auto y_row = [&](int r) { return (size_t)__shfl(at_row, r) * D; };
            if (p.y_bf16) leave(LatInt<2>{}, [&](int r) { return (uint16_t*)p.y + y_row(r); });
            else leave(LatInt<4>{}, [&](int r) { return (float*)p.y + y_row(r); });
        }
        if (odd) {
            lat_wait_vm<0>();
            auto sees = [&](int pos) { return pos < limit && (!kTree || (head_tree_bits(mask, p.words, pos - rq.before) & 1)); };
            head_put_odd<D>(p, b, g, tok0, kTileTokens, kTileTokens, end, sees, [&](int d, float v) {
                if (my0 + n >= rows || !(l < INFINITY)) return;
                if (!whole) p.part[(slot0 + 32 * wave + n) * D + d] = v;
                else if (p.y_bf16) ((__bf16*)p.y)[(size_t)at_row * D + d] = (__bf16)v;
                else ((float*)p.y)[(size_t)at_row * D + d] = v;
            });
        }
    }
#endif
}

template <int D>
hipError_t head_tile(const HeadParams& p, unsigned grid, int pieces, hipStream_t s) {
    auto run = [&](auto tree, auto rest) {
        hipLaunchKernelGGL((k_head_tile<D, decltype(tree)::value != 0, decltype(rest)::value != 0>), lat_grid(grid),
                           dim3(kTileThreads), 0, s, p, pieces);
    };
    auto trees = [&](auto rest) {
        if (p.tree) run(LatInt<1>{}, rest);
        else run(LatInt<0>{}, rest);
    };
    // Weights' remainders for 32-bit results only.
    if (p.y_bf16) trees(LatInt<0>{});
    else trees(LatInt<1>{});
    return hipGetLastError();
}

}  // namespace
}  // namespace caee
