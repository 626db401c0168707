// Attention with grouped heads, many rows: 128 query rows of a request and
// group (its new tokens' heads, head fastest) a workgroup, over all tokens that
// the rows see or a piece of them.
#pragma once

#include "heads.h"

namespace caee {
namespace {

constexpr int kTileThreads = 256;

// Steps of a piece at most.  A lane tries cutting the longest request's row tiles
// into lane + 1 pieces, others' as far as theirs are longer; what decides is
// the time that the CUs take for all pieces, with kStart steps for a piece's start
// and end and kJoin for the partial results.  (The next 259 tokens of
// 2 prompts behind 30000, 144 row tiles: 1008 pieces of 68 steps, 315 us; values of kStart and
// kJoin between half and twice these made no difference.)
__device__ inline int head_piece(const HeadParams& p, const HeadLine& line) {
    constexpr float kStart = 5.0f, kJoin = 8.0f;
    if (!p.part) return INT32_MAX / 2;
    const int lane = threadIdx.x & (kWave - 1);
    const int tiles = lane < p.B ? head_tiles(p, line.mine) : 0, n = tiles > 0 ? head_steps(line.mine) : 0;
    const int most = max(head_last(head_scan(n, 0, [](int a, int b) { return max(a, b); })), 1);
    const int least = head_last(head_scan(tiles > 0 ? n : INT32_MAX, INT32_MAX, [](int a, int b) { return min(a, b); }));
    const int all = head_last(head_scan(tiles, 0, head_add_units));
    if ((long long)all * p.G > kTilePieces) return most;
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
    const int rounds = (pieces + kTileSlots - 1) / kTileSlots;
    const float each = (float)per + kStart;
    const float mean = (units * (float)p.G + (float)pieces * kStart) * (1.0f / kTileSlots);
    // Pieces of one size run in rounds; others fill each other's gaps.
    float cost = least == most ? (float)rounds * each : fmaxf(each, mean + 0.5f * (float)per);
    if (lane > 0) cost = pieces <= kTilePieces ? cost + kJoin : INFINITY;
    // (costs are positive: their order is that of their bits)
    const int best = head_last(head_scan(__float_as_int(cost), INT32_MAX, [](int a, int b) { return min(a, b); }));
    return __builtin_amdgcn_readlane(per, __ffsll((unsigned long long)__ballot(__float_as_int(cost) == best)) - 1);
}

// Row tile q of all requests', by where it ends, the last first: those see the
// most tokens, and what starts last should be short.  Request b's tiles lie in
// places first .. first + n - 1, a place for each kTileRows rows before the end
// that is the last of all; a lane tries a place, all 64 at a time.
struct HeadAt {
    int b, rt;
};
// Whether that pays: while the CUs take the row tiles in a few rounds.  After more
// rounds they end together anyway, and neighbours of one request share its keys in
// the L2.  us, by place and by request, 32 heads, 8 groups, lengths at random up to:
// 8 prompts of 700 (2 rounds) 25.4 and 27.0, 24 (4) 78 and 81, 40 (7) 121 and 118; 61 of
// 400 (6) 104 and 85, of 1500 (22) 620 and 565; 16 of 1400 (5) 146 and 154.  Behind up to
// 4000 cached tokens 16 of 200 107 and 136, behind 2000 61 of 100 102 and 123, 3 of 2000 156
// and 151.
__device__ inline bool head_ordered(const HeadParams& p, int tiles) {
    return p.B > 1 && p.B <= kWave && (long long)tiles * p.G > kTileSlots &&
           (long long)tiles * p.G <= (p.B <= 16 ? 6 : 4) * kTileSlots;
}
__device__ inline HeadAt head_order(const HeadParams& p, const HeadLine& line, int q) {
    const int lane = threadIdx.x & (kWave - 1);
    const int n = line.n, end = n > 0 ? line.mine.before + line.mine.add : INT32_MIN;
    const auto larger = [](int a, int b) { return max(a, b); };
    const int latest = head_last(head_scan(end, INT32_MIN, larger));
    const int first = n > 0 ? min(latest - end, 1 << 20) * p.ratio / kTileRows : 0;
    int lo = 0, hi = head_last(head_scan(first + n, 0, larger)), before = 0;
    while (hi - lo > 1) {          // before: the tiles in places before lo; at most q, and in those before hi more
        const int step = (hi - lo + kWave - 1) / kWave, x = lo + (lane + 1) * step;
        int tiles = 0;
        for (int b0 = 0; b0 < p.B; b0 += 4)          // (lanes without a request have no tiles)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                tiles += min(max(x - __builtin_amdgcn_readlane(first, b0 + i), 0), __builtin_amdgcn_readlane(n, b0 + i));
        const int k = __popcll(__ballot(x < hi && tiles <= q));
        if (k > 0) before = __builtin_amdgcn_readlane(tiles, k - 1);
        hi = min(hi, lo + (k + 1) * step);
        lo += k * step;
    }
    // The requests that have a tile in place lo, by number.
    const bool here = lo >= first && lo - first < n;
    const unsigned long long all = __ballot(here);
    const int at = __popcll(all & ((1ull << lane) - 1));
    const int b = __ffsll((unsigned long long)__ballot(here && at == q - before)) - 1;
    return {b, __builtin_amdgcn_readlane(n - 1 - (lo - first), b)};
}

// Keys or values of 64 tokens, or the queries of two waves, 32 each: blocks of 8
// rows x 128 bytes, swizzled.
template <int G>
struct HeadTile {
    lat_u32x4 v[kTileTokens / 8][G][kWave];
};

// A row tile, or a piece of it: a wave has 32 rows, whose sums, statistics and
// queries stay in registers, the workgroup 64 tokens at a time in LDS, two tiles in
// turn.  As in k_head_few keys are the M side of the scores and the weights a
// fragment of the second product as they are.  The next tile's loads go out between
// the products with the keys, the next 16 tokens' weights are made between the
// products with the values: a wave's vector instructions run beside its own MFMAs
// (an MFMA of 32x32x16 takes 13.6 ns, with four vector instructions and an exponential
// beside it 15.5).  Weights are rounded to bf16, and l sums the rounded ones, so that
// their roundings cancel where one token dominates; for a 32-bit result they have three
// parts.  The log-sum-exp is of the weights themselves, whose sum is kept beside l where
// it is asked for (kSum: the long prompt below 520 and 537 us).
// Two workgroups a CU fill each other's gaps; one of 256 rows, which reads the keys
// and values half as often, has none to fill them (tree-shaped calls of 16 users
// 159 us, 97 with two; 8 ragged prompts 42 and 38, one of 7161 tokens 508 and 527).
// What bounds it: the matrix units at the clock that power leaves.  7161 tokens
// behind 1030, 32 heads: 535 us (1010 TFLOP/s; a large library product reaches 1217 on that
// card), MFMAs 50 % of the cycles at 1.9 GHz; of 567 that copies for timing began with,
// they took 516 without the loads, 452 without the products with the values, 433 without
// those with the keys.  Filling one stage in two parts at
// two barriers a step was slower (540 beside 527).  Short calls are bound by a tile's start
// and end (7 to 8 us: lengths 1.8, pages and queries 1.7, fetch 0.8, out 2) beside
// 1.6 us a step.
template <int D, bool kTree, bool kRest, bool kSum>
__global__ __launch_bounds__(kTileThreads, 2) void k_head_tile(HeadParams p, int tiles) {
#if defined(__HIP_DEVICE_COMPILE__)   // the buffer-descriptor type exists for the GPU target only
    constexpr int kG = D / 64, kJ = D / 16, NC = D / 32;
    constexpr int kAhead = 5;                  // fragments read from LDS ahead of their MFMAs
    constexpr int kEights = 2, kLoads = kEights * kG;      // blocks of 8 tokens that a wave fetches of a tile; loads
    using Stage = HeadTile<kG>;
    // An object per stage: the compiler can tell the reads of one from the
    // loads that fill the other.
    __shared__ Stage kt0, kt1, vt0, vt1;
    __shared__ int odd_values;                 // an infinity or NaN was taken out of the values
    const int lane = threadIdx.x & 63, n = lane & 31, hf = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int kp0 = (n >> 3) * (kG * kWave) + (n & 7) * 8 + (hf ^ lat_swz(n));
    const int vrow = 4 * hf + ((lane & 15) >> 2);
    const int vp0 = 2 * (vrow * 8 + ((2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) ^ lat_swz(vrow))) + (lane & 1);
    const uint32_t row_bytes = (uint32_t)p.c.row_stride * 2u;

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
    if (!cut && head_ordered(p, line.total)) {
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
        const bool whole = parts == 1;
        const int first = whole ? 0 : __builtin_amdgcn_readfirstlane(head_piece_at(steps_all, part, parts));
        const int last = whole ? steps_all : __builtin_amdgcn_readfirstlane(head_piece_at(steps_all, part + 1, parts));
        const int row0 = rt * kTileRows, my0 = row0 + 32 * wave;
        auto sees = [&](int r) { return head_sees(p, rq, head_over(min(r, rows - 1), p.by_ratio)); };
        const int row = min(my0 + n, rows - 1), tok = head_over(row, p.by_ratio);
        const int limit = head_sees(p, rq, tok);
        // Tokens from lim_min (lim_wg) on some row of the wave (the workgroup) does not see.
        const int lim_tree = min(max(rq.before, 0), rq.seq);
        const int lim_min = kTree ? lim_tree : sees(my0), lim_wg = kTree ? lim_tree : sees(row0);
        const int end = min(last * kTileTokens, sees(row0 + kTileRows - 1));
        const int tok0 = first * kTileTokens;
        const int steps = end > tok0 ? (end - tok0 + kTileTokens - 1) / kTileTokens : 0;
        const int at_row = (rq.t0 + tok) * p.H + g * p.ratio + row - tok * p.ratio;      // of y and lse
        const uint32_t* mask = kTree ? p.tree + (size_t)(rq.t0 + tok) * p.words : nullptr;

        // A wave fetches 16 tokens of a tile.
        auto place = [&](int s, int i) __attribute__((always_inline)) { return tok0 + s * kTileTokens + 8 * (kEights * wave + i); };
        constexpr int kLook = kHeadWindow / kEights;
        HeadWindow win = {};           // of kLook tiles
        auto look = [&](int s) __attribute__((always_inline)) { return head_look(p, b, rq.seq, place(s + lane / kEights, lane % kEights)); };
        HeadLook soon = {};            // of the next ones
        if (steps > 0) soon = look(0);

        if (threadIdx.x == 0) odd_values = 0;
        // A wave's queries, as its results at the end, go through a part of LDS of
        // its own, eight lanes a 128-byte line: the other stages than tile 0's,
        // fetched meanwhile.
        lat_u32x4* const own = &(wave < 2 ? kt1 : vt1).v[4 * (wave & 1)][0][0];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = 8 * i + (lane >> 3), rr = min(my0 + r, rows - 1), t = head_over(rr, p.by_ratio);
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
        float m = kNoScore, l = 0.0f, all = 0.0f;

        auto piece = [&](int i) __attribute__((always_inline)) { return 16u * ((lane & 7) ^ lat_swz(8 * i + (lane >> 3))); };
        const char *const k_base = head_base(p, p.k, g), *const v_base = head_base(p, p.v, g);
        // Load n of a wave's part of tile s, the keys' and then the values' eights.  (A
        // buffer of size 0 past the last tile: its loads cost no traffic, and their
        // number does not depend on a branch.)
        struct Eights {
            HeadEight e[kEights];
        };
        auto eights = [&](int s) __attribute__((always_inline)) {
            Eights x;
#pragma unroll
            for (int i = 0; i < kEights; ++i) x.e[i] = head_eight(win, s % kLook * kEights + i);
            return x;
        };
        auto load = [&](int n, const Eights& x, int s, Stage& k, Stage& v) __attribute__((always_inline)) {
            const int i = n % kLoads / kG, gg = n % kG;
            const HeadEight& e = x.e[i];
            const __amdgpu_buffer_rsrc_t buf = __builtin_amdgcn_make_buffer_rsrc((void*)((n < kLoads ? k_base : v_base) + e.off), 0,
                                                                                s < steps && e.span >= 0 ? kLatBufBytes : 0, kLatBufWord3);
            __builtin_amdgcn_raw_ptr_buffer_load_lds(buf, (lat_lds_void*)&(n < kLoads ? k : v).v[kEights * wave + i][gg][0], 16,
                                                     (uint32_t)min(lane >> 3, e.span) * row_bytes + piece(i), 128 * gg, 0, 0);
        };
        // Rows in several pages, each by an address of its own, after the loads above, which touch nothing there.
        auto load_far = [&](const Eights& x, int s, Stage& k, Stage& v) __attribute__((always_inline)) {
            if (s >= steps || (x.e[0].span >= 0 && x.e[1].span >= 0)) return;
            lat_wait_vm<0>();
#pragma unroll
            for (int i = 0; i < kEights; ++i) {
                if (x.e[i].span >= 0) continue;
                const long long row = head_row(p, b, min(place(s, i) + (lane >> 3), rq.seq - 1)) + piece(i);
#pragma unroll
                for (int gg = 0; gg < kG; ++gg) {
                    __builtin_amdgcn_global_load_lds((lat_g_void*)(k_base + row + 128 * gg), (lat_lds_void*)&k.v[kEights * wave + i][gg][0], 16, 0, 0);
                    __builtin_amdgcn_global_load_lds((lat_g_void*)(v_base + row + 128 * gg), (lat_lds_void*)&v.v[kEights * wave + i][gg][0], 16, 0, 0);
                }
            }
        };
        auto clear = [&](int tb, Stage& d) __attribute__((always_inline)) {
            // Tokens that some rows do not see may hold anything: infinities and NaNs
            // must not meet their zero weights, so a wave clears them from the
            // values that it loaded, before the barrier that publishes them.
#pragma unroll
            for (int i = 0; i < kEights; ++i)
                if (tb + 8 * (kEights * wave + i) + (lane >> 3) >= lim_wg) {
                    bool odd = false;
#pragma unroll
                    for (int gg = 0; gg < kG; ++gg) {
                        const lat_u32x4 v = d.v[kEights * wave + i][gg][lane];
                        lat_u32x4 w;
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            w[e] = lat_finite(v[e]);
                            odd |= w[e] != v[e];
                        }
                        d.v[kEights * wave + i][gg][lane] = w;
                    }
                    if (odd) odd_values = 1;
                }
            __builtin_amdgcn_s_waitcnt(15 | (7 << 4) | (0 << 8) | (3 << 14));
        };
        lat_u32x4 pf[4], pr[kRest ? 4 : 1], pl[kRest ? 4 : 1];       // weights, their remainders
        lat_f32x16 sc[2];
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
        // Tile s in k and v; the next one into k2 and v2.
        auto step = [&](int s, Stage& k, Stage& v, Stage& k2, Stage& v2) __attribute__((always_inline)) {
            const int tb = tok0 + s * kTileTokens;
            lat_wait_vm<0>();              // this wave's part of the tile is there; after the barrier all of it is,
            asm volatile("" ::: "memory"); // and nobody reads the other stage
            if (tb + kTileTokens > lim_wg) clear(tb, v);
            lat_barrier();
            // the window of tile s + 1 on, asked for half a window before
            if ((s + 1) % kLook == kLook / 2) soon = look((s + 1) / kLook * kLook + kLook);
            if ((s + 1) % kLook == 0) win = head_window(p, soon);
            const Eights x = eights(s + 1);
            // made here: the registers that a stage's addresses would take through the loop are not there
            int kp = kp0, vp = vp0;
            asm volatile("" : "+v"(kp), "+v"(vp));
            const lat_u32x4* keys = &k.v[0][0][0];
            auto key = [&](int i) __attribute__((always_inline)) {
                const int j = i >> 1, e = i & 1;
                return keys[(kp ^ (2 * (j % 4))) + (4 * e * kG + j / 4) * kWave];
            };
            __builtin_amdgcn_sched_barrier(0);
            lat_u32x4 fr[kAhead];
            sc[0] = sc[1] = lat_f32x16{};
#pragma unroll
            for (int i = 0; i < kAhead; ++i) fr[i] = key(i);
            lat_for<0, 2 * kJ>([&](auto ic) __attribute__((always_inline)) {
                constexpr int i = decltype(ic)::value;
                sc[i & 1] = lat_mma(fr[i % kAhead], qf[i >> 1], sc[i & 1]);
                if constexpr (i + kAhead < 2 * kJ) fr[i % kAhead] = key(i + kAhead);
                if constexpr (i % 2 == 1 && i / 2 < 2 * kLoads) load(i / 2, x, s + 1, k2, v2);
                __builtin_amdgcn_sched_barrier(0);
            });
            static_assert(kJ >= 2 * kLoads, "a load between two products");
            load_far(x, s + 1, k2, v2);
#pragma unroll
            for (int i = 0; i < kAhead; ++i) fr[i] = value(v, i, vp);
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
            // The running maximum moves only when a score exceeds it by more than kMaxSlack.
            float mt = fmaxf(sc[0][0], sc[1][0]);
#pragma unroll
            for (int i = 1; i < 16; ++i) mt = fmaxf(mt, fmaxf(sc[0][i], sc[1][i]));
            if (__any(mt * p.scale_log2 > m + kMaxSlack)) {
                mt = lat_max_pair(mt) * p.scale_log2;
                const float mn = fmaxf(m, mt), f = __builtin_amdgcn_exp2f(m - mn);
                l *= f;
                if constexpr (kSum) all *= f;
                m = mn;
#pragma unroll
                for (int c = 0; c < NC; ++c) o[c] *= f;
            }
            // Weights are powers of two of sc factor - base: the products go into the
            // multiply-add unrounded, which scales all weights of a row by what m lost to
            // rounding; from kFusedMax on, where that might be too much, they are rounded.
            float factor = p.scale_log2, base = m;
            if (__any(fabsf(m) > kFusedMax && m > kNoScore)) {
#pragma clang fp contract(off)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    sc[0][i] = sc[0][i] * factor - m;
                    sc[1][i] = sc[1][i] * factor - m;
                }
                factor = 1.0f;
                base = 0.0f;
            }
            auto weights = [&](auto kc, auto ic) __attribute__((always_inline)) {
                constexpr int k = decltype(kc)::value, i = decltype(ic)::value;
                const float a = head_weight(sc[k >> 1][8 * (k & 1) + 2 * i], factor, base);
                const float e = head_weight(sc[k >> 1][8 * (k & 1) + 2 * i + 1], factor, base);
                pf[k][i] = lat_pack(a, e);
                if constexpr (kRest) {
                    const lat_f32x2 rest = lat_rest(pf[k][i], a, e);
                    pr[k][i] = lat_pack(rest[0], rest[1]);
                    const lat_f32x2 last = lat_rest(pr[k][i], rest[0], rest[1]);
                    pl[k][i] = lat_pack(last[0], last[1]);
                    l += a + e;
                } else {
                    l = lat_sum2(pf[k][i], l);
                    if constexpr (kSum) all += a + e;
                }
            };
            lat_for<0, 4>([&](auto ic) __attribute__((always_inline)) { weights(LatInt<0>{}, ic); });
            __builtin_amdgcn_sched_barrier(0);
            // The sums, and the next 16 tokens' weights between them.
            lat_for<0, 4 * NC>([&](auto ic) __attribute__((always_inline)) {
                constexpr int i = decltype(ic)::value, k = i / NC, kPairs = 4 / NC;
                const lat_u32x4 f = fr[i % kAhead];
                o[i % NC] = lat_mma(f, pf[k], o[i % NC]);
                if constexpr (kRest) {
                    o[i % NC] = lat_mma(f, pr[k], o[i % NC]);
                    o[i % NC] = lat_mma(f, pl[k], o[i % NC]);
                }
                if constexpr (i + kAhead < 4 * NC) fr[i % kAhead] = value(v, i + kAhead, vp);
                if constexpr (k < 3)
                    lat_for<0, kPairs>([&](auto jc) __attribute__((always_inline)) {
                        weights(LatInt<(k < 3 ? k + 1 : 3)>{}, LatInt<i % NC * kPairs + decltype(jc)::value>{});
                    });
                __builtin_amdgcn_sched_barrier(0);
            });
        };
        if (steps > 0) {
            win = head_window(p, soon);
            const Eights x = eights(0);
#pragma unroll
            for (int n2 = 0; n2 < 2 * kLoads; ++n2) load(n2, x, 0, kt0, vt0);
            load_far(x, 0, kt0, vt0);
            lat_wait_vm<2 * kLoads>();
            asm volatile("" ::: "memory");
#pragma unroll
            for (int j = 0; j < kJ; ++j) qf[j] = own[(kp0 ^ (2 * (j & 3))) + (j >> 2) * kWave];
            __builtin_amdgcn_s_waitcnt(15 | (7 << 4) | (0 << 8) | (3 << 14));
            lat_barrier();                 // the stages the queries came through are free
            for (int s = 0; s < steps; s += 2) {
                step(s, kt0, vt0, kt1, vt1);
                if (s + 1 < steps) step(s + 1, kt1, vt1, kt0, vt0);
            }
        }

        lat_wait_vm<0>();
        __syncthreads();           // nobody reads the stages any more
        l = lat_sum_pair(l);
        all = kSum ? lat_sum_pair(all) : l;
        const bool odd = __builtin_amdgcn_readfirstlane(odd_values) || __any(head_odd(o, l));
        const size_t slot0 = ((size_t)g * line.total + at_b + rt * parts + part) * kTileRows;
        const float f = whole ? head_inverse(l) : 1.0f;
        if (hf == 0 && my0 + n < rows) {
            if (!whole) {
                *(float2*)(p.part_ml + 2 * (slot0 + 32 * wave + n)) = make_float2(steps > 0 ? m : kNoPart, l);
                if constexpr (kSum) p.part_sum[slot0 + 32 * wave + n] = all;
            } else if (p.lse) {
                p.lse[at_row] = lat_lse(m, all);
            }
        }
        // 8 (dim 64: 4) KiB a wave: as much of a row at a time as a bf16 row has, unit
        // u (16 bytes) of it at u ^ (row % units).
        lat_u32x4* const out = &(wave < 2 ? kt0 : vt0).v[4 * (wave & 1)][0][0];
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
                    char* const to = (char*)row_of(r) + 16 * kUnits * pass + 16 * un;      // (by a shuffle: all lanes take part)
                    if (my0 + r < rows) *(lat_u32x4*)to = v;
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
            head_put_odd<D>(p, b, g, tok0, kTileTokens, kTileTokens, end, sees, [&](int d, float v, bool again) {
                if (my0 + n >= rows || !(l < INFINITY)) return;
                if (!whole) {
                    float* at = p.part + (slot0 + 32 * wave + n) * D + d;
                    *at = again ? *at + v : v;
                } else if (p.y_bf16) {
                    __bf16* at = (__bf16*)p.y + (size_t)at_row * D + d;
                    *at = (__bf16)(again ? (float)*at + v : v);
                } else {
                    float* at = (float*)p.y + (size_t)at_row * D + d;
                    *at = again ? *at + v : v;
                }
            });
        }
    }
#endif
}

template <int D>
hipError_t head_tile(const HeadParams& p, unsigned grid, int pieces, hipStream_t s) {
    auto run = [&](auto tree, auto rest, auto sum) {
        hipLaunchKernelGGL((k_head_tile<D, decltype(tree)::value != 0, decltype(rest)::value != 0, decltype(sum)::value != 0>),
                           lat_grid(grid), dim3(kTileThreads), 0, s, p, pieces);
    };
    auto trees = [&](auto rest, auto sum) {
        if (p.tree) run(LatInt<1>{}, rest, sum);
        else run(LatInt<0>{}, rest, sum);
    };
    // Weights' remainders for 32-bit results only, whose l is of the weights themselves.
    if (!p.y_bf16) trees(LatInt<1>{}, LatInt<0>{});
    else if (p.lse) trees(LatInt<0>{}, LatInt<1>{});
    else trees(LatInt<0>{}, LatInt<0>{});
    return hipGetLastError();
}

}  // namespace
}  // namespace caee
