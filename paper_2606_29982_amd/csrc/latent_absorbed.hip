// Latent attention, absorbed form: queries in the latent space attend to the
// cache rows themselves, so that each row is read once for all heads.
//
//   k_absorb     q'_th = [W_uk[h]^T q_nope | q_rope]   (and the shares below)
//   k_attend     per 64 (token, head) rows: s = q' . row, o' = sum softmax(s) c
//   k_join       partial results of requests that several workgroups share
//   k_unabsorb   y_th = W_uv[h] o'_th
//
// The rows of a request are its new tokens' heads, (token, head) with the
// head running fastest; a workgroup takes 64 of them.  The work of all
// requests is one line of units (64 tokens of one row tile, or of two, each),
// cut into equal shares: any mix of lengths keeps all CUs busy to the end,
// one long request is split as far as it takes, and a share that lies within
// many short requests leaves no partial results.
#include "latent.h"

namespace caee {
namespace {

constexpr int kAbsThreads = 256;
constexpr int kAbsRows = kAbsTileRows;   // query rows of a workgroup
constexpr int kUnit = 64;                // tokens of a tile, the unit shares are counted in

// A workgroup's share of the units.  With pairs, two workgroups of one XCD
// (neighbours in its launch order) take the two row tiles of the same
// tokens, so that the second reads them from the L2 the first filled.
struct AbsShare {
    int u0, u1, member;
};
template <bool kPairs>
__device__ inline int abs_share(int total) {
    constexpr int kGroups = kPairs ? kAbsGroups / 2 : kAbsGroups;
    return max((total + kGroups - 1) / kGroups, 1);
}
template <bool kPairs>
__device__ inline AbsShare abs_share_of(int total, int wg) {
    const int per = abs_share<kPairs>(total);
    const int k = wg / kXcds;
    const int g = kPairs ? (k >> 1) * kXcds + wg % kXcds : wg;
    const int u0 = min((long long)g * per, (long long)total);
    return {u0, min(u0 + per, total), kPairs ? k & 1 : 0};
}
// Workgroup of member m of share g.
template <bool kPairs>
__device__ inline int abs_workgroup(int g, int m) {
    return kPairs ? (g / kXcds * 2 + m) * kXcds + g % kXcds : g;
}

// Barrier that waits for this wave's LDS operations, not for its loads in flight.
__device__ inline void lds_barrier() {
    __builtin_amdgcn_s_waitcnt(15 | (7 << 4) | (0 << 8) | (3 << 14));
    lat_barrier();
}

// First unit of each request's row tiles (meta[b]; meta[B] the total).
__device__ void absorbed_shares(const LatentParams& p, int rows) {
    __shared__ int part[kAbsThreads];
    const int tid = threadIdx.x;
    const int chunk = (p.B + kAbsThreads - 1) / kAbsThreads;
    const int b0 = min(tid * chunk, p.B), b1 = min(b0 + chunk, p.B);
    auto units = [&](int b) {
        const LatentReq r = lat_req(p, b);
        return ((r.add * p.H + rows - 1) / rows) * ((r.seq + kUnit - 1) / kUnit);
    };
    int n = 0;
    for (int b = b0; b < b1; ++b) n += units(b);
    part[tid] = n;
    __syncthreads();
    for (int d = 1; d < kAbsThreads; d <<= 1) {
        const int u = tid >= d ? part[tid - d] : 0;
        __syncthreads();
        part[tid] += u;
        __syncthreads();
    }
    int at = part[tid] - n;
    for (int b = b0; b < b1; ++b) {
        p.meta[b] = at;
        at += units(b);
    }
    if (tid == kAbsThreads - 1) p.meta[p.B] = part[kAbsThreads - 1];
}

// 128 components of q'_th for 32 tokens of one head per workgroup: W_uk[h]^T
// rows as the M side of the product, tokens as the N side, so that a lane ends
// with four consecutive latent components of one token.  Bound by the weights
// (2 nope latent bytes a head) while tokens are few.
template <int NOPE>
__global__ __launch_bounds__(kAbsThreads) void k_absorb(LatentParams p, int tile_rows) {
    if (blockIdx.x == (unsigned)p.H) {
        if (blockIdx.y == 0 && blockIdx.z == 0) absorbed_shares(p, tile_rows);
        return;
    }
    constexpr int KS = NOPE / 16;
    const int h = blockIdx.x, t0 = blockIdx.y * 32;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = lane & 31, hf = lane >> 5;
    const int t = t0 + n < p.T ? t0 + n : p.T - 1;
    const int width = p.latent + kRopeDim;
    const uint16_t* qt = p.q + (size_t)t * p.q_stride + (size_t)h * (NOPE + kRopeDim);
    lat_u32x4 qf[KS];
#pragma unroll
    for (int k = 0; k < KS; ++k) qf[k] = *(const lat_u32x4*)(qt + 16 * k + 8 * hf);
    const int c = blockIdx.z * (kAbsThreads / 64) + wave;
    const uint16_t* w = p.w_uk_t + ((size_t)h * p.latent + 32 * c + n) * NOPE + 8 * hf;
    lat_f32x16 acc = {};
#pragma unroll
    for (int k = 0; k < KS; ++k) acc = lat_mma(*(const lat_u32x4*)(w + 16 * k), qf[k], acc);
    // Through LDS, so that 16 lanes write 256 bytes of a token.
    __shared__ lat_u32x4 tile[32][17];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        lat_u32x2* at = (lat_u32x2*)&tile[n][4 * wave + i];
        at[hf] = lat_u32x2{lat_pack(acc[4 * i], acc[4 * i + 1]), lat_pack(acc[4 * i + 2], acc[4 * i + 3])};
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int r = 16 * i + (threadIdx.x >> 4), c8 = threadIdx.x & 15;
        if (t0 + r < p.T)
            *(lat_u32x4*)(p.qw + ((size_t)(t0 + r) * p.H + h) * width + 128 * blockIdx.z + 8 * c8) = tile[r][c8];
    }
    if (blockIdx.z > 0) return;
    // The rotary part goes along unchanged: 32 tokens x 8 pieces.
    const int rt = t0 + (threadIdx.x >> 3), q8 = threadIdx.x & 7;
    if (rt < p.T) {
        const uint16_t* src = p.q + (size_t)rt * p.q_stride + (size_t)h * (NOPE + kRopeDim) + NOPE + 8 * q8;
        *(lat_u32x4*)(p.qw + ((size_t)rt * p.H + h) * width + p.latent + 8 * q8) = *(const lat_u32x4*)src;
    }
}

// One KV tile: 64 cache rows as [row / 8][128-byte group][row % 8][16-byte
// piece, swizzled]: one direct-to-LDS load fills a block of 8 rows x 128
// bytes, so that a lane's addresses in all groups differ by constants.
template <int R>
struct AbsTile {
    static constexpr int kGroups = (R + kRopeDim) / 64;
    lat_u32x4 v[kUnit / 8][kGroups][kWave];
};

// What the waves hand each other in every step is written and read by these:
// the compiler lets an ordinary LDS access wait for all direct-to-LDS loads in
// flight unless it can tell that they go elsewhere.  The reads' waits are in
// the block, the writes' in lds_barrier.
__device__ inline void lds_put16(uint32_t at, const lat_u32x4& v) {
    asm volatile("ds_write_b128 %0, %1" ::"v"(at), "v"(v) : "memory");
}
__device__ inline void lds_put4(uint32_t at, uint32_t v) { asm volatile("ds_write_b32 %0, %1" ::"v"(at), "v"(v) : "memory"); }
__device__ inline void lds_get(uint32_t at, uint32_t flags, lat_u32x4 (&w)[4][2], lat_u32x4& f) {
    asm volatile(
        "ds_read_b128 %0, %9\n"
        "ds_read_b128 %1, %9 offset:4096\n"
        "ds_read_b128 %2, %9 offset:1024\n"
        "ds_read_b128 %3, %9 offset:5120\n"
        "ds_read_b128 %4, %9 offset:2048\n"
        "ds_read_b128 %5, %9 offset:6144\n"
        "ds_read_b128 %6, %9 offset:3072\n"
        "ds_read_b128 %7, %9 offset:7168\n"
        "ds_read_b128 %8, %10\n"
        "s_waitcnt lgkmcnt(0)"
        : "=&v"(w[0][0]), "=&v"(w[0][1]), "=&v"(w[1][0]), "=&v"(w[1][1]), "=&v"(w[2][0]), "=&v"(w[2][1]), "=&v"(w[3][0]),
          "=&v"(w[3][1]), "=&v"(f)
        : "v"(at), "v"(flags)
        : "memory");
}

// A workgroup holds 64 query rows and walks over the tiles of its share.
// Four waves, one per SIMD (a wave may use 512 registers), take two parts in
// turn:
//   scores: wave (rg, th) multiplies rows 32 rg .. + 31 (144 registers of
//     query fragments at latent 512) with tokens 32 th .. + 31 of the tile,
//     keys as the M side, so that a lane holds 16 scores of one row; the
//     weights it makes of them are, in that order, a fragment of the second
//     product and go through LDS as they are;
//   sums: wave w adds all 64 rows' weighted sums of a quarter of the latent
//     components, the values read from the same tile by transposed reads.
// A tile's row is then read once per 32 query rows for the scores and once
// for the sums.  (32 rows per wave with private sums would need 256
// accumulators beside the queries.  128 rows on eight waves, two per SIMD,
// fetch each row half as often, but their 256 registers a wave leave room for
// half the contraction only and cost one more exchange: 106 us for 64 users
// of 128 heads and 2048 tokens on average, 195 us for five of 120011 tokens
// and 64 rows; this takes 84 and 149.)
// It is bound by the fetches: the same loads with no work between them take
// 60 and 128 us (5.4 TB/s).  A CU takes 16 cycles for each load, so the next
// tile's go out between the scores' MFMAs, one to two of these (all at the
// start of the step: 96 and 155 us).
// A row's running maximum moves only when a weight exceeds 2^kMaxSlack; then
// the workgroup exchanges maxima and rescales its sums.
template <int R, bool kPairs>
__global__ __launch_bounds__(kAbsThreads, 1) void k_attend(LatentParams p) {
#if defined(__HIP_DEVICE_COMPILE__)   // the buffer-descriptor type exists for the GPU target only
    constexpr int kG = AbsTile<R>::kGroups;
    constexpr int kJ = 4 * kG;                 // 16-deep steps of the scores' contraction
    constexpr int NC = R / 128;                // 32-column tiles of the latent per wave
    constexpr int kAhead = 6, kVAhead = 3;     // fragments read from LDS ahead of their MFMAs
    constexpr int kRowBytes = (R + kRopeDim) * 2;
    // One object per stage, so that the compiler can tell the reads of one
    // from the loads that fill the other.
    __shared__ AbsTile<R> st0, st1;
    __shared__ lat_u32x4 pw[2][4][kWave];      // softmax weights: [row group][16 tokens][fragment]
    __shared__ float sm[2][kAbsRows], sf[kAbsRows];
    __shared__ int over[4];
    const int lane = threadIdx.x & 63, n = lane & 31, hf = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int rg = wave & 1, th = wave >> 1;
    int mine_at = 0;
    LatentReq mine = {};
    if (lane < p.B && p.B <= kWave) {
        mine_at = p.meta[lane];
        mine = lat_req(p, lane);
    }
    const AbsShare sh = abs_share_of<kPairs>(p.meta[p.B], blockIdx.x);
    const uint32_t pw_at = (uint32_t)(uintptr_t)(lat_lds_void*)&pw[0][0][0], over_at = (uint32_t)(uintptr_t)(lat_lds_void*)&over[0];
    // Fragment places in a tile.  Keys: row 32 th + n, piece 2 j + hf.
    // Transposed values: rows 16 ks + 8 e + 4 hf + (0 .. 3), four 16-byte
    // pieces per 32 components.
    const int kp0 = (4 * th + (n >> 3)) * (kG * kWave) + (n & 7) * 8 + (hf ^ lat_swz(n));
    const int vr = 4 * hf + ((lane & 15) >> 2);
    const int vp0 = 2 * (vr * 8 + ((2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) ^ lat_swz(vr))) + (lane & 1);

    for (int u = sh.u0; u < sh.u1;) {
        // Up to 64 requests: each lane has read one, all at once.
        int b, at_u;
        LatentReq rq;
        if (p.B <= kWave) {
            b = 63 - __clzll(__ballot(lane < p.B && mine_at <= u) | 1ull);
            at_u = __builtin_amdgcn_readlane(mine_at, b);
            rq = {__builtin_amdgcn_readlane(mine.t0, b), __builtin_amdgcn_readlane(mine.add, b),
                  __builtin_amdgcn_readlane(mine.seq, b)};
        } else {
            b = lat_find_wave(p.meta, p.B, u);
            rq = lat_req(p, b);
            at_u = p.meta[b];
        }
        const int rows = rq.add * p.H;
        const int n_u = (rq.seq + kUnit - 1) / kUnit;
        const int rel = u - at_u, rp = rel / n_u, first = rel - rp * n_u;
        const int rt = kPairs ? 2 * rp + sh.member : rp;
        const int last = min(n_u, first + (sh.u1 - u));
        const bool whole = first == 0 && last == n_u;
        const bool head = u == sh.u0;          // the share's first segment
        u += last - first;
        if (rt * kAbsRows >= rows) continue;   // a pair's second tile may not exist

        // This lane's query row and how many tokens it sees.
        const int row0 = rt * kAbsRows;
        const int row = min(row0 + 32 * rg + n, rows - 1);
        auto sees = [&](int r) { return p.causal ? min(max(rq.seq - rq.add + r / p.H + 1, 0), rq.seq) : rq.seq; };
        const int limit = sees(row);
        const int lim_min = __builtin_amdgcn_readfirstlane(sees(row0));
        const int tok0 = first * kUnit, tok1 = min(last * kUnit, sees(min(row0 + kAbsRows, rows) - 1));
        const int steps = tok1 > tok0 ? (tok1 - tok0 + kUnit - 1) / kUnit : 0;

        // Wave w fills the tile's rows 16 w .. 16 w + 15, eight by eight; a lane
        // reads piece lane % 8 (swizzled) of row lane / 8 in every group.  The
        // pages of its two rows come one tile ahead, used only after the wait
        // for that tile.  Past the request's tokens: its last row, masked later.
        struct Pages {
            int page[2], at[2];
        };
        auto pages_of = [&](int s) __attribute__((always_inline)) {
            Pages v;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const unsigned pos = min(tok0 + s * kUnit + 16 * wave + 8 * i + (lane >> 3), rq.seq - 1);
                const unsigned j = pos / (unsigned)p.block;
                v.page[i] = p.table[(size_t)b * p.max_blocks + min(j, (unsigned)p.max_blocks - 1u)];
                v.at[i] = (int)(pos - j * p.block);
            }
            return v;
        };
        // Buffer loads (the compiler counts the LDS reads apart from them): one
        // buffer per page, a lane's row a 32-bit offset in it.
        auto page_buf = [&](int page) __attribute__((always_inline)) {
            return __builtin_amdgcn_make_buffer_rsrc(
                (void*)((const char*)p.cache + (size_t)page * (uint32_t)p.block * kRowBytes), 0, kLatBufBytes, kLatBufWord3);
        };
        auto offset = [&](const Pages& v, int i) __attribute__((always_inline)) {
            return (uint32_t)v.at[i] * kRowBytes + 16 * ((lane & 7) ^ lat_swz(8 * i + (lane >> 3)));
        };
        auto page = [&](const Pages& v, int i) __attribute__((always_inline)) { return min(max(v.page[i], 0), p.n_blocks - 1); };
        // Eight rows in one page each; else row by row.
        auto one_page = [&](const Pages& v) __attribute__((always_inline)) {
            const int p0 = page(v, 0), p1 = page(v, 1);
            return __all(p0 == __builtin_amdgcn_readfirstlane(p0) && p1 == __builtin_amdgcn_readfirstlane(p1));
        };
        auto load = [&](const Pages& v, AbsTile<R>& t) __attribute__((always_inline)) {
            const bool one = one_page(v);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int pg = page(v, i);
                const uint32_t at = offset(v, i);
#pragma unroll 1
                for (int r = 0; r < (one ? 1 : 8); ++r) {
                    const __amdgpu_buffer_rsrc_t buf = page_buf(__builtin_amdgcn_readlane(pg, 8 * r));
                    if (one || lane >> 3 == r) {
#pragma unroll
                        for (int g = 0; g < kG; ++g)
                            __builtin_amdgcn_raw_ptr_buffer_load_lds(buf, (lat_lds_void*)&t.v[2 * wave + i][g][0], 16, at, 128 * g, 0, 0);
                    }
                }
            }
        };

        __syncthreads();       // the segment before is done with the tiles
        // The queries come through the other stage, laid out as a tile's rows
        // (a lane's piece of a row straight to its registers is a line of its
        // own, 64 cycles a load: 1.5 us more).
        {
            const __amdgpu_buffer_rsrc_t buf = __builtin_amdgcn_make_buffer_rsrc(
                (void*)(p.qw + ((size_t)rq.t0 * p.H + row0) * (R + kRopeDim)), 0, kLatBufBytes, kLatBufWord3);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int r = 16 * wave + 8 * i + (lane >> 3);
                const uint32_t at = (uint32_t)min(r, rows - 1 - row0) * kRowBytes + 16 * ((lane & 7) ^ lat_swz(8 * i + (lane >> 3)));
#pragma unroll
                for (int g = 0; g < kG; ++g)
                    __builtin_amdgcn_raw_ptr_buffer_load_lds(buf, (lat_lds_void*)&st1.v[2 * wave + i][g][0], 16, at, 128 * g, 0, 0);
            }
        }
        Pages ahead = {};
        if (steps > 0) {
            load(pages_of(0), st0);
            ahead = pages_of(1);
        }
        lat_wait_vm<0>();
        lat_barrier();
        lat_u32x4 qf[kJ];
        const int qp = kp0 + 4 * (rg - th) * (kG * kWave);
#pragma unroll
        for (int j = 0; j < kJ; ++j) qf[j] = (&st1.v[0][0][0])[(qp ^ (2 * (j & 3))) + (j >> 2) * kWave];
        __builtin_amdgcn_s_waitcnt(15 | (7 << 4) | (0 << 8) | (3 << 14));      // before the stage is filled again
        lat_f32x16 o[NC][2];
#pragma unroll
        for (int c = 0; c < NC; ++c) o[c][0] = o[c][1] = lat_f32x16{};
        float m = kNoScore, l = 0.0f;

        auto step = [&](int s, AbsTile<R>& t, AbsTile<R>& next) __attribute__((always_inline)) {
            const int tb = tok0 + s * kUnit;
            lat_wait_vm<0>();                  // this wave's part of the tile is there; after the barrier all of it is,
            lat_barrier();                     // and nobody reads the other stage
            lat_f32x16 sc = {};
            const lat_u32x4* keys = &t.v[0][0][0];
            // (made here: the registers that a stage's addresses would take
            // through the loop are not there)
            int kp = kp0, vp = vp0;
            asm volatile("" : "+v"(kp), "+v"(vp));
            auto key = [&](int j) __attribute__((always_inline)) { return keys[(kp ^ (2 * (j & 3))) + (j >> 2) * kWave]; };
            // Scores, key fragments kAhead steps ahead of their MFMA, with the
            // next tile's loads where its eight rows lie in one page each.
            const bool more_tiles = s + 1 < steps, spread = more_tiles && one_page(ahead);
            if (more_tiles && !spread) load(ahead, next);
            const __amdgpu_buffer_rsrc_t buf[2] = {page_buf(__builtin_amdgcn_readfirstlane(page(ahead, 0))),
                                                   page_buf(__builtin_amdgcn_readfirstlane(page(ahead, 1)))};
            const uint32_t at[2] = {offset(ahead, 0), offset(ahead, 1)};
            ahead = pages_of(s + 2);
            __builtin_amdgcn_sched_barrier(0);
            lat_u32x4 kf[kAhead];
#pragma unroll
            for (int j = 0; j < kAhead; ++j) kf[j] = key(j);
            lat_for<0, kJ>([&](auto jc) __attribute__((always_inline)) {
                constexpr int j = decltype(jc)::value;
                sc = lat_mma(kf[j % kAhead], qf[j], sc);
                if constexpr (j + kAhead < kJ) kf[j % kAhead] = key(j + kAhead);
                if constexpr (j % 2 == 0) {
                    constexpr int i = j / 2 / kG, g = j / 2 % kG;
                    if (spread)
                        __builtin_amdgcn_raw_ptr_buffer_load_lds(buf[i], (lat_lds_void*)&next.v[2 * wave + i][g][0], 16, at[i],
                                                                 128 * g, 0, 0);
                }
                __builtin_amdgcn_sched_barrier(0);
            });
            // Values: fragments (16 tokens ks, column tile c) in order, kVAhead
            // ahead of their MFMAs.
            const lat_u32x2* base = (const lat_u32x2*)&t.v[0][0][0];
            constexpr int kF = 4 * NC;
            auto value = [&](int i) __attribute__((always_inline)) {
                const int ks = i / NC, c = i % NC, cc = NC * wave + c;
                lat_u32x2 w[2];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const lat_u32x2* at = base + ((2 * ks + e) * kG + (cc >> 1)) * (2 * kWave) + (vp ^ (8 * (cc & 1) + 2 * e));
                    w[e] = __builtin_bit_cast(lat_u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lat_lds_s16x4*)at));
                }
                return lat_u32x4{w[0][0], w[0][1], w[1][0], w[1][1]};
            };
            lat_u32x4 vf[kVAhead];
#pragma unroll
            for (int i = 0; i < kVAhead; ++i) vf[i] = value(i);
            const bool masked = tb + kUnit > lim_min;
            if (masked) {
                asm volatile("");       // a branch, not selects in every step
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (tb + 32 * th + 8 * (i >> 2) + 4 * hf + (i & 3) >= limit) sc[i] = -INFINITY;
            }
            float more, big;
            auto weights = [&]() __attribute__((always_inline)) {
                more = big = 0.0f;
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    lat_u32x4 w;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float a = __builtin_amdgcn_exp2f(fmaf(sc[8 * k + 2 * i], p.scale_log2, -m));
                        const float e = __builtin_amdgcn_exp2f(fmaf(sc[8 * k + 2 * i + 1], p.scale_log2, -m));
                        big = fmaxf(fmaxf(big, a), e);
                        w[i] = lat_pack(a, e);
                        more = lat_sum2(w[i], more);
                    }
                    lds_put16(pw_at + ((rg * 4 + 2 * th + k) * kWave + lane) * 16, w);
                }
            };
            lat_u32x4 bw[4][2], ov;
            bool moves = s == 0;
            if (!moves) {
                weights();
                const bool over_it = __any(big > kMaxWeight);
                if (lane == 0) lds_put4(over_at + 4 * wave, over_it);
                lds_barrier();
                lds_get(pw_at + 16 * lane, over_at, bw, ov);
                moves = __builtin_amdgcn_readfirstlane(ov[0] | ov[1] | ov[2] | ov[3]);
            }
            if (moves) {
                // Some maxima move (all do in the first step): they and the factors go round.
                float mt = sc[0];
#pragma unroll
                for (int i = 1; i < 16; ++i) mt = fmaxf(mt, sc[i]);
                mt = lat_max_pair(mt) * p.scale_log2;
                if (hf == 0) sm[th][32 * rg + n] = mt;
                lds_barrier();
                const float mn = fmaxf(m, fmaxf(sm[0][32 * rg + n], sm[1][32 * rg + n]));
                const float f = __builtin_amdgcn_exp2f(m - mn);
                l *= f;
                m = mn;
                if (th == 0 && hf == 0) sf[32 * rg + n] = f;
                weights();
                lds_barrier();
                lds_get(pw_at + 16 * lane, over_at, bw, ov);
                if (s > 0) {
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        const float fr = sf[32 * r + n];
#pragma unroll
                        for (int c = 0; c < NC; ++c) {
                            // Out of the accumulator registers and back within this branch, not in every step.
                            asm volatile("" : "+a"(o[c][r]));
                            o[c][r] *= fr;
                            asm volatile("" : "+a"(o[c][r]));
                        }
                    }
                }
            }
            l += more;
            if (masked) {
                // Rows that some queries do not see may hold anything: their
                // infinities and NaNs must not meet the zero weights (queries
                // that see such a row have it in their scores).
                const int r0 = max(lim_min - tb, 0);
                for (int i = threadIdx.x; i < (kUnit - r0) * (R / 8); i += kAbsThreads) {
                    const int r = r0 + i / (R / 8), c = i % (R / 8);
                    lat_u32x4& v = t.v[r >> 3][c >> 3][(r & 7) * 8 + (c & 7)];
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[e] = lat_finite(v[e]);
                }
                lds_barrier();
#pragma unroll
                for (int i = 0; i < kVAhead; ++i) vf[i] = value(i);
            }
            __builtin_amdgcn_sched_barrier(0);
            lat_for<0, kF>([&](auto ic) __attribute__((always_inline)) {
                constexpr int i = decltype(ic)::value;
                o[i % NC][0] = lat_mma(vf[i % kVAhead], bw[i / NC][0], o[i % NC][0]);
                o[i % NC][1] = lat_mma(vf[i % kVAhead], bw[i / NC][1], o[i % NC][1]);
                if constexpr (i + kVAhead < kF) vf[i % kVAhead] = value(i + kVAhead);
                __builtin_amdgcn_sched_barrier(0);
            });
        };
        for (int s = 0; s < steps; s += 2) {
            step(s, st0, st1);
            if (s + 1 < steps) step(s + 1, st1, st0);
        }

        // Row sums: two halves of a lane pair, two token halves.
        l = lat_sum_pair(l);
        __syncthreads();
        if (hf == 0) sm[th][32 * rg + n] = l;
        if (th == 0 && hf == 0) sf[32 * rg + n] = m;
        __syncthreads();
        const size_t slot0 = ((size_t)blockIdx.x * 2 + (head ? 0 : 1)) * kAbsRows;
        if (wave == 0 && row0 + lane < rows) {
            const float lr = sm[0][lane] + sm[1][lane];
            if (!whole) *(float2*)(p.part_ml + 2 * (slot0 + lane)) = make_float2(sf[lane], lr);
            else if (p.lse) p.lse[(size_t)rq.t0 * p.H + row0 + lane] = lat_lse(sf[lane], lr);
        }
        // The sums leave through the stages, 32 rows each, unit c (16 bytes) of
        // a row at c ^ (row % 32): a store then writes 1 KiB of a row.
        float4* const out[2] = {(float4*)&st0, (float4*)&st1};
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            const float f = whole ? lat_inverse(sm[0][32 * r + n] + sm[1][32 * r + n]) : 1.0f;
#pragma unroll
            for (int c = 0; c < NC; ++c)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    out[r][n * (R / 4) + ((8 * (NC * wave + c) + 2 * i + hf) ^ n)] =
                        make_float4(o[c][r][4 * i] * f, o[c][r][4 * i + 1] * f, o[c][r][4 * i + 2] * f, o[c][r][4 * i + 3] * f);
        }
        __syncthreads();
        float* const dst = whole ? p.o + ((size_t)rq.t0 * p.H + row0) * R : p.part + slot0 * R;
        const int n_rows = min(kAbsRows, rows - row0);
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            const int n_here = min(max(n_rows - 32 * r, 0), 32) * (R / 4);
#pragma unroll 8
            for (int i = threadIdx.x; i < n_here; i += kAbsThreads)
                ((float4*)dst)[32 * r * (R / 4) + i] = out[r][i ^ (i / (R / 4))];
        }
    }
#endif
}

// kWaves waves per (token, head) row: rows whose request lies in one share
// are done; the others are the sum of their shares' partial results; rows
// that see no token are zero.  The shares' maxima and sums are read 64 at a
// time, a lane each; the partial results go over the waves in turn and the
// waves' sums are added in order.  The chain of lookups bounds it, so few
// rows, which have many partial results, take four waves each, and many rows
// one (512 partial tiles of 64 rows in all, so 16 a row at 2048 rows; 14 us
// instead of 18 for 8192 rows of three each).
constexpr int kJoinRows = 2048;
template <int R, bool kPairs, int kWaves>
__global__ __launch_bounds__(kAbsThreads) void k_join(LatentParams p) {
    constexpr int V = R / kWave;              // components of a lane
    __shared__ float red[kWaves == 1 ? 1 : kWaves - 1][V][kWave];
    const int lane = threadIdx.x & 63, wave_of_wg = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wave = kWaves == 1 ? 0 : wave_of_wg;
    const size_t at = kWaves == 1 ? (size_t)blockIdx.x * (kAbsThreads / kWave) + wave_of_wg : blockIdx.x;
    const int t = (int)(at / p.H);
    if (t >= p.T) return;
    float* dst = p.o + at * R + V * lane;
    const int end = p.B > 0 ? p.cu_new[p.B] : 0;
    bool none = t >= end || t < p.cu_new[0];
    int g0 = 0, g1 = 0, a = 0, rr = 0, rt = 0, per = 1;
    if (!none) {
        const int b = lat_find_wave(p.cu_new, p.B, t);
        const LatentReq rq = lat_req(p, b);
        const int n_u = (rq.seq + kUnit - 1) / kUnit;
        rr = (int)((long long)at - (long long)rq.t0 * p.H);
        rt = rr / kAbsRows;
        none = n_u == 0 || t - rq.t0 >= rq.add;
        if (!none) {
            per = abs_share<kPairs>(p.meta[p.B]);
            a = p.meta[b] + (kPairs ? rt >> 1 : rt) * n_u;
            g0 = a / per;
            g1 = (a + n_u - 1) / per;
        }
    }
    if (none) {
        if (wave == 0) {
#pragma unroll
            for (int v = 0; v < V; ++v) dst[v] = 0.0f;
            if (p.lse && lane == 0) p.lse[at] = -INFINITY;
        }
        return;
    }
    if (g0 == g1) return;
    // Share g's slot: its second when the row's tokens begin inside it.
    auto slot = [&](int g) {
        return ((size_t)abs_workgroup<kPairs>(g, rt & 1) * 2 + (g == g0 && a > g0 * per ? 1 : 0)) * kAbsRows + rr % kAbsRows;
    };
    const float2* ml = (const float2*)p.part_ml;
    float m = kNoScore, l = 0.0f;
    for (int g = g0; g <= g1; g += kWave) {
        const float2 v = g + lane <= g1 ? ml[slot(g + lane)] : make_float2(kNoScore, 0.0f);
        float mn = fmaxf(m, v.x);
#pragma unroll
        for (int d = 32; d >= 1; d >>= 1) mn = fmaxf(mn, __shfl_xor(mn, d));
        float s = v.y * __builtin_amdgcn_exp2f(v.x - mn);
#pragma unroll
        for (int d = 32; d >= 1; d >>= 1) s += __shfl_xor(s, d);
        l = l * __builtin_amdgcn_exp2f(m - mn) + s;
        m = mn;
    }
    float sum[V] = {};
    auto add = [&](int g, auto count) __attribute__((always_inline)) {
        constexpr int U = decltype(count)::value;       // partial rows in flight
        float w[U], x[U][V];
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const size_t sl = slot(g + kWaves * i);
            w[i] = ml[sl].x;
#pragma unroll
            for (int v = 0; v < V; ++v) x[i][v] = p.part[sl * R + V * lane + v];
        }
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const float f = __builtin_amdgcn_exp2f(w[i] - m);
#pragma unroll
            for (int v = 0; v < V; ++v) sum[v] += f > 0.0f ? x[i][v] * f : 0.0f;
        }
    };
    int g = g0 + wave;
    for (; g + 7 * kWaves <= g1; g += 8 * kWaves) add(g, LatInt<8>{});
    for (; g <= g1; g += kWaves) add(g, LatInt<1>{});
    if constexpr (kWaves > 1) {
        if (wave > 0) {
#pragma unroll
            for (int v = 0; v < V; ++v) red[wave - 1][v][lane] = sum[v];
        }
        __syncthreads();
        if (wave > 0) return;
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int i = 0; i < kWaves - 1; ++i) sum[v] += red[i][v][lane];
    }
    const float inv = lat_inverse(l);
#pragma unroll
    for (int v = 0; v < V; ++v) dst[v] = sum[v] * inv;
    if (p.lse && lane == 0) p.lse[at] = lat_lse(m, l);
}

// y_th for 32 tokens of one head per workgroup, W_uv rows as the M side: a
// wave has an eighth of the contraction and all outputs, so that the attended
// latents, in 32 bits the larger operand, are read once; the eighths are added
// through LDS in order.  Latency bounds it: each wave has all its loads in
// flight at once.
// The attended latents are split into two bf16 parts (value and remainder),
// which keeps them at 16 bits of mantissa for one more product per step of
// a kernel that the weights' and the latents' bytes bound.
constexpr int kUnThreads = 512;
template <int R, int NV>
__global__ __launch_bounds__(kUnThreads) void k_unabsorb(LatentParams p) {
    constexpr int kRanges = kUnThreads / kWave;
    __shared__ float4 red[kRanges][NV][4][kWave];
    const int h = blockIdx.x, t0 = blockIdx.y * 32;
    const int lane = threadIdx.x & 63, n = lane & 31, hf = lane >> 5;
    const int kr = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int t = t0 + n < p.T ? t0 + n : p.T - 1;
    constexpr int kLen = R / kRanges;
    const int k0 = kr * kLen;
    const float* src = p.o + ((size_t)t * p.H + h) * R + 8 * hf + k0;
    const uint16_t* w = p.w_uv + ((size_t)h * p.v + n) * R + 8 * hf + k0;
    lat_f32x16 acc[NV] = {};
#pragma unroll
    for (int k = 0; k < kLen; k += 16) {
        const float4 a = *(const float4*)(src + k), b = *(const float4*)(src + k + 4);
        lat_u32x4 wf[NV];
#pragma unroll
        for (int v = 0; v < NV; ++v) wf[v] = *(const lat_u32x4*)(w + (size_t)32 * v * R + k);
        const float x[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
        lat_u32x4 hi, lo;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            hi[i] = lat_pack(x[2 * i], x[2 * i + 1]);
            lo[i] = lat_pack(x[2 * i] - __uint_as_float(hi[i] << 16), x[2 * i + 1] - __uint_as_float(hi[i] & 0xFFFF0000u));
        }
#pragma unroll
        for (int v = 0; v < NV; ++v) acc[v] = lat_mma(wf[v], lo, lat_mma(wf[v], hi, acc[v]));
    }
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            red[kr][v][i][lane] = make_float4(acc[v][4 * i], acc[v][4 * i + 1], acc[v][4 * i + 2], acc[v][4 * i + 3]);
    __syncthreads();
    // Four outputs of a token a thread: 8 lanes write 32 consecutive ones.
    for (int j = threadIdx.x; j < 8 * NV * 32; j += kUnThreads) {
        const int tok = j / (8 * NV), c = j % (8 * NV), v = c >> 3, i = (c & 7) >> 1, from = tok + 32 * (c & 1);
        if (t0 + tok >= p.T) continue;
        float4 s = red[0][v][i][from];
#pragma unroll
        for (int r = 1; r < kRanges; ++r) {
            const float4 x = red[r][v][i][from];
            s.x += x.x;
            s.y += x.y;
            s.z += x.z;
            s.w += x.w;
        }
        const size_t o = ((size_t)(t0 + tok) * p.H + h) * p.v + 4 * c;
        if (p.y_bf16) *(lat_u32x2*)((uint16_t*)p.y + o) = lat_u32x2{lat_pack(s.x, s.y), lat_pack(s.z, s.w)};
        else *(float4*)((float*)p.y + o) = s;
    }
}

template <bool kPairs>
void attend_on(const LatentParams& p, hipStream_t s) {
    const long long rows = (long long)p.T * p.H;
    const dim3 grid(kAbsGroups), block(kAbsThreads);
    auto run = [&](auto latent) {
        constexpr int R = decltype(latent)::value;
        hipLaunchKernelGGL((k_attend<R, kPairs>), grid, block, 0, s, p);
        if (rows < kJoinRows) hipLaunchKernelGGL((k_join<R, kPairs, 4>), dim3((unsigned)rows), block, 0, s, p);
        else hipLaunchKernelGGL((k_join<R, kPairs, 1>), dim3((unsigned)((rows + 3) / 4)), block, 0, s, p);
        const dim3 heads(p.H, (p.T + 31) / 32);
        if (p.v == 128) hipLaunchKernelGGL((k_unabsorb<R, 4>), heads, dim3(kUnThreads), 0, s, p);
        else hipLaunchKernelGGL((k_unabsorb<R, 2>), heads, dim3(kUnThreads), 0, s, p);
    };
    if (p.latent == 512) run(LatInt<512>{});
    else if (p.latent == 256) run(LatInt<256>{});
    else run(LatInt<128>{});
}

}  // namespace

hipError_t launch_latent_absorbed(const LatentParams& p, hipStream_t s) {
    // Two row tiles per request or more: their workgroups run in pairs.
    const bool pairs = (long long)p.max_new * p.H > kAbsRows;
    const dim3 grid(p.H + 1, (p.T + 31) / 32, p.latent / 128), block(kAbsThreads);
    const int unit_rows = pairs ? 2 * kAbsRows : kAbsRows;
    if (p.nope == 128) hipLaunchKernelGGL(k_absorb<128>, grid, block, 0, s, p, unit_rows);
    else hipLaunchKernelGGL(k_absorb<64>, grid, block, 0, s, p, unit_rows);
    if (pairs) attend_on<true>(p, s);
    else attend_on<false>(p, s);
    return hipGetLastError();
}

}  // namespace caee
