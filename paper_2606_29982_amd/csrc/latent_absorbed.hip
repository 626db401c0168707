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
// tokens, so that the second reads them from the L2 the first filled (64 users
// of 128 heads: 72 us for k_attend, 79 without; both of plain bf16 weights).
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

// Units are counted up to this; no request has more (a limit of the host's,
// as is that of all requests while their lengths add up to max_kv at most).
constexpr int kMaxUnits = INT32_MAX / 2;
__device__ inline int add_units(int a, int b) { return min(a + b, kMaxUnits); }

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
    for (int b = b0; b < b1; ++b) n = add_units(n, units(b));
    part[tid] = n;
    __syncthreads();
    for (int d = 1; d < kAbsThreads; d <<= 1) {
        const int u = tid >= d ? part[tid - d] : 0;
        __syncthreads();
        part[tid] = add_units(part[tid], u);
        __syncthreads();
    }
    int at = tid > 0 ? part[tid - 1] : 0;
    for (int b = b0; b < b1; ++b) {
        p.meta[b] = at;
        at = add_units(at, units(b));
    }
    if (tid == kAbsThreads - 1) p.meta[p.B] = part[kAbsThreads - 1];
}

// 128 components of q'_th for 32 tokens of one head per workgroup: W_uk[h]^T
// rows as the M side of the product, tokens as the N side.  Both come through
// LDS, eight lanes a 128-byte line, and the outputs leave through it (straight
// from and to registers a lane's 16 bytes are a line of their own, 64 cycles a
// load: 15 us for 64 tokens of 128 heads where this takes 10).  Bound by
// the weights (2 nope latent bytes a head) while tokens are few.  q' is rounded
// to bf16 as the queries were: the scores' error of 2^-9 a product, random in
// sign, is that of the bf16 weights of the sums.
template <int NOPE>
__global__ __launch_bounds__(kAbsThreads) void k_absorb(LatentParams p, int tile_rows) {
    if (blockIdx.x == (unsigned)p.H) {
        if (blockIdx.y == 0 && blockIdx.z == 0) absorbed_shares(p, tile_rows);
        return;
    }
    constexpr int KS = NOPE / 16, G = NOPE / 64;
    __shared__ lat_u32x4 wt[16][G][kWave], qt[4][G][kWave];       // blocks of 8 rows x 128 bytes, swizzled
    const int h = blockIdx.x, t0 = blockIdx.y * 32;
    const int lane = threadIdx.x & 63, n = lane & 31, hf = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int width = p.latent + kRopeDim;
    const uint16_t* wrow = p.w_uk_t + ((size_t)h * p.latent + 128 * blockIdx.z) * NOPE;
#pragma unroll
    for (int i = 0; i < 5; ++i) {
        const int blk = i < 4 ? 4 * wave + i : wave, r = 8 * blk + (lane >> 3), c8 = 8 * ((lane & 7) ^ lat_swz(r));
        const uint16_t* src = i < 4 ? wrow + (size_t)r * NOPE
                                    : p.q + (size_t)min(t0 + r, p.T - 1) * p.q_stride + (size_t)h * (NOPE + kRopeDim);
#pragma unroll
        for (int g = 0; g < G; ++g)
            __builtin_amdgcn_global_load_lds((lat_g_void*)(src + 64 * g + c8),
                                             (lat_lds_void*)(i < 4 ? &wt[blk][g][0] : &qt[blk][g][0]), 16, 0, 0);
    }
    __syncthreads();
    lat_f32x16 acc = {};
    const int at = (n & 7) * 8 + (hf ^ lat_swz(n));
#pragma unroll
    for (int k = 0; k < KS; ++k)
        acc = lat_mma(wt[4 * wave + (n >> 3)][k / 4][at ^ (2 * (k % 4))], qt[n >> 3][k / 4][at ^ (2 * (k % 4))], acc);
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

// Half a KV tile: 32 cache rows as [row / 8][128-byte group][row % 8][16-byte
// piece, swizzled]: one direct-to-LDS load fills a block of 8 rows x 128
// bytes, so that a lane's addresses in all groups differ by constants.
constexpr int kHalf = kUnit / 2;
template <int R>
struct AbsHalf {
    static constexpr int kGroups = (R + kRopeDim) / 64;
    lat_u32x4 v[kHalf / 8][kGroups][kWave];
};

// What the waves hand each other in every step is written and read by these:
// the compiler lets an ordinary LDS access wait for all direct-to-LDS loads in
// flight unless it can tell that they go elsewhere.  The reads' waits are in
// the block, the writes' in lds_barrier.
__device__ inline void lds_put16(uint32_t at, const lat_u32x4& v) {
    asm volatile("ds_write_b128 %0, %1" ::"v"(at), "v"(v) : "memory");
}
__device__ inline void lds_put4(uint32_t at, uint32_t v) { asm volatile("ds_write_b32 %0, %1" ::"v"(at), "v"(v) : "memory"); }
__device__ inline void lds_get(uint32_t at, lat_u32x4 (&w)[4][2]) {
    asm volatile(
        "ds_read_b128 %0, %8\n"
        "ds_read_b128 %1, %8 offset:4 * 1024\n"
        "ds_read_b128 %2, %8 offset:1 * 1024\n"
        "ds_read_b128 %3, %8 offset:5 * 1024\n"
        "ds_read_b128 %4, %8 offset:2 * 1024\n"
        "ds_read_b128 %5, %8 offset:6 * 1024\n"
        "ds_read_b128 %6, %8 offset:3 * 1024\n"
        "ds_read_b128 %7, %8 offset:7 * 1024\n"
        "s_waitcnt lgkmcnt(0)"
        : "=&v"(w[0][0]), "=&v"(w[0][1]), "=&v"(w[1][0]), "=&v"(w[1][1]), "=&v"(w[2][0]), "=&v"(w[2][1]), "=&v"(w[3][0]),
          "=&v"(w[3][1])
        : "v"(at)
        : "memory");
}
__device__ inline void lds_put8(uint32_t at, const lat_u32x2& v) {
    asm volatile("ds_write_b64 %0, %1" ::"v"(at), "v"(v) : "memory");
}
__device__ inline void lds_get(uint32_t at, lat_u32x2 (&w)[4][2]) {
    asm volatile(
        "ds_read_b64 %0, %8\n"
        "ds_read_b64 %1, %8 offset:4 * 512\n"
        "ds_read_b64 %2, %8 offset:1 * 512\n"
        "ds_read_b64 %3, %8 offset:5 * 512\n"
        "ds_read_b64 %4, %8 offset:2 * 512\n"
        "ds_read_b64 %5, %8 offset:6 * 512\n"
        "ds_read_b64 %6, %8 offset:3 * 512\n"
        "ds_read_b64 %7, %8 offset:7 * 512\n"
        "s_waitcnt lgkmcnt(0)"
        : "=&v"(w[0][0]), "=&v"(w[0][1]), "=&v"(w[1][0]), "=&v"(w[1][1]), "=&v"(w[2][0]), "=&v"(w[2][1]), "=&v"(w[3][0]),
          "=&v"(w[3][1])
        : "v"(at)
        : "memory");
}
// Weights' remainders in 8 bits (e5m2, times 2^10: at most 2^10 for weights of
// up to kMaxWeight) and back as bf16.
constexpr float kRestScale = 1024.0f;
__device__ inline lat_u32x4 abs_rest(const lat_u32x2& v) {
    lat_u32x4 w;
    w[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(v[0], 1.0f / kRestScale, false));
    w[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(v[0], 1.0f / kRestScale, true));
    w[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(v[1], 1.0f / kRestScale, false));
    w[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(v[1], 1.0f / kRestScale, true));
    return w;
}
// The same and four flags.
__device__ inline uint32_t lds_get(uint32_t at, uint32_t flags, lat_u32x4 (&w)[4][2]) {
    lat_u32x4 f;
    asm volatile(
        "ds_read_b128 %0, %9\n"
        "ds_read_b128 %1, %9 offset:4 * 1024\n"
        "ds_read_b128 %2, %9 offset:1 * 1024\n"
        "ds_read_b128 %3, %9 offset:5 * 1024\n"
        "ds_read_b128 %4, %9 offset:2 * 1024\n"
        "ds_read_b128 %5, %9 offset:6 * 1024\n"
        "ds_read_b128 %6, %9 offset:3 * 1024\n"
        "ds_read_b128 %7, %9 offset:7 * 1024\n"
        "ds_read_b128 %8, %10\n"
        "s_waitcnt lgkmcnt(0)"
        : "=&v"(w[0][0]), "=&v"(w[0][1]), "=&v"(w[1][0]), "=&v"(w[1][1]), "=&v"(w[2][0]), "=&v"(w[2][1]), "=&v"(w[3][0]),
          "=&v"(w[3][1]), "=&v"(f)
        : "v"(at), "v"(flags)
        : "memory");
    return f[0] | f[1] | f[2] | f[3];
}

// Tokens of a request up to which its weights' remainders are multiplied too:
// rounding errors weigh most where few rows share a sum, over long contexts they
// average out.  Errors of the result (of its size, rms; rounding it to bf16 is
// 0.0017 of them) without and with, and us: 901 tokens 0.0025 and 0.0022, 23.6 and
// 24.0; 64 requests of 128 heads, 2048 tokens 0.0025 and 0.0023, 81 and 92; 32 of
// 8192 0.0024 and 0.0023, 115 and 137; 16 of 16384 0.0024 and 0.0023, 111 and 132;
// 8 of 32768 0.0024 and 0.0023, 112 and 133; 5 of 120013, 32 heads 0.0024 and
// 0.0023, 139 and 161.  (16384 and 32768 with 32 heads: 0.00237 and 0.00230,
// 0.00236 and 0.00232.)
constexpr int kRestTokens = 16384;

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
// and 64 rows; this takes 72 and 121.  These and the figures below are of
// plain bf16 weights; with remainders the 64 users take 83.)
// The five are bound by the fetches (5.8 TB/s).  The 64 users, whose rows go to
// two workgroups each by way of an L2, are not: 2.1 TB/s, L2 hits of 48 %,
// matrix units busy 26 % of the cycles, so a step's chain and the segments'
// starts and ends with one wave a SIMD.  A CU takes 16 cycles for each load, so
// they go out between the MFMAs: the second half of the next tile beside the
// scores, the first half of the one after as soon as the sums are done with
// this tile's (with whole tiles of lookahead, all loads at a step's start: 96
// and 155 us before other changes that gained 20; between the scores' MFMAs: 84
// and 149).  Rows that one workgroup reads are not kept in the caches: 121 us
// for the five where it was 137; for the 64 users' it changes nothing.
// A row's running maximum moves only when a weight exceeds 2^kMaxSlack; then
// the workgroup exchanges maxima and rescales its sums.
// Scores, maxima and sums are fp32.  The weights are rounded to bf16, the type of
// the rows they multiply.  Up to kRestTokens (by the request's own length) what
// the rounding left, in 8 bits, is multiplied too; past them a row's sum is of
// the rounded weights, so that the roundings' mean cancels.
template <int R, bool kPairs>
__global__ __launch_bounds__(kAbsThreads, 1) void k_attend(LatentParams p) {
#if defined(__HIP_DEVICE_COMPILE__)   // the buffer-descriptor type exists for the GPU target only
    constexpr int kG = AbsHalf<R>::kGroups;
    constexpr int kJ = 4 * kG;                 // 16-deep steps of the scores' contraction
    constexpr int NC = R / 128;                // 32-column tiles of the latent per wave
    constexpr int kAhead = 6, kVAhead = 3;     // fragments read from LDS ahead of their MFMAs
    constexpr int kRowBytes = (R + kRopeDim) * 2;
    constexpr int kOnce = kPairs ? 0 : 2;      // rows that one workgroup reads: non-temporal loads
    // One object per stage and half, so that the compiler can tell the reads of
    // one from the loads that fill another.
    __shared__ AbsHalf<R> st0a, st0b, st1a, st1b;
    __shared__ lat_u32x4 pw[2][4][kWave];      // softmax weights: [row group][16 tokens][fragment]
    __shared__ lat_u32x2 pr[2][4][kWave];      // their remainders
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
    const uint32_t pr_at = (uint32_t)(uintptr_t)(lat_lds_void*)&pr[0][0][0];
    // Fragment places in a half.  Keys: row n, piece 2 j + hf.  Transposed
    // values: rows 16 ks + 8 e + 4 hf + (0 .. 3), four 16-byte pieces per 32
    // components.
    const int kp0 = (n >> 3) * (kG * kWave) + (n & 7) * 8 + (hf ^ lat_swz(n));
    const int vr = 4 * hf + ((lane & 15) >> 2);
    const int vp0 = 2 * (vr * 8 + ((2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) ^ lat_swz(vr))) + (lane & 1);

    for (int u = sh.u0; u < sh.u1;) {
        // Up to 64 requests: each lane has read one, all at once (one user: 12.1
        // us, 12.8 by a search in memory; 64: 72 and 74).
        int b, at_u;
        LatentReq rq;
        if (p.B <= kWave) {
            b = 63 - __clzll(__ballot(lane < p.B && mine_at <= u) | 1ull);
            at_u = __builtin_amdgcn_readlane(mine_at, b);
            rq = {__builtin_amdgcn_readlane(mine.t0, b), __builtin_amdgcn_readlane(mine.add, b),
                  __builtin_amdgcn_readlane(mine.seq, b), __builtin_amdgcn_readlane(mine.before, b)};
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
        auto sees = [&](int r) { return lat_sees(p, rq, r / p.H); };
        const int limit = sees(row);
        const int lim_min = __builtin_amdgcn_readfirstlane(sees(row0));
        const int tok0 = first * kUnit, tok1 = min(last * kUnit, sees(min(row0 + kAbsRows, rows) - 1));
        const int steps = tok1 > tok0 ? (tok1 - tok0 + kUnit - 1) / kUnit : 0;

        // Wave w fills rows 8 w .. 8 w + 7 of a half; a lane reads piece lane % 8
        // (swizzled) of row lane / 8 in every group.  Where the eight lie in one
        // page, its number is read by a scalar load (a vector load's wait would
        // drain the tiles in flight) a step or more ahead; else row by row.
        // Past the request's tokens: its last row, masked later.
        struct Rows {
            int page, at, span;       // of the first row; the others follow up to at + span
            bool one;
        };
        auto entry = [&](int j) __attribute__((always_inline)) {
            const size_t i = (size_t)b * p.max_blocks + min((unsigned)j, (unsigned)p.max_blocks - 1u);
            return ((const __attribute__((address_space(4))) int32_t*)p.table)[i];
        };
        auto rows_of = [&](int s, int half) __attribute__((always_inline)) {
            const int pos = tok0 + s * kUnit + kHalf * half + 8 * wave;
            const int r0 = min(pos, rq.seq - 1), r1 = min(pos + 7, rq.seq - 1);
            const unsigned j = __builtin_amdgcn_readfirstlane((unsigned)r0 / (unsigned)p.block);
            const int at = r0 - (int)(j * (unsigned)p.block);
            return Rows{entry(j), at, r1 - r0, at + (r1 - r0) < p.block};
        };
        // Buffer loads (the compiler counts the LDS reads apart from them): one
        // buffer per page, a lane's row a 32-bit offset in it.
        // Of size 0 where nothing is to be loaded: its loads cost no memory
        // traffic, and their number does not depend on a branch (the compiler
        // would wait for the fewest).
        auto page_buf = [&](int page, bool there = true) __attribute__((always_inline)) {
            return __builtin_amdgcn_make_buffer_rsrc(
                (void*)((const char*)p.cache + (size_t)min(max(page, 0), p.n_blocks - 1) * (uint32_t)p.block * kRowBytes), 0,
                there ? kLatBufBytes : 0, kLatBufWord3);
        };
        auto piece = [&]() __attribute__((always_inline)) { return 16u * ((lane & 7) ^ lat_swz(8 * wave + (lane >> 3))); };
        auto offset = [&](const Rows& v) __attribute__((always_inline)) {
            return (uint32_t)(v.at + min(lane >> 3, v.span)) * kRowBytes + piece();
        };
        auto load_each = [&](int s, int half, AbsHalf<R>& t) __attribute__((always_inline)) {
            lat_wait_vm<0>();
#pragma unroll 1
            for (int r = 0; r < 8; ++r) {
                const int pos = min(tok0 + s * kUnit + kHalf * half + 8 * wave + r, rq.seq - 1);
                const unsigned j = __builtin_amdgcn_readfirstlane((unsigned)pos / (unsigned)p.block);
                const __amdgpu_buffer_rsrc_t buf = page_buf(entry(j));
                const uint32_t at = (uint32_t)(pos - (int)(j * (unsigned)p.block)) * kRowBytes + piece();
                if (lane >> 3 == r) {
#pragma unroll
                    for (int g = 0; g < kG; ++g)
                        __builtin_amdgcn_raw_ptr_buffer_load_lds(buf, (lat_lds_void*)&t.v[wave][g][0], 16, at, 128 * g, 0, 0);
                }
            }
            lat_wait_vm<0>();
        };
        auto load = [&](int s, int half, AbsHalf<R>& t) __attribute__((always_inline)) {
            const Rows v = rows_of(s, half);
            if (v.one) {
                const __amdgpu_buffer_rsrc_t buf = page_buf(v.page);
                const uint32_t at = offset(v);
#pragma unroll
                for (int g = 0; g < kG; ++g)
                    __builtin_amdgcn_raw_ptr_buffer_load_lds(buf, (lat_lds_void*)&t.v[wave][g][0], 16, at, 128 * g, 0, 0);
            } else {
                load_each(s, half, t);
            }
        };

        __syncthreads();       // the segment before is done with the stages
        // The queries come through the other stage, laid out as a tile's rows
        // (a lane's piece of a row straight to its registers is a line of its
        // own, 64 cycles a load: 1.5 us more).
        {
            const __amdgpu_buffer_rsrc_t buf = __builtin_amdgcn_make_buffer_rsrc(
                (void*)(p.qw + ((size_t)rq.t0 * p.H + row0) * (R + kRopeDim)), 0, kLatBufBytes, kLatBufWord3);
            const int r = 8 * wave + (lane >> 3);
            const uint32_t at0 = (uint32_t)min(r, rows - 1 - row0) * kRowBytes + piece();
            const uint32_t at1 = (uint32_t)min(kHalf + r, rows - 1 - row0) * kRowBytes + piece();
#pragma unroll
            for (int g = 0; g < kG; ++g) {
                __builtin_amdgcn_raw_ptr_buffer_load_lds(buf, (lat_lds_void*)&st1a.v[wave][g][0], 16, at0, 128 * g, 0, 0);
                __builtin_amdgcn_raw_ptr_buffer_load_lds(buf, (lat_lds_void*)&st1b.v[wave][g][0], 16, at1, 128 * g, 0, 0);
            }
        }
        if (steps > 0) {
            load(0, 0, st0a);
            load(0, 1, st0b);
        }
        Rows next_b = rows_of(1, 1);
        lat_wait_vm<0>();
        lat_barrier();
        lat_u32x4 qf[kJ];
        auto queries = [&](const AbsHalf<R>& t) __attribute__((always_inline)) {
#pragma unroll
            for (int j = 0; j < kJ; ++j) qf[j] = (&t.v[0][0][0])[(kp0 ^ (2 * (j & 3))) + (j >> 2) * kWave];
        };
        if (rg) queries(st1b);
        else queries(st1a);
        lds_barrier();                         // before the stage is filled again
        {
            const Rows v = rows_of(1, 0);
            const __amdgpu_buffer_rsrc_t buf = page_buf(v.page, steps > 1 && v.one);
            const uint32_t at = offset(v);
#pragma unroll
            for (int g = 0; g < kG; ++g)
                __builtin_amdgcn_raw_ptr_buffer_load_lds(buf, (lat_lds_void*)&st1a.v[wave][g][0], 16, at, 128 * g, 0, 0);
            if (steps > 1 && !v.one) load_each(1, 0, st1a);
        }
        lat_f32x16 o[NC][2];
#pragma unroll
        for (int c = 0; c < NC; ++c) o[c][0] = o[c][1] = lat_f32x16{};
        float m = kNoScore, l = 0.0f;

        // Step s: tile s in ta and tb, the other stage's second half nb for that
        // of tile s + 1 (its first half is on its way).
        auto step = [&](auto rest_too, int s, AbsHalf<R>& ta, AbsHalf<R>& tb, AbsHalf<R>& nb) __attribute__((always_inline)) {
            constexpr bool kRest = decltype(rest_too)::value;
            const int tok = tok0 + s * kUnit;
            // This wave's part of the tile is there (the first half of the next
            // may stay in flight); after the barrier all of it is, and nobody
            // reads the other stage.
            lat_wait_vm<kG>();
            lat_barrier();
            lat_f32x16 sc = {};
            // (made here: the registers that a stage's addresses would take
            // through the loop are not there)
            int kp = kp0, vp = vp0;
            asm volatile("" : "+v"(kp), "+v"(vp));
            // Scores, key fragments kAhead steps ahead of their MFMA, with the
            // loads where the eight rows lie in one page.
            const bool more_b = s + 1 < steps, one_b = next_b.one;
            const __amdgpu_buffer_rsrc_t buf_b = page_buf(next_b.page, more_b && one_b);
            const uint32_t at_b = offset(next_b);
            const Rows next_a = rows_of(s + 2, 0);
            next_b = rows_of(s + 2, 1);
            auto scores = [&](const AbsHalf<R>& t) __attribute__((always_inline)) {
                const lat_u32x4* keys = &t.v[0][0][0];
                auto key = [&](int j) __attribute__((always_inline)) { return keys[(kp ^ (2 * (j & 3))) + (j >> 2) * kWave]; };
                __builtin_amdgcn_sched_barrier(0);
                lat_u32x4 kf[kAhead];
#pragma unroll
                for (int j = 0; j < kAhead; ++j) kf[j] = key(j);
                lat_for<0, kJ>([&](auto jc) __attribute__((always_inline)) {
                    constexpr int j = decltype(jc)::value;
                    sc = lat_mma(kf[j % kAhead], qf[j], sc);
                    if constexpr (j + kAhead < kJ) kf[j % kAhead] = key(j + kAhead);
                    if constexpr (j % 4 == 0) {
                        __builtin_amdgcn_raw_ptr_buffer_load_lds(buf_b, (lat_lds_void*)&nb.v[wave][j / 4][0], 16, at_b,
                                                                 128 * (j / 4), 0, kOnce);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                });
            };
            if (th) scores(tb);
            else scores(ta);
            if (more_b && !one_b) load_each(s + 1, 1, nb);
            // Values: fragments (16 tokens ks, column tile c) in order, kVAhead
            // ahead of their MFMAs.
            constexpr int kF = 4 * NC;
            auto value = [&](int i) __attribute__((always_inline)) {
                const int ks = i / NC, c = i % NC, cc = NC * wave + c;
                lat_u32x2 w[2];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int place = ((2 * (ks & 1) + e) * kG + (cc >> 1)) * (2 * kWave) + (vp ^ (8 * (cc & 1) + 2 * e));
                    const lat_u32x2* at = (const lat_u32x2*)(ks < 2 ? &ta.v[0][0][0] : &tb.v[0][0][0]) + place;
                    w[e] = __builtin_bit_cast(lat_u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lat_lds_s16x4*)at));
                }
                return lat_u32x4{w[0][0], w[0][1], w[1][0], w[1][1]};
            };
            lat_u32x4 vf[kVAhead];
#pragma unroll
            for (int i = 0; i < kVAhead; ++i) vf[i] = value(i);
            const bool masked = tok + kUnit > lim_min;
            if (masked) {
                asm volatile("");       // a branch, not selects in every step
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (tok + 32 * th + 8 * (i >> 2) + 4 * hf + (i & 3) >= limit) sc[i] = -INFINITY;
            }
            float more, big;
            auto weights = [&]() __attribute__((always_inline)) {
                more = big = 0.0f;
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    lat_u32x4 w;
                    [[maybe_unused]] int rest[2] = {0, 0};
                    lat_for<0, 4>([&](auto ic) __attribute__((always_inline)) {
                        constexpr int i = decltype(ic)::value;
                        const float a = lat_weight(sc[8 * k + 2 * i], p.scale_log2, m);
                        const float e = lat_weight(sc[8 * k + 2 * i + 1], p.scale_log2, m);
                        big = fmaxf(fmaxf(big, a), e);
                        w[i] = lat_pack(a, e);
                        if constexpr (kRest) {
                            const lat_f32x2 r = lat_rest(w[i], a, e);
                            rest[i / 2] = __builtin_amdgcn_cvt_pk_bf8_f32(r[0] * kRestScale, r[1] * kRestScale, rest[i / 2], i & 1);
                            more += a + e;
                        } else {
                            more = lat_sum2(w[i], more);
                        }
                    });
                    const int at = (rg * 4 + 2 * th + k) * kWave + lane;
                    lds_put16(pw_at + at * 16, w);
                    if constexpr (kRest) lds_put8(pr_at + at * 8, lat_u32x2{(uint32_t)rest[0], (uint32_t)rest[1]});
                }
            };
            lat_u32x4 bw[4][2];
            bool moves = s == 0;
            if (!moves) {
                weights();
                const bool over_it = __any(big > kMaxWeight);
                if (lane == 0) lds_put4(over_at + 4 * wave, over_it);
                lds_barrier();
                moves = __builtin_amdgcn_readfirstlane(lds_get(pw_at + 16 * lane, over_at, bw));
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
                lds_get(pw_at + 16 * lane, bw);
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
            [[maybe_unused]] lat_u32x2 br[4][2];
            if constexpr (kRest) lds_get(pr_at + 8 * lane, br);
            l += more;
            if (masked) {
                // Rows that some queries do not see may hold anything: their
                // infinities and NaNs must not meet the zero weights (queries
                // that see such a row have it in their scores).
                auto clear = [&](AbsHalf<R>& t, int r0) __attribute__((always_inline)) {
                    for (int i = threadIdx.x; i < (kHalf - r0) * (R / 8); i += kAbsThreads) {
                        const int r = r0 + i / (R / 8), c = i % (R / 8);
                        lat_u32x4& v = t.v[r >> 3][c >> 3][(r & 7) * 8 + (c & 7)];
#pragma unroll
                        for (int e = 0; e < 4; ++e) v[e] = lat_finite(v[e]);
                    }
                };
                clear(ta, max(lim_min - tok, 0));
                clear(tb, max(lim_min - tok - kHalf, 0));
                lds_barrier();
#pragma unroll
                for (int i = 0; i < kVAhead; ++i) vf[i] = value(i);
            }
            __builtin_amdgcn_sched_barrier(0);
            const bool more_a = s + 2 < steps;
            const __amdgpu_buffer_rsrc_t buf_a = page_buf(next_a.page, more_a && next_a.one);
            const uint32_t at_a = offset(next_a);
            [[maybe_unused]] lat_u32x4 rest[2];
            lat_for<0, kF>([&](auto ic) __attribute__((always_inline)) {
                constexpr int i = decltype(ic)::value;
                if constexpr (kRest && i % NC == 0) {
                    rest[0] = abs_rest(br[i / NC][0]);
                    rest[1] = abs_rest(br[i / NC][1]);
                }
                if constexpr (i == kF / 2) lat_barrier();      // nobody reads the first half any more
                o[i % NC][0] = lat_mma(vf[i % kVAhead], bw[i / NC][0], o[i % NC][0]);
                o[i % NC][1] = lat_mma(vf[i % kVAhead], bw[i / NC][1], o[i % NC][1]);
                if constexpr (kRest) {
                    o[i % NC][0] = lat_mma(vf[i % kVAhead], rest[0], o[i % NC][0]);
                    o[i % NC][1] = lat_mma(vf[i % kVAhead], rest[1], o[i % NC][1]);
                }
                if constexpr (i + kVAhead < kF) vf[i % kVAhead] = value(i + kVAhead);
                if constexpr (i >= kF / 2) {
                    constexpr int n0 = (i - kF / 2) * kG / (kF / 2), n1 = (i + 1 - kF / 2) * kG / (kF / 2);
                    lat_for<n0, n1>([&](auto gc) __attribute__((always_inline)) {
                        constexpr int g = decltype(gc)::value;
                        __builtin_amdgcn_raw_ptr_buffer_load_lds(buf_a, (lat_lds_void*)&ta.v[wave][g][0], 16, at_a, 128 * g, 0, kOnce);
                    });
                }
                __builtin_amdgcn_sched_barrier(0);
            });
            if (more_a && !next_a.one) load_each(s + 2, 0, ta);
        };
        auto walk = [&](auto rest_too) __attribute__((always_inline)) {
            for (int s = 0; s < steps; s += 2) {
                step(rest_too, s, st0a, st0b, st1b);
                if (s + 1 < steps) step(rest_too, s + 1, st1a, st1b, st0b);
            }
        };
        if (rq.seq <= kRestTokens) walk(LatInt<1>{});
        else walk(LatInt<0>{});

        lat_wait_vm<0>();          // no load is on its way into the stages any more
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
        // The sums leave through the stages, 16 rows in each half, unit c (16
        // bytes) of a row at c ^ (row % 32): a store then writes 1 KiB of a row.
        auto out = [&](int r, int i32) __attribute__((always_inline)) {      // row 32 r + i32
            return (float4*)(r == 0 ? (i32 < 16 ? &st0a : &st0b) : (i32 < 16 ? &st1a : &st1b)) + (i32 & 15) * (R / 4);
        };
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            const float f = whole ? lat_inverse(sm[0][32 * r + n] + sm[1][32 * r + n]) : 1.0f;
            float4* const at = out(r, n);
#pragma unroll
            for (int c = 0; c < NC; ++c)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    at[(8 * (NC * wave + c) + 2 * i + hf) ^ n] =
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
                ((float4*)dst)[32 * r * (R / 4) + i] = out(r, i / (R / 4))[(i % (R / 4)) ^ (i / (R / 4))];
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
// one (512 partial tiles of 64 rows in all, so 16 a row at 2048 rows): one and
// four waves take 14 and 18 us for 8192 rows of three each, 14 and 11 for 320
// of a hundred.
constexpr int kJoinRows = 2048;
template <int R, bool kPairs, int kWaves>
__global__ __launch_bounds__(kAbsThreads) void k_join(LatentParams p) {
    constexpr int V = R / kWave;              // components of a lane
    __shared__ float red[kWaves == 1 ? 1 : kWaves - 1][V][kWave];
    const int lane = threadIdx.x & 63, wave_of_wg = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wave = kWaves == 1 ? 0 : wave_of_wg;
    const size_t at = kWaves == 1 ? (size_t)lat_workgroup() * (kAbsThreads / kWave) + wave_of_wg : lat_workgroup();
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
            constexpr int kLast = (kPairs ? kAbsGroups / 2 : kAbsGroups) - 1;
            g0 = min((int)((unsigned)a / (unsigned)per), kLast);
            g1 = min((int)((unsigned)(a + n_u - 1) / (unsigned)per), kLast);
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

// 64 components of y_th for 32 tokens of one head per workgroup, W_uv rows as
// the M side: a wave has 64 of the contraction, whose operands it fetches into
// its own part of LDS, eight lanes a 128-byte line (straight to registers a
// lane's 16 bytes are a line of their own, 64 cycles a load: 16 us for 64 tokens
// of 128 heads where this takes 12); the waves' sums are added through LDS in
// order.
// The attended latents are split into two bf16 parts (value and remainder),
// which keeps them at 16 bits of mantissa for one more product per step of
// a kernel that the weights' and the latents' bytes bound.
template <int R>
__global__ __launch_bounds__(R) void k_unabsorb(LatentParams p) {
    constexpr int kRanges = R / kWave;
    __shared__ lat_u32x4 wt[kRanges][8][kWave], ot[kRanges][2][4][kWave];      // blocks of 8 rows x 128 bytes, swizzled
    const int h = blockIdx.x, t0 = blockIdx.y * 32, v0 = blockIdx.z * 64;
    const int lane = threadIdx.x & 63, n = lane & 31, hf = lane >> 5;
    const int kr = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int r = 8 * i + (lane >> 3), c = (lane & 7) ^ lat_swz(r);
        const uint16_t* w = p.w_uv + ((size_t)h * p.v + v0 + r) * R + 64 * kr + 8 * c;
        __builtin_amdgcn_global_load_lds((lat_g_void*)w, (lat_lds_void*)&wt[kr][i][0], 16, 0, 0);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = 8 * i + (lane >> 3), c = (lane & 7) ^ lat_swz(r);
        const float* o = p.o + ((size_t)min(t0 + r, p.T - 1) * p.H + h) * R + 64 * kr + 4 * c;
#pragma unroll
        for (int g = 0; g < 2; ++g)
            __builtin_amdgcn_global_load_lds((lat_g_void*)(o + 32 * g), (lat_lds_void*)&ot[kr][g][i][0], 16, 0, 0);
    }
    lat_wait_vm<0>();          // what a wave reads it has loaded itself
    asm volatile("" ::: "memory");
    lat_f32x16 acc[2] = {};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int at = (n & 7) * 8, sw = lat_swz(n), c0 = 4 * (k & 1) + 2 * hf;
        const lat_u32x4 a = ot[kr][k >> 1][n >> 3][at + (c0 ^ sw)], b = ot[kr][k >> 1][n >> 3][at + ((c0 + 1) ^ sw)];
        lat_u32x4 hi, lo;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float x0 = __uint_as_float(i < 2 ? a[2 * i] : b[2 * i - 4]), x1 = __uint_as_float(i < 2 ? a[2 * i + 1] : b[2 * i - 3]);
            hi[i] = lat_pack(x0, x1);
            lo[i] = lat_pack(x0 - __uint_as_float(hi[i] << 16), x1 - __uint_as_float(hi[i] & 0xFFFF0000u));
        }
#pragma unroll
        for (int v = 0; v < 2; ++v) {
            const lat_u32x4 w = wt[kr][4 * v + (n >> 3)][at + ((2 * k + hf) ^ sw)];
            acc[v] = lat_mma(w, lo, lat_mma(w, hi, acc[v]));
        }
    }
    __syncthreads();
    float4(*const red)[2][4][kWave] = (float4(*)[2][4][kWave])&wt;
#pragma unroll
    for (int v = 0; v < 2; ++v)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            red[kr][v][i][lane] = make_float4(acc[v][4 * i], acc[v][4 * i + 1], acc[v][4 * i + 2], acc[v][4 * i + 3]);
    __syncthreads();
    // Four outputs of a token a thread, 16 threads a token.
    for (int j = threadIdx.x; j < 512; j += R) {
        const int tok = j >> 4, c = j & 15, v = c >> 3, i = (c & 7) >> 1, from = tok + 32 * (c & 1);
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
        const size_t o = ((size_t)(t0 + tok) * p.H + h) * p.v + v0 + 4 * c;
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
        if (rows < kJoinRows) hipLaunchKernelGGL((k_join<R, kPairs, 4>), lat_grid((unsigned)rows), block, 0, s, p);
        else hipLaunchKernelGGL((k_join<R, kPairs, 1>), lat_grid((unsigned)((rows + 3) / 4)), block, 0, s, p);
        hipLaunchKernelGGL(k_unabsorb<R>, dim3(p.H, (p.T + 31) / 32, p.v / 64), dim3(R), 0, s, p);
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
