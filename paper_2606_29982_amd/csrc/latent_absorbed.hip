// Latent attention, absorbed form: queries in the latent space attend to the
// cache rows themselves, so that each row is read once for all heads.
//
//   k_absorb     q'_th = [W_uk[h]^T q_nope | q_rope]   (and the shares below)
//   k_attend     per 32 (token, head) rows: s = q' . row, o' = sum softmax(s) c
//   k_join       partial results of requests that several workgroups share
//   k_unabsorb   y_th = W_uv[h] o'_th
//
// The rows of a request are its new tokens' heads, (token, head) with the
// head running fastest; a workgroup takes 64 of them.  The work of all
// requests is one line of units (64 tokens of one row tile, or pair of
// tiles, each), cut into equal shares: any mix of lengths keeps all CUs busy to the
// end, one long request is split as far as it takes, and a share that lies
// within many short requests leaves no partial results.
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
__device__ inline AbsShare abs_share(int total, int wg) {
    constexpr int kGroups = kPairs ? kAbsGroups / 2 : kAbsGroups;
    const int per = max((total + kGroups - 1) / kGroups, 1);
    const int k = wg / kXcds;
    const int g = kPairs ? (k >> 1) * kXcds + wg % kXcds : wg;
    const int u0 = min((long long)g * per, (long long)total);
    return {u0, min(u0 + per, total), kPairs ? k & 1 : 0};
}
// Workgroup of member m of share group g.
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
__device__ void absorbed_shares(const LatentParams& p, bool pairs) {
    __shared__ int part[kAbsThreads];
    const int tid = threadIdx.x;
    const int chunk = (p.B + kAbsThreads - 1) / kAbsThreads;
    const int b0 = min(tid * chunk, p.B), b1 = min(b0 + chunk, p.B);
    auto units = [&](int b) {
        const LatentReq r = lat_req(p, b);
        const int rows = pairs ? 2 * kAbsRows : kAbsRows;
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

// q'_th for 32 tokens of one head per workgroup: W_uk[h]^T rows as the M side
// of the product, tokens as the N side, so that a lane ends with four
// consecutive latent components of one token.  Bound by the weights
// (2 nope latent bytes a head) while tokens are few.
template <int NOPE>
__global__ __launch_bounds__(kAbsThreads) void k_absorb(LatentParams p, int pairs) {
    if (blockIdx.x == (unsigned)p.H) {
        if (blockIdx.y == 0) absorbed_shares(p, pairs != 0);
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
    uint16_t* out = p.qw + ((size_t)t * p.H + h) * width;
    for (int c = wave; c < p.latent / 32; c += kAbsThreads / 64) {
        const uint16_t* w = p.w_uk_t + ((size_t)h * p.latent + 32 * c + n) * NOPE + 8 * hf;
        lat_f32x16 acc = {};
#pragma unroll
        for (int k = 0; k < KS; ++k) acc = lat_mma(*(const lat_u32x4*)(w + 16 * k), qf[k], acc);
        if (t0 + n < p.T) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const lat_u32x2 v = {lat_pack(acc[4 * i], acc[4 * i + 1]), lat_pack(acc[4 * i + 2], acc[4 * i + 3])};
                *(lat_u32x2*)(out + 32 * c + 8 * i + 4 * hf) = v;
            }
        }
    }
    // The rotary part goes along unchanged: 32 tokens x 8 pieces.
    const int rt = t0 + (threadIdx.x >> 3), q8 = threadIdx.x & 7;
    if (rt < p.T) {
        const uint16_t* src = p.q + (size_t)rt * p.q_stride + (size_t)h * (NOPE + kRopeDim) + NOPE + 8 * q8;
        *(lat_u32x4*)(p.qw + ((size_t)rt * p.H + h) * width + p.latent + 8 * q8) = *(const lat_u32x4*)src;
    }
}

// One KV tile: 64 cache rows as [row / 8][128-byte group][row % 8][16-byte
// piece ^ lat_swz(row)]: one direct-to-LDS load fills a block of 8 rows x 128
// bytes, so that a lane's addresses in all groups differ by constants.
template <int R>
struct AbsTile {
    static constexpr int kGroups = (R + kRopeDim) / 64;
    lat_u32x4 v[kUnit / 8][kGroups][kWave];
};

// A workgroup holds 64 query rows and walks over the tiles of its share.
// Four waves, one per SIMD, take two parts in turn:
//   scores: wave (rg, th) multiplies rows 32 rg .. + 31 (144 registers of
//     query fragments at latent 512) with tokens 32 th .. + 31 of the tile,
//     keys as the M side, so that a lane holds 16 scores of one row; the
//     weights it makes of them are, in that order, a fragment of the second
//     product and go through LDS as they are;
//   sums: wave w adds all 64 rows' weighted sums of a quarter of the latent
//     components, the values read from the same tile by transposed reads.
// A tile's row is then read once per 32 query rows for the scores and once
// for the sums: 251 KB of LDS reads and writes against 2176 cycles of matrix
// work per tile at latent 512 (32 rows per wave with private sums would need
// 256 accumulators, more than a wave has beside the scores'; 16 rows per wave
// twice the LDS bytes).
// The running maximum is common to a row's waves and moves only when some
// row's scores exceed it by more than kMaxSlack: then, and only then, the
// workgroup exchanges maxima and rescales its sums.
template <int R, bool kPairs>
__global__ __launch_bounds__(kAbsThreads, 1) void k_attend(LatentParams p) {
    constexpr int kG = AbsTile<R>::kGroups;
    constexpr int kJ = 4 * kG;                 // 16-deep steps of the scores' contraction
    constexpr int NC = R / 128;                // 32-column tiles of the latent per wave
    // One object per stage, so that the compiler can tell the reads of one
    // from the loads that fill the other.
    __shared__ AbsTile<R> st0, st1;
    __shared__ lat_u32x4 pw[2][4][kWave];      // softmax weights: [row group][16 tokens][fragment]
    __shared__ float sm[2][kAbsRows], sf[kAbsRows];
    __shared__ int over[4];
    const int lane = threadIdx.x & 63, n = lane & 31, hf = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int rg = wave & 1, th = wave >> 1;
    const AbsShare sh = abs_share<kPairs>(p.meta[p.B], blockIdx.x);
    // Fragment places in a tile.  Keys: row 32 th + n, piece 2 j + hf.
    // Transposed values: rows 4 hf + r of each eight, four 16-byte pieces per
    // 32 components.
    int kpos[4], vpos[2];
#pragma unroll
    for (int j = 0; j < 4; ++j) kpos[j] = (4 * th + (n >> 3)) * (kG * kWave) + (n & 7) * 8 + ((2 * j + hf) ^ lat_swz(n));
    const int vrow = 4 * hf + ((lane & 15) >> 2);
#pragma unroll
    for (int j = 0; j < 2; ++j)
        vpos[j] = 2 * (vrow * 8 + ((4 * j + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) ^ lat_swz(vrow))) + (lane & 1);

    for (int u = sh.u0; u < sh.u1;) {
        const int b = lat_find(p.meta, p.B, u);
        const LatentReq rq = lat_req(p, b);
        const int rows = rq.add * p.H;
        const int n_u = (rq.seq + kUnit - 1) / kUnit;
        const int rel = u - p.meta[b], rp = rel / n_u, first = rel - rp * n_u;
        const int rt = kPairs ? 2 * rp + sh.member : rp;
        const int last = min(n_u, first + (sh.u1 - u));
        const bool whole = first == 0 && last == n_u;
        const bool head = u == sh.u0;          // the share's first segment
        u += last - first;
        if (rt * kAbsRows >= rows) continue;   // a pair's second tile may not exist

        // This lane's query row and how many tokens it sees.
        const int row0 = rt * kAbsRows + rg * 32;
        const int row = min(row0 + n, rows - 1);
        auto sees = [&](int r) { return p.causal ? min(max(rq.seq - rq.add + r / p.H + 1, 0), rq.seq) : rq.seq; };
        const int limit = sees(row);
        const int lim_min = __builtin_amdgcn_readfirstlane(sees(rt * kAbsRows));
        const int tok0 = first * kUnit, tok1 = min(last * kUnit, sees(min(rt * kAbsRows + kAbsRows, rows) - 1));
        const int steps = tok1 > tok0 ? (tok1 - tok0 + kUnit - 1) / kUnit : 0;
        lat_u32x4 qf[kJ];
        const uint16_t* qrow = p.qw + ((size_t)rq.t0 * p.H + row) * (R + kRopeDim) + 8 * hf;
#pragma unroll
        for (int j = 0; j < kJ; ++j) qf[j] = *(const lat_u32x4*)(qrow + 16 * j);

        lat_f32x16 o[NC][2];
#pragma unroll
        for (int c = 0; c < NC; ++c) o[c][0] = o[c][1] = lat_f32x16{};
        float m = kNoScore, l = 0.0f;

        // Wave w fills the tile's rows 16 w .. 16 w + 15; a lane reads piece
        // lane % 8 (swizzled) of two of them in every group.  Tokens past the
        // request's read its last row and are masked later.
        struct Rows {
            uint32_t r[2];
        };
        auto rows_of = [&](int s) {
            Rows v;
#pragma unroll
            for (int i = 0; i < 2; ++i)
                v.r[i] = lat_slot(p, b, min(tok0 + s * kUnit + 16 * wave + 8 * i + (lane >> 3), rq.seq - 1));
            return v;
        };
        const uint16_t* piece = p.cache + 8 * ((lane & 7) ^ lat_swz(lane >> 3));
        auto load = [&](const Rows& v, AbsTile<R>& t) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const uint16_t* src = piece + (size_t)v.r[i] * (R + kRopeDim);
#pragma unroll
                for (int g = 0; g < kG; ++g)
                    __builtin_amdgcn_global_load_lds((lat_g_void*)(src + 64 * g),
                                                     (lat_lds_void*)&t.v[2 * wave + i][g][0], 16, 0, 0);
            }
        };
        auto step = [&](int s, AbsTile<R>& t, AbsTile<R>& next, Rows& ahead) __attribute__((always_inline)) {
            const int tb = tok0 + s * kUnit;
            lat_wait_vm<0>();                  // this wave's part of the tile is there; after the barrier all of it is,
            lat_barrier();                     // and nobody reads the other stage
            if (s + 1 < steps) {
                load(ahead, next);
                ahead = rows_of(s + 2);
            }
            __builtin_amdgcn_sched_barrier(0);
            lat_f32x16 sc = {};
#pragma unroll
            for (int j = 0; j < kJ; ++j) {
                sc = lat_mma((&t.v[0][0][0])[kpos[j % 4] + (j / 4) * kWave], qf[j], sc);
                if (j % 4 == 3) __builtin_amdgcn_sched_barrier(0);
            }
            __builtin_amdgcn_sched_barrier(0);
            const bool masked = tb + kUnit > lim_min;
            float mt = -INFINITY;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                sc[i] *= p.scale_log2;
                if (masked && tb + 32 * th + 8 * (i >> 2) + 4 * hf + (i & 3) >= limit) sc[i] = -INFINITY;
                mt = fmaxf(mt, sc[i]);
            }
            mt = lat_max_pair(mt);
            auto weights = [&]() __attribute__((always_inline)) {
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    lat_u32x4 w;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float a = __builtin_amdgcn_exp2f(sc[8 * k + 2 * i] - m);
                        const float e = __builtin_amdgcn_exp2f(sc[8 * k + 2 * i + 1] - m);
                        l += a + e;
                        w[i] = lat_pack(a, e);
                    }
                    pw[rg][2 * th + k][lane] = w;
                }
            };
            const bool mine = __any(mt > m + kMaxSlack);
            if (!mine) weights();
            if (lane == 0) over[wave] = mine;
            lds_barrier();
            if (over[0] | over[1] | over[2] | over[3]) {
                // Move the maxima (the waves that had none over it undo their sums).
                if (!mine) {
                    float back = 0.0f;
#pragma unroll
                    for (int i = 0; i < 16; ++i) back += __builtin_amdgcn_exp2f(sc[i] - m);
                    l -= back;
                }
                if (hf == 0) sm[th][32 * rg + n] = mt;
                lds_barrier();
                const float mn = fmaxf(m, fmaxf(sm[0][32 * rg + n], sm[1][32 * rg + n]));
                const float f = __builtin_amdgcn_exp2f(m - mn);
                l *= f;
                m = mn;
                if (th == 0 && hf == 0) sf[32 * rg + n] = f;
                weights();
                lds_barrier();
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    const float fr = sf[32 * r + n];
#pragma unroll
                    for (int c = 0; c < NC; ++c) o[c][r] *= fr;
                }
            }
            __builtin_amdgcn_sched_barrier(0);
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
            }
            const lat_u32x2* base = (const lat_u32x2*)&t.v[0][0][0];
#pragma unroll
            for (int ks = 0; ks < 4; ++ks) {
                const lat_u32x4 b0 = pw[0][ks][lane], b1 = pw[1][ks][lane];
#pragma unroll
                for (int c = 0; c < NC; ++c) {
                    const int cc = NC * wave + c;
                    lat_u32x2 w[2];
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const lat_u32x2* at = base + ((2 * ks + e) * kG + (cc >> 1)) * (2 * kWave) + vpos[NC > 1 ? c & 1 : cc & 1];
                        w[e] = __builtin_bit_cast(lat_u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lat_lds_s16x4*)at));
                    }
                    const lat_u32x4 a = {w[0][0], w[0][1], w[1][0], w[1][1]};
                    o[c][0] = lat_mma(a, b0, o[c][0]);
                    o[c][1] = lat_mma(a, b1, o[c][1]);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        };
        __syncthreads();       // the segment before is done with the ring
        Rows ahead = {};
        if (steps > 0) {
            load(rows_of(0), st0);
            ahead = rows_of(1);
        }
        for (int s = 0; s < steps; s += 2) {
            step(s, st0, st1, ahead);
            if (s + 1 < steps) step(s + 1, st1, st0, ahead);
        }

        // Row sums: two halves of a lane pair, two token halves.
        l = lat_sum_pair(l);
        __syncthreads();
        if (hf == 0) sm[th][32 * rg + n] = l;
        if (th == 0 && hf == 0) sf[32 * rg + n] = m;
        __syncthreads();
        const size_t slot0 = ((size_t)blockIdx.x * 2 + (head ? 0 : 1)) * kAbsRows;
        if (wave == 0 && rt * kAbsRows + lane < rows) {
            const float lr = sm[0][lane] + sm[1][lane];
            if (!whole) {
                p.part_ml[2 * (slot0 + lane)] = sf[lane];
                p.part_ml[2 * (slot0 + lane) + 1] = lr;
            } else if (p.lse) {
                p.lse[(size_t)rq.t0 * p.H + rt * kAbsRows + lane] = lat_lse(sf[lane], lr);
            }
        }
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            const int at = rt * kAbsRows + 32 * r + n;
            if (at >= rows) continue;
            const float f = whole ? lat_inverse(sm[0][32 * r + n] + sm[1][32 * r + n]) : 1.0f;
            float* dst = (whole ? p.o + ((size_t)rq.t0 * p.H + at) * R : p.part + (slot0 + 32 * r + n) * R) + 4 * hf;
#pragma unroll
            for (int c = 0; c < NC; ++c)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    *(float4*)(dst + 32 * (NC * wave + c) + 8 * i) =
                        make_float4(o[c][r][4 * i] * f, o[c][r][4 * i + 1] * f, o[c][r][4 * i + 2] * f,
                                    o[c][r][4 * i + 3] * f);
        }
    }
}

// One wave per (token, head) row: rows whose request lies in one share are
// done; the others are the sum of their shares' partial results, in share
// order; rows that see no token are zero.
template <bool kPairs>
__global__ __launch_bounds__(kAbsThreads) void k_join(LatentParams p) {
    const int lane = threadIdx.x & 63;
    const long long at = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (at >= (long long)p.T * p.H) return;
    const int t = (int)(at / p.H);
    float* dst = p.o + at * p.latent;
    bool none = p.B == 0 || t >= p.cu_new[p.B] || t < p.cu_new[0];
    int g0 = 0, g1 = 0, a = 0, rt = 0, rr = 0, per = 1;
    if (!none) {
        const int b = lat_find(p.cu_new, p.B, t);
        const LatentReq rq = lat_req(p, b);
        const int n_u = (rq.seq + kUnit - 1) / kUnit;
        rr = (int)(at - (long long)rq.t0 * p.H);
        none = n_u == 0 || t - rq.t0 >= rq.add;
        if (!none) {
            constexpr int kGroups = kPairs ? kAbsGroups / 2 : kAbsGroups;
            per = max((p.meta[p.B] + kGroups - 1) / kGroups, 1);
            rt = rr / kAbsRows;
            a = p.meta[b] + (kPairs ? rt >> 1 : rt) * n_u;
            g0 = a / per;
            g1 = (a + n_u - 1) / per;
        }
    }
    if (none) {
        for (int c = 4 * lane; c < p.latent; c += 256) *(float4*)(dst + c) = make_float4(0.f, 0.f, 0.f, 0.f);
        if (p.lse && lane == 0) p.lse[at] = -INFINITY;
        return;
    }
    if (g0 == g1) return;
    auto slot = [&](int g) {
        return ((size_t)abs_workgroup<kPairs>(g, rt & 1) * 2 + (g == g0 && a > g0 * per ? 1 : 0)) * kAbsRows + rr % kAbsRows;
    };
    float m = kNoScore, l = 0.0f;
    for (int g = g0; g <= g1; ++g) m = fmaxf(m, p.part_ml[2 * slot(g)]);
    for (int g = g0; g <= g1; ++g) l += p.part_ml[2 * slot(g) + 1] * __builtin_amdgcn_exp2f(p.part_ml[2 * slot(g)] - m);
    const float inv = lat_inverse(l);
    for (int c = 4 * lane; c < p.latent; c += 256) {
        float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int g = g0; g <= g1; ++g) {
            const size_t sl = slot(g);
            const float f = __builtin_amdgcn_exp2f(p.part_ml[2 * sl] - m) * inv;
            const float4 v = *(const float4*)(p.part + sl * p.latent + c);
            s.x += v.x * f;
            s.y += v.y * f;
            s.z += v.z * f;
            s.w += v.w * f;
        }
        *(float4*)(dst + c) = s;
    }
    if (p.lse && lane == 0) p.lse[at] = lat_lse(m, l);
}

// y_th for 32 tokens of one head per workgroup, W_uv rows as the M side.
// The attended latents are split into two bf16 parts (value and remainder),
// which keeps them at 16 bits of mantissa for one more product per step of
// a kernel that the weights and the latents' bytes bound.
__global__ __launch_bounds__(kAbsThreads) void k_unabsorb(LatentParams p) {
    const int h = blockIdx.x, t0 = blockIdx.y * 32;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = lane & 31, hf = lane >> 5;
    if (wave * 32 >= p.v) return;
    const int t = t0 + n < p.T ? t0 + n : p.T - 1;
    const float* src = p.o + ((size_t)t * p.H + h) * p.latent + 8 * hf;
    const uint16_t* w = p.w_uv + ((size_t)h * p.v + 32 * wave + n) * p.latent + 8 * hf;
    lat_f32x16 acc = {};
    for (int k = 0; k < p.latent; k += 16) {
        const float4 a = *(const float4*)(src + k), b = *(const float4*)(src + k + 4);
        const float x[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
        lat_u32x4 hi, lo;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            hi[i] = lat_pack(x[2 * i], x[2 * i + 1]);
            lo[i] = lat_pack(x[2 * i] - __uint_as_float(hi[i] << 16), x[2 * i + 1] - __uint_as_float(hi[i] & 0xFFFF0000u));
        }
        const lat_u32x4 wf = *(const lat_u32x4*)(w + k);
        acc = lat_mma(wf, hi, acc);
        acc = lat_mma(wf, lo, acc);
    }
    if (t0 + n >= p.T) return;
    const size_t o = ((size_t)t * p.H + h) * p.v + 32 * wave + 4 * hf;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (p.y_bf16) {
            const lat_u32x2 v = {lat_pack(acc[4 * i], acc[4 * i + 1]), lat_pack(acc[4 * i + 2], acc[4 * i + 3])};
            *(lat_u32x2*)((uint16_t*)p.y + o + 8 * i) = v;
        } else {
            *(float4*)((float*)p.y + o + 8 * i) =
                make_float4(acc[4 * i], acc[4 * i + 1], acc[4 * i + 2], acc[4 * i + 3]);
        }
    }
}

template <bool kPairs>
void attend_and_join(const LatentParams& p, hipStream_t s) {
    const dim3 grid(kAbsGroups), block(kAbsThreads);
    if (p.latent == 512) hipLaunchKernelGGL((k_attend<512, kPairs>), grid, block, 0, s, p);
    else if (p.latent == 256) hipLaunchKernelGGL((k_attend<256, kPairs>), grid, block, 0, s, p);
    else hipLaunchKernelGGL((k_attend<128, kPairs>), grid, block, 0, s, p);
    const long long rows = (long long)p.T * p.H;
    hipLaunchKernelGGL(k_join<kPairs>, dim3((unsigned)((rows + 3) / 4)), block, 0, s, p);
}

}  // namespace

hipError_t launch_latent_absorbed(const LatentParams& p, hipStream_t s) {
    // Two row tiles per request or more: their workgroups run in pairs.
    const bool pairs = (long long)p.max_new * p.H > kAbsRows;
    const unsigned tt = (unsigned)((p.T + 31) / 32);
    const dim3 block(kAbsThreads);
    if (p.nope == 128) hipLaunchKernelGGL(k_absorb<128>, dim3(p.H + 1, tt), block, 0, s, p, pairs ? 1 : 0);
    else hipLaunchKernelGGL(k_absorb<64>, dim3(p.H + 1, tt), block, 0, s, p, pairs ? 1 : 0);
    if (pairs) attend_and_join<true>(p, s);
    else attend_and_join<false>(p, s);
    hipLaunchKernelGGL(k_unabsorb, dim3(p.H, tt), block, 0, s, p);
    return hipGetLastError();
}

}  // namespace caee
