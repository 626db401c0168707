// Latent attention, absorbed form: queries in the latent space attend to the
// cache rows themselves, so that each row is read once for all heads.
//
//   k_absorb     q'_th = [W_uk[h]^T q_nope | q_rope]   (and the shares below)
//   k_attend     per 32 (token, head) rows: s = q' . row, o' = sum softmax(s) c
//   k_join       partial results of requests that several workgroups share
//   k_unabsorb   y_th = W_uv[h] o'_th
//
// The rows of a request are its new tokens' heads, (token, head) with the
// head running fastest; a workgroup takes 32, 64 or 128 of them.  The work of
// all requests is one line of units (32 tokens of one row tile each), cut into
// equal shares: any mix of lengths keeps all CUs busy to the
// end, one long request is split as far as it takes, and a share that lies
// within many short requests leaves no partial results.
#include "latent.h"

namespace caee {
namespace {

constexpr int kAbsThreads = 256;
constexpr int kAttendThreads = 512;

constexpr int kUnit = 32;                // tokens of a tile, the unit shares are counted in

// Units per share (shares are kAbsGroups consecutive ranges).
__device__ inline int abs_share(int total) { return max((total + kAbsGroups - 1) / kAbsGroups, 1); }

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
    uint16_t* out = p.qw + ((size_t)t * p.H + h) * width;
    const int c = blockIdx.z * (kAbsThreads / 64) + wave;
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
    if (blockIdx.z > 0) return;
    // The rotary part goes along unchanged: 32 tokens x 8 pieces.
    const int rt = t0 + (threadIdx.x >> 3), q8 = threadIdx.x & 7;
    if (rt < p.T) {
        const uint16_t* src = p.q + (size_t)rt * p.q_stride + (size_t)h * (NOPE + kRopeDim) + NOPE + 8 * q8;
        *(lat_u32x4*)(p.qw + ((size_t)rt * p.H + h) * width + p.latent + 8 * q8) = *(const lat_u32x4*)src;
    }
}

// One KV tile: 32 cache rows as [row / 8][128-byte group][row % 8][16-byte
// piece, swizzled]: one direct-to-LDS load fills a block of 8 rows x 128
// bytes, so that a lane's addresses in all groups differ by constants.
template <int R>
struct AbsTile {
    static constexpr int kGroups = (R + kRopeDim) / 64;
    lat_u32x4 v[kUnit / 8][kGroups][kWave];
};

// A workgroup holds 32 NR query rows (128 at most: all heads of a
// DeepSeek-R1 token) and walks over the tiles of its share.  Its 8 waves take
// two parts in turn:
//   scores: wave w multiplies rows 16 w .. + 15 (72 registers of query
//     fragments at latent 512) with the tile's 32 tokens, keys as the M side,
//     so that a lane holds 8 scores of one row and a row's maximum and sum
//     stay within a wave; the weights go to LDS as fragments of the second
//     product;
//   sums: wave w adds all rows' weighted sums of an eighth of the latent
//     components (128 accumulators), the values read from the same tile by
//     transposed reads.
// So a cache row is fetched once per 128 query rows, the rate at which a CU
// can fetch being what bounds a split with fewer (64 rows per workgroup:
// twice the bytes and 92 us where this takes XX for 64 users of 128 heads),
// and the accumulators and queries fit the register file without a copy.
// Tiles are fetched three ahead into a ring of four.
// A row's running maximum moves only when its scores exceed it by more than
// kMaxSlack; then the workgroup exchanges the factors and rescales its sums.
template <int R, int NR>
__global__ __launch_bounds__(kAttendThreads) void k_attend(LatentParams p) {
    constexpr int kG = AbsTile<R>::kGroups;
    constexpr int kJ = 2 * kG;                 // 32-deep steps of the scores' contraction
    constexpr int NC = R / 32;                 // 32-column tiles of the latent
    constexpr int kTiles = NC * NR;            // accumulator tiles of the workgroup
    // Waves over columns, the remaining factor over row tiles.
    constexpr int kCw = NC >= 8 ? 8 : NC, kRw = 8 / kCw;
    constexpr int MC = NC / kCw, MR = NR >= kRw ? NR / kRw : 1;
    constexpr int kSlotTiles = kAttendThreads / kUnit;
    constexpr int kAhead = 3;                  // key fragments read from LDS ahead of their MFMAs
    static_assert(kTiles > 0, "tiles");
    // One object per stage, so that the compiler can tell the reads of one
    // from the loads that fill the others.
    __shared__ AbsTile<R> st0, st1, st2, st3;
    __shared__ lat_u32x4 pw[NR][2][kWave];     // softmax weights: [row tile][16 tokens][fragment]
    __shared__ uint32_t slots[2][kAttendThreads];
    __shared__ float sf[32 * NR], sl[32 * NR];
    __shared__ int over[8];
    const int lane = threadIdx.x & 63, n = lane & 31, hf = lane >> 5, r16 = lane & 15, g4 = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const bool scorer = 16 * wave < 32 * NR;
    const int cw = wave % kCw, rw = wave / kCw;         // this wave's column and row part of the sums
    const bool summer = rw * MR < NR;
    const int total = p.meta[p.B], per = abs_share(total);
    const int share0 = min((long long)blockIdx.x * per, (long long)total), share1 = min(share0 + per, total);
    // Fragment places in a tile.  Keys: row r16 (+ 16), piece 4 j + g4.
    // Transposed values: rows 16 ks + 8 hf + 4 u + (0 .. 3), pieces 4 c + ...
    // A step of the piece's place by 4 (keys, values) or of four rows (values)
    // is an exclusive-or, so one register each serves all.
    const int kpos0 = (r16 >> 3) * (kG * kWave) + (r16 & 7) * 8 + (g4 ^ lat_swz(r16));
    const int vr = 8 * hf + (r16 >> 2);
    const int vpos0 = hf * (kG * 2 * kWave) +
                      2 * ((vr & 7) * 8 + ((2 * (g4 & 1) + ((lane & 3) >> 1)) ^ lat_swz(vr))) + (lane & 1);
    // Waves 2 i and 2 i + 1 fetch the tile's rows 8 i .. 8 i + 7, half of the
    // groups each; a lane reads piece lane % 8 (swizzled) of row lane / 8.
    constexpr int kEven = (kG + 1) / 2, kOdd = kG - kEven;
    const int blk = wave >> 1;
    const bool odd = wave & 1;
    const uint16_t* piece = p.cache + 8 * ((lane & 7) ^ lat_swz(8 * blk + (lane >> 3))) + (odd ? 64 * kEven : 0);

    for (int u = share0; u < share1;) {
        const int b = lat_find_wave(p.meta, p.B, u);
        const LatentReq rq = lat_req(p, b);
        const int rows = rq.add * p.H;
        const int n_u = (rq.seq + kUnit - 1) / kUnit;
        const int rel = u - p.meta[b], rt = rel / n_u, first = rel - rt * n_u;
        const int last = min(n_u, first + (share1 - u));
        const bool whole = first == 0 && last == n_u;
        const bool head = u == share0;         // the share's first segment
        u += last - first;

        const int row0 = rt * 32 * NR;
        const int row = min(row0 + 16 * wave + r16, rows - 1);      // this lane's row of the scores
        auto sees = [&](int r) { return p.causal ? min(max(rq.seq - rq.add + r / p.H + 1, 0), rq.seq) : rq.seq; };
        const int limit = sees(row), lim_min = sees(row0);
        const int tok0 = first * kUnit, tok1 = min(last * kUnit, sees(min(row0 + 32 * NR, rows) - 1));
        const int steps = tok1 > tok0 ? (tok1 - tok0 + kUnit - 1) / kUnit : 0;

        // Cache rows of 16 tiles' tokens at a time wait in LDS (a page number
        // used straight from its load would drain the loads in flight); past
        // the request's tokens that of its last row, masked later.
        auto fill_slots = [&](int chunk) __attribute__((always_inline)) {
            slots[chunk & 1][threadIdx.x] =
                lat_slot(p, b, min(tok0 + chunk * kAttendThreads + (int)threadIdx.x, rq.seq - 1));
        };
        auto load = [&](int s, AbsTile<R>& t) __attribute__((always_inline)) {
            const uint32_t slot = slots[(s / kSlotTiles) & 1][s % kSlotTiles * kUnit + 8 * blk + (lane >> 3)];
            const uint16_t* src = piece + (size_t)slot * (R + kRopeDim);
            if (odd) {
#pragma unroll
                for (int g = 0; g < kOdd; ++g)
                    __builtin_amdgcn_global_load_lds((lat_g_void*)(src + 64 * g), (lat_lds_void*)&t.v[blk][kEven + g][0], 16, 0, 0);
            } else {
#pragma unroll
                for (int g = 0; g < kEven; ++g)
                    __builtin_amdgcn_global_load_lds((lat_g_void*)(src + 64 * g), (lat_lds_void*)&t.v[blk][g][0], 16, 0, 0);
            }
        };
        // This wave's part of a tile has landed: the loads of the `later`
        // tiles that follow may stay in flight.
        auto landed = [&](int later) __attribute__((always_inline)) {
            if (later >= 2) {
                if (odd) lat_wait_vm<2 * kOdd>();
                else lat_wait_vm<2 * kEven>();
            } else if (later == 1) {
                if (odd) lat_wait_vm<kOdd>();
                else lat_wait_vm<kEven>();
            } else {
                lat_wait_vm<0>();
            }
        };
        __syncthreads();       // the segment before is done with the ring
        if (steps > 0) fill_slots(0);
        if (steps > kSlotTiles) fill_slots(1);
        __syncthreads();
        if (steps > 0) load(0, st0);
        if (steps > 1) load(1, st1);
        if (steps > 2) load(2, st2);
        lat_u32x4 qf[kJ];
        const uint16_t* qrow = p.qw + ((size_t)rq.t0 * p.H + row) * (R + kRopeDim) + 8 * g4;
        if (scorer) {
#pragma unroll
            for (int j = 0; j < kJ; ++j) qf[j] = *(const lat_u32x4*)(qrow + 32 * j);
        }
        lat_f32x16 o[MC][MR];
#pragma unroll
        for (int c = 0; c < MC; ++c)
#pragma unroll
            for (int r = 0; r < MR; ++r) o[c][r] = lat_f32x16{};
        float m = kNoScore, l = 0.0f;

        auto step = [&](int s, AbsTile<R>& t, AbsTile<R>& ahead) __attribute__((always_inline)) {
            const int tb = tok0 + s * kUnit;
            landed(steps - 1 - s);
            lat_barrier();                     // all of the tile is there, nobody reads the stage of the tile before
            if (s + 3 < steps) load(s + 3, ahead);
            if (s % kSlotTiles == 0 && s > 0 && s + kSlotTiles < steps) fill_slots(s / kSlotTiles + 1);
            const bool masked = tb + kUnit > lim_min;
            lat_f32x4 sc[2] = {};
            float mt = -INFINITY;
            bool mine = false;
            auto weight = [&](int i) __attribute__((always_inline)) {
                return __builtin_amdgcn_exp2f(fmaf(sc[i >> 2][i & 3], p.scale_log2, -m));
            };
            // Lane (r16, g4) holds tokens 16 k + 4 g4 .. + 3 of its row: half
            // of the fragment that lane (row % 32, g4 / 2) of the sums reads.
            auto weights = [&]() __attribute__((always_inline)) {
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const float a = weight(4 * k), e = weight(4 * k + 1), c = weight(4 * k + 2), d = weight(4 * k + 3);
                    l += (a + e) + (c + d);
                    lat_u32x2* dst = (lat_u32x2*)&pw[wave >> 1][k][16 * (wave & 1) + r16 + 32 * (g4 >> 1)];
                    dst[g4 & 1] = lat_u32x2{lat_pack(a, e), lat_pack(c, d)};
                }
            };
            if (scorer) {
                __builtin_amdgcn_sched_barrier(0);
                const lat_u32x4* keys = &t.v[0][0][0];
                int kp = kpos0;
                asm volatile("" : "+v"(kp));        // the stage's addresses are made here, not kept through the loop
                auto key = [&](int i) __attribute__((always_inline)) {     // step i / 2, 16 tokens i % 2
                    return keys[(kp ^ (4 * ((i >> 1) & 1))) + (i >> 2) * kWave + (i & 1) * (2 * kG * kWave)];
                };
                lat_u32x4 kf[kAhead];
#pragma unroll
                for (int i = 0; i < kAhead; ++i) kf[i] = key(i);
#pragma unroll
                for (int i = 0; i < 2 * kJ; ++i) {
                    sc[i & 1] = lat_mma16(kf[i % kAhead], qf[i >> 1], sc[i & 1]);
                    if (i + kAhead < 2 * kJ) kf[i % kAhead] = key(i + kAhead);
                }
                __builtin_amdgcn_sched_group_barrier(0x100, kAhead, 0);
#pragma unroll
                for (int i = 0; i < 2 * kJ; ++i) {
                    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                    if (i + kAhead < 2 * kJ) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
                }
                __builtin_amdgcn_sched_barrier(0);
                if (masked) {
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        if (tb + 16 * (i >> 2) + 4 * g4 + (i & 3) >= limit) sc[i >> 2][i & 3] = -INFINITY;
                }
#pragma unroll
                for (int i = 0; i < 8; ++i) mt = fmaxf(mt, sc[i >> 2][i & 3]);
                mt = fmaxf(mt, __shfl_xor(mt, 16));
                mt = lat_max_pair(mt) * p.scale_log2;
                mine = __any(mt > m + kMaxSlack);
                if (!mine) weights();
            }
            if (lane == 0) over[wave] = mine;
            lds_barrier();
            const int4 ov0 = *(const int4*)&over[0], ov1 = *(const int4*)&over[4];
            if (ov0.x | ov0.y | ov0.z | ov0.w | ov1.x | ov1.y | ov1.z | ov1.w) {
                // Some maxima move: their rows' factors go round, the others' are 1.
                if (scorer) {
                    float f = 1.0f;
                    if (mine) {
                        const float mn = fmaxf(m, mt);
                        f = __builtin_amdgcn_exp2f(m - mn);
                        l *= f;
                        m = mn;
                        weights();
                    }
                    if (g4 == 0) sf[16 * wave + r16] = f;
                }
                lds_barrier();
#pragma unroll
                for (int r = 0; r < MR; ++r) {
                    const float fr = sf[32 * ((rw * MR + r) % NR) + n];
#pragma unroll
                    for (int c = 0; c < MC; ++c) o[c][r] *= fr;
                }
            }
            if (masked) {
                // Rows that some queries do not see may hold anything: their
                // infinities and NaNs must not meet the zero weights (queries
                // that see such a row have it in their scores).
                const int r0 = max(lim_min - tb, 0);
                for (int i = threadIdx.x; i < (kUnit - r0) * (R / 8); i += kAttendThreads) {
                    const int r = r0 + i / (R / 8), c = i % (R / 8);
                    lat_u32x4& v = t.v[r >> 3][c >> 3][(r & 7) * 8 + (c & 7)];
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[e] = lat_finite(v[e]);
                }
                lds_barrier();
            }
            if (summer) {
                __builtin_amdgcn_sched_barrier(0);
                const lat_u32x2* base = (const lat_u32x2*)&t.v[0][0][0];
                int vp = vpos0;
                asm volatile("" : "+v"(vp));
#pragma unroll
                for (int ks = 0; ks < 2; ++ks) {
                    lat_u32x4 wf[MR], vf[MC];
#pragma unroll
                    for (int c = 0; c < MC; ++c) {
                        const int cc = MC * cw + c;
                        lat_u32x2 w[2];
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            const lat_u32x2* at = base + (2 * ks * kG + (cc >> 1)) * (2 * kWave) + (vp ^ (8 * ((MC > 1 ? c : cc) & 1) + 4 * e)) + 64 * e;
                            w[e] = __builtin_bit_cast(lat_u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lat_lds_s16x4*)at));
                        }
                        vf[c] = lat_u32x4{w[0][0], w[0][1], w[1][0], w[1][1]};
                    }
#pragma unroll
                    for (int r = 0; r < MR; ++r) wf[r] = pw[(rw * MR + r) % NR][ks][lane];
#pragma unroll
                    for (int r = 0; r < MR; ++r)
#pragma unroll
                        for (int c = 0; c < MC; ++c) o[c][r] = lat_mma(vf[c], wf[r], o[c][r]);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        };
        for (int s = 0; s < steps; s += 4) {
            step(s, st0, st3);
            if (s + 1 < steps) step(s + 1, st1, st0);
            if (s + 2 < steps) step(s + 2, st2, st1);
            if (s + 3 < steps) step(s + 3, st3, st2);
        }

        // Row sums over the four lanes of a row.
        l += __shfl_xor(l, 16);
        l = lat_sum_pair(l);
        __syncthreads();
        const size_t slot0 = ((size_t)blockIdx.x * 2 + (head ? 0 : 1)) * (32 * NR);
        if (scorer && g4 == 0) {
            const int at = 16 * wave + r16;
            sl[at] = whole ? lat_inverse(l) : 1.0f;
            if (row0 + at < rows) {
                if (!whole) *(float2*)(p.part_ml + 2 * (slot0 + at)) = make_float2(m, l);
                else if (p.lse) p.lse[(size_t)rq.t0 * p.H + row0 + at] = lat_lse(m, l);
            }
        }
        __syncthreads();
        if (summer) {
#pragma unroll
            for (int r = 0; r < MR; ++r) {
                const int at = 32 * (rw * MR + r) + n;
                if (row0 + at >= rows) continue;
                const float f = sl[at];
                float* dst = (whole ? p.o + ((size_t)rq.t0 * p.H + row0 + at) * R : p.part + (slot0 + at) * R) + 4 * hf;
#pragma unroll
                for (int c = 0; c < MC; ++c)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        *(float4*)(dst + 32 * (MC * cw + c) + 8 * i) =
                            make_float4(o[c][r][4 * i] * f, o[c][r][4 * i + 1] * f, o[c][r][4 * i + 2] * f,
                                        o[c][r][4 * i + 3] * f);
            }
        }
    }
}

// One workgroup per (token, head) row: rows whose request lies in one share
// are done; the others are the sum of their shares' partial results; rows
// that see no token are zero.  The shares' maxima and sums are read 64 at a
// time, a lane each; the partial results go over the waves in turn and the
// waves' sums are added in order.
template <int R>
__global__ __launch_bounds__(kAbsThreads) void k_join(LatentParams p, int tile_rows) {
    constexpr int V = R / kWave;              // components of a lane
    constexpr int kWaves = kAbsThreads / kWave;
    __shared__ float red[kWaves - 1][V][kWave];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const size_t at = blockIdx.x;
    const int t = (int)(at / p.H);
    float* dst = p.o + at * R + V * lane;
    const int end = p.B > 0 ? p.cu_new[p.B] : 0;
    bool none = t >= end || t < p.cu_new[0];
    int g0 = 0, g1 = 0, a = 0, rr = 0, per = 1;
    if (!none) {
        const int b = lat_find_wave(p.cu_new, p.B, t);
        const LatentReq rq = lat_req(p, b);
        const int n_u = (rq.seq + kUnit - 1) / kUnit;
        rr = (int)((long long)at - (long long)rq.t0 * p.H);
        none = n_u == 0 || t - rq.t0 >= rq.add;
        if (!none) {
            per = abs_share(p.meta[p.B]);
            a = p.meta[b] + rr / tile_rows * n_u;
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
    const size_t first = ((size_t)g0 * 2 + (a > g0 * per ? 1 : 0)) * tile_rows + rr % tile_rows;
    auto slot = [&](int g) { return g == g0 ? first : (size_t)g * 2 * tile_rows + rr % tile_rows; };
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
    constexpr int U = 8;                      // partial rows in flight per wave
    for (int g = g0 + wave; g <= g1; g += kWaves * U) {
        float w[U], x[U][V];
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const int gi = min(g + kWaves * i, g1);
            const size_t sl = slot(gi);
            w[i] = ml[sl].x;
#pragma unroll
            for (int v = 0; v < V; ++v) x[i][v] = g + kWaves * i <= g1 ? p.part[sl * R + V * lane + v] : 0.0f;
        }
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const float f = g + kWaves * i <= g1 ? __builtin_amdgcn_exp2f(w[i] - m) : 0.0f;
#pragma unroll
            for (int v = 0; v < V; ++v) sum[v] += f > 0.0f ? x[i][v] * f : 0.0f;
        }
    }
    if (wave > 0) {
#pragma unroll
        for (int v = 0; v < V; ++v) red[wave - 1][v][lane] = sum[v];
    }
    __syncthreads();
    if (wave > 0) return;
    const float inv = lat_inverse(l);
#pragma unroll
    for (int v = 0; v < V; ++v) {
        float s = sum[v];
#pragma unroll
        for (int i = 0; i < kWaves - 1; ++i) s += red[i][v][lane];
        dst[v] = s * inv;
    }
    if (p.lse && lane == 0) p.lse[at] = lat_lse(m, l);
}

// y_th for 32 tokens of one head per workgroup, W_uv rows as the M side: v /
// 32 tiles of outputs x a range of the contraction per wave, the ranges' sums
// added through LDS in order (latency bounds it, so each wave has all its
// loads in flight at once).
// The attended latents are split into two bf16 parts (value and remainder),
// which keeps them at 16 bits of mantissa for one more product per step of
// a kernel that the weights' and the latents' bytes bound.
constexpr int kUnThreads = 1024;
template <int NV>
__global__ __launch_bounds__(kUnThreads) void k_unabsorb(LatentParams p) {
    constexpr int kRanges = kUnThreads / kWave / NV;
    __shared__ float red[kRanges - 1][NV][4][kWave][4];
    const int h = blockIdx.x, t0 = blockIdx.y * 32;
    const int lane = threadIdx.x & 63, n = lane & 31, hf = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), vt = wave % NV, kr = wave / NV;
    const int t = t0 + n < p.T ? t0 + n : p.T - 1;
    const int len = p.latent / kRanges, k0 = kr * len;      // 16, 32, 64 or 128
    const float* src = p.o + ((size_t)t * p.H + h) * p.latent + 8 * hf + k0;
    const uint16_t* w = p.w_uv + ((size_t)h * p.v + 32 * vt + n) * p.latent + 8 * hf + k0;
    lat_f32x16 acc = {};
#pragma unroll 8
    for (int k = 0; k < len; k += 16) {
        const float4 a = *(const float4*)(src + k), b = *(const float4*)(src + k + 4);
        const lat_u32x4 wf = *(const lat_u32x4*)(w + k);
        const float x[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
        lat_u32x4 hi, lo;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            hi[i] = lat_pack(x[2 * i], x[2 * i + 1]);
            lo[i] = lat_pack(x[2 * i] - __uint_as_float(hi[i] << 16), x[2 * i + 1] - __uint_as_float(hi[i] & 0xFFFF0000u));
        }
        acc = lat_mma(wf, hi, acc);
        acc = lat_mma(wf, lo, acc);
    }
    if (kr > 0) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            *(float4*)red[kr - 1][vt][i][lane] = make_float4(acc[4 * i], acc[4 * i + 1], acc[4 * i + 2], acc[4 * i + 3]);
    }
    __syncthreads();
    if (kr > 0 || t0 + n >= p.T) return;
    const size_t o = ((size_t)t * p.H + h) * p.v + 32 * vt + 4 * hf;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float4 s = make_float4(acc[4 * i], acc[4 * i + 1], acc[4 * i + 2], acc[4 * i + 3]);
#pragma unroll
        for (int r = 0; r < kRanges - 1; ++r) {
            const float4 v = *(const float4*)red[r][vt][i][lane];
            s.x += v.x;
            s.y += v.y;
            s.z += v.z;
            s.w += v.w;
        }
        if (p.y_bf16) *(lat_u32x2*)((uint16_t*)p.y + o + 8 * i) = lat_u32x2{lat_pack(s.x, s.y), lat_pack(s.z, s.w)};
        else *(float4*)((float*)p.y + o + 8 * i) = s;
    }
}

template <int R>
void attend_and_join(const LatentParams& p, int row_tiles, hipStream_t s) {
    const dim3 grid(kAbsGroups), block(kAttendThreads);
    if (row_tiles == 1) hipLaunchKernelGGL((k_attend<R, 1>), grid, block, 0, s, p);
    else if (row_tiles == 2) hipLaunchKernelGGL((k_attend<R, 2>), grid, block, 0, s, p);
    else hipLaunchKernelGGL((k_attend<R, 4>), grid, block, 0, s, p);
    hipLaunchKernelGGL(k_join<R>, dim3((unsigned)((long long)p.T * p.H)), dim3(kAbsThreads), 0, s, p, 32 * row_tiles);
}

}  // namespace

hipError_t launch_latent_absorbed(const LatentParams& p, int row_tiles, hipStream_t s) {
    const unsigned tt = (unsigned)((p.T + 31) / 32);
    const dim3 grid(p.H + 1, tt, p.latent / 128), block(kAbsThreads);
    if (p.nope == 128) hipLaunchKernelGGL(k_absorb<128>, grid, block, 0, s, p, 32 * row_tiles);
    else hipLaunchKernelGGL(k_absorb<64>, grid, block, 0, s, p, 32 * row_tiles);
    if (p.latent == 512) attend_and_join<512>(p, row_tiles, s);
    else if (p.latent == 256) attend_and_join<256>(p, row_tiles, s);
    else attend_and_join<128>(p, row_tiles, s);
    if (p.v == 128) hipLaunchKernelGGL(k_unabsorb<4>, dim3(p.H, tt), dim3(kUnThreads), 0, s, p);
    else hipLaunchKernelGGL(k_unabsorb<2>, dim3(p.H, tt), dim3(kUnThreads), 0, s, p);
    return hipGetLastError();
}

}  // namespace caee
