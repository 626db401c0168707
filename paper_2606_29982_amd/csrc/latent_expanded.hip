// Latent attention, expanded form: every head's keys and values are formed
// from the cache rows first, then attended to as in ordinary attention.
//
//   k_expand   [k_nope | v] of every cached token and head = W c, rotary keys
//              copied next to them in token order (and the query tiles below)
//   k_prompt   per head and 256 query rows of one request: softmax attention
//              over its tokens, tile by tile
#include "latent.h"

namespace caee {
namespace {

constexpr int kExpandThreads = 256;
constexpr int kPromptThreads = 512;
constexpr int kKvTile = 64;            // tokens of a KV tile

// First query tile (kExpRows new tokens) of each request: meta[b].
__device__ void prompt_tiles(const LatentParams& p) {
    __shared__ int part[kExpandThreads];
    const int tid = threadIdx.x;
    const int chunk = (p.B + kExpandThreads - 1) / kExpandThreads;
    const int b0 = min(tid * chunk, p.B), b1 = min(b0 + chunk, p.B);
    int n = 0;
    for (int b = b0; b < b1; ++b) n += (lat_req(p, b).add + kExpRows - 1) / kExpRows;
    part[tid] = n;
    __syncthreads();
    for (int d = 1; d < kExpandThreads; d <<= 1) {
        const int u = tid >= d ? part[tid - d] : 0;
        __syncthreads();
        part[tid] += u;
        __syncthreads();
    }
    int at = part[tid] - n;
    for (int b = b0; b < b1; ++b) {
        p.meta[b] = at;
        at += (lat_req(p, b).add + kExpRows - 1) / kExpRows;
    }
    if (tid == kExpandThreads - 1) p.meta[p.B] = part[kExpandThreads - 1];
}

// 64 contraction elements of 128 weight rows and 128 tokens: blocks of 8
// rows x 128 bytes, piece c of row r at 8 (r % 8) + (c ^ lat_swz(r)).
struct ExpandStage {
    lat_u32x4 a[16][kWave], b[16][kWave];
};

// A product of 128 outputs (of the heads' nope + v rows, in that order) and
// 128 cached tokens per workgroup: weight rows as the M side, tokens, looked
// up in the block tables, as the N side; 2 x 2 waves of 64 x 64.
__global__ __launch_bounds__(kExpandThreads) void k_expand(LatentParams p) {
    const int ft = blockIdx.x;
    if (ft == (int)gridDim.x - 1) {
        if (blockIdx.y == 0) prompt_tiles(p);
        return;
    }
    __shared__ ExpandStage st0, st1;
    const int lane = threadIdx.x & 63, n = lane & 31, hf = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave & 1, wn = wave >> 1;
    const int total = p.B > 0 ? (int)min((long long)p.cu_kv[p.B], p.max_kv) : 0;
    const int s0 = blockIdx.y * 128;
    if (s0 >= total) return;
    const int hw = p.nope + p.v, row_bytes = p.latent + kRopeDim;
    // Cache row of token s of all requests' tokens.
    auto cache_row = [&](int s) {
        s = min(s, total - 1);
        const int b = lat_find(p.cu_kv, p.B, s);
        return p.cache + (size_t)lat_slot(p, b, s - p.cu_kv[b]) * row_bytes;
    };
    const int swz = 8 * ((lane & 7) ^ lat_swz(lane >> 3));
    const uint16_t *wsrc[4], *xsrc[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int j = ft * 128 + 32 * wave + 8 * i + (lane >> 3), h = j / hw, jj = j - h * hw;
        wsrc[i] = (jj < p.nope ? p.w_uk + ((size_t)h * p.nope + jj) * p.latent
                               : p.w_uv + ((size_t)h * p.v + jj - p.nope) * p.latent) + swz;
        xsrc[i] = cache_row(s0 + 32 * wave + 8 * i + (lane >> 3)) + swz;
    }
    if (ft == 0) {
        for (int i = threadIdx.x; i < 128 * 8; i += kExpandThreads) {
            const int s = s0 + (i >> 3);
            if (s < total)
                *(lat_u32x4*)(p.kr + (size_t)s * kRopeDim + 8 * (i & 7)) =
                    *(const lat_u32x4*)(cache_row(s) + p.latent + 8 * (i & 7));
        }
    }
    auto load = [&](int k, ExpandStage& t) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            __builtin_amdgcn_global_load_lds((lat_g_void*)(wsrc[i] + 64 * k), (lat_lds_void*)&t.a[4 * wave + i][0], 16, 0, 0);
            __builtin_amdgcn_global_load_lds((lat_g_void*)(xsrc[i] + 64 * k), (lat_lds_void*)&t.b[4 * wave + i][0], 16, 0, 0);
        }
    };
    lat_f32x16 acc[2][2] = {};
    const int steps = p.latent / 64;
    auto step = [&](int k, ExpandStage& t, ExpandStage& next) __attribute__((always_inline)) {
        lat_wait_vm<0>();
        lat_barrier();
        if (k + 1 < steps) load(k + 1, next);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int at = (n & 7) * 8 + ((2 * j + hf) ^ lat_swz(n));
            lat_u32x4 a[2], b[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                a[i] = t.a[8 * wm + 4 * i + (n >> 3)][at];
                b[i] = t.b[8 * wn + 4 * i + (n >> 3)][at];
            }
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int e = 0; e < 2; ++e) acc[i][e] = lat_mma(a[i], b[e], acc[i][e]);
        }
    };
    load(0, st0);
    for (int k = 0; k < steps; k += 2) {
        step(k, st0, st1);
        step(k + 1, st1, st0);      // latent is a multiple of 128
    }
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        const int s = s0 + 64 * wn + 32 * e + n;
        if (s >= total) continue;
        uint16_t* dst = p.kv + (size_t)s * p.H * hw + ft * 128 + 64 * wm + 4 * hf;
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const lat_u32x2 v = {lat_pack(acc[i][e][4 * q], acc[i][e][4 * q + 1]),
                                     lat_pack(acc[i][e][4 * q + 2], acc[i][e][4 * q + 3])};
                *(lat_u32x2*)(dst + 32 * i + 8 * q) = v;
            }
    }
}

// One KV tile of a head: keys (nope groups, then the rotary one) and values,
// blocks of 8 tokens x 128 bytes as above.
template <int NOPE, int V>
struct PromptTile {
    static constexpr int kGk = NOPE / 64 + 1, kGv = V / 64;
    lat_u32x4 k[kKvTile / 8][kGk][kWave];
    lat_u32x4 v[kKvTile / 8][kGv][kWave];
};

template <int NOPE, int V>
__global__ __launch_bounds__(kPromptThreads) void k_prompt(LatentParams p, int tiles) {
    using Tile = PromptTile<NOPE, V>;
    constexpr int kGk = Tile::kGk, kGv = Tile::kGv;
    constexpr int kJ = 4 * kGk, NC = V / 32;
    constexpr int kLoads = kGk + kGv;          // loads of a wave per tile: one block of 8 tokens
    __shared__ Tile st0, st1, st2;
    const int lane = threadIdx.x & 63, n = lane & 31, hf = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // Workgroups go to the XCDs round robin: all tiles of a head run on one
    // XCD, whose L2 holds the head's keys and values; the last tiles, which
    // see the most tokens, first.
    int h, q;
    if (p.H % kXcds == 0) {
        const int k = blockIdx.x / kXcds;
        h = blockIdx.x % kXcds + kXcds * (k / tiles);
        q = k % tiles;
    } else {
        h = blockIdx.x / tiles;
        q = blockIdx.x % tiles;
    }
    const int tile = p.meta[p.B] - 1 - q;
    if (tile < 0) return;
    const int b = lat_find(p.meta, p.B, tile);
    const LatentReq rq = lat_req(p, b);
    const int row0 = (tile - p.meta[b]) * kExpRows;
    const int kv0 = p.cu_kv[b];
    auto sees = [&](int r) { return p.causal ? min(max(rq.seq - rq.add + r + 1, 0), rq.seq) : rq.seq; };
    const int my0 = row0 + 32 * wave;
    const int row = min(my0 + n, rq.add - 1);
    const int limit = sees(row);
    const int lim_min = sees(min(my0, rq.add - 1)), lim_max = sees(min(my0 + 31, rq.add - 1));
    const int lim_wg = sees(row0);
    const int end = sees(min(row0 + kExpRows, rq.add) - 1);
    const int steps = (end + kKvTile - 1) / kKvTile;
    const int t = rq.t0 + row;

    lat_u32x4 qf[kJ];
    const uint16_t* qrow = p.q + (size_t)t * p.q_stride + (size_t)h * (NOPE + kRopeDim) + 8 * hf;
#pragma unroll
    for (int j = 0; j < kJ; ++j) qf[j] = *(const lat_u32x4*)(qrow + 16 * j);
    lat_f32x16 o[NC];
#pragma unroll
    for (int c = 0; c < NC; ++c) o[c] = lat_f32x16{};
    float m = kNoScore, l = 0.0f;

    int kpos[4], vpos[2];
#pragma unroll
    for (int j = 0; j < 4; ++j) kpos[j] = (n >> 3) * (kGk * kWave) + (n & 7) * 8 + ((2 * j + hf) ^ lat_swz(n));
    const int vrow = 4 * hf + ((lane & 15) >> 2);
#pragma unroll
    for (int j = 0; j < 2; ++j)
        vpos[j] = 2 * (vrow * 8 + ((4 * j + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) ^ lat_swz(vrow))) + (lane & 1);

    const int swz = 8 * ((lane & 7) ^ lat_swz(lane >> 3));
    const size_t kv_row = (size_t)p.H * (NOPE + V);
    auto load = [&](int s, Tile& d) __attribute__((always_inline)) {
        const int tok = min(s * kKvTile + 8 * wave + (lane >> 3), rq.seq - 1);
        const long long at = min((long long)kv0 + tok, p.max_kv - 1);
        const uint16_t* src = p.kv + (size_t)at * kv_row + (size_t)h * (NOPE + V) + swz;
#pragma unroll
        for (int g = 0; g < NOPE / 64; ++g)
            __builtin_amdgcn_global_load_lds((lat_g_void*)(src + 64 * g), (lat_lds_void*)&d.k[wave][g][0], 16, 0, 0);
        __builtin_amdgcn_global_load_lds((lat_g_void*)(p.kr + (size_t)at * kRopeDim + swz),
                                         (lat_lds_void*)&d.k[wave][kGk - 1][0], 16, 0, 0);
#pragma unroll
        for (int g = 0; g < kGv; ++g)
            __builtin_amdgcn_global_load_lds((lat_g_void*)(src + NOPE + 64 * g), (lat_lds_void*)&d.v[wave][g][0], 16, 0, 0);
    };
    auto step = [&](int s, Tile& d, Tile& next) __attribute__((always_inline)) {
        const int tb = s * kKvTile;
        // The loads of one later tile may stay in flight; the barrier says that
        // the tile is whole and that nobody reads the stage `next` fills.
        if (s + 1 < steps) lat_wait_vm<kLoads>();
        else lat_wait_vm<0>();
        lat_barrier();
        if (s + 2 < steps) load(s + 2, next);
        if (tb + kKvTile > lim_wg) {
            // Tokens that some rows do not see may hold anything: infinities
            // and NaNs must not meet their zero weights (rows that see such
            // a token have it in their scores).
            const int r0 = max(lim_wg - tb, 0);
            for (int i = threadIdx.x; i < (kKvTile - r0) * (V / 8); i += kPromptThreads) {
                const int r = r0 + i / (V / 8), c = i % (V / 8);
                lat_u32x4& v = d.v[r >> 3][c >> 3][(r & 7) * 8 + (c & 7)];
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = lat_finite(v[e]);
            }
            __builtin_amdgcn_s_waitcnt(15 | (7 << 4) | (0 << 8) | (3 << 14));
            lat_barrier();
        }
        if (tb >= lim_max || my0 >= rq.add) return;    // this wave's rows see none of it
        lat_f32x16 sc[2] = {};
#pragma unroll
        for (int j = 0; j < kJ; ++j)
#pragma unroll
            for (int e = 0; e < 2; ++e)
                sc[e] = lat_mma((&d.k[0][0][0])[kpos[j % 4] + (4 * e * kGk + j / 4) * kWave], qf[j], sc[e]);
        const bool masked = tb + kKvTile > lim_min;
        float mt = -INFINITY;
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                sc[e][i] *= p.scale_log2;
                if (masked && tb + 32 * e + 8 * (i >> 2) + 4 * hf + (i & 3) >= limit) sc[e][i] = -INFINITY;
                mt = fmaxf(mt, sc[e][i]);
            }
        mt = lat_max_pair(mt);
        if (__any(mt > m + kMaxSlack)) {
            const float mn = fmaxf(m, mt), f = __builtin_amdgcn_exp2f(m - mn);
            l *= f;
            m = mn;
#pragma unroll
            for (int c = 0; c < NC; ++c) o[c] *= f;
        }
        lat_u32x4 pf[4];
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float a = __builtin_amdgcn_exp2f(sc[k >> 1][8 * (k & 1) + 2 * i] - m);
                const float e = __builtin_amdgcn_exp2f(sc[k >> 1][8 * (k & 1) + 2 * i + 1] - m);
                l += a + e;
                pf[k][i] = lat_pack(a, e);
            }
        const lat_u32x2* base = (const lat_u32x2*)&d.v[0][0][0];
#pragma unroll
        for (int ks = 0; ks < 4; ++ks)
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                lat_u32x2 w[2];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const lat_u32x2* at = base + ((2 * ks + e) * kGv + (c >> 1)) * (2 * kWave) + vpos[c & 1];
                    w[e] = __builtin_bit_cast(lat_u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lat_lds_s16x4*)at));
                }
                const lat_u32x4 a = {w[0][0], w[0][1], w[1][0], w[1][1]};
                o[c] = lat_mma(a, pf[ks], o[c]);
            }
    };
    if (steps > 0) load(0, st0);
    if (steps > 1) load(1, st1);
    for (int s = 0; s < steps; s += 3) {
        step(s, st0, st2);
        if (s + 1 < steps) step(s + 1, st1, st0);
        if (s + 2 < steps) step(s + 2, st2, st1);
    }

    l = lat_sum_pair(l);
    if (my0 + n >= rq.add) return;
    const float f = lat_inverse(l);
    const size_t at = (size_t)t * p.H + h;
    if (p.lse && hf == 0) p.lse[at] = lat_lse(m, l);
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const size_t y = at * V + 32 * c + 8 * i + 4 * hf;
            const float v0 = o[c][4 * i] * f, v1 = o[c][4 * i + 1] * f, v2 = o[c][4 * i + 2] * f, v3 = o[c][4 * i + 3] * f;
            if (p.y_bf16) {
                const lat_u32x2 v = {lat_pack(v0, v1), lat_pack(v2, v3)};
                *(lat_u32x2*)((uint16_t*)p.y + y) = v;
            } else {
                *(float4*)((float*)p.y + y) = make_float4(v0, v1, v2, v3);
            }
        }
}

// Rows of no request (padding) are zero, their lse -inf.
__global__ __launch_bounds__(256) void k_blank_rows(LatentParams p) {
    const int end = p.B > 0 ? min(max(p.cu_new[p.B], 0), p.T) : 0;
    const long long words = (long long)p.H * p.v * (p.y_bf16 ? 2 : 4) / 16;
    const long long n = (p.T - end) * words;
    const lat_u32x4 zero = {0, 0, 0, 0};
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < n; i += (long long)gridDim.x * 256)
        ((lat_u32x4*)p.y)[end * words + i] = zero;
    if (p.lse)
        for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < (long long)(p.T - end) * p.H;
             i += (long long)gridDim.x * 256)
            p.lse[(long long)end * p.H + i] = -INFINITY;
}

template <int NOPE>
void prompt(const LatentParams& p, unsigned grid, int tiles, hipStream_t s) {
    if (p.v == 128) hipLaunchKernelGGL((k_prompt<NOPE, 128>), dim3(grid), dim3(kPromptThreads), 0, s, p, tiles);
    else hipLaunchKernelGGL((k_prompt<NOPE, 64>), dim3(grid), dim3(kPromptThreads), 0, s, p, tiles);
}

}  // namespace

hipError_t launch_latent_expanded(const LatentParams& p, hipStream_t s) {
    const unsigned ft = (unsigned)((long long)p.H * (p.nope + p.v) / 128);
    const unsigned st = (unsigned)((p.max_kv + 127) / 128);
    hipLaunchKernelGGL(k_expand, dim3(ft + 1, st > 0 ? st : 1), dim3(kExpandThreads), 0, s, p);
    hipLaunchKernelGGL(k_blank_rows, dim3(64), dim3(256), 0, s, p);
    long long tiles = (long long)p.B * ((p.max_new + kExpRows - 1) / kExpRows);
    if (tiles > p.T / kExpRows + p.B) tiles = p.T / kExpRows + p.B;
    if (tiles > 0) {
        const unsigned grid = (unsigned)(tiles * p.H);
        if (p.nope == 128) prompt<128>(p, grid, (int)tiles, s);
        else prompt<64>(p, grid, (int)tiles, s);
    }
    return hipGetLastError();
}

}  // namespace caee
