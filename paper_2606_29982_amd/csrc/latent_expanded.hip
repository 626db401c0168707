// Latent attention, expanded form: every head's keys and values are formed
// from the cache rows first, then attended to as in ordinary attention.
//
//   k_expand   [k_nope | v] of every cached token and head = W c, rotary keys
//              copied next to them in token order (and the query tiles below;
//              rows of no request are zeroed)
//   k_prompt   per head and 256 query rows of one request: softmax attention
//              over its tokens, tile by tile
#include "latent.h"

namespace caee {
namespace {

constexpr int kExpandThreads = 512;
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

// Rows of no request (padding) are zero, their lse -inf; `groups` workgroups.
__device__ void blank_rows(const LatentParams& p, int group, int groups) {
    const int end = p.B > 0 ? min(max(p.cu_new[p.B], 0), p.T) : 0;
    const long long words = (long long)p.H * p.v * (p.y_bf16 ? 2 : 4) / 16, n = (p.T - end) * words;
    const long long first = (long long)group * kExpandThreads + threadIdx.x, by = (long long)groups * kExpandThreads;
    const lat_u32x4 zero = {0, 0, 0, 0};
    for (long long i = first; i < n; i += by) ((lat_u32x4*)p.y)[end * words + i] = zero;
    if (p.lse)
        for (long long i = first; i < (long long)(p.T - end) * p.H; i += by) p.lse[(long long)end * p.H + i] = -INFINITY;
}

// 64 contraction elements of 256 weight rows and 256 tokens: blocks of 8
// rows x 128 bytes, piece c of row r at 8 (r % 8) + (c ^ lat_swz(r)).
constexpr int kExpandTile = 256;
struct ExpandStage {
    lat_u32x4 a[kExpandTile / 8][kWave], b[kExpandTile / 8][kWave];
};

// A product of 256 outputs (of the heads' nope + v rows, in that order) and
// 256 cached tokens per workgroup: weight rows as the M side, tokens, looked
// up in the block tables, as the N side; 2 x 4 waves of 128 x 64.  Two stages,
// the next one's loads between the first half of a stage's MFMAs; workgroups
// that run together share weight tiles by XCD (they are numbered weights
// first) and the outputs leave through LDS, 512 bytes of a token at a time.
// 8191 tokens of 64 heads take 183 us, 0.75 PFLOP/s (100 us of products at the
// rate of a large one): bound by the fetches into LDS, 173 us without the
// products, 159 without the outputs, which pass the caches by (kept there: 201).
// Neither 128 x 128 tiles with outputs straight from the registers (264 us) nor
// 128 x 256 ones of half the depth, two workgroups a CU and a third stage (212)
// are faster.
__global__ __launch_bounds__(kExpandThreads) void k_expand(LatentParams p) {
#if defined(__HIP_DEVICE_COMPILE__)   // the buffer-descriptor type exists for the GPU target only
    const int ft = blockIdx.x;
    constexpr int kWaves = kExpandThreads / kWave, kBlocks = kExpandTile / 8 / kWaves;     // blocks of 8 rows a wave fetches
    __shared__ ExpandStage st0, st1;
    const int lane = threadIdx.x & 63, n = lane & 31, hf = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave & 1, wn = wave >> 1;
    const int total = p.B > 0 ? (int)min((long long)p.cu_kv[p.B], p.max_kv) : 0;
    // Cache row of token s of all requests' tokens.
    auto cache_row = [&](int s) {
        s = min(s, total - 1);
        const int b = lat_find(p.cu_kv, p.B, s);
        return lat_slot(p, b, s - p.cu_kv[b]);
    };
    if (blockIdx.y == gridDim.y - 1) {
        if (ft == 0) prompt_tiles(p);
        blank_rows(p, ft, gridDim.x);
        // The rotary keys, 8 lanes a token.
        for (int i0 = ft * kExpandThreads; i0 < total * 8; i0 += gridDim.x * kExpandThreads) {
            const int s = (i0 + (int)threadIdx.x) >> 3, q8 = threadIdx.x & 7;
            if (s < total)
                *(lat_u32x4*)(p.kr + (size_t)s * kRopeDim + 8 * q8) =
                    *(const lat_u32x4*)(p.cache + (size_t)cache_row(s) * (p.latent + kRopeDim) + p.latent + 8 * q8);
        }
        return;
    }
    const int s0 = blockIdx.y * kExpandTile;
    if (s0 >= total) return;
    const int hw = p.nope + p.v, outs = p.H * hw, row_bytes = (p.latent + kRopeDim) * 2;
    // Buffer loads (the compiler counts the LDS reads apart from them).  Eight
    // weight rows lie in one head's keys or values.  A token's row is a 32-bit
    // offset where the cache has at most 4 GiB, else rows go one by one, each
    // with a descriptor of its own.
    const bool near = (unsigned long long)p.n_blocks * p.block * row_bytes < 0xFFFFFFFFull;
    const char* wbase[kBlocks];
    uint32_t xrow[kBlocks];
#pragma unroll
    for (int i = 0; i < kBlocks; ++i) {
        const int r = 8 * (kBlocks * wave + i);
        const int j = min(ft * kExpandTile + r, outs - 8), h = j / hw, jj = j - h * hw;
        wbase[i] = (const char*)(jj < p.nope ? p.w_uk + ((size_t)h * p.nope + jj) * p.latent
                                             : p.w_uv + ((size_t)h * p.v + jj - p.nope) * p.latent);
        xrow[i] = cache_row(s0 + r + (lane >> 3));
    }
    auto piece = [&](int i) { return 16u * ((lane & 7) ^ lat_swz(8 * i + (lane >> 3))); };     // kBlocks is even
    // Load i of a wave's part of stage k: weight blocks, then token blocks.
    auto load = [&](int k, int i, ExpandStage& t) __attribute__((always_inline)) {
        if (i < kBlocks) {
            const __amdgpu_buffer_rsrc_t buf = __builtin_amdgcn_make_buffer_rsrc((void*)wbase[i], 0, kLatBufBytes, kLatBufWord3);
            __builtin_amdgcn_raw_ptr_buffer_load_lds(buf, (lat_lds_void*)&t.a[kBlocks * wave + i][0], 16,
                                                     (uint32_t)(lane >> 3) * (uint32_t)(p.latent * 2) + piece(i), 128 * k, 0, 0);
        } else {
            const int e = i - kBlocks;
            const __amdgpu_buffer_rsrc_t buf = __builtin_amdgcn_make_buffer_rsrc((void*)p.cache, 0, -1, kLatBufWord3);
            __builtin_amdgcn_raw_ptr_buffer_load_lds(buf, (lat_lds_void*)&t.b[kBlocks * wave + e][0], 16,
                                                     xrow[e] * (uint32_t)row_bytes + piece(e), 128 * k, 0, 0);
        }
    };
    auto load_far = [&](int k, ExpandStage& t) __attribute__((always_inline)) {
#pragma unroll
        for (int e = 0; e < kBlocks; ++e) {
#pragma unroll 1
            for (int r = 0; r < 8; ++r) {
                const uint32_t row = __builtin_amdgcn_readlane(xrow[e], 8 * r);
                const __amdgpu_buffer_rsrc_t buf = __builtin_amdgcn_make_buffer_rsrc(
                    (void*)((const char*)p.cache + (size_t)row * (uint32_t)row_bytes), 0, kLatBufBytes, kLatBufWord3);
                if (lane >> 3 == r)
                    __builtin_amdgcn_raw_ptr_buffer_load_lds(buf, (lat_lds_void*)&t.b[kBlocks * wave + e][0], 16, piece(e),
                                                             128 * k, 0, 0);
            }
        }
    };
    lat_f32x16 acc[4][2] = {};
    const int steps = p.latent / 64;
    auto step = [&](int k, ExpandStage& t, ExpandStage& next) __attribute__((always_inline)) {
        lat_wait_vm<0>();                  // this wave's part of the stage is there; after the barrier all of it is,
        lat_barrier();                     // and nobody reads the other
        const bool more = k + 1 < steps;
        if (more && !near) load_far(k + 1, next);
        const int loads = !more ? 0 : near ? 2 * kBlocks : kBlocks;
        auto a_at = [&](int j, int i) __attribute__((always_inline)) {
            return t.a[16 * wm + 4 * i + (n >> 3)][(n & 7) * 8 + ((2 * j + hf) ^ lat_swz(n))];
        };
        auto b_at = [&](int j, int i) __attribute__((always_inline)) {
            return t.b[8 * wn + 4 * i + (n >> 3)][(n & 7) * 8 + ((2 * j + hf) ^ lat_swz(n))];
        };
        lat_u32x4 a[2][4], b[2][2];
        auto fetch = [&](int j) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < 2; ++i) b[j & 1][i] = b_at(j, i);
#pragma unroll
            for (int i = 0; i < 4; ++i) a[j & 1][i] = a_at(j, i);
        };
        __builtin_amdgcn_sched_barrier(0);
        fetch(0);
        lat_for<0, 4>([&](auto jc) __attribute__((always_inline)) {
            constexpr int j = decltype(jc)::value;
            if constexpr (j < 3) fetch(j + 1);
            lat_for<0, 8>([&](auto ic) __attribute__((always_inline)) {
                constexpr int i = decltype(ic)::value, op = 8 * j + i;
                acc[i >> 1][i & 1] = lat_mma(a[j & 1][i >> 1], b[j & 1][i & 1], acc[i >> 1][i & 1]);
                if constexpr (op % 2 == 1 && op / 2 < 2 * kBlocks) {
                    if (op / 2 < loads) load(k + 1, op / 2, next);
                }
                __builtin_amdgcn_sched_barrier(0);
            });
        });
    };
    for (int i = 0; i < (near ? 2 * kBlocks : kBlocks); ++i) load(0, i, st0);
    if (!near) load_far(0, st0);
    for (int k = 0; k < steps; k += 2) {
        step(k, st0, st1);
        step(k + 1, st1, st0);      // latent is a multiple of 128
    }
    // The tile's tokens, 512 bytes each, half in either stage; piece c of token
    // r at c ^ (r % 32).
    __syncthreads();
    lat_u32x4* const half = wn < 2 ? &st0.a[0][0] : &st1.a[0][0];
#pragma unroll
    for (int e = 0; e < 2; ++e)
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                lat_u32x2* at = (lat_u32x2*)&half[(64 * (wn & 1) + 32 * e + n) * 32 + ((16 * wm + 4 * i + q) ^ n)];
                at[hf] = lat_u32x2{lat_pack(acc[i][e][4 * q], acc[i][e][4 * q + 1]),
                                   lat_pack(acc[i][e][4 * q + 2], acc[i][e][4 * q + 3])};
            }
    __syncthreads();
    const int c8 = threadIdx.x & 31, out = ft * kExpandTile + 8 * c8;
    if (out >= outs) return;
    uint16_t* dst = p.kv + (size_t)s0 * outs + out;
    constexpr int kRows = kExpandThreads / 32;
#pragma unroll
    for (int i = 0; i < kExpandTile / kRows; i += 4) {
        lat_u32x4 v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int r = kRows * (i + e) + (threadIdx.x >> 5);
            v[e] = (r < 128 ? &st0.a[0][0] : &st1.a[0][0])[(r & 127) * 32 + (c8 ^ (r & 31))];
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int r = kRows * (i + e) + (threadIdx.x >> 5);
            if (s0 + r < total) __builtin_nontemporal_store(v[e], (lat_u32x4*)(dst + (size_t)r * outs));
        }
    }
#endif
}

// One tile of a head's keys (nope groups, then the rotary one) or values: G
// groups of 128 bytes of 64 tokens, blocks of 8 tokens x 128 bytes as above.
template <int G>
struct PromptTile {
    lat_u32x4 v[kKvTile / 8][G][kWave];
};
// The query rows of W waves, 32 each, in the same blocks.
template <int G, int W>
struct QueryRows {
    lat_u32x4 v[4 * W][G][kWave];
};

// Softmax attention of 256 query rows of one head, 32 a wave, over 64-token
// tiles: keys as the M side, so that a lane holds a row's scores, whose weights
// are, in that order, a fragment of the second product, without a trip through
// LDS.  Bound by the matrix units at the clock that power leaves them (40 MFMAs
// of 32 x 32 x 16 a step and wave, 59 % of the cycles): 7161 tokens behind 1030,
// 64 heads, take 1.2 ms among other calls, 1.1 PFLOP/s (1.36 in a trace).  Short prompts are bound by their longest
// tile (2.7 us a step): eight of up to 700 tokens, 16 heads, 33 us.
// Keys, values and weights are bf16, the cache's type (the result's error is
// 0.0028 of its size, rms, of which rounding the result to bf16 is 0.0017).
template <int NOPE, int V>
__global__ __launch_bounds__(kPromptThreads) void k_prompt(LatentParams p, int tiles) {
#if defined(__HIP_DEVICE_COMPILE__)   // the buffer-descriptor type exists for the GPU target only
    constexpr int kGk = NOPE / 64 + 1, kGv = V / 64;
    using Keys = PromptTile<kGk>;
    using Values = PromptTile<kGv>;
    constexpr int kJ = 4 * kGk, NC = V / 32;
    constexpr int kAhead = 5;                  // fragments read from LDS ahead of their MFMAs
    constexpr int kLoads = kGk + kGv;          // loads of a wave per tile: one block of 8 tokens
    // An object per stage: the compiler can tell the reads of one from the
    // loads that fill another.
    __shared__ Keys kt0, kt1, kt2;
    __shared__ Values vt0, vt1, vt2;
    constexpr int kExtra = V == 128 ? 2 : 4;   // waves whose queries no free stage holds
    __shared__ QueryRows<kGk, kExtra> extra;
    const int lane = threadIdx.x & 63, n = lane & 31, hf = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // Workgroups go to the XCDs round robin: all tiles of a head run on one
    // XCD, whose L2 holds the head's keys and values, where the heads divide
    // evenly (64 heads, 7161 tokens behind 1030: 1312 us; in plain order, as with
    // other numbers of heads, 1486; 16 heads, short prompts: 32 and 49); the last
    // tiles, which see the most tokens, first.
    const int wg = (int)lat_workgroup();
    int h, q;
    if (p.H % kXcds == 0) {
        const int k = wg / kXcds;
        h = wg % kXcds + kXcds * (k / tiles);
        q = k % tiles;
    } else {
        h = wg / tiles;
        q = wg % tiles;
    }
    if (h >= p.H) return;      // the last line of a long grid
    const int tile = p.meta[p.B] - 1 - q;
    if (tile < 0) return;
    const int b = lat_find_wave(p.meta, p.B, tile);
    const LatentReq rq = lat_req(p, b);
    const int row0 = (tile - p.meta[b]) * kExpRows;
    const int kv0 = p.cu_kv[b];
    auto sees = [&](int r) { return lat_sees(p, rq, r); };
    const int my0 = row0 + 32 * wave;
    const int row = min(my0 + n, rq.add - 1);
    const int limit = sees(row);
    const int lim_min = sees(min(my0, rq.add - 1)), lim_wg = sees(row0);
    const int end = sees(min(row0 + kExpRows, rq.add) - 1);
    const int steps = (end + kKvTile - 1) / kKvTile;
    const int t = rq.t0 + row;

    // A wave's queries, as its results at the end, go through a part of LDS of
    // its own, eight lanes a 128-byte line: straight from memory a lane's 16
    // bytes are a line of their own, 64 cycles a load (34.4 us where this takes
    // 32.4, eight prompts of up to 700 tokens, 16 heads).  The stages of
    // tile 0, fetched meanwhile, are left out.
    lat_u32x4* const own = wave < 2                ? &kt1.v[4 * wave][0][0]
                           : wave < 4              ? &kt2.v[4 * (wave - 2)][0][0]
                           : wave < 4 + kExtra     ? &extra.v[4 * (wave - 4)][0][0]
                           : wave == 6             ? &vt1.v[0][0][0]
                                                   : &vt2.v[0][0][0];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = 8 * i + (lane >> 3);
        const uint16_t* src = p.q + (size_t)(rq.t0 + min(my0 + r, rq.add - 1)) * p.q_stride +
                              (size_t)h * (NOPE + kRopeDim) + 8 * ((lane & 7) ^ lat_swz(r));
#pragma unroll
        for (int g = 0; g < kGk; ++g)
            __builtin_amdgcn_global_load_lds((lat_g_void*)(src + 64 * g), (lat_lds_void*)(own + (kGk * i + g) * kWave), 16, 0, 0);
    }
    lat_u32x4 qf[kJ];
    lat_f32x16 o[NC];
#pragma unroll
    for (int c = 0; c < NC; ++c) o[c] = lat_f32x16{};
    float m = kNoScore, l = 0.0f;

    int kpos[4], vpos[2][2];       // [piece], [column tile parity][eight of a 16-token step]
#pragma unroll
    for (int j = 0; j < 4; ++j) kpos[j] = (n >> 3) * (kGk * kWave) + (n & 7) * 8 + ((2 * j + hf) ^ lat_swz(n));
    const int vrow = 4 * hf + ((lane & 15) >> 2);
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int e = 0; e < 2; ++e)
            vpos[j][e] = 2 * (vrow * 8 + ((4 * j + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) ^ lat_swz(8 * e + vrow))) + (lane & 1);

    // A wave fetches 8 tokens of a tile: descriptors begin at the tile's first
    // row (uniform), lanes at piece lane % 8 (swizzled) of row lane / 8.
    // (Buffer loads: the compiler counts the LDS reads apart from them.)
    const uint32_t kv_row = (uint32_t)p.H * (NOPE + V) * 2u;
    const int swz = 16 * ((lane & 7) ^ lat_swz(8 * wave + (lane >> 3)));
    struct Source {
        const char *kv, *kr;      // uniform: the tile's first row (this head's part), its rotary row
        uint32_t row;             // this lane's row
    };
    const char* kv_head = (const char*)p.kv + (size_t)h * (NOPE + V) * 2;
    auto source = [&](int s) __attribute__((always_inline)) {
        const int first = (int)min((long long)kv0 + s * kKvTile, p.max_kv - 1);
        const int most = min(rq.seq - 1 - s * kKvTile, (int)p.max_kv - 1 - first);
        return Source{kv_head + (size_t)first * kv_row, (const char*)p.kr + (size_t)first * (kRopeDim * 2),
                      (uint32_t)max(min(8 * wave + (lane >> 3), most), 0)};
    };
    // Load i of the wave's part of a tile: the groups of the keys (the rotary
    // one last), then of the values.
    auto load = [&](auto ic, const Source& from, Keys& k, Values& v) __attribute__((always_inline)) {
        constexpr int i = decltype(ic)::value;
        const char* base = i == kGk - 1 ? from.kr : from.kv;
        const __amdgpu_buffer_rsrc_t buf = __builtin_amdgcn_make_buffer_rsrc((void*)base, 0, kLatBufBytes, kLatBufWord3);
        if constexpr (i == kGk - 1) {
            __builtin_amdgcn_raw_ptr_buffer_load_lds(buf, (lat_lds_void*)&k.v[wave][i][0], 16,
                                                     from.row * (kRopeDim * 2) + swz, 0, 0, 0);
        } else if constexpr (i < kGk - 1) {
            __builtin_amdgcn_raw_ptr_buffer_load_lds(buf, (lat_lds_void*)&k.v[wave][i][0], 16, from.row * kv_row + swz,
                                                     128 * i, 0, 0);
        } else {
            __builtin_amdgcn_raw_ptr_buffer_load_lds(buf, (lat_lds_void*)&v.v[wave][i - kGk][0], 16,
                                                     from.row * kv_row + swz, 128 * (i - 1), 0, 0);
        }
    };
    // Step s has two phases: X multiplies the keys of tile s and sums the
    // values of tile s - 1 (40 MFMAs at 128 + 64, 128), Y makes the weights of
    // tile s (exponentials) and starts loads.  The two waves of a SIMD take
    // turns: waves 4 .. 7 run one barrier behind waves 0 .. 3, so that one is in
    // X while the other is in Y.  Keys of tile s are read in phases 2 s (waves
    // 0 .. 3) and 2 s + 1 (4 .. 7), values in 2 s + 2 and 2 s + 3; so in Y(s) the
    // first waves, in phase 2 s + 1, may load the keys of tile s + 2 and the
    // values of tile s + 1 into rings of three, the others, in phase 2 s + 2,
    // those of one tile more.  At the end of the odd phases (Y of the first
    // waves, X of the others) a wave waits for all but its latest step's loads:
    // what the next phase reads is then there.  Past the last tile the loads
    // read it again, for nobody.  (The loads among the MFMAs of X instead: 1645
    // us where this takes 1448, a prompt of 7161 tokens behind 1030, 64 heads.)
    const bool second = wave >= 4;
    // Tokens that some rows do not see may hold anything: infinities and NaNs
    // must not meet their zero weights, so a wave clears them from the values
    // that it loaded, before the barrier that publishes them (rows that see
    // such a token have it in their scores).
    auto clear = [&](int s, Values& d) __attribute__((always_inline)) {
        if (s >= steps || (s + 1) * kKvTile <= lim_wg) return;
        if (s * kKvTile + 8 * wave + (lane >> 3) >= lim_wg) {
#pragma unroll
            for (int g = 0; g < kGv; ++g) {
                lat_u32x4 v = d.v[wave][g][lane];
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = lat_finite(v[e]);
                d.v[wave][g][lane] = v;
            }
        }
        __builtin_amdgcn_s_waitcnt(15 | (7 << 4) | (0 << 8) | (3 << 14));
    };
    auto odd_end = [&](int s, Values& values) __attribute__((always_inline)) {
        lat_wait_vm<kLoads>();
        asm volatile("" ::: "memory");
        clear(s, values);
    };
    lat_u32x4 pf[4] = {};          // weights of the tile before
    lat_f32x16 sc[2];
    // X's MFMAs, 2 kJ of the scores and 4 NC of the sums, evenly mixed (two
    // chains of sums alone would wait for each other), their fragments read
    // kAhead before they are used.
    constexpr int kOps = 2 * kJ + 4 * NC;
    auto sums_before = [](int i) constexpr { return i * (4 * NC) / kOps; };
    auto value = [&](const Values& d, int i) __attribute__((always_inline)) {
        const lat_u32x2* base = (const lat_u32x2*)&d.v[0][0][0];
        const int ks = i / NC, c = i % NC;
        lat_u32x2 w[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const lat_u32x2* at = base + ((2 * ks + e) * kGv + (c >> 1)) * (2 * kWave) + vpos[c & 1][e];
            w[e] = __builtin_bit_cast(lat_u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lat_lds_s16x4*)at));
        }
        return lat_u32x4{w[0][0], w[0][1], w[1][0], w[1][1]};
    };
    auto load_tiles = [&](const Source& from_k, const Source& from_v, Keys& k, Values& v) __attribute__((always_inline)) {
        lat_for<0, kLoads>([&](auto ic) __attribute__((always_inline)) {
            load(ic, decltype(ic)::value < kGk ? from_k : from_v, k, v);
        });
    };
    // k, k2: the keys of tile s (their stage then takes those of tile s + 3)
    // and the stage for those of tile s + 2; v0, v1, v2: the values of tiles
    // s - 1 (their stage then takes those of tile s + 2) and s and the stage
    // for those of tile s + 1.
    auto step = [&](int s, Keys& k, Keys& k2, Values& v0, Values& v1, Values& v2) __attribute__((always_inline)) {
        const int tb = s * kKvTile;
        const lat_u32x4* keys = &k.v[0][0][0];
        auto fetch = [&](auto ic) __attribute__((always_inline)) {
            constexpr int i = decltype(ic)::value, v = sums_before(i);
            if constexpr (sums_before(i + 1) > v) {
                return value(v0, v);
            } else {
                constexpr int j = (i - v) >> 1, e = (i - v) & 1;
                return keys[kpos[j % 4] + (4 * e * kGk + j / 4) * kWave];
            }
        };
        __builtin_amdgcn_sched_barrier(0);
        lat_u32x4 fr[kAhead];
        sc[0] = sc[1] = lat_f32x16{};
        lat_for<0, kAhead>([&](auto ic) __attribute__((always_inline)) { fr[decltype(ic)::value] = fetch(ic); });
        lat_for<0, kOps>([&](auto ic) __attribute__((always_inline)) {
            constexpr int i = decltype(ic)::value, v = sums_before(i), j = i - v;
            if constexpr (sums_before(i + 1) > v) o[v % NC] = lat_mma(fr[i % kAhead], pf[v / NC], o[v % NC]);
            else sc[j & 1] = lat_mma(fr[i % kAhead], qf[j >> 1], sc[j & 1]);
            if constexpr (i + kAhead < kOps) fr[i % kAhead] = fetch(LatInt<i + kAhead>{});
            __builtin_amdgcn_sched_barrier(0);
        });
        if (second) odd_end(s, v1);
        lat_barrier();
        const int more_k = second ? 3 : 2;
        const Source from_k = source(min(s + more_k, steps - 1)), from_v = source(min(s + more_k - 1, steps - 1));
        if (second) load_tiles(from_k, from_v, k, v0);
        else load_tiles(from_k, from_v, k2, v2);
        if (tb + kKvTile > lim_min) {
            asm volatile("");       // a branch, not 32 selects in every step
#pragma unroll
            for (int e = 0; e < 2; ++e)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (tb + 32 * e + 8 * (i >> 2) + 4 * hf + (i & 3) >= limit) sc[e][i] = -INFINITY;
        }
        // The weights by the running maximum; where one exceeds the slack the
        // maximum moves and they are made again.
        float big = 0.0f, more = 0.0f;
        auto weights = [&]() __attribute__((always_inline)) {
#pragma unroll
            for (int k = 0; k < 4; ++k)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float a = lat_weight(sc[k >> 1][8 * (k & 1) + 2 * i], p.scale_log2, m);
                    const float e = lat_weight(sc[k >> 1][8 * (k & 1) + 2 * i + 1], p.scale_log2, m);
                    big = fmaxf(fmaxf(big, a), e);
                    pf[k][i] = lat_pack(a, e);
                    more = lat_sum2(pf[k][i], more);
                }
        };
        weights();
        if (__any(big > kMaxWeight)) {
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
            weights();
        }
        l += more;
        if (!second) odd_end(s, v1);
        lat_barrier();
    };
    if (steps > 0) {
        // Tile 0, the keys of tile 1 (and what the second waves' Y(-1) would
        // have loaded); the values of "tile -1" are zeros.
        const Source from0 = source(0), from1 = source(min(1, steps - 1)), from2 = source(min(2, steps - 1));
        load_tiles(from0, from0, kt0, vt0);
        lat_wait_vm<kLoads>();
        asm volatile("" ::: "memory");
#pragma unroll
        for (int j = 0; j < kJ; ++j)
            qf[j] = own[((n >> 3) * kGk + (j >> 2)) * kWave + (n & 7) * 8 + ((2 * (j & 3) + hf) ^ lat_swz(n))];
        __builtin_amdgcn_s_waitcnt(15 | (7 << 4) | (0 << 8) | (3 << 14));
        lat_barrier();             // the stages the queries came through are free
        lat_for<0, kGk>([&](auto ic) __attribute__((always_inline)) { load(ic, from1, kt1, vt1); });
        if (second) load_tiles(from2, from1, kt2, vt1);
#pragma unroll
        for (int g = 0; g < kGv; ++g) vt2.v[wave][g][lane] = lat_u32x4{0, 0, 0, 0};
        // Tile 0 is there; the keys of tile 1 are waited for at the end of phase 1.
        if (second) lat_wait_vm<kGk + kLoads>();
        else lat_wait_vm<kGk>();
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
        auto finish = [&](const Values& d) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < 4 * NC; ++i) o[i % NC] = lat_mma(value(d, i), pf[i / NC], o[i % NC]);
        };
        const int at = (steps - 1) % 3;
        if (at == 0) finish(vt0);
        else if (at == 1) finish(vt1);
        else finish(vt2);
    }

    lat_wait_vm<0>();
    lat_barrier();             // nobody's loads are on their way into the stages any more
    l = lat_sum_pair(l);
    const float f = lat_inverse(l);
    if (p.lse && hf == 0 && my0 + n < rq.add) p.lse[(size_t)t * p.H + h] = lat_lse(m, l);
    // 8 KiB a wave: 256 bytes of a row at a time, unit u (16 bytes) of a row at
    // u ^ (row % units).
    lat_u32x4* const out = wave < 6 ? (lat_u32x4*)(wave < 2 ? &kt0 : wave < 4 ? &kt1 : &kt2) + 512 * (wave & 1)
                                    : (lat_u32x4*)&extra + 512 * (wave - 6);
    auto leave = [&](auto bytes_of) __attribute__((always_inline)) {
        constexpr int kSize = decltype(bytes_of)::value, kUnits = V * kSize < 256 ? V * kSize / 16 : 16;
        constexpr int kPasses = V * kSize / (16 * kUnits), kTiles = NC / kPasses;
#pragma unroll
        for (int pass = 0; pass < kPasses; ++pass) {
#pragma unroll
            for (int c = 0; c < kTiles; ++c)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const lat_f32x16& v = o[kTiles * pass + c];
                    const float v0 = v[4 * i] * f, v1 = v[4 * i + 1] * f, v2 = v[4 * i + 2] * f, v3 = v[4 * i + 3] * f;
                    const int unit = kSize == 2 ? 4 * c + i : 8 * c + 2 * i + hf;
                    lat_u32x4* const at = out + n * kUnits + (unit ^ (n & (kUnits - 1)));
                    if constexpr (kSize == 2) ((lat_u32x2*)at)[hf] = lat_u32x2{lat_pack(v0, v1), lat_pack(v2, v3)};
                    else *at = lat_u32x4{__float_as_uint(v0), __float_as_uint(v1), __float_as_uint(v2), __float_as_uint(v3)};
                }
            __builtin_amdgcn_s_waitcnt(15 | (7 << 4) | (0 << 8) | (3 << 14));
            asm volatile("" ::: "memory");
#pragma unroll
            for (int i = 0; i < kUnits / 2; ++i) {
                const int r = (64 * i + lane) / kUnits, u = (64 * i + lane) % kUnits;
                const lat_u32x4 v = out[r * kUnits + (u ^ (r & (kUnits - 1)))];
                if (my0 + r < rq.add)
                    *(lat_u32x4*)((char*)p.y + ((size_t)(rq.t0 + my0 + r) * p.H + h) * (V * kSize) + 256 * pass + 16 * u) = v;
            }
            __builtin_amdgcn_s_waitcnt(15 | (7 << 4) | (0 << 8) | (3 << 14));
            asm volatile("" ::: "memory");
        }
    };
    if (p.y_bf16) leave(LatInt<2>{});
    else leave(LatInt<4>{});
#endif
}

template <int NOPE>
void prompt(const LatentParams& p, unsigned grid, int tiles, hipStream_t s) {
    if (p.v == 128) hipLaunchKernelGGL((k_prompt<NOPE, 128>), lat_grid(grid), dim3(kPromptThreads), 0, s, p, tiles);
    else hipLaunchKernelGGL((k_prompt<NOPE, 64>), lat_grid(grid), dim3(kPromptThreads), 0, s, p, tiles);
}

}  // namespace

hipError_t launch_latent_expanded(const LatentParams& p, hipStream_t s) {
    const unsigned ft = (unsigned)(((long long)p.H * (p.nope + p.v) + kExpandTile - 1) / kExpandTile);
    const unsigned st = (unsigned)((p.max_kv + kExpandTile - 1) / kExpandTile);
    hipLaunchKernelGGL(k_expand, dim3(ft, st + 1), dim3(kExpandThreads), 0, s, p);
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
