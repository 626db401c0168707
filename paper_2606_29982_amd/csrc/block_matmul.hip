// y = x W^T with e4m3 weights and activations and fp32 scales: one per
// 128 x 128 weight block, one per activation row and 128-deep block
// (caee_block_matmul).
//
// Per 128-deep block the code products are summed by scaled MFMAs with unit
// E8M0 scales; the block's sum times (weight scale x row scale) is added in
// fp32.  The 8-bit MFMAs keep about 16 bits of such a sum (measured: relative
// error 1.4e-5 of 128 products, the same for all their shapes), which a bf16
// result does not show.  Where it would show, the codes are converted to
// bf16, which holds them exactly, and multiplied by the bf16 MFMAs at half the
// rate (kExact): fp32 results, and contractions of up to 256, where the error
// has no further blocks to average over and the output's bytes are the cost.
#include "caee_internal.h"
#include "fp8_codec.h"

#include <math.h>

#include <type_traits>

namespace caee {
namespace {

typedef uint32_t bm_u32x4 __attribute__((ext_vector_type(4)));
typedef int bm_i32x8 __attribute__((ext_vector_type(8)));
typedef float bm_f32x4 __attribute__((ext_vector_type(4)));
typedef float bm_f32x16 __attribute__((ext_vector_type(16)));
typedef float bm_f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bm_bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bm_bf16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t bm_u32x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) void bm_lds_void;

constexpr int kBmMaxK = 65536;
constexpr int kBmMaxStride = 1 << 22;  // elements from row to row of x: 256 rows stay within 2^32 bytes
constexpr int kBmBufBytes = 0x7FFFFFFF, kBmBufWord3 = 0x00020000;   // buffer descriptor: size, raw 32-bit access
// Row tiles of a band of k_bm_many's tile order (8000 x 7168, K = 4096, calls back to back: 2 303 us, 4 297,
// 8 298, 16 303, one band 310; 3000 x 7168, K = 7168: 219, 214, 214, 220, 216).
constexpr int kBmBand = 8;
constexpr int kUnitScale = 127;       // E8M0 1.0

struct BmParams {
    int M, N, K, kb;                  // kb: 128-deep blocks
    const void* x;                    // bf16 or fp32 rows (quantised first)
    const uint8_t* xq;                // e4m3 rows, xq_stride bytes apart
    const float* xs;                  // [M][kb]
    const uint8_t* w;
    const float* ws;                  // [ceil(N / 128)][kb]
    void* y;
    long long x_stride, xq_stride, y_stride;
    int tiled, y_bf16, vec;           // vec: four consecutive outputs are stored together
    uint8_t* xq_out;
    float* xs_out;
};

__device__ inline bm_i32x8 bm_join(const bm_u32x4& a, const bm_u32x4& b) {
    return bm_i32x8{(int)a[0], (int)a[1], (int)a[2], (int)a[3], (int)b[0], (int)b[1], (int)b[2], (int)b[3]};
}

template <int N>
using BmInt = std::integral_constant<int, N>;
// f(BmInt<B>{}), ..., f(BmInt<E - 1>{}).
template <int B, int E, class F>
__device__ __attribute__((always_inline)) inline void bm_for(F&& f) {
    if constexpr (B < E) {
        f(BmInt<B>{});
        bm_for<B + 1, E>(f);
    }
}

__device__ inline uint32_t bm_pack(float a, float b) {
    const bm_f32x2 t = {a, b};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(t, bm_bf16x2));
}

// Eight codes (two words) as bf16.
__device__ inline bm_bf16x8 bm_wide(uint32_t lo, uint32_t hi) {
    const bm_bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, false);
    const bm_bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, true);
    const bm_bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, false);
    const bm_bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, true);
    return bm_bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// Outputs n .. n + 3 of row m.
__device__ inline void bm_store4(const BmParams& p, int m, int n, float a, float b, float c, float d) {
    const size_t o = (size_t)m * p.y_stride + n;
    const float v[4] = {a, b, c, d};
    if (p.vec && n + 3 < p.N) {
        if (p.y_bf16) *(bm_u32x2*)((uint16_t*)p.y + o) = bm_u32x2{bm_pack(a, b), bm_pack(c, d)};
        else *(float4*)((float*)p.y + o) = make_float4(a, b, c, d);
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (n + i >= p.N) continue;
        if (p.y_bf16) ((uint16_t*)p.y)[o + i] = (uint16_t)bm_pack(v[i], v[i]);
        else ((float*)p.y)[o + i] = v[i];
    }
}

// Rows of x to codes and block scales, as caee_quantize_rows but rows
// x_stride apart.
template <class T>
__global__ __launch_bounds__(256) void k_bm_quant(BmParams p) {
    const int l = threadIdx.x & (kQuantLanes - 1);
    const long long n = (long long)p.M * p.kb;
    const long long step = (long long)gridDim.x * (256 / kQuantLanes);
    for (long long i = (long long)blockIdx.x * (256 / kQuantLanes) + threadIdx.x / kQuantLanes; i < n; i += step) {
        const int m = (int)(i / p.kb), b = (int)(i - (long long)m * p.kb);
        float v[8];
        load8((const T*)p.x + (size_t)m * p.x_stride + 128 * b + 8 * l, v);
        const float sc = quant_block(v, p.xq_out + (size_t)m * p.K + 128 * b, l);
        if (l == 0) p.xs_out[i] = sc;
    }
}

// Bytes from a 128-deep block of a weight row to the next.
__device__ inline int bm_block(const BmParams& p) { return p.tiled ? 2048 : 128; }

// Blocks of 8 rows x 128 bytes in LDS have piece c of row r at
// 8 (r % 8) + (c ^ bm_swz(r)): 16 rows' reads of a piece hit all 64 banks.
__device__ inline int bm_swz(int r) { return (r >> 1) & 7; }

// Few outputs: 32 T x 32 T outputs and rows per workgroup, its waves a range
// of the contraction's blocks each, so that small products fill the chip too.
// A wave keeps its own two stages in LDS (no barriers), one filled by direct
// loads while the other is multiplied; the waves' sums are added through LDS
// in wave order.  Bound by the weights of few rows (5 rows, 4096 outputs, K =
// 7168: 7.3 us, 4.0 TB/s), else by the lines a CU's requests take: eight lanes
// read one, 16 cycles a load.  (Straight to registers a lane's 16-byte piece is
// a line of its own, 64 cycles a load: 8 and 20 us for 5 and 131 rows x 576
// outputs, K = 7168, 57 for 512 x 2048, K = 4096, where this takes 6, 10, 14.)
template <int T, int WAVES>
struct BmSplitStage {
    bm_u32x4 w[WAVES][4 * T][kWave], x[WAVES][4 * T][kWave];
};
template <int T, int WAVES, bool kExact>
__global__ __launch_bounds__(WAVES * 64, 2) void k_bm_split(BmParams p) {
#if defined(__HIP_DEVICE_COMPILE__)   // the buffer-descriptor type exists for the GPU target only
    using Stage = BmSplitStage<T, WAVES>;
    __shared__ Stage st0, st1;
    constexpr int kTile = 32 * T;
    const int lane = threadIdx.x & 63, n = lane & 31, hf = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n0 = blockIdx.x * kTile, m0 = blockIdx.y * kTile;
    const int b0 = (int)((long long)p.kb * wave / WAVES), b1 = (int)((long long)p.kb * (wave + 1) / WAVES);
    // Tiled weights have 8 rows' pieces c next to each other: block slots
    // 8 (c ^ (r / 8) % 2) + r % 8 keep lanes and lines together.
    const size_t first = p.tiled ? (size_t)(n0 >> 4) * (p.K / 64) * 1024 : (size_t)n0 * p.K;
    const __amdgpu_buffer_rsrc_t wbuf =
        __builtin_amdgcn_make_buffer_rsrc((void*)(p.w + first), 0, kBmBufBytes, kBmBufWord3);
    const __amdgpu_buffer_rsrc_t xbuf =
        __builtin_amdgcn_make_buffer_rsrc((void*)(p.xq + (size_t)m0 * p.xq_stride), 0, kBmBufBytes, kBmBufWord3);
    uint32_t woff[4 * T], xoff[4 * T];
#pragma unroll
    for (int i = 0; i < 4 * T; ++i) {
        const int r = 8 * i + (lane >> 3), c = (lane & 7) ^ bm_swz(r);
        xoff[i] = (uint32_t)min(r, p.M - 1 - m0) * (uint32_t)p.xq_stride + 16u * c;
        const int wr = min(p.tiled ? 8 * i + (lane & 7) : r, p.N - 1 - n0), wc = p.tiled ? (lane >> 3) ^ (i & 1) : c;
        woff[i] = p.tiled ? (uint32_t)((wr >> 4) * (p.K / 64) * 1024 + (wc >> 2) * 1024 + ((wr & 15) + 16 * (wc & 3)) * 16)
                          : (uint32_t)(wr * p.K + 16 * wc);
    }
    const float* xs[T];
#pragma unroll
    for (int e = 0; e < T; ++e) xs[e] = p.xs + (size_t)min(m0 + 32 * e + n, p.M - 1) * p.kb;
    // (an address of the lane's own, so that this is a vector load and counts as one)
    int zero_lane = 0;
    asm volatile("" : "+v"(zero_lane));
    const float* wsc = p.ws + (size_t)(n0 >> 7) * p.kb + zero_lane;
    const int wstep = bm_block(p);
    // A fragment's pieces 2 q + hf of row n: at xat ^ 2 q and wat ^ wq q.
    const int xat = (n >> 3) * kWave + 8 * (n & 7) + (hf ^ bm_swz(n));
    const int wat = p.tiled ? (n >> 3) * kWave + 8 * (hf ^ ((n >> 3) & 1)) + (n & 7) : xat, wq = p.tiled ? 16 : 2;
    struct Scales {
        float x[T], w;
    } c0, c1;
    auto fetch = [&](Stage& t, Scales& c, int b) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 4 * T; ++i) {
            __builtin_amdgcn_raw_ptr_buffer_load_lds(wbuf, (bm_lds_void*)&t.w[wave][i][0], 16, woff[i], b * wstep, 0, 0);
            __builtin_amdgcn_raw_ptr_buffer_load_lds(xbuf, (bm_lds_void*)&t.x[wave][i][0], 16, xoff[i], b * 128, 0, 0);
        }
#pragma unroll
        for (int e = 0; e < T; ++e) c.x[e] = xs[e][b];
        c.w = wsc[b];
        __builtin_amdgcn_sched_barrier(0);
    };
    bm_f32x16 acc[T][T] = {};
    const bm_f32x16 zero = {};
    // `later`: another stage's loads were issued after this one's.
    auto mul = [&](Stage& t, const Scales& c, auto later) __attribute__((always_inline)) {
        constexpr int kLater = decltype(later)::value ? 9 * T + 1 : 0;
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_waitcnt((kLater & 15) | (7 << 4) | (15 << 8) | ((kLater >> 4) << 14));
        asm volatile("" ::: "memory");
        bm_u32x4 w[T][4], x[T][4];
#pragma unroll
        for (int i = 0; i < T; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                w[i][q] = (&t.w[wave][4 * i][0])[wat ^ (wq * q)];
                x[i][q] = (&t.x[wave][4 * i][0])[xat ^ (2 * q)];
            }
#pragma unroll
        for (int i = 0; i < T; ++i)
#pragma unroll
            for (int e = 0; e < T; ++e) {
                bm_f32x16 s = zero;
                if constexpr (kExact) {
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(bm_wide(w[i][q][0], w[i][q][1]),
                                                                    bm_wide(x[e][q][0], x[e][q][1]), s, 0, 0, 0);
                        s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(bm_wide(w[i][q][2], w[i][q][3]),
                                                                    bm_wide(x[e][q][2], x[e][q][3]), s, 0, 0, 0);
                    }
                } else {
#pragma unroll
                    for (int q = 0; q < 4; q += 2)
                        s = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(bm_join(w[i][q], w[i][q + 1]),
                                                                            bm_join(x[e][q], x[e][q + 1]), s, 0, 0, 0,
                                                                            kUnitScale, 0, kUnitScale);
                }
                const float f = c.w * c.x[e];
#pragma unroll
                for (int v = 0; v < 16; ++v) acc[i][e][v] += s[v] * f;
            }
        // The stage's reads are over before it is filled again.
        __builtin_amdgcn_s_waitcnt(15 | (7 << 4) | (0 << 8) | (3 << 14));
        asm volatile("" ::: "memory");
    };
    if (b0 < b1) {
        fetch(st0, c0, b0);
        int b = b0;
        for (; b + 2 < b1; b += 2) {
            fetch(st1, c1, b + 1);
            mul(st0, c0, BmInt<1>{});
            fetch(st0, c0, b + 2);
            mul(st1, c1, BmInt<1>{});
        }
        if (b + 1 < b1) {
            fetch(st1, c1, b + 1);
            mul(st0, c0, BmInt<1>{});
            mul(st1, c1, BmInt<0>{});
        } else {
            mul(st0, c0, BmInt<0>{});
        }
    }
    __syncthreads();
    float4* const red = (float4*)&st0;          // [wave][tile][eight outputs][lane]
    auto place = [](int wv, int tile, int q, int ln) { return ((wv * T * T + tile) * 4 + q) * kWave + ln; };
#pragma unroll
    for (int i = 0; i < T; ++i)
#pragma unroll
        for (int e = 0; e < T; ++e)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                red[place(wave, T * i + e, q, lane)] = make_float4(acc[i][e][4 * q], acc[i][e][4 * q + 1],
                                                                   acc[i][e][4 * q + 2], acc[i][e][4 * q + 3]);
    __syncthreads();
    // Four outputs of a row a thread, 8 T threads a row.
    for (int j = threadIdx.x; j < 256 * T * T; j += WAVES * 64) {
        const int row = j / (8 * T), c = j % (8 * T), e = row >> 5, i = c >> 3, q = (c & 7) >> 1, from = (row & 31) + 32 * (c & 1);
        float4 s = red[place(0, T * i + e, q, from)];
#pragma unroll
        for (int v = 1; v < WAVES; ++v) {
            const float4 x = red[place(v, T * i + e, q, from)];
            s.x += x.x;
            s.y += x.y;
            s.z += x.z;
            s.w += x.w;
        }
        if (m0 + row < p.M) bm_store4(p, m0 + row, n0 + 4 * c, s.x, s.y, s.z, s.w);
    }
#endif
}

// Many rows: 256 outputs x 32 NT rows per workgroup, a 128-deep
// block per stage, both operands two stages ahead.  Each of the 8 waves owns
// 32 outputs, whose codes go straight to its registers (three sets in turn);
// the rows' codes and scales go global -> LDS directly into a ring of three
// and every wave reads all of them.  (Both operands through LDS leave room for
// two stages only, and one stage of lookahead does not cover a fetch: 345 us
// for 8000 rows, K = 4096, N = 7168, of which the loads alone take 244.)
template <int NT>
struct BmStage {
    bm_u32x4 b[4 * NT][kWave];
    float xs[8][kWave];
};
struct BmCodes {
    bm_u32x4 v[4];        // pieces hf, 2 + hf, 4 + hf, 6 + hf of a block of this lane's weight row
};

template <int NT, bool kExact>
__global__ __launch_bounds__(512) void k_bm_many(BmParams p, int n_tiles, int m_tiles) {
#if defined(__HIP_DEVICE_COMPILE__)   // the buffer-descriptor type exists for the GPU target only
    using Stage = BmStage<NT>;
    __shared__ Stage st0, st1, st2;
    __shared__ float wscale[2][kBmMaxK / 128];
    const int lane = threadIdx.x & 63, n = lane & 31, hf = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // Workgroups go to the XCDs round robin; each XCD takes a contiguous run
    // of tiles, ordered by bands of kBmBand row tiles, so that the about 32
    // that run there at a time share few rows and few outputs in its L2.
    const int total = n_tiles * m_tiles, run = (total + kXcds - 1) / kXcds;
    const int id = blockIdx.x % kXcds * run + blockIdx.x / kXcds;
    if ((int)blockIdx.x / kXcds >= run || id >= total) return;
    const int band = id / (kBmBand * n_tiles), high = min(kBmBand, m_tiles - band * kBmBand);
    const int in_band = id - band * kBmBand * n_tiles;
    const int n0 = in_band / high * 256, m0 = (band * kBmBand + in_band % high) * (32 * NT);
    // Sources: buffers that begin at the workgroup's first row, 32-bit
    // offsets of this lane's rows (clamped to the last; 256 rows span less
    // than 2^31 bytes) and a uniform offset that moves with the block.
    const uint8_t* wbase = p.w + (p.tiled ? (size_t)(n0 >> 4) * (p.K / 64) * 1024 : (size_t)n0 * p.K);
    const uint8_t* xbase = p.xq + (size_t)m0 * p.xq_stride;
    const __amdgpu_buffer_rsrc_t wbuf = __builtin_amdgcn_make_buffer_rsrc((void*)wbase, 0, kBmBufBytes, kBmBufWord3);
    const __amdgpu_buffer_rsrc_t xbuf = __builtin_amdgcn_make_buffer_rsrc((void*)xbase, 0, kBmBufBytes, kBmBufWord3);
    const __amdgpu_buffer_rsrc_t sbuf =
        __builtin_amdgcn_make_buffer_rsrc((void*)(p.xs + (size_t)m0 * p.kb), 0, kBmBufBytes, kBmBufWord3);
    const int wr = min(32 * wave + n, p.N - 1 - n0);
    uint32_t aoff = p.tiled ? (uint32_t)((wr >> 4) * (p.K / 64) * 1024 + ((wr & 15) + 16 * hf) * 16)
                            : (uint32_t)(wr * p.K + 16 * hf);
    const int half_step = p.tiled ? 1024 : 64, pair_step = p.tiled ? 512 : 32;    // pieces + 4, + 2
    constexpr int kBLoads = (NT + 1) / 2;      // row blocks a wave fetches per stage (odd NT: the last ones twice)
    uint32_t boff[kBLoads];
#pragma unroll
    for (int i = 0; i < kBLoads; ++i) {
        const int blk = min(kBLoads * wave + i, 4 * NT - 1), rr = 8 * blk + (lane >> 3), c = (lane & 7) ^ bm_swz(rr);
        boff[i] = (uint32_t)min(rr, p.M - 1 - m0) * (uint32_t)p.xq_stride + 16u * c;
        asm volatile("" : "+v"(boff[i]));       // one register from here on
    }
    asm volatile("" : "+v"(aoff));
    // Row scales: wave w loads rows 32 w .. + 31 (lanes 32 .. 63 repeat them).
    const uint32_t xsoff = (uint32_t)min(32 * (wave % NT) + n, p.M - 1 - m0) * (uint32_t)p.kb * 4u;
    const int wstep = bm_block(p);
    constexpr int kLoads = 4 + kBLoads + 1;
    // Load i of this wave's share of a stage.
    auto load = [&](auto ic, int k, Stage& t, BmCodes& w) __attribute__((always_inline)) {
        constexpr int i = decltype(ic)::value;
        if constexpr (i < 4) {
            w.v[i] = __builtin_bit_cast(bm_u32x4, __builtin_amdgcn_raw_buffer_load_b128(
                wbuf, aoff, k * wstep + (i >> 1) * half_step + (i & 1) * pair_step, 0));
        } else if constexpr (i < 4 + kBLoads) {
            __builtin_amdgcn_raw_ptr_buffer_load_lds(xbuf, (bm_lds_void*)&t.b[min(kBLoads * wave + i - 4, 4 * NT - 1)][0], 16, boff[i - 4], k * 128, 0, 0);
        } else {
            __builtin_amdgcn_raw_ptr_buffer_load_lds(sbuf, (bm_lds_void*)&t.xs[wave][0], 4, xsoff, k * 4, 0, 0);
        }
    };
    // This lane's fragments of a 32-row tile: row n, pieces 2 q + hf of a
    // block, at base ^ 2 q.
    const int base = (n >> 3) * kWave + (n & 7) * 8 + (hf ^ bm_swz(n));
    bm_f32x16 acc[NT] = {};
    const bm_f32x16 zero = {};
    const int wrow = (32 * wave) >> 7;
    auto step = [&](int k, Stage& t, const BmCodes& w, Stage& tn, BmCodes& wn) __attribute__((always_inline)) {
        // All but the next stage's loads have landed; after the barrier
        // everybody's have, and nobody reads the stage `tn` any more.
        __builtin_amdgcn_s_waitcnt((kLoads & 15) | (7 << 4) | (15 << 8) | ((kLoads >> 4) << 14));
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        const int ahead = min(k + 2, p.kb - 1);     // past the end the last block again, read by nobody
        const float ws = wscale[wrow][k];
        int at[4];
        at[0] = base;
        asm volatile("" : "+v"(at[0]));     // the other three are made in the step, not kept through the loop
#pragma unroll
        for (int q = 1; q < 4; ++q) at[q] = at[0] ^ (2 * q);
        auto rows = [&](int i, int q) __attribute__((always_inline)) { return t.b[4 * i][at[q]]; };
        auto scale = [&](int i) __attribute__((always_inline)) { return t.xs[i][n]; };
        auto add = [&](bm_f32x16& c, const bm_f32x16& q, float f) __attribute__((always_inline)) {
#pragma unroll
            for (int v = 0; v < 16; ++v) c[v] += q[v] * f;
        };
        if constexpr (kExact) {
            bm_bf16x8 a[8];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                a[2 * q] = bm_wide(w.v[q][0], w.v[q][1]);
                a[2 * q + 1] = bm_wide(w.v[q][2], w.v[q][3]);
            }
            bm_for<0, NT>([&](auto ic) __attribute__((always_inline)) {
                constexpr int i = decltype(ic)::value;
                bm_f32x16 s = zero;
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const bm_u32x4 v = rows(i, q);
                    s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[2 * q], bm_wide(v[0], v[1]), s, 0, 0, 0);
                    s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[2 * q + 1], bm_wide(v[2], v[3]), s, 0, 0, 0);
                }
                bm_for<i * kLoads / NT, (i + 1) * kLoads / NT>(
                    [&](auto lc) __attribute__((always_inline)) { load(lc, ahead, tn, wn); });
                add(acc[i], s, scale(i) * ws);
                __builtin_amdgcn_sched_barrier(0);
            });
        } else {
            // Tile by tile: the next tile's rows are read and one of the loads
            // of the stage after next issued while this one is multiplied
            // (a CU takes only so many requests at a time, and a wave waits at
            // a load that is not taken).
            const bm_i32x8 a0 = bm_join(w.v[0], w.v[1]), a1 = bm_join(w.v[2], w.v[3]);
            bm_u32x4 bq[2][4];
            float f[2];
#pragma unroll
            for (int q = 0; q < 4; ++q) bq[0][q] = rows(0, q);
            f[0] = scale(0);
            bm_for<0, NT>([&](auto ic) __attribute__((always_inline)) {
                constexpr int i = decltype(ic)::value;
                bm_f32x16 q = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a0, bm_join(bq[i & 1][0], bq[i & 1][1]), zero,
                                                                             0, 0, 0, kUnitScale, 0, kUnitScale);
                q = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a1, bm_join(bq[i & 1][2], bq[i & 1][3]), q, 0, 0, 0,
                                                                    kUnitScale, 0, kUnitScale);
                if constexpr (i + 1 < NT) {
#pragma unroll
                    for (int v = 0; v < 4; ++v) bq[(i + 1) & 1][v] = rows(i + 1, v);
                    f[(i + 1) & 1] = scale(i + 1);
                }
                bm_for<i * kLoads / NT, (i + 1) * kLoads / NT>(
                    [&](auto lc) __attribute__((always_inline)) { load(lc, ahead, tn, wn); });
                add(acc[i], q, f[i & 1] * ws);
                __builtin_amdgcn_sched_barrier(0);
            });
        }
    };
    BmCodes w0, w1, w2;
    bm_for<0, kLoads>([&](auto ic) __attribute__((always_inline)) { load(ic, 0, st0, w0); });
    bm_for<0, kLoads>([&](auto ic) __attribute__((always_inline)) { load(ic, min(1, p.kb - 1), st1, w1); });
    for (int i = threadIdx.x; i < 2 * p.kb; i += 512) {
        const int h = i / p.kb;
        wscale[h][i - h * p.kb] = p.ws[(size_t)min((n0 >> 7) + h, (p.N - 1) >> 7) * p.kb + i - h * p.kb];
    }
    __syncthreads();
    for (int k = 0; k < p.kb; k += 3) {
        step(k, st0, w0, st2, w2);
        if (k + 1 < p.kb) step(k + 1, st1, w1, st0, w0);
        if (k + 2 < p.kb) step(k + 2, st2, w2, st1, w1);
    }
    __builtin_amdgcn_s_waitcnt((0) | (7 << 4) | (15 << 8));      // the last blocks' second readings have landed
#pragma unroll
    for (int e = 0; e < NT; ++e) {
        int m = m0 + 32 * e + n;
        asm volatile("" : "+v"(m));     // keeps the address arithmetic here, out of the stage loop
        if (m >= p.M) continue;
#pragma unroll
        for (int q = 0; q < 4; ++q)
            bm_store4(p, m, n0 + 32 * wave + 8 * q + 4 * hf, acc[e][4 * q], acc[e][4 * q + 1], acc[e][4 * q + 2],
                      acc[e][4 * q + 3]);
    }
#endif
}

size_t up256(size_t n) { return (n + 255) & ~(size_t)255; }

size_t bm_ws(const caee_block_matmul_desc_t& d) {
    if (d.x_dtype == CAEE_FP8_E4M3) return 0;
    return up256((size_t)d.M * d.K) + up256((size_t)d.M * (d.K / 128) * 4);
}

caee_status_t check_bm(const caee_block_matmul_desc_t* d) {
    if (!d) return fail(CAEE_ERR_INVALID_ARG, "desc is NULL");
    if (d->M < 0) return fail(CAEE_ERR_INVALID_ARG, "M=%d must be >= 0", d->M);
    if (d->N < 1) return fail(CAEE_ERR_INVALID_ARG, "N=%d must be >= 1", d->N);
    if (d->K < 128 || d->K % 128) return fail(CAEE_ERR_INVALID_ARG, "K=%d must be a positive multiple of 128", d->K);
    if (d->x_dtype != CAEE_F32 && d->x_dtype != CAEE_BF16 && d->x_dtype != CAEE_FP8_E4M3)
        return fail(CAEE_ERR_INVALID_ARG, "unknown x_dtype=%d", d->x_dtype);
    if (d->y_dtype != CAEE_F32 && d->y_dtype != CAEE_BF16)
        return fail(CAEE_ERR_INVALID_ARG, "y_dtype=%d must be CAEE_F32 or CAEE_BF16", d->y_dtype);
    if (d->layout != CAEE_LAYOUT_ROWMAJOR && d->layout != CAEE_LAYOUT_TILED)
        return fail(CAEE_ERR_INVALID_ARG, "unknown weight layout=%d", d->layout);
    if (d->layout == CAEE_LAYOUT_TILED && d->N % 16)
        return fail(CAEE_ERR_INVALID_ARG, "N=%d must be a multiple of 16 for tiled weights", d->N);
    if (d->x_stride < d->K || d->x_stride * elem_bytes(d->x_dtype) % 16)
        return fail(CAEE_ERR_INVALID_ARG, "x_stride=%lld must be >= K=%d and keep rows 16-byte aligned",
                    (long long)d->x_stride, d->K);
    if (d->y_stride < d->N) return fail(CAEE_ERR_INVALID_ARG, "y_stride=%lld must be >= N=%d", (long long)d->y_stride, d->N);
    // Limits of this build.
    if (d->x_stride > kBmMaxStride)
        return fail(CAEE_ERR_UNSUPPORTED, "x_stride=%lld exceeds %d", (long long)d->x_stride, kBmMaxStride);
    if (d->K > kBmMaxK || d->M > (1 << 24) || d->N > (1 << 24))
        return fail(CAEE_ERR_UNSUPPORTED, "M=%d, N=%d or K=%d exceeds %d, %d, %d", d->M, d->N, d->K, 1 << 24, 1 << 24,
                    kBmMaxK);
    return CAEE_OK;
}

constexpr int kBmExactK = 256;
constexpr int kBmCus = 256;            // CUs of the chip, one workgroup of k_bm_many each at a time

// Row tiles per workgroup: the height whose whole rounds of the chip's CUs
// take the least (8000 rows x 7168 outputs: 4 rounds of 8, 4 of 7, 5 of 6).
int bm_height(const BmParams& p) {
    int best = 8;
    long long least = 0;
    for (int nt = 8; nt >= 4; --nt) {
        const long long tiles = (long long)((p.M + 32 * nt - 1) / (32 * nt)) * ((p.N + 255) / 256);
        const long long cost = (tiles + kBmCus - 1) / kBmCus * (nt + 1);     // a workgroup's fixed part: about a tile row
        if (least == 0 || cost < least) {
            least = cost;
            best = nt;
        }
    }
    return best;
}

template <int NT, bool kExact>
void launch_many(const BmParams& p, hipStream_t s) {
    const int n_tiles = (p.N + 255) / 256, m_tiles = (p.M + 32 * NT - 1) / (32 * NT);
    const unsigned grid = (unsigned)((n_tiles * m_tiles + kXcds - 1) / kXcds * kXcds);
    hipLaunchKernelGGL((k_bm_many<NT, kExact>), dim3(grid), dim3(512), 0, s, p, n_tiles, m_tiles);
}

// By the number of 64 x 64 tiles, in rounds of the CUs.  Up to half a round 32 x
// 32 tiles, which make two of them, are about as fast or faster (K = 4096, 32 and
// 64, us: 5 x 4096 7 and 10 of K = 7168, 256 x 2048 10.5 and 10.8, 64 x 7168 12.5
// and 10.8; fp32 results 11.8 and 13.3, 13.2 and 13.6; past it 1024 x 576 16.2 and
// 13.9, 128 x 7168 20.9 and 11.9).  k_bm_many takes K / 128 + 2 steps for any
// product of one round of its own and then gains; its steps are 0.85 us, with the
// bf16 MFMAs of kExact 1.5.  64 x 64 tiles and k_bm_many, m x 4096:
//                    2 rounds (m = 512)   3 (m = 768)   4 (m = 1024)
//   bf16,  K =  512     9.7 and  9.7      13.3    9.9   17.4   10.3
//          K = 2048    15.0     17.8      21.3   18.1   28.1   18.7
//          K = 7168    35.3     51.4      51.1   51.6   66.7   52.1
//   exact, K =  512    10.7     13.1      15.1   13.7   19.3   14.5
//          K = 2048    18.2     31.2      25.9   32.0   33.1   32.7
//          K = 7168    44.5     93.0      63.6   93.7   82.1   94.1
template <bool kExact>
hipError_t launch_bm(const BmParams& p, hipStream_t s) {
    const long long nt = (p.N + 63) / 64, mt = (p.M + 63) / 64, tiles = nt * mt;
    if (tiles <= kBmCus / 2) {
        const dim3 grid((p.N + 31) / 32, (p.M + 31) / 32);
        hipLaunchKernelGGL((k_bm_split<1, 8, kExact>), grid, dim3(512), 0, s, p);
    } else if (tiles <= (!kExact ? 2 : p.K < 2048 ? 3 : 4) * kBmCus) {
        hipLaunchKernelGGL((k_bm_split<2, 4, kExact>), dim3((unsigned)nt, (unsigned)mt), dim3(256), 0, s, p);
    } else if constexpr (kExact) {
        launch_many<4, true>(p, s);
    } else {
        switch (bm_height(p)) {
            case 4: launch_many<4, false>(p, s); break;
            case 5: launch_many<5, false>(p, s); break;
            case 6: launch_many<6, false>(p, s); break;
            case 7: launch_many<7, false>(p, s); break;
            default: launch_many<8, false>(p, s); break;
        }
    }
    return hipGetLastError();
}

}  // namespace
}  // namespace caee

using namespace caee;

extern "C" {

caee_status_t caee_block_matmul_workspace_size(const caee_block_matmul_desc_t* desc, size_t* bytes) {
    clear_last_error();
    if (!bytes) return fail(CAEE_ERR_INVALID_ARG, "bytes is NULL");
    CAEE_TRY(check_bm(desc));
    *bytes = bm_ws(*desc);
    return CAEE_OK;
}

caee_status_t caee_block_matmul(const caee_block_matmul_desc_t* desc, const void* x, const float* x_scale,
                                const void* w, const float* w_scale, void* y, void* ws, size_t ws_bytes,
                                void* stream) {
    clear_last_error();
    CAEE_TRY(check_bm(desc));
    const caee_block_matmul_desc_t& d = *desc;
    const bool any = d.M > 0, given = d.x_dtype == CAEE_FP8_E4M3;
    CAEE_TRY(check_ptr(x, "x", any));
    CAEE_TRY(check_ptr(x_scale, "x_scale", any && given));
    if (!given && x_scale) return fail(CAEE_ERR_INVALID_ARG, "x_scale given for x that the call quantises");
    CAEE_TRY(check_ptr(w, "w", true));
    CAEE_TRY(check_ptr(w_scale, "w_scale", true));
    CAEE_TRY(check_ptr(y, "y", any));
    if (!any) return CAEE_OK;
    const size_t need = bm_ws(d);
    if (need) {
        if (!ws) return fail(CAEE_ERR_WORKSPACE, "workspace is NULL");
        if (((uintptr_t)ws & 255u) != 0) return fail(CAEE_ERR_WORKSPACE, "workspace is not 256-byte aligned");
        if (ws_bytes < need) return fail(CAEE_ERR_WORKSPACE, "workspace has %zu bytes, %zu needed", ws_bytes, need);
    }
    BmParams p{};
    p.M = d.M;
    p.N = d.N;
    p.K = d.K;
    p.kb = d.K / 128;
    p.x = x;
    p.w = (const uint8_t*)w;
    p.ws = w_scale;
    p.y = y;
    p.x_stride = d.x_stride;
    p.y_stride = d.y_stride;
    p.tiled = d.layout == CAEE_LAYOUT_TILED;
    p.y_bf16 = d.y_dtype == CAEE_BF16;
    p.vec = d.y_stride % 4 == 0;
    hipStream_t s = (hipStream_t)stream;
    if (given) {
        p.xq = (const uint8_t*)x;
        p.xs = x_scale;
        p.xq_stride = d.x_stride;
    } else {
        p.xq_out = (uint8_t*)ws;
        p.xs_out = (float*)((char*)ws + up256((size_t)d.M * d.K));
        p.xq = p.xq_out;
        p.xs = p.xs_out;
        p.xq_stride = d.K;
        const long long groups = ((long long)d.M * p.kb + 15) / 16;
        const dim3 grid((unsigned)(groups < 65536 ? groups : 65536));
        CAEE_TRY(timed_launch(CAEE_KERNEL_QUANT, s, "quantise x", [&] {
            if (d.x_dtype == CAEE_BF16) hipLaunchKernelGGL(k_bm_quant<uint16_t>, grid, dim3(256), 0, s, p);
            else hipLaunchKernelGGL(k_bm_quant<float>, grid, dim3(256), 0, s, p);
            return hipGetLastError();
        }));
    }
    return timed_launch(CAEE_KERNEL_MATMUL, s, "block matmul", [&] {
        return !p.y_bf16 || p.K <= kBmExactK ? launch_bm<true>(p, s) : launch_bm<false>(p, s);
    });
}

}  // extern "C"
