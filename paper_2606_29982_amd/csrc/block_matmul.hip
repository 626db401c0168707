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
typedef const __attribute__((address_space(1))) void bm_g_void;
typedef const __attribute__((address_space(1))) bm_u32x4 bm_g_u32x4;

constexpr int kBmMaxK = 65536;
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

// Byte offset of 16-byte piece c of block 0 of weight row n; the next block
// is bm_block bytes further.
__device__ inline size_t bm_piece(const BmParams& p, int n, int c) {
    if (p.tiled) return (((size_t)(n >> 4) * (p.K / 64) + (c >> 2)) * 64 + (n & 15) + 16 * (c & 3)) * 16;
    return (size_t)n * p.K + 16 * c;
}
__device__ inline int bm_block(const BmParams& p) { return p.tiled ? 2048 : 128; }

// Few rows: the weight stream bounds it.  A workgroup takes 16 outputs and
// up to 16 NT rows, its waves a range of blocks each; a wave's weights go
// straight to registers, U blocks of loads in flight, and the waves' sums
// are added through LDS in wave order.
template <int NT, int WAVES, bool kExact>
__global__ __launch_bounds__(WAVES * 64) void k_bm_few(BmParams p) {
    constexpr int U = 4;
    __shared__ float red[WAVES][NT][16 * 17];
    const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n0 = blockIdx.x * 16, m0 = blockIdx.y * 16 * NT;
    const int b0 = (int)((long long)p.kb * wave / WAVES), b1 = (int)((long long)p.kb * (wave + 1) / WAVES);
    const int n = min(n0 + r, p.N - 1);
    const uint8_t* w0 = p.w + bm_piece(p, n, g);
    const uint8_t* w1 = p.w + bm_piece(p, n, 4 + g);
    const int wstep = bm_block(p);
    const uint8_t* xr[NT];
    const float* xs[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const int m = min(m0 + 16 * t + r, p.M - 1);
        xr[t] = p.xq + (size_t)m * p.xq_stride + 16 * g;
        xs[t] = p.xs + (size_t)m * p.kb;
    }
    const float* wsc = p.ws + (size_t)(n0 >> 7) * p.kb;
    bm_f32x4 acc[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) acc[t] = bm_f32x4{0.f, 0.f, 0.f, 0.f};
    const bm_f32x4 zero = {0.f, 0.f, 0.f, 0.f};
    bm_u32x4 cw[U][2], nw[U][2];
    auto fetch = [&](bm_u32x4 (&d)[U][2], int b) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const size_t o = (size_t)min(b + u, p.kb - 1) * wstep;
            d[u][0] = __builtin_nontemporal_load((bm_g_u32x4*)(w0 + o));
            d[u][1] = __builtin_nontemporal_load((bm_g_u32x4*)(w1 + o));
        }
    };
    auto mul = [&](const bm_u32x4 (&d)[U][2], int b) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (b + u >= b1) continue;
            const bm_i32x8 a = bm_join(d[u][0], d[u][1]);
            const float sc = wsc[b + u];
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const uint8_t* x = xr[t] + (size_t)(b + u) * 128;
                const bm_i32x8 c = bm_join(*(const bm_u32x4*)x, *(const bm_u32x4*)(x + 64));
                bm_f32x4 q = zero;
                if constexpr (kExact) {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        q = __builtin_amdgcn_mfma_f32_16x16x32_bf16(bm_wide(a[2 * i], a[2 * i + 1]),
                                                                    bm_wide(c[2 * i], c[2 * i + 1]), q, 0, 0, 0);
                } else {
                    q = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, c, zero, 0, 0, 0, kUnitScale, 0, kUnitScale);
                }
                const float f = sc * xs[t][b + u];
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[t][i] += q[i] * f;
            }
        }
    };
    fetch(cw, b0);
    for (int b = b0; b < b1; b += 2 * U) {
        fetch(nw, b + U);
        mul(cw, b);
        if (b + U >= b1) break;
        fetch(cw, b + 2 * U);
        mul(nw, b + U);
    }
    // Lane (r, g) holds outputs n0 + 4 g .. + 3 of row m0 + 16 t + r.
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) red[wave][t][r * 17 + 4 * g + i] = acc[t][i];
    __syncthreads();
    for (int i = threadIdx.x; i < NT * 64; i += WAVES * 64) {
        const int t = i >> 6, rr = (i >> 2) & 15, q = i & 3;
        float s[4] = {0.f, 0.f, 0.f, 0.f};
        for (int v = 0; v < WAVES; ++v)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[e] += red[v][t][rr * 17 + 4 * q + e];
        const int m = m0 + 16 * t + rr;
        if (m < p.M) bm_store4(p, m, n0 + 4 * q, s[0], s[1], s[2], s[3]);
    }
}

// Many rows: 256 outputs x 256 rows per workgroup, 8 waves of 128 x 64, one
// 128-deep block per stage; both operands go global -> LDS directly, one
// block ahead.  Blocks of 8 rows x 128 bytes, piece c of row r at
// 8 (r % 8) + (c ^ (r % 8)).
struct BmStage {
    bm_u32x4 a[32][kWave], b[32][kWave];
    float xs[256];
};

template <bool kExact>
__global__ __launch_bounds__(512) void k_bm_many(BmParams p, int n_tiles) {
    __shared__ BmStage st0, st1;
    const int lane = threadIdx.x & 63, n = lane & 31, hf = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave & 1, wn = wave >> 1;
    const int n0 = (blockIdx.x % n_tiles) * 256, m0 = (blockIdx.x / n_tiles) * 256;
    const uint8_t *asrc[4], *bsrc[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = 32 * wave + 8 * i + (lane >> 3), c = (lane & 7) ^ (lane >> 3);
        asrc[i] = p.w + bm_piece(p, min(n0 + r, p.N - 1), c);
        bsrc[i] = p.xq + (size_t)min(m0 + r, p.M - 1) * p.xq_stride + 16 * c;
    }
    const float* xsrc = p.xs + (size_t)min(m0 + 64 * (wave & 3) + lane, p.M - 1) * p.kb;
    const int wstep = bm_block(p);
    const float* wsc = p.ws + (size_t)min((n0 + 128 * wm) >> 7, (p.N - 1) >> 7) * p.kb;
    auto load = [&](int k, BmStage& t) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            __builtin_amdgcn_global_load_lds((bm_g_void*)(asrc[i] + (size_t)k * wstep), (bm_lds_void*)&t.a[4 * wave + i][0], 16, 0, 0);
            __builtin_amdgcn_global_load_lds((bm_g_void*)(bsrc[i] + (size_t)k * 128), (bm_lds_void*)&t.b[4 * wave + i][0], 16, 0, 0);
        }
        if (wave < 4)
            __builtin_amdgcn_global_load_lds((bm_g_void*)(xsrc + k), (bm_lds_void*)&t.xs[64 * wave], 4, 0, 0);
    };
    bm_f32x16 acc[4][2] = {};
    const bm_f32x16 zero = {};
    auto step = [&](int k, BmStage& t, BmStage& next) __attribute__((always_inline)) {
        __builtin_amdgcn_s_waitcnt((0) | (7 << 4) | (15 << 8));
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        if (k + 1 < p.kb) load(k + 1, next);
        auto frag = [&](const bm_u32x4* row, int kk) __attribute__((always_inline)) {
            return bm_join(row[(n & 7) * 8 + ((4 * kk + hf) ^ (n & 7))], row[(n & 7) * 8 + ((4 * kk + 2 + hf) ^ (n & 7))]);
        };
        bm_i32x8 b[2][2];
        float f[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
#pragma unroll
            for (int kk = 0; kk < 2; ++kk) b[e][kk] = frag(t.b[8 * wn + 4 * e + (n >> 3)], kk);
            f[e] = t.xs[64 * wn + 32 * e + n] * wsc[k];
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const bm_u32x4* row = t.a[16 * wm + 4 * i + (n >> 3)];
            const bm_i32x8 a0 = frag(row, 0), a1 = frag(row, 1);
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                bm_f32x16 q = zero;
                if constexpr (kExact) {
#pragma unroll
                    for (int kk = 0; kk < 2; ++kk) {
                        const bm_i32x8& a = kk ? a1 : a0;
#pragma unroll
                        for (int v = 0; v < 4; ++v)
                            q = __builtin_amdgcn_mfma_f32_32x32x16_bf16(bm_wide(a[2 * v], a[2 * v + 1]),
                                                                        bm_wide(b[e][kk][2 * v], b[e][kk][2 * v + 1]), q,
                                                                        0, 0, 0);
                    }
                } else {
                    q = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a0, b[e][0], zero, 0, 0, 0, kUnitScale, 0,
                                                                        kUnitScale);
                    q = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a1, b[e][1], q, 0, 0, 0, kUnitScale, 0,
                                                                        kUnitScale);
                }
#pragma unroll
                for (int v = 0; v < 16; ++v) acc[i][e][v] += q[v] * f[e];
            }
        }
    };
    load(0, st0);
    for (int k = 0; k < p.kb; k += 2) {
        step(k, st0, st1);
        if (k + 1 < p.kb) step(k + 1, st1, st0);
    }
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        const int m = m0 + 64 * wn + 32 * e + n;
        if (m >= p.M) continue;
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                bm_store4(p, m, n0 + 128 * wm + 32 * i + 8 * q + 4 * hf, acc[i][e][4 * q], acc[i][e][4 * q + 1],
                          acc[i][e][4 * q + 2], acc[i][e][4 * q + 3]);
    }
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
    if (d->K > kBmMaxK || d->M > (1 << 24) || d->N > (1 << 24))
        return fail(CAEE_ERR_UNSUPPORTED, "M=%d, N=%d or K=%d exceeds %d, %d, %d", d->M, d->N, d->K, 1 << 24, 1 << 24,
                    kBmMaxK);
    return CAEE_OK;
}

constexpr int kBmExactK = 256;

template <int WAVES, bool kExact>
void launch_few(const BmParams& p, hipStream_t s) {
    const unsigned nt = (unsigned)((p.N + 15) / 16);
    const dim3 block(WAVES * 64);
    if (p.M <= 16) hipLaunchKernelGGL((k_bm_few<1, WAVES, kExact>), dim3(nt, 1), block, 0, s, p);
    else if (p.M <= 32) hipLaunchKernelGGL((k_bm_few<2, WAVES, kExact>), dim3(nt, 1), block, 0, s, p);
    else hipLaunchKernelGGL((k_bm_few<4, WAVES, kExact>), dim3(nt, (unsigned)((p.M + 63) / 64)), block, 0, s, p);
}

template <bool kExact>
hipError_t launch_bm(const BmParams& p, hipStream_t s) {
    const long long tiles = (long long)((p.M + 255) / 256) * ((p.N + 255) / 256);
    if (p.M > 64 && (tiles >= 128 || p.M > 1024)) {
        hipLaunchKernelGGL(k_bm_many<kExact>, dim3((unsigned)tiles), dim3(512), 0, s, p, (p.N + 255) / 256);
    } else {
        launch_few<8, kExact>(p, s);
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
