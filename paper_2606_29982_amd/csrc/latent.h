// Shared by the latent-attention kernels: parameter blocks, the workspace
// layout and the device helpers of both forms.
#pragma once

#include "caee_internal.h"

#include <type_traits>

namespace caee {

constexpr int kRopeDim = 64;          // rotary part of a query and of a cache row
// Absorbed form: workgroups of the attention launch (one per CU of the chip:
// its LDS tiles fill a CU), each with an equal share of the tokens of all
// requests; a share begins and ends inside a request, so a workgroup leaves
// at most two partial results.
constexpr int kAbsGroups = 256;
constexpr int kAbsTileRows = 64;      // query rows of such a workgroup
constexpr int kExpRows = 256;         // query rows of a workgroup of the expanded form

struct LatentWs {
    size_t meta;          // [B + 1] unit (absorbed) or query tile (expanded) prefix sums
    size_t q;             // absorbed: [T][heads][latent + rope] bf16 queries
    size_t o;             // absorbed: [T][heads][latent] fp32 attended latents
    size_t part, part_ml; // absorbed: [2 groups][rows][latent] partial sums and [..][rows][2] (maximum, sum)
    size_t kv, kr;        // expanded: [max_kv][heads][nope + v] keys and values, [max_kv][rope] rotary keys
    size_t total;
    bool expanded;
};

struct LatentParams {
    int T, B, H, nope, latent, v, block, n_blocks, max_blocks, max_new, causal, y_bf16;
    long long max_kv, q_stride;
    float scale;
    float scale_log2;     // scale * log2(e): softmax in powers of two
    const uint16_t* q;
    const uint16_t* w_uk;
    const uint16_t* w_uk_t;
    const uint16_t* w_uv;
    const uint16_t* cache;
    const int32_t* table;
    const int32_t* cu_new;
    const int32_t* cu_kv;
    const int32_t* seq_len;
    void* y;
    float* lse;
    int32_t* meta;
    uint16_t* qw;
    float* o;
    float* part;
    float* part_ml;
    uint16_t* kv;
    uint16_t* kr;
};

// A launch has fewer than 2^32 threads in x: past kLatGridX workgroups (a
// multiple of the XCDs) a grid goes on in y, as one line of workgroups.
constexpr unsigned kLatGridX = 1u << 22;
inline dim3 lat_grid(unsigned n) { return n <= kLatGridX ? dim3(n) : dim3(kLatGridX, (n + kLatGridX - 1) / kLatGridX); }
__device__ inline unsigned lat_workgroup() { return blockIdx.y * gridDim.x + blockIdx.x; }

hipError_t launch_latent_absorbed(const LatentParams& p, hipStream_t s);
hipError_t launch_latent_expanded(const LatentParams& p, hipStream_t s);

typedef uint32_t lat_u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t lat_u32x2 __attribute__((ext_vector_type(2)));
typedef short lat_s16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 lat_bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 lat_bf16x2 __attribute__((ext_vector_type(2)));
typedef float lat_f32x2 __attribute__((ext_vector_type(2)));
typedef float lat_f32x16 __attribute__((ext_vector_type(16)));
typedef __attribute__((address_space(3))) lat_s16x4 lat_lds_s16x4;
typedef __attribute__((address_space(3))) void lat_lds_void;
typedef const __attribute__((address_space(1))) void lat_g_void;

constexpr int kLatBufBytes = 0x7FFFFFFF, kLatBufWord3 = 0x00020000;   // buffer descriptor: size, raw 32-bit access
template <int N>
using LatInt = std::integral_constant<int, N>;
// f(LatInt<B>{}), ..., f(LatInt<E - 1>{}).
template <int B, int E, class F>
__device__ __attribute__((always_inline)) inline void lat_for(F&& f) {
    if constexpr (B < E) {
        f(LatInt<B>{});
        lat_for<B + 1, E>(f);
    }
}

constexpr float kNoScore = -3.40282347e38f;    // running maximum of a row that has seen nothing: the lowest finite score
// Softmax weight of score s where the running maximum is m (a product s
// scale_log2 of fp32).  The product is rounded before m is taken off, as m's
// was: in one multiply-add a score past 2^30 would leave its product's rounding,
// up to any power of two, as the weight of the maximum itself.
__device__ inline float lat_weight(float s, float scale_log2, float m) {
#pragma clang fp contract(off)
    const float t = s * scale_log2;
    return __builtin_amdgcn_exp2f(t - m);
}
// The running maximum moves only when a score exceeds it by more than
// kMaxSlack (in powers of two): the weights are then at most 2^8, which costs
// neither fp32 sums nor bf16 weights any precision, and the accumulators are
// rescaled a few times per row instead of at every new maximum.
constexpr float kMaxSlack = 8.0f, kMaxWeight = 256.0f;

template <int N>
__device__ inline void lat_wait_vm() {
    __builtin_amdgcn_s_waitcnt((N & 15) | (7 << 4) | (15 << 8) | (((N >> 4) & 3) << 14));
}
__device__ inline void lat_barrier() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

__device__ inline lat_f32x16 lat_mma(const lat_u32x4& a, const lat_u32x4& b, const lat_f32x16& c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(lat_bf16x8, a),
                                                   __builtin_bit_cast(lat_bf16x8, b), c, 0, 0, 0);
}

// Two floats rounded to bf16 (nearest even), a in the low half.
__device__ inline uint32_t lat_pack(float a, float b) {
    const lat_f32x2 t = {a, b};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(t, lat_bf16x2));
}

// What rounding a and b to the bf16 pair v left.
__device__ inline lat_f32x2 lat_rest(uint32_t v, float a, float b) {
    return lat_f32x2{a - __uint_as_float(v << 16), b - __uint_as_float(v & 0xFFFF0000u)};
}

// sum + both bf16 values of v.
__device__ inline float lat_sum2(uint32_t v, float sum) {
    const lat_bf16x2 one = {(__bf16)1.0f, (__bf16)1.0f};
    return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(lat_bf16x2, v), one, sum, false);
}

// KV tiles in LDS are blocks of 8 rows x 128 bytes; piece c (16 bytes) of row
// r is at 8 (r % 8) + (c ^ lat_swz(r)).  A 16-byte read takes 16 lanes at a
// time over 64 banks: 16 rows' piece c, of which the even and the odd rows
// fall into different halves of the banks and the eight of each half into
// different places by the three bits that lat_swz permutes.  A transposed
// read takes four pieces of each of four rows: rows r and r + 2 (4 | r) differ
// in the swizzle's top bit, so in different quarters.
__device__ inline int lat_swz(int r) { return ((r & 2) << 1) | ((r & 4) >> 1) | ((r & 8) >> 3); }

// Maximum, or sum, over a lane and its partner 32 lanes away (the two halves
// of a 32 x 32 tile's column).
__device__ inline float lat_max_pair(float v) { return fmaxf(v, __shfl_xor(v, 32)); }
__device__ inline float lat_sum_pair(float v) { return v + __shfl_xor(v, 32); }

// Two bf16 values with infinities and NaNs replaced by zero.
__device__ inline uint32_t lat_finite(uint32_t v) {
    if ((v & 0x7F80u) == 0x7F80u) v &= 0xFFFF0000u;
    if ((v & 0x7F800000u) == 0x7F800000u) v &= 0x0000FFFFu;
    return v;
}

// 1 / l; 0 for a row that sees nothing; NaN stays.
__device__ inline float lat_inverse(float l) { return l > 0.0f ? 1.0f / l : l; }
__device__ inline float lat_lse(float m, float l) {
    return l == 0.0f ? -INFINITY : 0.6931471805599453f * m + logf(l);
}

// Largest i in [0, n) with a[i] <= x (a ascending, a[0] <= x).
__device__ inline int lat_find(const int32_t* a, int n, int x) {
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (a[mid] <= x) lo = mid;
        else hi = mid;
    }
    return lo;
}

// The same for an x that the wave's lanes share, 64 entries at a time.
__device__ inline int lat_find_wave(const int32_t* a, int n, int x) {
    const int lane = threadIdx.x & (kWave - 1);
    int lo = 0, len = n;
    while (len > 1) {
        const int step = (len + kWave - 1) / kWave, at = lane * step;
        const unsigned long long le = __ballot(at < len && a[lo + min(at, len - 1)] <= x);
        const int k = (63 - __clzll(le | 1ull)) * step;
        lo += k;
        len = min(step, len - k);
    }
    return __builtin_amdgcn_readfirstlane(lo);
}

// Cache row of token `pos` of request b.
__device__ inline uint32_t lat_slot(const LatentParams& p, int b, int pos) {
    const unsigned j = (unsigned)pos / (unsigned)p.block;
    const unsigned at = j < (unsigned)p.max_blocks ? j : (unsigned)p.max_blocks - 1u;
    int page = p.table[(size_t)b * p.max_blocks + at];
    page = page < 0 ? 0 : page >= p.n_blocks ? p.n_blocks - 1 : page;
    return (uint32_t)page * (uint32_t)p.block + ((unsigned)pos - j * (unsigned)p.block);
}

// New tokens and length of request b as the kernels use them: 0 <= new <=
// max_new, rows within [0, T), 0 <= seq <= max_kv (the host's bounds size the
// workspace and the counters, so lengths past them are cut), and the tokens
// before its new ones, by the lengths as they are: what a causal row sees does
// not change where the rows end inside a request.
struct LatentReq {
    int t0, add, seq, before;
};
// Tokens that new token i of the request sees.
__device__ inline int lat_sees(const LatentParams& p, const LatentReq& r, int i) {
    return p.causal ? min(max(r.before + i + 1, 0), r.seq) : r.seq;
}
__device__ inline LatentReq lat_req(const LatentParams& p, int b) {
    LatentReq r;
    const int a = p.cu_new[b], e = p.cu_new[b + 1];
    r.t0 = min(max(a, 0), p.T);
    r.add = min(max(min(e, p.T) - r.t0, 0), p.max_new);
    const int len = max(p.seq_len[b], 0);
    r.seq = min(len, (int)p.max_kv);
    r.before = len - (e - a);
    return r;
}

}  // namespace caee
