// Shared by the kernels of attention with grouped heads over a paged cache of
// keys and values: parameter block, workspace layout and device helpers.
#pragma once

#include "latent.h"

namespace caee {

// Where a head's keys (and values, in an array of the same strides) of a page lie.
struct HeadCache {
    int block, n_blocks;
    long long page_stride, row_stride, head_stride;    // elements; 0 where there is one page, row or head
};
// Checks the cache fields that both entry points have; *c gets the strides that the kernels use.
caee_status_t head_cache(int kv_heads, int dim, int block_size, int n_blocks, long long page_stride,
                         long long row_stride, long long head_stride, HeadCache* c);

// Both kernels of attention go over the tokens once.  With m the largest score so
// far (in powers of two: c = scale log2 e), l = sum 2^(c s_j - m) and o = sum
// 2^(c s_j - m) v_j, a tile of tokens adds to l and o, and where its scores exceed m
// by much, m moves to m' and l and o are multiplied by 2^(m - m') first.  Results
// over parts of the tokens are joined by the same rule; y = o / l at the end.
//
// Few rows (k_head_few): the work of all requests is one line
// of units, kFewTokens tokens of one row tile (kFewRows rows of a request, its new
// tokens' heads of one group) each, by request, group, row tile and token.  It is
// cut into equal shares, one a workgroup; a share begins and ends inside a row
// tile's line, so a workgroup leaves at most two partial results.  A row tile's
// start and end take as long as some tokens and count as units before them
// (few_start).
constexpr int kFewRows = 32, kFewTokens = 128;
constexpr int kFewGroups = 512;                    // two workgroups a CU
// Many rows (k_head_tile): row tiles of kTileRows rows, a workgroup each, or,
// where that leaves CUs idle, one for each of equal pieces of the row tile's
// tokens, which leave partial results: at most kTilePieces pieces then.
constexpr int kTileRows = 128, kTileTokens = 64;
constexpr int kTileSlots = 512;                    // workgroups that run at a time, two a CU
constexpr int kTilePieces = 2 * kTileSlots;
constexpr unsigned kHeadBlank = 64;                // workgroups that blank the rows of no request (whole form)
// A quotient of uniform numbers, in a scalar register.
__device__ inline int head_div(int a, int b) { return __builtin_amdgcn_readfirstlane(a / b); }
__device__ inline int head_share(int total) { return max((total + kFewGroups - 1) / kFewGroups, 1); }
// Neighbouring shares, which have row tiles of the same tokens, run on one XCD.
__device__ inline int head_group(int wg) { return wg % kXcds * (kFewGroups / kXcds) + wg / kXcds; }
__device__ inline int head_workgroup(int g) { return g % (kFewGroups / kXcds) * kXcds + g / (kFewGroups / kXcds); }

struct HeadWs {
    size_t meta;           // [B + 1] unit or piece prefix sums, of more than 64 requests; [1] steps of a piece
    size_t part, part_ml;  // split: [two a share, or a piece][rows][dim] partial sums and [..][rows][2] (maximum, sum)
    size_t part_sum;       // [piece][rows] sums of the weights before their rounding
    size_t total;
};

// Division of 0 <= n < 2^31 by d: n m / 2^(31 + shift), rounded down, with m =
// 2^(31 + shift) / d, rounded up, and 2^shift >= d > 2^(shift - 1): m is off by less
// than 2^shift / d of n's step, so the quotient is right.
struct HeadBy {
    uint32_t m;
    int shift;
};
inline HeadBy head_by(int d) {
    int shift = 0;
    while (1 << shift < d) ++shift;
    return {(uint32_t)(((1ull << (31 + shift)) + (unsigned)d - 1) / (unsigned)d), shift};
}
__device__ inline int head_over(int n, const HeadBy& d) { return (int)(__umulhi(2u * (unsigned)n, d.m) >> d.shift); }

struct HeadParams {
    int T, B, H, G, ratio, dim, max_blocks, max_new, causal, y_bf16, words, few_start;
    HeadCache c;
    HeadBy by_ratio, by_block;
    long long max_kv;     // no request is longer (what max_kv and the table's rows allow)
    long long q_stride;
    float scale_log2;     // scale * log2(e): softmax in powers of two
    const uint16_t* q;
    const uint16_t* k;
    const uint16_t* v;
    const int32_t* table;
    const int32_t* cu_new;
    const int32_t* seq_len;
    const uint32_t* tree;
    void* y;
    float* lse;
    int32_t* meta;
    float* part;          // NULL: whole form
    float* part_ml;
    float* part_sum;      // NULL: those of part_ml are of weights that are not rounded, or there is no lse
};

// New tokens and length of request b as the kernels use them: 0 <= new <=
// max_new, rows within [0, T), 0 <= seq <= max_kv, and the tokens before its
// new ones, by the lengths as they are (within bounds whose sums and differences
// 32 bits hold, whatever the arrays do).
__device__ inline LatentReq head_req(const HeadParams& p, int b) {
    LatentReq r;
    const int a = max(p.cu_new[b], 0), e = max(p.cu_new[b + 1], 0);
    r.t0 = min(a, p.T);
    r.add = min(max(min(e, p.T) - r.t0, 0), p.max_new);
    const int len = min(max(p.seq_len[b], 0), 1 << 30);
    r.seq = min(len, (int)p.max_kv);
    r.before = max(len - max(e - a, 0), -(1 << 29));
    return r;
}
// Tokens up to which new token i of the request may see some; with a tree not all of them.
__device__ inline int head_sees(const HeadParams& p, const LatentReq& r, int i) {
    return p.causal && !p.tree ? min(max(r.before + i + 1, 0), r.seq) : r.seq;
}

// Units and pieces are counted up to this; requests within the host's bounds have
// no more, one by one and together.
constexpr int kHeadMaxUnits = INT32_MAX / 2;
__device__ inline int head_add_units(int a, int b) { return min(a + b, kHeadMaxUnits); }
// Units of a list: those of a row tile's tokens, and few_start.
__device__ inline int head_few_list(const HeadParams& p, const LatentReq& r) {
    return r.seq > 0 ? (r.seq + kFewTokens - 1) / kFewTokens + p.few_start : 0;
}
__device__ inline int head_few_units(const HeadParams& p, const LatentReq& r) {
    const long long n = (long long)(p.G * ((r.add * p.ratio + kFewRows - 1) / kFewRows)) * head_few_list(p, r);
    return (int)min(n, (long long)kHeadMaxUnits);
}
__device__ inline int head_tiles(const HeadParams& p, const LatentReq& r) { return (r.add * p.ratio + kTileRows - 1) / kTileRows; }
__device__ inline int head_steps(const LatentReq& r) { return (r.seq + kTileTokens - 1) / kTileTokens; }
// Pieces of a row tile of n steps.
__device__ inline int head_cut(int n, int per) { return max((n + per - 1) / per, 1); }
// Step that piece `part` of `parts` of n steps begins with (part == parts: n), n part / parts:
// that product passes 32 bits for 2^28 tokens in 512 pieces, these do not.
__host__ __device__ inline int head_piece_at(int n, int part, int parts) {
    const int each = n / parts;
    return each * part + (n - each * parts) * part / parts;
}

// Inclusive scan over the lanes, in registers (a shuffle through LDS takes ten
// times as long, and a workgroup begins with a chain of these), and its last.
template <int C, int ROWS, class Op>
__device__ inline int head_scan_step(int v, int none, Op&& op) {
    return op(v, __builtin_amdgcn_update_dpp(none, v, C, ROWS, 0xF, false));
}
template <class Op>
__device__ inline int head_scan(int v, int none, Op&& op) {
    v = head_scan_step<0x111, 0xF>(v, none, op);       // 1, 2, 4 and 8 lanes down a row of 16
    v = head_scan_step<0x112, 0xF>(v, none, op);
    v = head_scan_step<0x114, 0xF>(v, none, op);
    v = head_scan_step<0x118, 0xF>(v, none, op);
    v = head_scan_step<0x142, 0xA>(v, none, op);       // the rows' last lanes to the next row, the second's to both after it
    return head_scan_step<0x143, 0xC>(v, none, op);
}
__device__ inline int head_last(int v) { return __builtin_amdgcn_readlane(v, kWave - 1); }

// Prefix sums over the requests of a number each has.  Up to 64 requests every
// wave makes them by itself, a lane each; of more, p.meta has them.
struct HeadLine {
    LatentReq mine;      // lane b: request b
    int n, at, total;    // its number and the sum of those before; all requests'
};
__device__ inline HeadLine head_line(const HeadParams& p) {
    HeadLine h = {};
    if (p.B > kWave) h.total = __builtin_amdgcn_readfirstlane(p.meta[p.B]);
    else if ((int)(threadIdx.x & (kWave - 1)) < p.B) h.mine = head_req(p, threadIdx.x & (kWave - 1));
    return h;
}
__device__ inline void head_line_sum(const HeadParams& p, HeadLine* h, int n) {
    if (p.B > kWave) return;
    const int lane = threadIdx.x & (kWave - 1);
    h->n = lane < p.B ? n : 0;
    const int sum = head_scan(h->n, 0, head_add_units);
    h->at = sum - h->n;
    h->total = head_last(sum);
}
// Request b of the line: its lengths and what is before it.
__device__ inline LatentReq head_line_req(const HeadParams& p, const HeadLine& h, int b, int* at) {
    if (p.B > kWave) {
        *at = __builtin_amdgcn_readfirstlane(p.meta[b]);
        const LatentReq r = head_req(p, b);
        return {__builtin_amdgcn_readfirstlane(r.t0), __builtin_amdgcn_readfirstlane(r.add),
                __builtin_amdgcn_readfirstlane(r.seq), __builtin_amdgcn_readfirstlane(r.before)};
    }
    *at = __builtin_amdgcn_readlane(h.at, b);
    return {__builtin_amdgcn_readlane(h.mine.t0, b), __builtin_amdgcn_readlane(h.mine.add, b),
            __builtin_amdgcn_readlane(h.mine.seq, b), __builtin_amdgcn_readlane(h.mine.before, b)};
}
// Request that number u of the line is of (u below the total).
__device__ inline int head_line_find(const HeadParams& p, const HeadLine& h, int u) {
    if (p.B > kWave) return lat_find_wave(p.meta, p.B, u);
    return 63 - __clzll(__ballot((int)(threadIdx.x & (kWave - 1)) < p.B && h.at <= u) | 1ull);
}

// Bits of a token's tree mask for new tokens bit .. bit + 31 of its request;
// tokens before the new ones are seen.
__device__ inline uint32_t head_tree_bits(const uint32_t* mask, int words, int bit) {
    const int w = bit >> 5, sh = bit & 31;
    const uint32_t a = w < 0 ? ~0u : w < words ? mask[w] : 0u;
    const uint32_t b = w + 1 < 0 ? ~0u : w + 1 < words ? mask[w + 1] : 0u;
    return sh ? (a >> sh) | (b << (32 - sh)) : a;
}

// Where the tokens that a wave fetches lie: eights of them, whose rows one load
// gets where they lie in one page, E of a tile.  A lane looks up one eight, so
// that a look covers kHeadWindow / E tiles and a step reads lanes (in scalar
// instructions, a tile's addresses take as long as its products).
constexpr int kHeadWindow = kWave;
struct HeadWindow {
    uint32_t lo, hi;      // byte offset of the eight's first row from the cache's (of the group)
    int span;             // the others follow up to this row after it; -1: they lie in several pages
};
// The eight that begins at token `pos` (tokens past the request's are its last
// one), in two parts: what the first asks for may be on its way for a while.
struct HeadLook {
    int entry, at, span;
};
__device__ inline HeadLook head_look(const HeadParams& p, int b, int seq, int pos) {
    const int r0 = min(pos, seq - 1), span = min(pos + 7, seq - 1) - r0;
    const unsigned j = (unsigned)head_over(r0, p.by_block);
    return {p.table[(size_t)b * p.max_blocks + min(j, (unsigned)p.max_blocks - 1u)], r0 - (int)(j * (unsigned)p.c.block), span};
}
__device__ inline HeadWindow head_window(const HeadParams& p, const HeadLook& l) {
    const unsigned long long off =
        2ull * (unsigned long long)(min(max(l.entry, 0), p.c.n_blocks - 1) * p.c.page_stride + l.at * p.c.row_stride);
    return {(uint32_t)off, (uint32_t)(off >> 32), l.at + l.span < p.c.block ? l.span : -1};
}
// Byte offset of row `pos` of request b.
__device__ inline long long head_row(const HeadParams& p, int b, int pos) {
    const HeadWindow w = head_window(p, head_look(p, b, pos + 1, pos));
    return (long long)((unsigned long long)w.hi << 32 | w.lo);
}
struct HeadEight {
    unsigned long long off;
    int span;
};
__device__ inline HeadEight head_eight(const HeadWindow& w, int i) {
    return {(unsigned long long)(uint32_t)__builtin_amdgcn_readlane(w.hi, i) << 32 | (uint32_t)__builtin_amdgcn_readlane(w.lo, i),
            __builtin_amdgcn_readlane(w.span, i)};
}
__device__ inline const char* head_base(const HeadParams& p, const uint16_t* cache, int g) {
    return (const char*)(cache + g * p.c.head_stride);
}

// Softmax weight of score s where the running maximum is m, by one multiply-add:
// what m's product with scale_log2 lost to rounding is a factor that all weights
// of the row have in common.  Up to kFusedMax it is at most 2^64 (half a step of
// m), and neither it nor the sums leave the range of 32 bits.
constexpr float kFusedMax = 0x1p30f;
__device__ inline float head_weight(float s, float scale_log2, float m) { return __builtin_amdgcn_exp2f(fmaf(s, scale_log2, -m)); }
// While the weights of a lane's tile add up to no more than kMaxWeight none of
// them exceeds it, and the maximum need not move; past 2^20 it moves with every
// tile, so that the weights are made by lat_weight, whose products are rounded.
__device__ inline bool head_moves(float more, float m) { return more > kMaxWeight || !(fabsf(m) <= 0x1p20f); }

// Adds a partial result (sums x of weights by the maximum w.x, whose total is w.y, and
// `all` before the weights were rounded) to one.  An infinity or NaN among the sums, of a
// value that the row sees, stays however little its part of the tokens weighs (kOdd); without,
// it is no number afterwards, whatever its factor, and that is looked for once, at the end
// (looked for at every sum, 31.4 us of a call became 40.0).
template <bool kOdd>
__device__ inline float head_join(float a, float f, float x, float e) {
    const float r = fmaf(x, e, a * f);
    if (!kOdd || fabsf(r) < INFINITY) return r;        // (a row's numbers do not change by an infinity beside them)
    return (fabsf(a) < INFINITY ? a * f : a) + (fabsf(x) < INFINITY ? x * e : x);
}
template <bool kOdd>
__device__ inline void head_merge(float4& v, float& m, float& l, float& sum, const float4& x, const float2& w, float all) {
    const float mn = fmaxf(m, w.x), f = __builtin_amdgcn_exp2f(m - mn), e = __builtin_amdgcn_exp2f(w.x - mn);
    v = make_float4(head_join<kOdd>(v.x, f, x.x, e), head_join<kOdd>(v.y, f, x.y, e), head_join<kOdd>(v.z, f, x.z, e),
                    head_join<kOdd>(v.w, f, x.w, e));
    l = fmaf(w.y, e, l * f);           // (in every kernel the same rounding)
    sum = fmaf(all, e, sum * f);
    m = mn;
}
__device__ inline bool head_finite(const float4& v) { return fabsf(v.x) + fabsf(v.y) + fabsf(v.z) + fabsf(v.w) < INFINITY; }
// Maximum of a partial result without sums: none of its tokens is one that the row may see.
constexpr float kNoPart = -INFINITY;
// Factor of a row's sums: 1 / l.  Where no weight is left they are zero, but for infinities
// and NaNs, which stay.
__device__ inline float head_inverse(float l) { return l == 0.0f ? 1.0f : 1.0f / l; }

// Whether values that are no numbers may have met weights of zero, or weights'
// remainders, in a lane's sums o of a row whose weights add up to l.
template <int NC>
__device__ inline bool head_odd(const lat_f32x16 (&o)[NC], float l) {
    float t = 0.0f;
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int i = 0; i < 16; ++i) t += fabsf(o[c][i]);
    return !(t < INFINITY) && l < INFINITY;
}
// Puts that right after the sums of row n (a lane of each half) were written: where
// values of tokens that the row sees (spans of `width` tokens, `step` apart, from
// tok0 to end) are infinities or NaNs, the sum is theirs: put(d, value, false), then
// put(d, value, true) for what adds to it.  Each lane looks through a token's values.
template <int D, class Sees, class Put>
__device__ inline void head_put_odd(const HeadParams& p, int b, int g, int tok0, int width, int step, int end, Sees&& sees,
                                    Put&& put) {
    const int lane = threadIdx.x & (kWave - 1), hf = lane >> 5;
    const char* base = head_base(p, p.v, g);
    unsigned long long touched = 0;
    const int per = kWave / width;       // spans at a time
#pragma unroll 1
    for (int t0 = tok0; t0 < end; t0 += per * step) {
        const int mine = t0 + lane / width * step + lane % width;
        bool odd = false;
        if (mine < end) {
            const lat_u32x4* row = (const lat_u32x4*)(base + head_row(p, b, mine));
#pragma unroll
            for (int c = 0; c < D / 8; ++c) {
                const lat_u32x4 v = row[c];
#pragma unroll
                for (int e = 0; e < 4; ++e) odd |= lat_finite(v[e]) != v[e];
            }
        }
        unsigned long long found = __ballot(odd);
#pragma unroll 1
        while (found) {
            const int i = __ffsll(found) - 1, pos = t0 + i / width * step + i % width;
            found &= found - 1;
            const lat_u32x2* row = (const lat_u32x2*)(base + head_row(p, b, pos));
            if (!sees(pos)) continue;
#pragma unroll 1
            for (int c = hf; c < D / 4; c += 2) {
                const lat_u32x2 v = row[c];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float x = __uint_as_float(e & 1 ? v[e >> 1] & 0xFFFF0000u : v[e >> 1] << 16);
                    const unsigned long long bit = 1ull << (4 * (c >> 1) + e);
                    if (!(fabsf(x) < INFINITY)) {
                        put(4 * c + e, x, (touched & bit) != 0);
                        touched |= bit;
                    }
                }
            }
        }
    }
}

// The kernel of few rows and its join; that of many, with a join where p.part is
// there, and without (whole).
hipError_t launch_head_few(const HeadParams& p, hipStream_t s);
hipError_t launch_head_many(const HeadParams& p, hipStream_t s);
hipError_t launch_head_tile_64(const HeadParams& p, unsigned grid, int pieces, hipStream_t s);
hipError_t launch_head_tile_128(const HeadParams& p, unsigned grid, int pieces, hipStream_t s);

}  // namespace caee
