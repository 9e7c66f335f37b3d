// What the attention kernels share: widening of codes, shares of the work, rows that have nothing to read.
#pragma once

#include "pag_kv.h"

namespace pagkv {

constexpr float LOWEST = -3.0e38f;        // M before the first key
constexpr float HEADROOM = 15.f;          // weights stay below 2^15
constexpr float START = 7.f;              // and are 2^7 at most when M moves: 16-bit floats then hold 2^-31 of the largest
constexpr float LOG2E = 1.44269504088896340736f;
constexpr float LN2 = 0.69314718055994530942f;

// Up to this cap a capped score is cap - 2 cap / (1 + e^(2 score / cap)), one exponential and one reciprocal, whose error is 2^-22 of the cap (of 64 a
// twentieth of what a weight's rounding to 11 bits does).  Above it the error has to be the score's own, see capped().
constexpr float NEAR_CAP = 64.f;

// cap * tanh(x / cap), by: 1 / cap; x and cap are a score and its cap, both times log2 e.  Below half the cap by tanh's series, x - x^3 / 3 + ..., whose
// first term left out is 2^-23 of x there; above it as for small caps.  A cap beyond all scores leaves x as it is.
__device__ __forceinline__ float capped(float x, float cap, float by) {
    const float y = x * by, u = y * y;
    float p = 21844.f / 6081075.f;
    p = __builtin_fmaf(p, u, -1382.f / 155925.f);
    p = __builtin_fmaf(p, u, 62.f / 2835.f);
    p = __builtin_fmaf(p, u, -17.f / 315.f);
    p = __builtin_fmaf(p, u, 2.f / 15.f);
    p = __builtin_fmaf(p, u, -1.f / 3.f);
    const float low = __builtin_fmaf(x, u * p, x), high = __builtin_fmaf(-2.f * cap, __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(2.f * LOG2E * y)), cap);
    return fabsf(y) < 0.5f ? low : high;
}

__device__ __forceinline__ u32 perm(u32 hi, u32 lo, u32 sel) { return __builtin_amdgcn_perm(hi, lo, sel); }

// A weight is carried with its values' scale, w = 2^(t) with t = score * log2 e + e - M, and 2^-e takes that off again in the weights' sum.  32 bits hold
// weights down to 2^-126, so that a key whose e lies 120 below the largest would be missing there: once a wave has seen an e above this one
// (values of 2^31 and more; e is -64 at least), 2^(t - e) itself is summed up, in the narrow kernels beside the weights, in the wide one once all keys are added.
constexpr int FAR_EXPONENT = 24;

// sum + x * 2^d, d <= 0 or so, also where 2^d alone leaves 32 bits
__device__ __forceinline__ float add_scaled(float sum, float x, float d) {
    const bool far = d < -100.f;
    return __builtin_fmaf(x * (far ? 0x1p-100f : 1.f), __builtin_amdgcn_exp2f(far ? d + 100.f : d), sum);
}

// two codes, bytes 0 and 2 of a word whose other bytes are zero, as 16-bit floats: 1024 + (code + 128) has the code's bits, with the
// sign turned, as its lowest
__device__ __forceinline__ half2_t widen_int8(u32 w) {
    const half2_t bias = { (_Float16)1152.f, (_Float16)1152.f };
    return __builtin_bit_cast(half2_t, w ^ 0x64806480u) - bias;
}

// eight codes in their order
template <int FMT>
__device__ __forceinline__ half8_t widen8(u32 lo, u32 hi) {
    half2_t h[4];
    if constexpr (FMT == PAG_KV_INT8) {
        h[0] = widen_int8(perm(0, lo, 0x0c010c00));
        h[1] = widen_int8(perm(0, lo, 0x0c030c02));
        h[2] = widen_int8(perm(0, hi, 0x0c010c00));
        h[3] = widen_int8(perm(0, hi, 0x0c030c02));
    } else {
        h[0] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.f, false);
        h[1] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.f, true);
        h[2] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.f, false);
        h[3] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.f, true);
    }
    return half8_t{ h[0].x, h[0].y, h[1].x, h[1].y, h[2].x, h[2].y, h[3].x, h[3].y };
}

// byte c of eight words, c = 0 .. 3: a column of eight tokens for each of four numbers of a row
template <int FMT>
__device__ __forceinline__ void columns(const u32* w, half8_t* out) {
    if constexpr (FMT == PAG_KV_INT8) {
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            half2_t h[4];
#pragma unroll
            for (int p = 0; p < 4; ++p) h[p] = widen_int8(perm(w[2 * p + 1], w[2 * p], 0x0c040c00u + 0x00010001u * c));
            out[c] = half8_t{ h[0].x, h[0].y, h[1].x, h[1].y, h[2].x, h[2].y, h[3].x, h[3].y };
        }
    } else {
        u32 lo[2][2], t[2][4];                       // pairs of bytes of two words, then four bytes of four words
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            lo[0][0] = perm(w[4 * q + 1], w[4 * q], 0x05010400);
            lo[0][1] = perm(w[4 * q + 1], w[4 * q], 0x07030602);
            lo[1][0] = perm(w[4 * q + 3], w[4 * q + 2], 0x05010400);
            lo[1][1] = perm(w[4 * q + 3], w[4 * q + 2], 0x07030602);
            t[q][0] = perm(lo[1][0], lo[0][0], 0x05040100);
            t[q][1] = perm(lo[1][0], lo[0][0], 0x07060302);
            t[q][2] = perm(lo[1][1], lo[0][1], 0x05040100);
            t[q][3] = perm(lo[1][1], lo[0][1], 0x07060302);
        }
#pragma unroll
        for (int c = 0; c < 4; ++c) out[c] = widen8<FMT>(t[0][c], t[1][c]);
    }
}

// LDS traffic only: loads from memory stay in flight
__device__ __forceinline__ void lds_barrier() {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// what fits 32 bits is divided in 32 bits, in a tenth of the instructions
__device__ __forceinline__ u64 divide(u64 a, u64 b) {
    if ((a | b) >> 32) return a / b;
    return (u32)a / (u32)b;
}

__device__ __forceinline__ u64 share(u64 total, u32 parts, u32 i) { return divide(total * i, parts); }

// zeros for the heads of tokens [t0, t1)
__device__ __forceinline__ void write_empty(const Attend& a, u32 t0, u32 t1) {
    const u32 pieces = a.c.dim / 8;
    const u64 n = (u64)(t1 - t0) * a.heads * pieces;
    for (u64 i = threadIdx.x; i < n; i += blockDim.x) {
        const u32 at = (u32)(i % pieces) * 8, head = (u32)(i / pieces % a.heads), t = t0 + (u32)(i / pieces / a.heads);
        *(uint4*)((uint16_t*)a.out + (int64_t)t * a.o_ts + (int64_t)head * a.o_hs + at) = make_uint4(0, 0, 0, 0);
        if (at == 0) {
            if (a.lse) a.lse[(u64)t * a.heads + head] = -INFINITY;
            if (a.joined) a.joined[(u64)t * a.heads + head] = make_int2(-1, -1);
        }
    }
}

// rows of a request, tokens that it holds (no more than its row of the table), and where its first new token stands: counted from all of its new
// tokens, also where the step has rows for some of them only
struct Span {
    u32 t0, tokens;
    int context, first;
};

__device__ __forceinline__ Span span_of(const Attend& a, u32 b) {
    Span s;
    const int32_t from = a.s.offsets[b], to = a.s.offsets[b + 1];
    s.t0 = min((u32)max(from, 0), a.s.tokens);
    const u32 end = max((u32)max(to, 0), s.t0);
    s.tokens = min(end, a.s.tokens) - s.t0;
    s.context = (int)min((u64)(u32)max(a.s.context[b], 0), (u64)a.s.max_pages * a.c.page_tokens);
    s.first = s.context - (int)(end - s.t0);
    return s;
}

// The first position that a row at `position` reads.  Positions are negative where a request holds fewer tokens than it has rows: such a row reads
// nothing, and position - window would leave 32 bits.
__device__ __forceinline__ int oldest_of(const Attend& a, int position) {
    return a.window && position >= 0 && (u32)position >= a.window ? position - (int)a.window + 1 : 0;
}

// zeros for tokens before the first request and behind the last one; this workgroup's part of them
__device__ __forceinline__ void write_padding(const Attend& a) {
    const u32 last = min((u32)max(a.s.offsets[a.s.requests], 0), a.s.tokens), first = min((u32)max(a.s.offsets[0], 0), last), pad = first + a.s.tokens - last;
    const u32 from = (u32)((u64)pad * blockIdx.x / gridDim.x), to = (u32)((u64)pad * (blockIdx.x + 1) / gridDim.x);
    if (from < min(to, first)) write_empty(a, from, min(to, first));
    if (max(from, first) < to) write_empty(a, max(from, first) - first + last, to - first + last);
}

// shapes of the kernels for few query rows to a key
constexpr u32 ROWS = 16;                  // query rows of a tile
constexpr u32 TILE = 32;                  // keys of a tile
constexpr u32 SPLIT_WAVES = 4;            // waves of a workgroup whose keys are a share of all,
constexpr u32 UNIT = SPLIT_WAVES * TILE;  // and keys of the smallest share

// What beginning and ending a piece costs, in units: shares count it, or workgroups with many short requests end last (64 requests of 300 to
// 12,000 tokens with 1, 2, 4, 8: 122, 117, 112, 117 us; heads of 64: 64, 57, 51, 54)
constexpr u32 PIECE = 4;

// workgroups of a CU: as many as its registers and LDS last for
constexpr u32 groups_per_cu(u32 width, int t) { return width > 128 ? 1 : width == 64 && t == 1 ? 3 : 2; }

u64 narrow_groups(const Attend& a);        // workgroups, where one reads all keys of its rows
template <int FMT, int C>
void launch_narrow(hipStream_t st, const Attend& a, int num_cu, bool whole);

}  // namespace pagkv
