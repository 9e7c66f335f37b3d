// Attention of many query rows over the same keys: pag_kv_attend for chunks of prompts and wide groups.
//
// The mathematics is that of pag_kv_narrow.h; what bounds it is different.  With 16 rows a tile a key is widened to 16-bit floats
// once for each of them, and the vector units are what a long chunk waits for.  Here four waves have 32 rows each, and 64 keys are
// widened once for all 128, into LDS: keys row by row, values transposed, in the order in which the scores leave the matrix unit,
// so that weights go back in from their registers as in the narrow kernel.  The next 64 keys are on their way from memory
// meanwhile.  Shares are counted in steps of 64 keys of the tiles' own causal lengths: tile j and the j-th from the end make a pair,
// and all pairs of a request are equally long, so that a share is found without adding up tiles.
// 4 chunks of 700 to 2,000 tokens that end at 2,500 to 9,000, 32 heads over 8 of 128 numbers: 540 us, 810 TFLOP/s, with the cap's tanh 640 us; a product of
// 8192 x 8192 x 8192 reaches 1,160.  The matrix units are busy for 40 % of it and the vector units for 50 %: in a wave scores, weights and values' products
// follow one another, and all waves meet every 64 keys, so that the two waves of a SIMD overlap in part only.  (No third wave: 250 of 256 registers are taken;
// the four-wave kernel for 72 to 128 numbers spills 8 to 17.)  Of 4 bits the same chunks take 555 and 696 us: a conversion and a scale for every two numbers, where 8-bit codes are widened two
// at a time without one.  (Two lanes with four numbers of four tokens each, rather than two of eight, make half as many scales, and take 15 us more: twice as many stores.)
#pragma once

#include <algorithm>

#include "pag_kv_attend.h"

namespace pagkv {
namespace {

constexpr u32 STEP = 64;                    // keys of a step, one block of 16 a wave to fetch

typedef float float16_t __attribute__((ext_vector_type(16)));

struct Tiles {
    Span s;
    u32 rows, count, pairs, pair_units, mid_units;
    u64 units;                              // of one key/value head
};

struct Range { int start, stop, p0, p1; u32 units; };

template <int NW>
__device__ __forceinline__ Range range_of(const Attend& a, const Span& s, u32 rows, u32 tile) {
    Range r;
    r.p0 = s.first + (int)(tile * (NW * WROWS) / a.group);
    r.p1 = s.first + (int)(min(tile * (NW * WROWS) + (NW * WROWS) - 1, rows - 1) / a.group);
    r.start = oldest_of(a, r.p0) & ~(int)(BLOCK - 1);
    r.stop = max(r.p1 + 1, r.start);
    r.units = max(((u32)(r.stop - r.start) + STEP - 1) / STEP, 1u);
    return r;
}

template <int NW>
__device__ __forceinline__ Tiles tiles_of(const Attend& a, u32 b) {
    Tiles t;
    t.s = span_of(a, b);
    t.rows = t.s.tokens * a.group;
    t.count = t.s.context ? (t.rows + (NW * WROWS) - 1) / (NW * WROWS) : 0;
    t.pairs = t.count / 2;
    t.mid_units = t.count & 1 ? range_of<NW>(a, t.s, t.rows, t.pairs).units : 0;
    // no pair is longer: two ends of tiles that lie opposite add up to the same, and each is rounded up once
    u64 most = (2 * (u64)max(t.s.first + 1, 0) + ((u64)(NW * WROWS) * (t.count ? t.count - 1 : 0) + 2 * ((NW * WROWS) - 1)) / a.group + 1) / STEP + 2;
    if (a.window) most = min(most, 2 * (((u64)a.window + ((NW * WROWS) - 1) / a.group + 1 + BLOCK - 1 + STEP - 1) / STEP));
    t.pair_units = (u32)max(most, (u64)2);
    t.units = (u64)t.pairs * t.pair_units + t.mid_units;
    return t;
}

// halves of a row of keys, in pieces of 8; of a row of values (64 tokens of a number), likewise.  Rows that a wave reads together lie in
// different banks.
template <int C>
__device__ __forceinline__ u32 key_at(u32 token, u32 piece) {
    const u32 turn = C % 2 ? token >> 1 & 7u : token & (C == 2 ? 15u : 7u);
    return token * (64 * C) + (piece ^ turn) * 8;
}

__device__ __forceinline__ u32 value_at(u32 d, u32 piece) { return d * STEP + (piece ^ (d >> 2 & 7u) ^ (d & 2u)) * 8; }

// What a thread fetches of the next 64 keys.  NW waves share them, NW / 4 of them a block of 16: 64 C / NW bytes of a key, and words of eight
// tokens' values.  With four waves a word's four numbers are one lane's, with eight two lanes have the same word and two numbers each.
template <int C, int NW>
struct Share {
    static constexpr int PIECES = 8 * C / NW;            // of 8 numbers of a key
    static constexpr int N = (32 * C + 63) / 64;         // words of values a lane has at most
    static constexpr int COLUMNS = 16 / NW;              // numbers of a word
};

template <int FMT, int C, int NW>
struct Fetch : Share<C, NW> {
    uint2 k[Share<C, NW>::PIECES];
    u32 v[Share<C, NW>::N][8];
};

// 4-bit codes: half as wide, with the exponents of their parts; a part is four pieces, and two pieces that begin at an even number lie in one
template <int C, int NW>
struct Fetch<PAG_KV_FP4, C, NW> : Share<C, NW> {
    static constexpr int PARTS = Share<C, NW>::PIECES % 4 ? (Share<C, NW>::PIECES + 1) / 2 : Share<C, NW>::PIECES / 4, EACH = (Share<C, NW>::PIECES + PARTS - 1) / PARTS;
    u32 k[Share<C, NW>::PIECES];
    int ke[PARTS];
    u32 v[Share<C, NW>::N][8];
    u32 ve[Share<C, NW>::N][2];                          // of the word's first four tokens and its last four
};

// bytes first and first + 1 of eight words: columns of eight tokens
template <int FMT>
__device__ __forceinline__ void two_columns(const u32* w, u32 first, half8_t* out) {
    if constexpr (FMT == PAG_KV_INT8) {
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            const u32 pick = 0x0c040c00u + 0x00010001u * (first + c);
            half2_t h[4];
#pragma unroll
            for (int p = 0; p < 4; ++p) h[p] = widen_int8(perm(w[2 * p + 1], w[2 * p], pick));
            out[c] = half8_t{ h[0].x, h[0].y, h[1].x, h[1].y, h[2].x, h[2].y, h[3].x, h[3].y };
        }
    } else {
        const u32 pick = 0x05010400u + 0x02020202u * (first / 2);
        u32 t[2][2];
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const u32 lo = perm(w[4 * q + 1], w[4 * q], pick), hi = perm(w[4 * q + 3], w[4 * q + 2], pick);
            t[q][0] = perm(hi, lo, 0x05040100);
            t[q][1] = perm(hi, lo, 0x07060302);
        }
#pragma unroll
        for (int c = 0; c < 2; ++c) out[c] = widen8<FMT>(t[0][c], t[1][c]);
    }
}

// two 4-bit codes, byte 0 of eight words, each word with a scale of its own: columns of eight tokens
__device__ __forceinline__ void two_columns_fp4(const u32 (&w)[8], const float (&scale)[8], half8_t* out) {
    u32 lo[4], hi[4];
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        const u32 x = __builtin_bit_cast(u32, widen2_fp4<0>(w[2 * p], scale[2 * p])), y = __builtin_bit_cast(u32, widen2_fp4<0>(w[2 * p + 1], scale[2 * p + 1]));
        lo[p] = perm(y, x, 0x05040100);
        hi[p] = perm(y, x, 0x07060302);
    }
    out[0] = __builtin_bit_cast(half8_t, make_uint4(lo[0], lo[1], lo[2], lo[3]));
    out[1] = __builtin_bit_cast(half8_t, make_uint4(hi[0], hi[1], hi[2], hi[3]));
}

// What far_sum looks at: a piece's keys and this lane's row.
struct FarRows {
    const uint8_t* data;
    const int8_t* exponents;
    const int32_t* table;
    const uint16_t* q;                      // row lane % 32; null: no such row
    u32 dim, dtype, page_blocks, kv_heads, kv_head, page_tokens, num_pages;
    int start, stop, position, oldest;
    float scale, cap, slope, M;
};

__device__ __forceinline__ FarRows far_rows(const Attend& a, const int32_t* table, u32 kv_head, const uint16_t* q, int start, int stop, int position, float slope, float M) {
    return FarRows{ a.c.data, a.c.exponents, table, q, a.c.dim, a.dtype, a.c.page_blocks, a.c.kv_heads, kv_head, a.c.page_tokens, a.c.num_pages,
                    start, stop, position, oldest_of(a, position), a.scale, a.softcap, slope, M };
}

// This lane's part, every other four keys, of the sum of 2^(score log2 e - M) over keys start .. stop - 1, straight from memory: for
// pieces with values' exponents above FAR_EXPONENT.  A call of its own: with this code, or a sum of its own, in a kernel's loop the loop's
// registers are shared out otherwise (4 chunks of 700 to 2,000 tokens, heads of 64: 455 -> 471 us, with the call 456 to 462).
template <int FMT, int C>
__device__ __attribute__((noinline)) float far_sum(FarRows r) {
    constexpr u32 W = 64 * C;
    const u32 lane = threadIdx.x & 63, col = lane & 31, hi = lane >> 5;
    const auto numbers = [&](int n, float* x) {
        if (r.q && n * 16 + hi * 8 < r.dim) return load8(r.q, n * 16 + hi * 8, r.dtype, x);
        for (int j = 0; j < 8; ++j) x[j] = 0.f;
    };
    float x[8], most = 0.f;
    for (int n = 0; n < 4 * C; ++n) {
        numbers(n, x);
        for (int j = 0; j < 8; ++j) most = fmaxf(most, fabsf(x[j]));
    }
    most = fmaxf(most, __shfl_xor(most, 32));
    const int up = min(max((int)(__float_as_uint(most) >> 23) - 127 - 7, -100), 100);       // as the loop's rows
    const float down = power(-up), factor = r.scale * power(up) * LOG2E, cap = r.cap * LOG2E;
    float sum = 0.f;
    for (int from = r.start; from < r.stop; from += 32) {
        const int first = from + (int)(col & BLOCK);
        const u32 page = first < r.stop ? (u32)r.table[(u32)first / BLOCK / r.page_blocks] : 0xFFFFFFFFu;
        const bool ok = page < r.num_pages;
        const u32 row = ok ? (page * r.kv_heads + r.kv_head) * r.page_tokens + (u32)first / BLOCK % r.page_blocks * BLOCK : 0;
        // of 4-bit codes e is the key's own: the largest of its parts'
        int e = 0;
        const int8_t* parts = r.exponents + (u64)(row / BLOCK) * (4 * C * BLOCK) + (col & (BLOCK - 1));
        if constexpr (FMT == PAG_KV_FP4) {
            e = LOWEST_EXPONENT;
            for (int b = 0; b < 2 * C; ++b) e = max(e, (int)parts[b * BLOCK]);
        } else {
            e = ok ? r.exponents[(u64)(row / BLOCK) * 2] : 0;
        }
        const u64 there = __ballot(ok);
        const uint8_t* k = r.data + (u64)(row + (col & (BLOCK - 1))) * (2 * row_bytes<FMT, C>()) + hi * (FMT == PAG_KV_FP4 ? 4 : 8);
        float16_t S;
#pragma unroll
        for (int i = 0; i < 16; ++i) S[i] = 0.f;
        for (int n = 0; n < 4 * C; ++n) {
            half8_t q, key;
            if constexpr (FMT == PAG_KV_FP4) {
                key = widen8_fp4(*(const u32*)(k + 8 * n), power((int)parts[n / 2 * BLOCK]) * power(-e));
            } else {
                const uint2 codes = *(const uint2*)(k + 16 * n);
                key = widen8<FMT>(codes.x, codes.y);
            }
            numbers(n, x);
#pragma unroll
            for (int j = 0; j < 8; ++j) q[j] = (_Float16)(x[j] * down);
            S = __builtin_amdgcn_mfma_f32_32x32x16_f16(key, q, S, 0, 0, 0);
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int key = from + 8 * (i >> 2) + 4 * (int)hi + (i & 3);
            const int e_of = FMT == PAG_KV_FP4 ? __shfl(e, 8 * (i >> 2) + 4 * (int)hi + (i & 3)) : __builtin_amdgcn_readlane(e, (i >> 3) * (int)BLOCK);
            float t = S[i] * (factor * power(e_of));
            if (r.cap > 0.f) t = capped(t, cap, 1.f / cap);
            t -= r.slope * (float)(r.position - key);
            if ((there >> ((i >> 3) * BLOCK) & 1u) && key <= r.position && key >= r.oldest) sum += __builtin_amdgcn_exp2f(t - r.M);
        }
    }
    return sum;
}

// CAP: 0 none, 1 up to NEAR_CAP, 2 above it
template <int FMT, int C, int CAP, int NW>
__global__ void __launch_bounds__(64 * NW, C <= 2 ? 2 : 1) k_attend_wide(Attend a, Head* heads) {
    constexpr u32 W = 64 * C, KEYS = STEP * W, VALUES = W * STEP;
    constexpr int KEY_TURNS = C == 2 ? 7 : 3;             // which pairs of pieces trade places in key_at
    extern __shared__ __align__(16) _Float16 lds[];       // two buffers of keys and values
    __shared__ float sh_scale[2][4][2];                   // 2^e of the keys' block, e of the values'
    __shared__ u32 sh_there[2][4];
    __shared__ u32 sh_far[2];                             // this piece, and the next: a block's values have an e above FAR_EXPONENT
    __shared__ u64 sh_sum[NW];
    __shared__ u64 sh_begin;
    __shared__ u32 sh_b;
    const u32 lane = threadIdx.x & 63, wave = wave_of(), col = lane & 31, hi = lane >> 5;

    // Workgroups go to the chip's parts (each with an L2 of its own) in turn; neighbouring shares, which read the same keys, go to one part
    const u32 self = gridDim.x % 8 ? blockIdx.x : blockIdx.x % 8 * (gridDim.x / 8) + blockIdx.x / 8;

    // this workgroup's share
    const u32 per = (a.s.requests + 64 * NW - 1) / (64 * NW), b0 = min(threadIdx.x * per, a.s.requests), b1 = min(b0 + per, a.s.requests);
    u64 mine = 0;
    for (u32 b = b0; b < b1; ++b) mine += tiles_of<NW>(a, b).units * a.c.kv_heads;
    u64 upto = mine;
#pragma unroll
    for (u32 o = 1; o < 64; o <<= 1) {
        const u64 y = __shfl_up(upto, o);
        if (lane >= o) upto += y;
    }
    if (lane == 63) sh_sum[wave] = upto;
    __syncthreads();
    u64 total = 0;
    for (u32 x = 0; x < NW; ++x) {
        if (x < wave) upto += sh_sum[x];
        total += sh_sum[x];
    }
    const u32 parts = (u32)min((u64)gridDim.x, total);
    const u64 begin = self < parts ? share(total, parts, self) : total, end = self < parts ? share(total, parts, self + 1) : total;
    if (begin < end && begin >= upto - mine && begin < upto) {
        u64 before = upto - mine;
        u32 b = b0;
        for (;; ++b) {
            const u64 n = tiles_of<NW>(a, b).units * a.c.kv_heads;
            if (begin < before + n) break;
            before += n;
        }
        sh_b = b;
        sh_begin = before;
    }
    for (u32 b = self; b < a.s.requests; b += gridDim.x) {
        const Span s = span_of(a, b);
        if (s.tokens && !s.context) write_empty(a, s.t0, s.t0 + s.tokens);
    }
    write_padding(a);
    if (threadIdx.x == 0) {
        heads[self].last = -1;
        sh_far[0] = sh_far[1] = 0;
    }
    if (begin >= end) return;
    __syncthreads();
    u32 b = sh_b;
    u64 before = sh_begin, at = begin;
    u32 turn = 0;                                           // of sh_far
    Tiles q = tiles_of<NW>(a, b);

    while (at < end) {
        while (at >= before + q.units * a.c.kv_heads) {
            before += q.units * a.c.kv_heads;
            ++b;
            q = tiles_of<NW>(a, b);
        }
        const u32 kv_head = (u32)((at - before) / q.units);
        const u64 in = (at - before) % q.units;
        u32 tile, u0, skip = 0;
        Range r;
        if (in >= (u64)q.pairs * q.pair_units) {
            tile = q.pairs;
            u0 = (u32)(in - (u64)q.pairs * q.pair_units);
            r = range_of<NW>(a, q.s, q.rows, tile);
        } else {
            const u32 pair = (u32)(in / q.pair_units);
            u0 = (u32)(in % q.pair_units);
            tile = q.count - 1 - pair;                      // the longer one first
            r = range_of<NW>(a, q.s, q.rows, tile);
            if (u0 >= r.units) {
                u0 -= r.units;
                tile = pair;
                r = range_of<NW>(a, q.s, q.rows, tile);
                if (u0 >= r.units) skip = (u32)(q.pair_units - in % q.pair_units);
            }
        }
        if (skip) {                                         // what the pair was rounded up by
            at += skip;
            continue;
        }
        const u32 u1 = (u32)min((u64)r.units, u0 + (end - at));
        const int start = r.start + (int)(u0 * STEP), stop = min(r.stop, start + (int)((u1 - u0) * STEP));

        // this wave's rows
        const u32 row = tile * (NW * WROWS) + wave * WROWS + col, token = row / a.group, head = kv_head * a.group + row % a.group;
        const bool real = row < q.rows;
        const int position = real ? q.s.first + (int)token : -1;
        const u32 w_row = tile * (NW * WROWS) + wave * WROWS;
        const bool busy = w_row < q.rows;                   // the wave has rows
        const int w_p0 = q.s.first + (int)(min(w_row, q.rows - 1) / a.group), w_p1 = q.s.first + (int)(min(w_row + WROWS - 1, q.rows - 1) / a.group);
        const int oldest = oldest_of(a, position);
        const int w_first = oldest_of(a, w_p0);
        const int w_full = oldest_of(a, w_p1);      // keys from here on are in the window of all rows
        const float slope = real && a.slopes ? a.slopes[head] * LOG2E : 0.f;

        half8_t Q[4 * C];                                   // numbers 16 n + 8 hi + 0 .. 7 in Q[n]
        float factor;
        {
            // scaled by a power of two, so that 16-bit floats hold it; two sweeps over the row rather than all of it in 32 bits
            float most = 0.f;
            const u64 from = (u64)(q.s.t0 + token) * (u64)a.q_ts + head * (u64)a.q_hs;
#pragma unroll
            for (int n = 0; n < 4 * C; ++n) {
                const u32 d = n * 16 + hi * 8;
                float x[8] = { 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f };
                if (real && d < a.c.dim) load8(a.q, from + d, a.dtype, x);
#pragma unroll
                for (int j = 0; j < 8; ++j) most = fmaxf(most, fabsf(x[j]));
            }
            most = fmaxf(most, __shfl_xor(most, 32));
            int e = (int)(__float_as_uint(most) >> 23) - 127 - 7;
            e = min(max(e, -100), 100);
            const float down = power(-e);
#pragma unroll
            for (int n = 0; n < 4 * C; ++n) {
                const u32 d = n * 16 + hi * 8;
                float x[8] = { 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f };
                if (real && d < a.c.dim) load8(a.q, from + d, a.dtype, x);
#pragma unroll
                for (int j = 0; j < 8; ++j) Q[n][j] = (_Float16)(x[j] * down);
            }
            factor = a.scale * power(e);
        }
        float M = LOWEST, sum = 0.f;
        float16_t acc[2 * C];
#pragma unroll
        for (int n = 0; n < 2 * C; ++n) {
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[n][i] = 0.f;
        }

        const int32_t* table = a.s.table + b * a.s.table_stride;
        // this wave's blocks of the next 64 steps, a lane each; NW / 4 waves share one
        const u32 block = wave / (NW / 4), part = wave % (NW / 4);
        u32 block_row = 0;
        int ek_mine = 0, ev_mine = 0;
        u64 there = 0;
        u64 far = 0;
        const auto look_up = [&](int from) {
            const int at_key = from + (int)(lane * STEP + block * BLOCK);
            bool ok = false;
            block_row = 0;
            ek_mine = ev_mine = 0;
            if (at_key < stop) {
                const u32 blk = (u32)at_key / BLOCK, page = (u32)table[blk / a.c.page_blocks];
                if (page < a.c.num_pages) {
                    ok = true;
                    block_row = row_of(a.c, page, kv_head, blk % a.c.page_blocks * BLOCK);
                    if constexpr (FMT == PAG_KV_FP4) {
                        Parts<C> parts;
                        load_parts<C>(parts_of<C>(a.c, block_row / BLOCK, 0), parts);
                        ek_mine = most_of_parts<C>(parts, stop - at_key);
                        load_parts<C>(parts_of<C>(a.c, block_row / BLOCK, 1), parts);
                        ev_mine = most_of_parts<C>(parts, stop - at_key);
                    } else {
                        const int8_t* e = a.c.exponents + (u64)(block_row / BLOCK) * 2;
                        ek_mine = e[0];
                        ev_mine = e[1];
                    }
                }
            }
            there = __ballot(ok);
        };
        Fetch<FMT, C, NW> f;
        const u32 key = part * (64 / NW) + lane / NW, key_piece0 = lane % NW * Share<C, NW>::PIECES;
        const auto word_of = [&](int i, u32& word, u32& half, u32& first) -> bool {
            const u32 item = lane + 64 * i;
            if (NW == 4) {
                word = item % (16 * C); half = item / (16 * C); first = 0;
                return half < 2;
            }
            word = item / 2; half = part; first = item % 2 * 2;
            return word < 16 * C;
        };
        const auto fetch = [&](u32 n) {
            if constexpr (FMT == PAG_KV_FP4) {
                typedef Fetch<FMT, C, NW> F;
                const u32 row = (u32)__builtin_amdgcn_readlane((int)block_row, (int)(n & 63));
                const uint8_t *rows = a.c.data + (u64)row * W, *k = rows + key * W + key_piece0 * 4;
                const int8_t *ke = parts_of<C>(a.c, row / BLOCK, 0) + key, *ve = parts_of<C>(a.c, row / BLOCK, 1);
                if constexpr (F::PIECES % 4 == 0) {
#pragma unroll
                    for (int i = 0; i < F::PIECES; i += 4) {
                        const uint4 x = *(const uint4*)(k + 4 * i);
                        f.k[i] = x.x; f.k[i + 1] = x.y; f.k[i + 2] = x.z; f.k[i + 3] = x.w;
                    }
                } else if constexpr (F::PIECES % 2 == 0) {
#pragma unroll
                    for (int i = 0; i < F::PIECES; i += 2) {
                        const uint2 x = *(const uint2*)(k + 4 * i);
                        f.k[i] = x.x; f.k[i + 1] = x.y;
                    }
                } else {
                    f.k[0] = *(const u32*)k;
                }
#pragma unroll
                for (int i = 0; i < F::PARTS; ++i) f.ke[i] = ke[(key_piece0 + F::EACH * i) / 4 * BLOCK];
#pragma unroll
                for (int i = 0; i < F::N; ++i) {
                    u32 word, half, first;
                    if (word_of(i, word, half, first)) {
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            const uint8_t* p = rows + (8 * (j >> 2) + 4 * half + (j & 3)) * W + W / 2 + word * 2;
                            f.v[i][j] = NW == 4 ? *(const uint16_t*)p : p[first / 2];
                        }
#pragma unroll
                        for (int j = 0; j < 2; ++j) f.ve[i][j] = *(const u32*)(ve + word / 8 * BLOCK + 8 * j + 4 * half);
                    }
                }
                return;
            } else {
            const uint8_t* rows = a.c.data + (u64)(u32)__builtin_amdgcn_readlane((int)block_row, (int)(n & 63)) * (2 * W);
            const uint8_t* k = rows + key * (2 * W) + key_piece0 * 8;
#pragma unroll
            for (int i = 0; i < Share<C, NW>::PIECES; ++i) f.k[i] = *(const uint2*)(k + 8 * i);
#pragma unroll
            for (int i = 0; i < Share<C, NW>::N; ++i) {
                u32 word, half, first;
                if (word_of(i, word, half, first)) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) f.v[i][j] = *(const u32*)(rows + (8 * (j >> 2) + 4 * half + (j & 3)) * (2 * W) + W + word * 4);
                }
            }
            }
        };
        const auto stage = [&](u32 n, int from, u32 buffer) {
            _Float16* keys = lds + buffer * (KEYS + VALUES);
            _Float16* values = keys + KEYS;
            const int ek_most = __builtin_amdgcn_readlane(ek_mine, (int)(n & 63)), ev_most = __builtin_amdgcn_readlane(ev_mine, (int)(n & 63));
            if constexpr (FMT == PAG_KV_FP4) {
                if (ek_most > MOST_PLAIN || ev_most > MOST_PLAIN) {
#pragma unroll
                    for (int i = 0; i < Fetch<FMT, C, NW>::PARTS; ++i) f.ke[i] = max(f.ke[i], ek_most - 127);
#pragma unroll
                    for (int i = 0; i < Share<C, NW>::N; ++i) {
                        f.ve[i][0] = raised_bytes(f.ve[i][0], ev_most - 127);
                        f.ve[i][1] = raised_bytes(f.ve[i][1], ev_most - 127);
                    }
                }
            }
#pragma unroll
            for (int i = 0; i < Share<C, NW>::PIECES; ++i) {
                half8_t wide;
                if constexpr (FMT == PAG_KV_FP4) wide = widen8_fp4(f.k[i], power_less(f.ke[i / Fetch<FMT, C, NW>::EACH], less_of(ek_most)));
                else wide = widen8<FMT>(f.k[i].x, f.k[i].y);
                *(half8_t*)(keys + key_at<C>(block * BLOCK + key, key_piece0 + i)) = wide;
            }
            const bool ok = there >> (n & 63) & 1;
            const int base = from + (int)(block * BLOCK);
#pragma unroll
            for (int i = 0; i < Share<C, NW>::N; ++i) {
                u32 word, half, first;
                if (word_of(i, word, half, first)) {
                    half8_t v[4];
                    if constexpr (FMT == PAG_KV_FP4) {
                        float scale[8];
                        powers_of_bytes(f.ve[i][0], less_of(ev_most), scale);
                        powers_of_bytes(f.ve[i][1], less_of(ev_most), scale + 4);
                        if (!ok || base + (int)BLOCK > stop) {
#pragma unroll
                            for (int j = 0; j < 8; ++j)
                                if (!ok || base + (int)(8 * (j >> 2) + 4 * half + (j & 3)) >= stop) scale[j] = 0.f;
                        }
                        if constexpr (NW == 4) columns_fp4<0>(f.v[i], scale, v);
                        else two_columns_fp4(f.v[i], scale, v);
                    } else {
                        if (!ok || base + (int)BLOCK > stop) {      // the memory behind the last token may hold anything
#pragma unroll
                            for (int j = 0; j < 8; ++j)
                                if (!ok || base + (int)(8 * (j >> 2) + 4 * half + (j & 3)) >= stop) f.v[i][j] = 0;
                        }
                        if constexpr (NW == 4) columns<FMT>(f.v[i], v);
                        else two_columns<FMT>(f.v[i], first, v);
                    }
#pragma unroll
                    for (int c = 0; c < Share<C, NW>::COLUMNS; ++c) *(half8_t*)(values + value_at(word * 4 + first + c, block * 2 + half)) = v[c];
                }
            }
            if (lane == 0 && part == 0) {
                sh_scale[buffer][block][0] = power(ek_most);
                sh_scale[buffer][block][1] = (float)ev_most;
                sh_there[buffer][block] = ok && base < stop ? 1u : 0u;
            }
        };

        // where this lane's pieces of keys and values lie: the piece's number turns bits of the address, the token's or number's group adds to it
        const u32 k_lds = key_at<C>(col, hi) * 2, v_lds = value_at(col, hi) * 2;
        const u32 steps = (u32)(max(stop - start, 0) + (int)STEP - 1) / STEP;
        __syncthreads();                                        // the piece before has been read
        if (threadIdx.x == 0) sh_far[turn ^ 1] = 0;
        // step n + 1 into LDS, and step n + 2 on its way
        const auto prepare = [&](u32 n) {
            if (n + 1 < steps) stage(n + 1, start + (int)((n + 1) * STEP), (n + 1) & 1);
            if (n + 2 < steps) {
                if (((n + 2) & 63) == 0) {
                    far |= __ballot(ev_mine > FAR_EXPONENT);
                    look_up(start + (int)((n + 2) * STEP));
                }
                fetch(n + 2);
            }
        };
        // Two waves of eight are on a SIMD: one widens the next keys before its products, the other after them, so that one has the vector unit
        // while the other has the matrix unit (4 chunks of 700 to 2,000 tokens 547 us with all of them after, this way 536; 8-bit integers 590, 567).
        const bool early = NW == 8 && wave >= 4;
        if (steps) {
            look_up(start);
            fetch(0);
            stage(0, start, 0);
            if (steps > 1) fetch(1);
        }
        __syncthreads();
        for (u32 n = 0; n < steps; ++n) {
            const int from = start + (int)(n * STEP);
            const u32 buffer = n & 1;
            if (early) prepare(n);
            if (busy && from <= w_p1 && from + (int)STEP > w_first) {
                const char* keys = (const char*)(lds + buffer * (KEYS + VALUES));
                const char* values = keys + KEYS * 2;
                float ek[4], ev[4];
                u32 found = 0;
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    ek[x] = sh_scale[buffer][x][0];
                    ev[x] = sh_scale[buffer][x][1];
                    found |= sh_there[buffer][x] << x;
                }
                // Both halves' scores are under way before the first of them is used: the matrix unit works on one half while the vector unit has
                // the other.  Pieces are asked for AHEAD of their products; left alone, the compiler asks for each right before it, to save
                // registers, and a product then waits for LDS every time (4 chunks of 700 to 2,000 tokens with a cap
                // 735 us, with this order 715; 256 numbers a head 957 and 854).
                constexpr int AHEAD = 4, PRODUCTS = 8 * C;
                const auto key_piece = [&](int n) {
                    const int h = n / (4 * C), i = n % (4 * C);
                    return *(const half8_t*)(keys + (k_lds ^ (i & KEY_TURNS) * 32) + (i & ~KEY_TURNS) * 32 + h * (32 * W * 2));
                };
                float16_t S[2];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) S[h][i] = 0.f;
                }
                {
                    half8_t piece[AHEAD];
#pragma unroll
                    for (int n = 0; n < AHEAD; ++n) piece[n] = key_piece(n);
                    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                    for (int n = 0; n < PRODUCTS; ++n) {
                        S[n / (4 * C)] = __builtin_amdgcn_mfma_f32_32x32x16_f16(piece[n % AHEAD], Q[n % (4 * C)], S[n / (4 * C)], 0, 0, 0);
                        if (n + AHEAD < PRODUCTS) piece[n % AHEAD] = key_piece(n + AHEAD);
                        __builtin_amdgcn_sched_barrier(0);
                    }
                }
                const bool masked = found != 15u || from + (int)STEP > w_p0 + 1 || from < w_full;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const auto value_piece = [&](int n) { return *(const half8_t*)(values + (v_lds ^ (2 * h + n / (2 * C)) * 32) + n % (2 * C) * (32 * STEP * 2)); };
                    half8_t piece[AHEAD];
#pragma unroll
                    for (int n = 0; n < (AHEAD < 4 * C ? AHEAD : 4 * C); ++n) piece[n] = value_piece(n);
                    // key 32 h + 8 (i / 4) + 4 hi + i % 4 in S[h][i]; i / 8 is its block's half.  S becomes the weights' exponents.
                    const float base = M == LOWEST ? 0.f : M;
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        if constexpr (CAP == 2) {
                            const float by = factor * LOG2E * ek[2 * h + x], add = ev[2 * h + x] - base, cap = a.softcap * LOG2E, per = 1.f / cap;
#pragma unroll
                            for (int i = 8 * x; i < 8 * x + 8; ++i) S[h][i] = capped(S[h][i] * by, cap, per) + add;
                        } else if constexpr (CAP == 1) {
                            const float by = 2.f * LOG2E * factor / a.softcap * ek[2 * h + x], cap = a.softcap * LOG2E, top = cap + (ev[2 * h + x] - base);
#pragma unroll
                            for (int i = 8 * x; i < 8 * x + 8; ++i)
                                S[h][i] = __builtin_fmaf(-2.f * cap, __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(S[h][i] * by)), top);
                        } else {
                            const float by = factor * LOG2E * ek[2 * h + x], add = ev[2 * h + x] - base;
#pragma unroll
                            for (int i = 8 * x; i < 8 * x + 8; ++i) S[h][i] = __builtin_fmaf(S[h][i], by, add);
                        }
                    }
                    if (a.slopes) {
#pragma unroll
                        for (int i = 0; i < 16; ++i) S[h][i] -= slope * (float)(position - (from + h * 32 + 8 * (i >> 2) + 4 * (int)hi + (i & 3)));
                    }
                    if (masked) {
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const int k = from + h * 32 + 8 * (i >> 2) + 4 * (int)hi + (i & 3);
                            if (!(found >> (2 * h + (i >> 3)) & 1u) || k > position || k < oldest) S[h][i] = -INFINITY;
                        }
                    }
                    float most = fmaxf(S[h][0], S[h][1]);
#pragma unroll
                    for (int i = 2; i < 16; ++i) most = fmaxf(most, S[h][i]);
                    if (__ballot(most > (M == LOWEST ? LOWEST : HEADROOM))) {
                        most = fmaxf(most, __shfl_xor(most, 32));
                        if (most > (M == LOWEST ? LOWEST : HEADROOM)) {
                            const float up = most - START, to = base + up, alpha = __builtin_amdgcn_exp2f(M - to);
#pragma unroll
                            for (int i = 0; i < 16; ++i) S[h][i] -= up;
                            sum *= alpha;
#pragma unroll
                            for (int d = 0; d < 2 * C; ++d) acc[d] *= alpha;
                            M = to;
                        }
                    }
                    half8_t P[2];
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        float part = 0.f;
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            const float y = __builtin_amdgcn_exp2f(S[h][8 * x + i]);
                            part = i ? part + y : y;
                            P[x][i] = (_Float16)y;
                        }
                        sum = __builtin_fmaf(part, power(-(int)ev[2 * h + x]), sum);
                    }
                    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                    for (int n = 0; n < 4 * C; ++n) {
                        acc[n % (2 * C)] = __builtin_amdgcn_mfma_f32_32x32x16_f16(piece[n % AHEAD], P[n / (2 * C)], acc[n % (2 * C)], 0, 0, 0);
                        if (n + AHEAD < 4 * C) piece[n % AHEAD] = value_piece(n + AHEAD);
                        __builtin_amdgcn_sched_barrier(0);
                    }
                }
            }
            if (!early) prepare(n);
            lds_barrier();
        }

        if (far | __ballot(ev_mine > FAR_EXPONENT)) sh_far[turn] = 1;
        lds_barrier();
        if (__builtin_amdgcn_readfirstlane((int)sh_far[turn])) {
            const uint16_t* row_at = real ? (const uint16_t*)a.q + (int64_t)(q.s.t0 + token) * a.q_ts + (int64_t)head * a.q_hs : nullptr;
            sum = far_sum<FMT, C>(far_rows(a, table, kv_head, row_at, start, busy ? min(stop, w_p1 + 1) : start, position, slope, M));
        }
        turn ^= 1;
        sum += __shfl_xor(sum, 32);
        const bool begun = u0 == 0, ended = u1 == r.units;
        if (begun && ended) {
            if (real) {
                const float by = sum != 0.f ? 1.f / sum : 0.f;
                uint16_t* out = (uint16_t*)a.out + (int64_t)(q.s.t0 + token) * a.o_ts + (int64_t)head * a.o_hs;
#pragma unroll
                for (int n = 0; n < 2 * C; ++n) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const u32 d = n * 32 + 8 * i + 4 * hi;
                        if (d < a.c.dim)
                            *(uint2*)(out + d) = make_uint2(pack2(finite(acc[n][4 * i] * by), finite(acc[n][4 * i + 1] * by), a.dtype),
                                                               pack2(finite(acc[n][4 * i + 2] * by), finite(acc[n][4 * i + 3] * by), a.dtype));
                    }
                }
                if (a.lse && hi == 0) a.lse[(u64)(q.s.t0 + token) * a.heads + head] = sum != 0.f ? LN2 * (M + __builtin_amdgcn_logf(sum)) : -INFINITY;
            }
        } else {
            float* partial = a.partial + (2 * (u64)self + (begun ? 1 : 0)) * ((NW * WROWS) * (W + 2));
            const u32 r_here = wave * WROWS + col;
            if (hi == 0) { partial[r_here] = M; partial[(NW * WROWS) + r_here] = sum; }
#pragma unroll
            for (int n = 0; n < 2 * C; ++n) {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    *(float4*)(partial + 2 * (NW * WROWS) + r_here * W + n * 32 + 8 * i + 4 * hi) = make_float4(acc[n][4 * i], acc[n][4 * i + 1], acc[n][4 * i + 2], acc[n][4 * i + 3]);
            }
            if (begun && threadIdx.x == 0) {
                Head h;
                h.t0 = q.s.t0; h.rows = q.rows; h.row0 = tile * (NW * WROWS); h.head0 = kv_head * a.group;
                h.last = (int)(((at + r.units) * parts - 1) / total);       // the workgroup of the tile's last unit
                heads[self] = h;
            }
        }
        at += u1 - u0;
    }
}

// Adds up the pieces of a tile that several workgroups had: workgroup (y, g) the rows 4 y to 4 y + 3 of the tile that g began.  Its waves take
// every fourth piece, four of them asked for at a time (a request's 32 rows over 20,000 keys are in hundreds of pieces).  The rows come first in
// the grid: workgroups go to the chip's parts in turn, and the tiles that have pieces begin at every 64th workgroup where a few requests
// are as long as the rest of the chip's work, so that with g first one part alone adds up (both kernels, 128 rows over 30,000 keys: 89 us, this way 52).
template <int C, int NW>
__global__ void __launch_bounds__(256) k_join_wide(Attend a, const Head* heads) {
    constexpr u32 W = 64 * C, SLOT = (NW * WROWS) * (W + 2), N = 4 * C, THREADS = 16;      // numbers of a lane, lanes of a row
    __shared__ float sh_m[4][4], sh_s[4][4];
    __shared__ __align__(16) float sh_acc[4][4][W];
    const Head h = heads[blockIdx.y];
    if (h.last <= (int)blockIdx.y || h.last >= (int)gridDim.y) return;
    const u32 lane = threadIdx.x & 63, wave = wave_of(), r = lane / THREADS, row0 = blockIdx.x * 4, first = lane % THREADS * N;
    if (h.row0 + row0 >= h.rows) return;
    const int pieces = h.last - (int)blockIdx.y + 1;
    float M = LOWEST, sum = 0.f, acc[N];
#pragma unroll
    for (u32 n = 0; n < N; ++n) acc[n] = 0.f;
    for (int i = (int)wave; i < pieces; i += 16) {
        float m[4], s[4];
        float4 y[4][C];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int k = min(i + 4 * u, pieces - 1);
            const float* p = a.partial + (2 * ((u64)blockIdx.y + (u32)k) + (k == 0 ? 1 : 0)) * SLOT;
            m[u] = i + 4 * u < pieces ? p[row0 + r] : LOWEST;
            s[u] = p[(NW * WROWS) + row0 + r];
#pragma unroll
            for (int c = 0; c < C; ++c) y[u][c] = *(const float4*)(p + 2 * (NW * WROWS) + (row0 + r) * W + first + 4 * c);
        }
        float top = M;
#pragma unroll
        for (int u = 0; u < 4; ++u) top = fmaxf(top, m[u]);
        const float was = __builtin_amdgcn_exp2f(M - top);
        sum = add_scaled(0.f, sum, M - top);
#pragma unroll
        for (u32 n = 0; n < N; ++n) acc[n] *= was;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            if (i + 4 * u >= pieces) break;
            const float is = __builtin_amdgcn_exp2f(m[u] - top);
            sum = add_scaled(sum, s[u], m[u] - top);
#pragma unroll
            for (int c = 0; c < C; ++c) {
                acc[4 * c] = __builtin_fmaf(y[u][c].x, is, acc[4 * c]);
                acc[4 * c + 1] = __builtin_fmaf(y[u][c].y, is, acc[4 * c + 1]);
                acc[4 * c + 2] = __builtin_fmaf(y[u][c].z, is, acc[4 * c + 2]);
                acc[4 * c + 3] = __builtin_fmaf(y[u][c].w, is, acc[4 * c + 3]);
            }
        }
        M = top;
    }
    if (lane % THREADS == 0) { sh_m[wave][r] = M; sh_s[wave][r] = sum; }
#pragma unroll
    for (int c = 0; c < C; ++c) *(float4*)&sh_acc[wave][r][first + 4 * c] = make_float4(acc[4 * c], acc[4 * c + 1], acc[4 * c + 2], acc[4 * c + 3]);
    __syncthreads();
    // a wave a row
    const u32 row = h.row0 + row0 + wave;
    if (row >= h.rows) return;
    const float top = fmaxf(fmaxf(sh_m[0][wave], sh_m[1][wave]), fmaxf(sh_m[2][wave], sh_m[3][wave]));
    float by[4], all = 0.f;
#pragma unroll
    for (int x = 0; x < 4; ++x) {
        by[x] = __builtin_amdgcn_exp2f(sh_m[x][wave] - top);
        all = add_scaled(all, sh_s[x][wave], sh_m[x][wave] - top);
    }
    const u32 t = h.t0 + row / a.group, head = h.head0 + row % a.group;
    const float f = all != 0.f ? 1.f / all : 0.f;
    uint16_t* out = (uint16_t*)a.out + (int64_t)t * a.o_ts + (int64_t)head * a.o_hs;
    for (u32 d = 2 * lane; d < a.c.dim; d += 128) {
        float o[2] = { 0.f, 0.f };
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            o[0] = __builtin_fmaf(sh_acc[x][wave][d], by[x], o[0]);
            o[1] = __builtin_fmaf(sh_acc[x][wave][d + 1], by[x], o[1]);
        }
        *(u32*)(out + d) = pack2(finite(o[0] * f), finite(o[1] * f), a.dtype);
    }
    if (a.lse && lane == 0) a.lse[(u64)t * a.heads + head] = all != 0.f ? LN2 * (top + __builtin_amdgcn_logf(all)) : -INFINITY;
}

constexpr u32 lds_bytes(u32 width) { return 2 * 2 * STEP * width * 2; }

// Eight waves share a step's keys where there are rows for them, and registers: they are widened half as often.  Four and eight waves, in us: 4 chunks of
// 700 to 2,000 tokens 605, 587; 256 rows over 30,000 keys 70, 65; 32 requests of 256 rows over 3,000 keys 155, 140;
// where a request has up to 128 rows half of the waves have none (32 requests of 64 rows, 300 to 12,000 keys: 118, 165).
constexpr int MANY = (int)MANY_WAVES;

template <int FMT, int C, int CAP, int NW>
int run_wide(hipStream_t st, const Attend& a, int num_cu) {
    const u32 grid = (u32)num_cu * wide_groups_per_cu(64 * C, NW);
    Head* heads = (Head*)(a.partial + 2ull * grid * (NW * WROWS) * (64 * C + 2));
    if (lds_bytes(64 * C) >= 65536) {
        const hipError_t e = hipFuncSetAttribute((const void*)k_attend_wide<FMT, C, CAP, NW>, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds_bytes(64 * C));
        if (e != hipSuccess) { pag_set_error(std::string("hipFuncSetAttribute: ") + hipGetErrorString(e)); return PAG_EHIP; }
    }
    k_attend_wide<FMT, C, CAP, NW><<<grid, 64 * NW, lds_bytes(64 * C), st>>>(a, heads);
    k_join_wide<C, NW><<<dim3(NW * WROWS / 4, grid), 256, 0, st>>>(a, heads);
    return PAG_OK;
}

template <int FMT, int C, int CAP>
int run(hipStream_t st, const Attend& a, int num_cu) {
    if constexpr (C <= 2) {
        if (a.many_rows) return run_wide<FMT, C, CAP, MANY>(st, a, num_cu);
    }
    return run_wide<FMT, C, CAP, 4>(st, a, num_cu);
}

template <int FMT, int CAP>
int run_format(hipStream_t st, const Attend& a, int num_cu) {
    const u32 n = a.c.width / 64;
    if (n == 1) return run<FMT, 1, CAP>(st, a, num_cu);
    if (n == 2) return run<FMT, 2, CAP>(st, a, num_cu);
    if (n == 3) return run<FMT, 3, CAP>(st, a, num_cu);
    return run<FMT, 4, CAP>(st, a, num_cu);
}

}  // namespace

template <int FMT>
int launch_wide(hipStream_t st, const Attend& a, int num_cu) {
    return a.softcap > NEAR_CAP ? run_format<FMT, 2>(st, a, num_cu) : a.softcap > 0.f ? run_format<FMT, 1>(st, a, num_cu) : run_format<FMT, 0>(st, a, num_cu);
}

}  // namespace pagkv
