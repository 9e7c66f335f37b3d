// Attention over the cache: the kernels of pag_kv_attend for few query rows to a key, and of pag_kv_attend_selected.
//
// Rows of a token's heads that read the same keys (a group, and a request's neighbouring tokens) are taken 16 at a time, as the columns of
// a matrix product.  Per tile of 32 keys a wave computes S^T = K Q^T (the keys are rows: a lane ends up with 8 scores of one query row), the
// softmax weights of these scores, and O^T += V^T P^T.  The product's inner index may number the keys in any order that both operands
// share, so the weights are its second operand in the registers in which the scores came out, without an exchange between lanes,
// and each lane has its row's running maximum and scale beside that row's sums.
// The 8-bit codes are widened to 16-bit floats, which hold every code exactly; rows of Q are scaled by a power of two so that 16-bit floats
// hold them as well as the 16-bit input does.  Scales of the blocks are powers of two: the keys' multiply the scores, the
// values' are added to the weights' exponents.
// Weights are 2^(t - M) with t = score * log2 e + exponent of the values' block and M a running offset: the weights lie below
// 2^15 and M moves only when one would not, so that most tiles need no rescaling and no exchange between lanes.
// A workgroup's four waves take every fourth tile of its piece, and add up their sums in LDS.
// Work is split evenly over a fixed number of workgroups, in units of 128 keys, across requests of any lengths: each finds its share by
// one sum over the requests' lengths.  A row block whose keys went to several workgroups is joined by a second kernel.
// Bound by memory: 64 requests of 300 to 12,000 tokens, 8 heads of 128 numbers, 485 MB in 103 us with the joining, 400,000 tokens of one request 819 MB in
// 146 us with it (5.6 TB/s; a kernel that only reads reaches 6.0).  Up to 16 rows cost what one costs.
#pragma once

#include <algorithm>

#include "pag_kv_attend.h"

namespace pagkv {
namespace {

// a lane's part of 32 keys: of row lane % 16 of both halves the 16-byte pieces lane / 16 + 4 h, and of tokens 4 (lane / 16) + 0 .. 3
// of both halves the values' numbers 4 C (lane % 16) + 0 .. 4 C - 1
template <int FMT, int C>
struct Tile {
    uint4 k[2][C];
    u32 v[8][C];
};

// 4-bit codes: pieces of 16 bytes, one part each, where rows are a multiple of 64 bytes, and of 8 bytes otherwise
template <int C>
struct Tile<PAG_KV_FP4, C> {
    static constexpr int PIECES = C % 2 ? C : C / 2, WORDS = 2 * C / PIECES;       // of a lane's row of keys, words of a piece
    static constexpr int PARTS = C == 3 ? 3 : 1;                                   // parts that a lane's numbers of a row of values lie in
    u32 k[2][2 * C];
    u32 v[8][(C + 1) / 2];
    int ke[2][PIECES];         // exponents of the pieces' parts; of listed keys less their largest
    u32 ve[2][PARTS];          // of tokens 4 (lane / 16) + 0 .. 3
};

// the first number of eight that a lane with g = lane / 16 has of a row for its product number n
template <int FMT, int C>
__device__ __forceinline__ u32 number_of(int n, u32 g) {
    if constexpr (FMT == PAG_KV_FP4 && C % 2 == 0) return (n >> 2) * 128 + g * 32 + (n & 3) * 8;
    else return (n >> 1) * 64 + g * 16 + (n & 1) * 8;
}

template <int C>
__device__ __forceinline__ void load_words(const uint8_t* p, u32* w) {
    if constexpr (C == 1) {
        w[0] = *(const u32*)p;
    } else if constexpr (C == 2) {
        const uint2 x = *(const uint2*)p;
        w[0] = x.x; w[1] = x.y;
    } else if constexpr (C == 3) {
        const uint3 x = *(const uint3*)p;
        w[0] = x.x; w[1] = x.y; w[2] = x.z;
    } else {
        const uint4 x = *(const uint4*)p;
        w[0] = x.x; w[1] = x.y; w[2] = x.z; w[3] = x.w;
    }
}

// 4-bit codes: 2 C bytes of a row of values, at a multiple of 2 C, in the low ends of words
template <int C>
__device__ __forceinline__ void load_halves(const uint8_t* p, u32* w) {
    if constexpr (C == 1) {
        w[0] = *(const uint16_t*)p;
    } else if constexpr (C == 2) {
        w[0] = *(const u32*)p;
    } else if constexpr (C == 3) {
        // 6 bytes at 6 (lane % 16): of an odd lane behind two others in the 8 bytes that begin at a multiple of 4 (as three pieces of 2 bytes 64 ragged requests of
        // 192 numbers a row 147 us, this way 137)
        typedef u32 words __attribute__((ext_vector_type(2), aligned(4)));
        const u32 odd = threadIdx.x & 1;
        const words x = *(const words*)(p - 2 * odd);
        w[0] = __builtin_amdgcn_alignbit(x.y, x.x, 16 * odd);
        w[1] = x.y >> (16 * odd);
    } else {
        const uint2 x = *(const uint2*)p;
        w[0] = x.x; w[1] = x.y;
    }
}

// A lane's part of half a tile of 4-bit codes.  k: its first piece of its row of keys; v(j): its numbers of the values of token j of its 4
template <int C, typename V>
__device__ __forceinline__ void load_codes(Tile<PAG_KV_FP4, C>& tile, int s, const uint8_t* k, V&& v) {
    typedef Tile<PAG_KV_FP4, C> Tile4;
#pragma unroll
    for (int h = 0; h < Tile4::PIECES; ++h) {
        if constexpr (Tile4::WORDS == 4) {
            const uint4 x = *(const uint4*)(k + h * 64);
            tile.k[s][4 * h] = x.x; tile.k[s][4 * h + 1] = x.y; tile.k[s][4 * h + 2] = x.z; tile.k[s][4 * h + 3] = x.w;
        } else {
            const uint2 x = *(const uint2*)(k + h * 32);
            tile.k[s][2 * h] = x.x; tile.k[s][2 * h + 1] = x.y;
        }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) load_halves<C>(v(j), tile.v[4 * s + j]);
}

// parts of a lane's pieces of keys and numbers of values
template <int C>
__device__ __forceinline__ u32 key_part(int h, u32 g) { return C % 2 ? 2 * h + g / 2 : g + 4 * h; }
template <int C>
__device__ __forceinline__ u32 value_part(int w, u32 col) { return C == 3 ? (3 * col + w) / 8 : C * col / 8; }

// what a wave knows of its 16 rows and has summed up
template <int C>
struct Rows {
    half8_t q[2 * C];          // row lane % 16, numbers number_of(n, lane / 16) + 0 .. 7 in q[n]
    float factor;              // of this row: scale, and the power of two that q was divided by
    float slope;               // times log2 e
    int position;              // -1: no such row
    float M, sum;              // offset; this lane's part of the sum of 2^(score log2 e - M)
    float4_t acc[4 * C];       // [c][i]: number (4 (lane / 16) + i) * 4 C + c of row lane % 16
};

// which rows a workgroup works on
struct Where {
    u32 t0, rows, row0, head0, kv_head;      // first token, rows of the block's request and group, first row of this tile, first query head, its keys' head
};

// the numbers of row lane % 16 as they come
template <int C>
struct RawRows { uint4 x[2 * C]; };

template <int FMT, int C>
__device__ __forceinline__ void fetch_rows(const Attend& a, const Where& w, RawRows<C>& raw) {
    const u32 lane = threadIdx.x & 63, row = w.row0 + (lane & 15), g = lane >> 4;
    const u64 from = (u64)(w.t0 + row / a.group) * (u64)a.q_ts + (w.head0 + row % a.group) * (u64)a.q_hs;
#pragma unroll
    for (int n = 0; n < 2 * C; ++n) {
        const u32 at = number_of<FMT, C>(n, g);
        raw.x[n] = make_uint4(0, 0, 0, 0);
        if (row < w.rows && at < a.c.dim) raw.x[n] = *(const uint4*)((const uint16_t*)a.q + from + at);
    }
}

template <int C>
__device__ __forceinline__ void start_rows(const Attend& a, const Where& w, int first_position, const RawRows<C>& raw, Rows<C>& r) {
    const u32 lane = threadIdx.x & 63, row = w.row0 + (lane & 15);
    const bool real = row < w.rows;
    r.position = real ? first_position + (int)(row / a.group) : -1;
    r.slope = real && a.slopes ? a.slopes[w.head0 + row % a.group] * LOG2E : 0.f;
    float most = 0.f;
#pragma unroll
    for (int n = 0; n < 2 * C; ++n) {
        float x[8];
        widen_row8(raw.x[n], a.dtype, x);
#pragma unroll
        for (int j = 0; j < 8; ++j) most = fmaxf(most, fabsf(x[j]));
    }
    most = fmaxf(most, __shfl_xor(most, 16));
    most = fmaxf(most, __shfl_xor(most, 32));
    // the largest number of the row comes to lie between 2^7 and 2^8
    int e = (int)(__float_as_uint(most) >> 23) - 127 - 7;
    e = min(max(e, -100), 100);
    const float down = power(-e);
#pragma unroll
    for (int n = 0; n < 2 * C; ++n) {
        float x[8];
        widen_row8(raw.x[n], a.dtype, x);
#pragma unroll
        for (int j = 0; j < 8; ++j) r.q[n][j] = (_Float16)(x[j] * down);
    }
    r.factor = a.scale * power(e);
    r.M = LOWEST;
    r.sum = 0.f;
#pragma unroll
    for (int c = 0; c < 4 * C; ++c) r.acc[c] = float4_t{ 0.f, 0.f, 0.f, 0.f };
}

// What this lane's 8 keys are scaled by: 2^e of the keys, e of the values and 2^-e of the values (0 where the sum takes none, see FAR_EXPONENT).
// LISTED: every key has its own and its position; otherwise keys 0 .. 3 and 4 .. 7 share theirs, and at holds the first one's position
template <bool LISTED>
struct Scales {
    static constexpr int N = LISTED ? 8 : 2;
    float ek[N], ev[N], down[N];
    int at[N];
    int less[2][2];            // 4-bit codes: what power_less takes, of the keys and of the values of either half (of listed ones, whose exponents are relative, of 0)
};

// T tiles of rows against one of keys.  keep: bit j set if the row may read key j; looked at only if `masked`.  far: the
// sum takes weights without their values' scale.  SLOPES: of lists, whether the call has slopes; otherwise that is looked up.  CAPPED: by a cap above
// NEAR_CAP.  Both are kernels of their own: code that a call does not run lies between code that it does, and short calls wait for
// its fetch (one request of 500 tokens 10.1 us with the large caps' code, 9.6 without).
// BLOCKS: listed blocks of tokens.
template <int FMT, int C, int T, bool LISTED, bool SLOPES, bool CAPPED, bool BLOCKS = false>
__device__ __forceinline__ void add_tile(const Attend& a, const Tile<FMT, C>& tile, Rows<C> (&rows)[T], const Scales<LISTED>& x, bool masked, const u32 (&keep)[T], bool far) {
    float4_t s[T][2];
#pragma unroll
    for (int y = 0; y < T; ++y) s[y][0] = s[y][1] = float4_t{ 0.f, 0.f, 0.f, 0.f };
    if constexpr (FMT == PAG_KV_FP4) {
#pragma unroll
        for (int b = 0; b < 2; ++b) {
#pragma unroll
            for (int n = 0; n < 2 * C; ++n) {
                const half8_t k = widen8_fp4(tile.k[b][n], power_less(tile.ke[b][n / Tile<FMT, C>::WORDS], x.less[b][0]));
#pragma unroll
                for (int y = 0; y < T; ++y) s[y][b] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k, rows[y].q[n], s[y][b], 0, 0, 0);
            }
        }
    } else {
#pragma unroll
        for (int h = 0; h < C; ++h) {
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                const half8_t k0 = widen8<FMT>(tile.k[b][h].x, tile.k[b][h].y), k1 = widen8<FMT>(tile.k[b][h].z, tile.k[b][h].w);
#pragma unroll
                for (int y = 0; y < T; ++y) {
                    s[y][b] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k0, rows[y].q[2 * h], s[y][b], 0, 0, 0);
                    s[y][b] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k1, rows[y].q[2 * h + 1], s[y][b], 0, 0, 0);
                }
            }
        }
    }
    half8_t p[T];
#pragma unroll
    for (int y = 0; y < T; ++y) {
        Rows<C>& r = rows[y];
        // t = score * log2 e + e of the values - offset.  Listed keys may all be far away, slope * distance 10^5 and more, of which the distances from each
        // other are a small part: with slopes of lists the difference from the offset comes out of one rounding, before the score is added.
        constexpr bool APART = (LISTED || BLOCKS) && SLOPES;
        float t[8];
        const auto exponents = [&](float base) {
            if constexpr (CAPPED) {
                const float f = r.factor * LOG2E, cap = a.softcap * LOG2E, by = 1.f / cap;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int n = LISTED ? j : j >> 2;
                    t[j] = capped(s[y][j >> 2][j & 3] * (f * x.ek[n]), cap, by) + (APART ? 0.f : x.ev[n] - base);
                }
            } else if (a.softcap > 0.f) {
                // tanh(y) = 1 - 2 / (1 + e^(2 y))
                const float in = 2.f * LOG2E * r.factor / a.softcap, cap = a.softcap * LOG2E;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int n = LISTED ? j : j >> 2;
                    const float z = __builtin_amdgcn_exp2f(s[y][j >> 2][j & 3] * (in * x.ek[n]));
                    t[j] = __builtin_fmaf(-2.f * cap, __builtin_amdgcn_rcpf(1.f + z), cap + (APART ? 0.f : x.ev[n] - base));
                }
            } else {
                const float f = r.factor * LOG2E;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int n = LISTED ? j : j >> 2;
                    t[j] = __builtin_fmaf(s[y][j >> 2][j & 3], f * x.ek[n], APART ? 0.f : x.ev[n] - base);
                }
            }
            if constexpr (APART) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int distance = r.position - (LISTED ? x.at[LISTED ? j : 0] : x.at[j >> 2] + (j & 3));          // in two parts that a float holds
                    t[j] += __builtin_fmaf(-r.slope, (float)(distance & 4095), __builtin_fmaf(-r.slope, (float)(distance & ~4095), -base)) + x.ev[LISTED ? j : j >> 2];
                }
            } else if (!LISTED && a.slopes) {
#pragma unroll
                for (int j = 0; j < 8; ++j) t[j] -= r.slope * (float)(r.position - (x.at[LISTED ? 0 : j >> 2] + (j & 3)));
            }
            if (masked) {
#pragma unroll
                for (int j = 0; j < 8; ++j) t[j] = keep[y] >> j & 1u ? t[j] : -INFINITY;
            }
        };
        const auto largest = [&]() {
            float most = fmaxf(t[0], t[1]);
#pragma unroll
            for (int j = 2; j < 8; ++j) most = fmaxf(most, t[j]);
            return most;
        };
        const auto of_row = [&](float most) {
            most = fmaxf(most, __shfl_xor(most, 16));
            return fmaxf(most, __shfl_xor(most, 32));
        };
        const auto move = [&](float M) {
            const float alpha = __builtin_amdgcn_exp2f(r.M - M);
            r.sum = add_scaled(0.f, r.sum, r.M - M);
#pragma unroll
            for (int c = 0; c < 4 * C; ++c) r.acc[c] *= alpha;
            r.M = M;
        };
        const float base = r.M == LOWEST ? 0.f : r.M;
        exponents(base);
        float most = largest();
        if (__ballot(most > (r.M == LOWEST ? LOWEST : HEADROOM))) {
            most = of_row(most);
            // rows that need not move stay as they are: a row's result does not depend on its neighbours in the tile
            if (most > (r.M == LOWEST ? LOWEST : HEADROOM)) {
                const float up = most - START, M = base + up, by = APART ? M - base : up;
                move(M);
#pragma unroll
                for (int j = 0; j < 8; ++j) t[j] -= by;
                if constexpr (APART) {
                    // numbers of 512 and more were rounded to 2^-15 and more: once again, from the offset where it is now.  Beyond 2^20 the offset is
                    // off by that rounding itself and is put right first; beyond 2^28 its own is more than the weights have room for.
                    if (fabsf(up) > 512.f) {
                        exponents(r.M);
                        if (fabsf(r.M) > 0x1p20f) {
                            move(r.M + (of_row(largest()) - START));
                            exponents(r.M);
#pragma unroll
                            for (int j = 0; j < 8; ++j) t[j] = fminf(t[j], HEADROOM);
                        }
                    }
                }
            }
        }
        if (far) {
#pragma unroll
            for (int j = 0; j < 8; ++j) r.sum += __builtin_amdgcn_exp2f(t[j] - x.ev[LISTED ? j : j >> 2]);
        }
#pragma unroll
        for (int n = 0; n < Scales<LISTED>::N; ++n) {
            constexpr int EACH = 8 / Scales<LISTED>::N;
            float part = 0.f;
#pragma unroll
            for (int i = 0; i < EACH; ++i) {
                const float w = __builtin_amdgcn_exp2f(t[n * EACH + i]);
                part = i ? part + w : w;
                p[y][n * EACH + i] = (_Float16)w;
            }
            r.sum = __builtin_fmaf(part, x.down[n], r.sum);
        }
    }
    if constexpr (FMT == PAG_KV_FP4) {
        float scale[8];
#pragma unroll
        for (int w = 0; w < C; ++w) {
            if (w < Tile<FMT, C>::PARTS) {
                powers_of_bytes(tile.ve[0][w], x.less[0][1], scale);
                powers_of_bytes(tile.ve[1][w], x.less[1][1], scale + 4);
            }
            u32 words[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) words[j] = tile.v[j][w / 2];
            half8_t v[4];
            if (w % 2) columns_fp4<1>(words, scale, v);
            else columns_fp4<0>(words, scale, v);
#pragma unroll
            for (int c = 0; c < 4; ++c) {
#pragma unroll
                for (int y = 0; y < T; ++y) rows[y].acc[4 * w + c] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v[c], p[y], rows[y].acc[4 * w + c], 0, 0, 0);
            }
        }
    } else {
#pragma unroll
        for (int w = 0; w < C; ++w) {
            u32 words[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) words[j] = tile.v[j][w];
            half8_t v[4];
            columns<FMT>(words, v);
#pragma unroll
            for (int c = 0; c < 4; ++c) {
#pragma unroll
                for (int y = 0; y < T; ++y) rows[y].acc[4 * w + c] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v[c], p[y], rows[y].acc[4 * w + c], 0, 0, 0);
            }
        }
    }
}

// a wave's y-th tile of rows
__device__ __forceinline__ Where tile_of(const Where& w, u32 y) {
    Where x = w;
    x.row0 += y * ROWS;
    return x;
}

template <int C, int NW>
struct Exchange {
    static constexpr u32 STRIDE = 64 * C + 4;
    float m[NW][ROWS], sum[NW][ROWS];
    float acc[NW][ROWS][STRIDE];
};

// The waves' sums, into LDS, of the rows that there are.  All waves call it; the rows are free afterwards.
template <int C, int NW>
__device__ __forceinline__ void exchange(const Rows<C>& r, const Where& w, Exchange<C, NW>& x) {
    const u32 lane = threadIdx.x & 63, wave = wave_of(), col = lane & 15, g = lane >> 4;
    float sum = r.sum;
    sum += __shfl_xor(sum, 16);
    sum += __shfl_xor(sum, 32);
    if (w.row0 + col < w.rows) {
        if (g == 0) {
            x.m[wave][col] = r.M;
            x.sum[wave][col] = sum;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
#pragma unroll
            for (int q = 0; q < C; ++q)
                *(float4*)&x.acc[wave][col][(4 * g + i) * 4 * C + 4 * q] = make_float4(r.acc[4 * q][i], r.acc[4 * q + 1][i], r.acc[4 * q + 2][i], r.acc[4 * q + 3][i]);
        }
    }
    lds_barrier();
}

// Adds them up and writes the rows' results, or the piece's sums for the second kernel.  partial: null, or
// [16] offsets, [16] sums, [16][width]
template <int C, int NW>
__device__ __forceinline__ void finish(const Attend& a, const Where& w, const Exchange<C, NW>& x, float* partial) {
    constexpr u32 W = 64 * C, THREADS = 64 * NW / ROWS, N = W / THREADS;      // threads of a row, numbers of a thread
    const u32 row = threadIdx.x / THREADS, first = threadIdx.x % THREADS * N;
    if (w.row0 + row < w.rows) {
        float M = x.m[0][row];
#pragma unroll
        for (u32 v = 1; v < NW; ++v) M = fmaxf(M, x.m[v][row]);
        float sum = 0.f, o[N];
#pragma unroll
        for (u32 n = 0; n < N; ++n) o[n] = 0.f;
#pragma unroll
        for (u32 v = 0; v < NW; ++v) {
            const float by = __builtin_amdgcn_exp2f(x.m[v][row] - M);
            sum = add_scaled(sum, x.sum[v][row], x.m[v][row] - M);
#pragma unroll
            for (u32 n = 0; n < N; n += 2) {
                const float2 y = *(const float2*)&x.acc[v][row][first + n];
                o[n] = __builtin_fmaf(y.x, by, o[n]);
                o[n + 1] = __builtin_fmaf(y.y, by, o[n + 1]);
            }
        }
        if (partial) {
            if (first == 0) { partial[row] = M; partial[ROWS + row] = sum; }
#pragma unroll
            for (u32 n = 0; n < N; n += 2) *(float2*)(partial + 2 * ROWS + row * W + first + n) = make_float2(o[n], o[n + 1]);
        } else {
            const u32 t = w.t0 + (w.row0 + row) / a.group, head = w.head0 + (w.row0 + row) % a.group;
            const float f = sum != 0.f ? 1.f / sum : 0.f;
            uint16_t* out = (uint16_t*)a.out + (int64_t)t * a.o_ts + (int64_t)head * a.o_hs + first;
#pragma unroll
            for (u32 n = 0; n < N; n += 2) {
                if (first + n < a.c.dim) *(u32*)(out + n) = pack2(finite(o[n] * f), finite(o[n + 1] * f), a.dtype);
            }
            if (a.lse && first == 0) a.lse[(u64)t * a.heads + head] = sum != 0.f ? LN2 * (M + __builtin_amdgcn_logf(sum)) : -INFINITY;
        }
    }
    lds_barrier();
}

// ---- attention over all tokens --------------------------------------------------------------------------------------

struct Request {
    Span s;
    u32 tiles, units;      // units of one row tile
};

template <int T>
__device__ __forceinline__ Request request_of(const Attend& a, u32 b) {
    Request r;
    r.s = span_of(a, b);
    r.tiles = (r.s.tokens * a.group + T * ROWS - 1) / (T * ROWS);
    // with a window a tile's first token begins `window` before itself, at the edge of a block
    const u32 span = a.window ? (u32)min((u64)r.s.context, (u64)a.window + (T * ROWS - 1) / a.group + 1 + BLOCK - 1) : (u32)r.s.context;
    r.units = r.s.tokens ? (span + UNIT - 1) / UNIT : 0;
    return r;
}

__device__ __forceinline__ u64 units_of(const Attend& a, const Request& r) { return r.units ? (u64)r.tiles * (r.units + PIECE) * a.c.kv_heads : 0; }

__device__ __forceinline__ void write_joined(const Attend& a, const Where& w, u32 count, int2 j) {
    if (threadIdx.x < count && w.row0 + threadIdx.x < w.rows) {
        const u32 row = w.row0 + threadIdx.x;
        a.joined[(u64)(w.t0 + row / a.group) * a.heads + w.head0 + row % a.group] = j;
    }
}

// A piece of a workgroup's share: rows of a tile, keys start .. stop - 1.
struct Piece {
    Where w;
    Span s;
    u32 b, units, u0, u1;
    int p0, p1, start, stop;   // positions of the first and last row; keys
    int last;                  // the workgroup that ends the tile
    // listed blocks: keys are numbered through them, and through the window behind them, from its block of 16 on
    const int32_t* ids;
    u32 listed;                // keys of the list
    int near;                  // the window's first block
};

// rows, first and last key of the piece with units u0 to u1 - 1, of `unit` keys each, of row tile `tile`
template <int T>
__device__ __forceinline__ void place_piece(const Attend& a, Piece& p, const Span& s, u32 tile, u32 kv_head, u32 unit) {
    p.s = s;
    p.w.t0 = s.t0;
    p.w.rows = s.tokens * a.group;
    p.w.row0 = tile * (T * ROWS);
    p.w.kv_head = kv_head;
    p.w.head0 = kv_head * a.group;
    p.p0 = s.first + (int)(p.w.row0 / a.group);
    p.p1 = s.first + (int)(min(p.w.row0 + T * ROWS - 1, p.w.rows - 1) / a.group);
    p.start = (oldest_of(a, p.p0) & ~(int)(BLOCK - 1)) + (int)(p.u0 * unit);
    p.stop = (int)min((int64_t)p.p1 + 1, (int64_t)p.start + (int64_t)(p.u1 - p.u0) * unit);
}

// The pieces that next(p) gives, one after the other.  A wave has T tiles of rows: keys are widened once for all of them.  WHOLE: the pieces
// are whole row tiles.  BLOCKS: the keys of listed blocks and of a window, one token's; SLOPES is for them.
template <int FMT, int C, int T, int NW, bool WHOLE, bool CAPPED, bool BLOCKS, bool SLOPES, typename Next>
__device__ __forceinline__ void attend_pieces(const Attend& a, Exchange<C, NW>& sh, Next&& next) {
    // One tile at a time where that leaves registers for two workgroups a CU, whose waits overlap instead: 64 ragged requests of 192 numbers in 4 bits 137 us
    // with two tiles and one workgroup, 113 this way; of 256 numbers, where 70 registers are spilled for it, 143 and 172
    constexpr bool ALONE = one_tile(FMT, 64 * C, T);
    const u32 lane = threadIdx.x & 63, wave = wave_of(), col = lane & 15, g = lane >> 4;
    Piece p;
    Rows<C> rows[T];
    RawRows<C> raw;
    // 64 blocks of this wave's tiles at a time: lane 2 i + s has block s of tile i
    const int mine_at = (int)(lane >> 1) * (int)(NW * TILE) + (int)(lane & 1) * (int)BLOCK;
    int from = 0;
    u32 page = 0, block_row = 0;
    uint16_t exponents = 0;
    u64 there = 0;
    bool far = false;
    int first = 0, first_next = 0;            // BLOCKS: position of the first token of lane's block
    const auto page_of = [&](int at_key) -> u32 {
        if constexpr (BLOCKS) {
            first_next = -1;
            if (at_key < p.stop) {
                if ((u32)at_key < p.listed) {
                    const int id = p.ids[(u32)at_key / a.block];
                    // a block of tokens that lie in the window or behind it is none
                    if (id >= 0 && (int64_t)id * a.block <= (int64_t)p.p0 - a.window) first_next = id * (int)a.block + (int)((u32)at_key % a.block);
                    if (first_next > p.p0 - (int)a.window) first_next = -1;
                } else {
                    first_next = p.near + (at_key - (int)p.listed);
                }
            }
            return first_next >= 0 ? (u32)a.s.table[p.b * a.s.table_stride + (u32)first_next / BLOCK / a.c.page_blocks] : 0xFFFFFFFFu;
        }
        return at_key < p.stop ? (u32)a.s.table[p.b * a.s.table_stride + (u32)at_key / BLOCK / a.c.page_blocks] : 0xFFFFFFFFu;
    };
    const auto ask = [&]() {                  // what does not depend on each other is asked for together: pages and rows,
        from = p.start + (int)(wave * TILE);
        page = page_of(from + mine_at);
        far = false;
        if (T == 1) fetch_rows<FMT, C>(a, p.w, raw);
    };
    // then exponents and, by then(), the first tile; the next 64 blocks' pages
    const auto look_up = [&](auto&& then) {
        const bool ok = page < a.c.num_pages;
        if (BLOCKS) first = first_next;
        const int at_key = BLOCKS ? first : from + mine_at;
        block_row = ok ? row_of(a.c, page, p.w.kv_head, (u32)at_key / BLOCK % a.c.page_blocks * BLOCK) : 0;
        there = __ballot(ok);
        if constexpr (FMT == PAG_KV_FP4) {
            // the parts' exponents are asked for, then the tile, before the largest are looked for
            Parts<C> k, v;
            load_parts<C>(parts_of<C>(a.c, block_row / BLOCK, 0), k);
            load_parts<C>(parts_of<C>(a.c, block_row / BLOCK, 1), v);
            then();
            const int tokens = ok ? (BLOCKS ? p.p0 + 1 : p.stop) - at_key : 0;
            exponents = (uint16_t)((most_of_parts<C>(k, tokens) & 255) | most_of_parts<C>(v, tokens) << 8);
            page = page_of(from + 32 * (int)(NW * TILE) + mine_at);
        } else {
            exponents = ok ? *(const uint16_t*)(a.c.exponents + (u64)(block_row / BLOCK) * 2) : 0;
            page = page_of(from + 32 * (int)(NW * TILE) + mine_at);
            then();
        }
    };
    // a lane's offset from where a block begins; what is added to it is the same for all lanes
    constexpr u32 HALF = FMT == PAG_KV_FP4 ? 1 : 2;          // bytes of two numbers
    const u32 k_at = col * (64 * C * HALF) + g * (FMT == PAG_KV_FP4 && C % 2 ? 8 : 16), v_at = 4 * g * (64 * C * HALF) + 32 * C * HALF + col * (2 * C * HALF);
    const auto load = [&](Tile<FMT, C>& tile, int i) {
        if constexpr (FMT == PAG_KV_FP4) {
            typedef Tile<FMT, C> T4;
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                const u32 row = (u32)__builtin_amdgcn_readlane((int)block_row, 2 * i + s);
                const uint8_t* rows_at = a.c.data + (u64)row * (64 * C);
                load_codes<C>(tile, s, rows_at + k_at, [&](int j) { return rows_at + v_at + j * (64 * C); });
                const int8_t* parts = parts_of<C>(a.c, row / BLOCK, 0);
#pragma unroll
                for (int h = 0; h < T4::PIECES; ++h) tile.ke[s][h] = parts[key_part<C>(h, g) * BLOCK + col];
#pragma unroll
                for (int w = 0; w < T4::PARTS; ++w) tile.ve[s][w] = *(const u32*)(parts + ((2 * C + value_part<C>(w, col)) * BLOCK + 4 * g));
            }
            return;
        } else {
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                const uint8_t* rows_at = a.c.data + (u64)(u32)__builtin_amdgcn_readlane((int)block_row, 2 * i + s) * (128 * C);
#pragma unroll
                for (int h = 0; h < C; ++h) tile.k[s][h] = *(const uint4*)(rows_at + k_at + h * 64);
#pragma unroll
                for (int j = 0; j < 4; ++j) load_words<C>(rows_at + v_at + j * (128 * C), tile.v[4 * s + j]);
            }
        }
    };
    const auto add = [&](Tile<FMT, C>& tile, int i) {
        const int pos = from + i * (int)(NW * TILE);
        Scales<false> x;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const int e = __builtin_amdgcn_readlane((int)exponents, 2 * i + s), ev = (int)(int8_t)(e >> 8);
            x.ek[s] = power((int)(int8_t)e);
            x.ev[s] = (float)ev;
            far = far || ev > FAR_EXPONENT;
            x.down[s] = power(-ev);
            if constexpr (FMT == PAG_KV_FP4) {
                x.less[s][0] = less_of((int)(int8_t)e);
                x.less[s][1] = less_of(ev);
                if ((int)(int8_t)e > MOST_PLAIN || ev > MOST_PLAIN) {
#pragma unroll
                    for (int h = 0; h < Tile<FMT, C>::PIECES; ++h) tile.ke[s][h] = max(tile.ke[s][h], (int)(int8_t)e - 127);
#pragma unroll
                    for (int w = 0; w < Tile<FMT, C>::PARTS; ++w) tile.ve[s][w] = raised_bytes(tile.ve[s][w], ev - 127);
                }
            }
            x.at[s] = (BLOCKS ? __builtin_amdgcn_readlane(first, 2 * i + s) : pos + s * (int)BLOCK) + 4 * (int)g;
        }
        if (far) x.down[0] = x.down[1] = 0.f;
        const u32 two = (u32)(there >> (2 * i)) & 3u;
        // behind the last token there may be anything
        const auto no_value = [&](int j) {
            if constexpr (FMT == PAG_KV_FP4) {                // nor may its exponent be anything
#pragma unroll
                for (int w = 0; w < Tile<FMT, C>::PARTS; ++w) tile.ve[j >> 2][w] &= ~(255u << (8 * (j & 3)));
            }
#pragma unroll
            for (int y = 0; y < (FMT == PAG_KV_FP4 ? (C + 1) / 2 : C); ++y) tile.v[j][y] = 0;
        };
        if constexpr (BLOCKS) {
            // listed tokens end where the window begins, the window's end with the token itself
            int oldest[2], newest[2];
            bool whole = two == 3u;
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                const bool listed = (u32)(pos + s * (int)BLOCK) < p.listed;
                const int block = x.at[s] - 4 * (int)g;
                oldest[s] = listed ? 0 : p.p0 - (int)a.window + 1;
                newest[s] = listed ? p.p0 - (int)a.window : p.p0;
                whole = whole && block >= oldest[s] && block + (int)BLOCK - 1 <= newest[s];
            }
            u32 keep[1] = { 0xFF };
            if (!whole) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int k = x.at[j >> 2] + (j & 3);
                    const bool exists = (two >> (j >> 2) & 1u) && k <= p.p0;
                    if (!exists || k < oldest[j >> 2] || k > newest[j >> 2]) keep[0] &= ~(1u << j);
                    if (!exists) no_value(j);
                }
            }
            add_tile<FMT, C, 1, false, SLOPES, CAPPED, true>(a, tile, rows, x, !whole, keep, far);
            return;
        } else {
            const bool masked = two != 3u || pos + (int)TILE > p.p0 + 1 || pos < oldest_of(a, p.p1);
            u32 keep[T];
#pragma unroll
            for (int y = 0; y < T; ++y) keep[y] = 0xFF;
            if (masked) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int k = x.at[j >> 2] + (j & 3);
                    const bool exists = (two >> (j >> 2) & 1u) && k < p.stop;
#pragma unroll
                    for (int y = 0; y < T; ++y) {
                        if (!exists || k > rows[y].position || k < oldest_of(a, rows[y].position)) keep[y] &= ~(1u << j);
                    }
                    if (!exists) no_value(j);
                }
            }
            add_tile<FMT, C, T, false, false, CAPPED>(a, tile, rows, x, masked, keep, far);
        }
    };
    const auto start = [&]() {
#pragma unroll
        for (int y = 0; y < T; ++y) {
            if (T > 1) fetch_rows<FMT, C>(a, tile_of(p.w, y), raw);
            start_rows<C>(a, tile_of(p.w, y), BLOCKS ? p.p0 : p.s.first, raw, rows[y]);
        }
    };
    constexpr u32 SLOT = ROWS * (64 * C + 2);

    if constexpr (WHOLE || T > 1) {
        // WHOLE: few tiles a wave; their latency is what counts, and a fetch of instructions that are used once costs more than a fetch of
        // keys.  T > 1: there are no registers for a second tile of keys.
        while (next(p)) {
            ask();
            start();
            while (from < p.stop) {
                const int count = min(32, (p.stop - from + (int)(NW * TILE) - 1) / (int)(NW * TILE));
                if constexpr (FMT == PAG_KV_FP4) {
                    Tile<FMT, C> tile;
                    look_up([&]() { load(tile, 0); });
                    for (int i = 0; i < count; ++i) {
                        if (i) load(tile, i);
                        add(tile, i);
                    }
                } else {
                    look_up([]() {});
                    for (int i = 0; i < count; ++i) {
                        Tile<FMT, C> tile;
                        load(tile, i);
                        add(tile, i);
                    }
                }
                from += 32 * (int)(NW * TILE);
            }
            const bool begun = p.u0 == 0, ended = p.u1 == p.units;
            float* partial = nullptr;
            if (!WHOLE) {
                if (!begun || !ended) partial = a.partial + (2 * (u64)blockIdx.x + (begun ? 1 : 0)) * (T * SLOT);
                if (begun) write_joined(a, p.w, T * ROWS, p.last >= 0 ? make_int2((int)blockIdx.x, p.last) : make_int2(-1, -1));
            }
#pragma unroll
            for (int y = 0; y < T; ++y) {
                exchange(rows[y], tile_of(p.w, y), sh);
                finish(a, tile_of(p.w, y), sh, partial ? partial + y * SLOT : nullptr);
            }
        }
        return;
    }
    Tile<FMT, C> even, odd;
    bool more = next(p);
    if (more) {
        ask();
        if (from < p.stop) {
            look_up([&]() { load(even, 0); });
        }
    }
    while (more) {
        start();
        while (from < p.stop) {
            // a tile is on its way while the one before it is added; behind the last one the last is asked for again, which the cache has
            const int count = min(32, (p.stop - from + (int)(NW * TILE) - 1) / (int)(NW * TILE));
            for (int i = 0; ALONE && i < count; ++i) {
                if (i) load(even, i);
                add(even, i);
            }
            for (int i = 0; !ALONE && i < count; i += 2) {
                load(odd, min(i + 1, count - 1));
                add(even, i);
                if (i + 1 < count) {
                    load(even, min(i + 2, count - 1));
                    add(odd, i + 1);
                }
            }
            from += 32 * (int)(NW * TILE);
            if (from < p.stop) {
                look_up([&]() { load(even, 0); });
            }
        }
        // the next piece's first tile is on its way while this one's waves are added up
        const Where w = p.w;
        const bool begun = p.u0 == 0, ended = p.u1 == p.units;
        float* partial = !begun || !ended ? a.partial + (2 * (u64)blockIdx.x + (begun ? 1 : 0)) * SLOT : nullptr;
        if (begun) write_joined(a, w, ROWS, p.last >= 0 ? make_int2((int)blockIdx.x, p.last) : make_int2(-1, -1));
        more = next(p);
        if (more) ask();
        exchange(rows[0], w, sh);
        if (more && from < p.stop) {
            look_up([&]() { load(even, 0); });
        }
        finish(a, w, sh, partial);
    }
}

template <int FMT, int C, int T, bool CAPPED>
__global__ void __launch_bounds__(256, groups_per_cu(FMT, 64 * C, T)) k_attend(Attend a) {
    __shared__ __align__(16) Exchange<C, SPLIT_WAVES> sh;
    __shared__ u64 sh_sum[SPLIT_WAVES];
    __shared__ u64 sh_begin;
    __shared__ u32 sh_b;
    const u32 lane = threadIdx.x & 63, wave = wave_of();

    // this workgroup's share of all units
    const u32 per = (a.s.requests + 255) / 256, b0 = min(threadIdx.x * per, a.s.requests), b1 = min(b0 + per, a.s.requests);
    u64 mine = 0;
    for (u32 b = b0; b < b1; ++b) mine += units_of(a, request_of<T>(a, b));
    u64 upto = mine;
#pragma unroll
    for (u32 o = 1; o < 64; o <<= 1) {
        const u64 y = __shfl_up(upto, o);
        if (lane >= o) upto += y;
    }
    if (lane == 63) sh_sum[wave] = upto;
    __syncthreads();
    u64 total = 0;
    for (u32 x = 0; x < SPLIT_WAVES; ++x) {
        if (x < wave) upto += sh_sum[x];
        total += sh_sum[x];
    }
    const u32 parts = (u32)min((u64)gridDim.x, total);
    const u64 begin = blockIdx.x < parts ? share(total, parts, blockIdx.x) : total, end = blockIdx.x < parts ? share(total, parts, blockIdx.x + 1) : total;
    if (begin < end && begin >= upto - mine && begin < upto) {
        u64 before = upto - mine;
        u32 b = b0;
        for (;; ++b) {
            const u64 n = units_of(a, request_of<T>(a, b));
            if (begin < before + n) break;
            before += n;
        }
        sh_b = b;
        sh_begin = before;
    }
    // tokens that have nothing to read, and padding
    for (u32 b = blockIdx.x; b < a.s.requests; b += gridDim.x) {
        const Request r = request_of<T>(a, b);
        if (r.s.tokens && !r.units) write_empty(a, r.s.t0, r.s.t0 + r.s.tokens);
    }
    write_padding(a);
    if (begin >= end) return;
    __syncthreads();

    u32 b = sh_b;
    u64 before = sh_begin, at = begin;
    Request q = request_of<T>(a, b);
    u64 n = units_of(a, q);
    const auto next_piece = [&](Piece& p) -> bool {
        while (at < end) {
            while (at >= before + n) {
                before += n;
                ++b;
                q = request_of<T>(a, b);
                n = units_of(a, q);
            }
            const u32 cost = q.units + PIECE;
            const u64 in = at - before;
            const u32 part = (u32)divide(in, cost), c0 = (u32)(in - (u64)part * cost), c1 = (u32)min((u64)cost, c0 + (end - at));
            at += c1 - c0;
            // the units of a row tile come after the cost of beginning it
            p.u0 = max(c0, PIECE) - PIECE;
            p.u1 = max(c1, PIECE) - PIECE;
            if (p.u0 == p.u1) continue;
            p.b = b;
            p.units = q.units;
            p.last = p.u0 == 0 && p.u1 < p.units ? (int)divide((before + (u64)(part + 1) * cost) * parts - 1, total) : -1;
            place_piece<T>(a, p, q.s, part % q.tiles, part / q.tiles, UNIT);
            return true;
        }
        return false;
    };
    attend_pieces<FMT, C, T, SPLIT_WAVES, false, CAPPED, false, false>(a, sh, next_piece);
}

// A workgroup for each request and key/value head, which reads all of its keys: nothing to share out and nothing to join.
template <int FMT, int C, int T, int NW, bool CAPPED>
__global__ void __launch_bounds__(64 * NW, C <= 2 ? 2 : 1) k_attend_whole(Attend a) {
    __shared__ __align__(16) Exchange<C, NW> sh;
    const u32 b = blockIdx.x / a.c.kv_heads, kv_head = blockIdx.x % a.c.kv_heads;
    const Span s = span_of(a, b);
    write_padding(a);
    if (s.tokens == 0) return;
    if (s.context == 0) {
        if (kv_head == 0) write_empty(a, s.t0, s.t0 + s.tokens);
        return;
    }
    const u32 tiles = (s.tokens * a.group + T * ROWS - 1) / (T * ROWS);
    u32 tile = 0;
    attend_pieces<FMT, C, T, NW, true, CAPPED, false, false>(a, sh, [&](Piece& p) -> bool {
        if (tile == tiles) return false;
        p.b = b;
        p.units = p.u1 = 1;
        p.u0 = 0;
        p.last = -1;
        place_piece<T>(a, p, s, tile++, kv_head, 0x7FFFFFFFu);
        return true;
    });
}

// ---- attention over listed tokens -----------------------------------------------------------------------------------

// what a wave knows of 64 keys that it will add or is adding
template <int FMT, int C>
struct Entries {
    u32 row[64];
    float ek[64], ev[64], down[64];
    int at[64];
};

template <int C>
struct Entries<PAG_KV_FP4, C> {
    u32 row[64];
    float ek[64], ev[64], down[64];
    int at[64];
    int8_t parts[2][2 * C][64];          // exponents of keys and values, less the largest of their row; -127: no such key
};

// a token's list, or a part of it
struct ListPiece : Where {
    u32 id_head, u0, u1;
    int last;
};

__device__ __forceinline__ void place_list(const Attend& a, ListPiece& p, u64 list, u32 tile) {
    p.t0 = (u32)divide(list, a.id_heads);
    p.id_head = (u32)(list - (u64)p.t0 * a.id_heads);
    p.rows = a.group;
    p.row0 = tile * ROWS;
    p.head0 = p.id_head * a.group;
    p.kv_head = p.id_head / (a.id_heads / a.c.kv_heads);
}

// The pieces that next(p) gives; a list has `units` units of 32 NW entries.
template <int FMT, int C, int NW, bool WHOLE, bool SLOPES, bool CAPPED, typename Next>
__device__ __forceinline__ void attend_lists(const Attend& a, Exchange<C, NW>& sh, Entries<FMT, C> (&sh_entries)[NW][2], u32 units, Next&& next) {
    const u32 lane = threadIdx.x & 63, wave = wave_of(), col = lane & 15, g = lane >> 4;
    const u32 entries = a.k + a.window;
    ListPiece w = {};
    Rows<C> rows[1];
    RawRows<C> raw;
    u32 from = 0, stop = 0;                      // this wave's next entries
    int request = -1, position = -1;
    int64_t id = -1;                             // of the entries two batches on,
    int key = -1;                                // the positions and pages of the next one
    u32 page = 0;
    u64 there = 0;                               // which of this batch are keys
    bool far = false;
    const u32 mine = (lane & 31) + (lane >> 5) * (NW * TILE);
    const auto id_of = [&](u32 n) -> int64_t { return n < a.k && n < stop ? a.ids[(int64_t)w.t0 * a.ids_ts + (int64_t)w.id_head * a.ids_hs + n] : -1; };
    const auto key_of = [&](u32 n) {             // from id
        int64_t k = id;
        if (n >= a.k) k = (int64_t)position - (int64_t)(n - a.k);
        else if (k > (int64_t)position - (int64_t)a.window) k = -1;
        key = n < stop && position >= 0 && k >= 0 ? (int)k : -1;
        page = key >= 0 ? (u32)a.s.table[(u64)(u32)request * a.s.table_stride + (u32)key / BLOCK / a.c.page_blocks] : 0xFFFFFFFFu;
    };
    const auto ask = [&]() {
        from = w.u0 * (NW * TILE) + wave * TILE;
        stop = min(entries, w.u1 * (NW * TILE));
        id = id_of(from + mine);
        request = a.s.request[w.t0];
        position = a.s.positions[w.t0];
        fetch_rows<FMT, C>(a, w, raw);
    };
    const auto check = [&]() {
        if (request < 0 || (u32)request >= a.s.requests || (u64)(u32)max(position, 0) >= (u64)a.s.max_pages * a.c.page_tokens) position = -1;
    };
    // the 64 entries whose pages have been asked for, into LDS; the pages of the next and the ids after those are asked for
    const auto look_up = [&](u32 buffer) {
        Entries<FMT, C>& x = sh_entries[wave][buffer];
        const bool ok = page < a.c.num_pages;
        const u32 row = ok ? row_of(a.c, page, w.kv_head, (u32)key / BLOCK % a.c.page_blocks * BLOCK + ((u32)key & (BLOCK - 1))) : 0;
        u32 e = 0;
        if constexpr (FMT == PAG_KV_FP4) {
#pragma unroll
            for (int kind = 0; kind < 2; ++kind) {
                const int8_t* parts = parts_of<C>(a.c, row / BLOCK, kind) + row % BLOCK;
                int y[2 * C], most = LOWEST_EXPONENT;
#pragma unroll
                for (int b = 0; b < 2 * C; ++b) {
                    y[b] = parts[b * BLOCK];
                    most = max(most, y[b]);
                }
#pragma unroll
                for (int b = 0; b < 2 * C; ++b) x.parts[kind][b][lane] = (int8_t)(ok ? max(y[b] - most, -127) : -127);
                if (ok) e |= (u32)(most & 255) << (8 * kind);
            }
        } else {
            e = ok ? *(const uint16_t*)(a.c.exponents + (u64)(row / BLOCK) * 2) : 0;
        }
        there = __ballot(ok);
        far = far || __ballot((int)(int8_t)(e >> 8) > FAR_EXPONENT);
        x.row[lane] = row;
        x.at[lane] = key;
        const u32 next = from + 2 * (NW * TILE) + mine;
        if (from + 2 * (NW * TILE) < stop) {
            key_of(next);
            id = id_of(next + 2 * (NW * TILE));
        }
        const int ev = (int)(int8_t)(e >> 8);
        x.ek[lane] = power((int)(int8_t)e);
        x.ev[lane] = (float)ev;
        x.down[lane] = far ? 0.f : power(-ev);
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    };
    const auto load = [&](Tile<FMT, C>& tile, u32 buffer, int i) {
        const Entries<FMT, C>& x = sh_entries[wave][buffer];
        if constexpr (FMT == PAG_KV_FP4) {
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                const uint4 r = *(const uint4*)&x.row[32 * i + 16 * s + 4 * g];
                const u32 rows_at[4] = { r.x, r.y, r.z, r.w };
                load_codes<C>(tile, s, a.c.data + (u64)x.row[32 * i + 16 * s + col] * (64 * C) + g * (C % 2 ? 8 : 16),
                              [&](int j) { return a.c.data + (u64)rows_at[j] * (64 * C) + 32 * C + col * (2 * C); });
#pragma unroll
                for (int h = 0; h < Tile<FMT, C>::PIECES; ++h) tile.ke[s][h] = x.parts[0][key_part<C>(h, g)][32 * i + 16 * s + col];
#pragma unroll
                for (int w = 0; w < Tile<FMT, C>::PARTS; ++w) tile.ve[s][w] = *(const u32*)&x.parts[1][value_part<C>(w, col)][32 * i + 16 * s + 4 * g];
            }
            return;
        } else {
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                const uint8_t* k = a.c.data + (u64)x.row[32 * i + 16 * s + col] * (128 * C) + g * 16;
                const uint4 r = *(const uint4*)&x.row[32 * i + 16 * s + 4 * g];
                const u32 v[4] = { r.x, r.y, r.z, r.w };
#pragma unroll
                for (int h = 0; h < C; ++h) tile.k[s][h] = *(const uint4*)(k + h * 64);
#pragma unroll
                for (int j = 0; j < 4; ++j) load_words<C>(a.c.data + (u64)v[j] * (128 * C) + 64 * C + col * (4 * C), tile.v[4 * s + j]);
            }
        }
    };
    const auto add = [&](Tile<FMT, C>& tile, u32 buffer, int i, u32 found, bool far_now) {
        const Entries<FMT, C>& x = sh_entries[wave][buffer];
        Scales<true> scales;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const u32 at0 = 32 * i + 16 * s + 4 * g;
            const float4 ek = *(const float4*)&x.ek[at0], ev = *(const float4*)&x.ev[at0], down = *(const float4*)&x.down[at0];
            const int4 pos = *(const int4*)&x.at[at0];
            scales.ek[4 * s] = ek.x; scales.ek[4 * s + 1] = ek.y; scales.ek[4 * s + 2] = ek.z; scales.ek[4 * s + 3] = ek.w;
            scales.ev[4 * s] = ev.x; scales.ev[4 * s + 1] = ev.y; scales.ev[4 * s + 2] = ev.z; scales.ev[4 * s + 3] = ev.w;
            scales.down[4 * s] = down.x; scales.down[4 * s + 1] = down.y; scales.down[4 * s + 2] = down.z; scales.down[4 * s + 3] = down.w;
            scales.at[4 * s] = pos.x; scales.at[4 * s + 1] = pos.y; scales.at[4 * s + 2] = pos.z; scales.at[4 * s + 3] = pos.w;
        }
        scales.less[0][0] = scales.less[0][1] = scales.less[1][0] = scales.less[1][1] = less_of(0);
        const bool masked = found != 0xFFFFFFFFu;
        const u32 keep[1] = { (found >> (4 * g) & 15u) | (found >> (16 + 4 * g) & 15u) << 4 };
        if constexpr (FMT != PAG_KV_FP4) {           // which have an exponent for keys that are none
            if (masked) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    if (!(keep[0] >> j & 1u)) {
#pragma unroll
                        for (int y = 0; y < C; ++y) tile.v[j][y] = 0;
                    }
                }
            }
        }
        add_tile<FMT, C, 1, true, SLOPES, CAPPED>(a, tile, rows, scales, masked, keep, far_now);
    };
    Tile<FMT, C> even, odd;
    u32 buffer = 0;
    const auto begin_piece = [&]() {
        check();
        far = false;
        key_of(from + mine);
        id = id_of(from + 2 * (NW * TILE) + mine);
        look_up(buffer);
        load(even, buffer, 0);
    };

    bool more = next(w);
    if (more) {
        ask();
        if (from < stop) begin_piece();
    }
    while (more) {
        start_rows<C>(a, w, position, raw, rows[0]);
        while (from < stop) {
            const u32 lo = (u32)there, hi = (u32)(there >> 32), now = buffer;
            const bool far_now = far;
            load(odd, now, 1);
            if (lo) add(even, now, 0, lo, far_now);
            from += 2 * (NW * TILE);
            if (from < stop) {
                buffer ^= 1;
                look_up(buffer);
                load(even, buffer, 0);
            }
            if (hi) add(odd, now, 1, hi, far_now);
        }
        const Where done = w;
        float* partial = nullptr;
        if (!WHOLE) {
            const bool begun = w.u0 == 0, ended = w.u1 == units;
            if (!begun || !ended) partial = a.partial + (2 * (u64)blockIdx.x + (begun ? 1 : 0)) * (ROWS * (64 * C + 2));
            if (begun) write_joined(a, done, ROWS, w.last >= 0 ? make_int2((int)blockIdx.x, w.last) : make_int2(-1, -1));
        }
        more = next(w);
        if (more) ask();
        exchange(rows[0], done, sh);
        if (more && from < stop) begin_piece();
        finish(a, done, sh, partial);
    }
}

// Slopes need registers that three workgroups a CU leave none of: 8 lists of 5,064 keys of 64 numbers, 4 of 40,000, in us, three 24.9, 44.7, two 20.3, 39.9
constexpr u32 list_groups_per_cu(u32 fmt, u32 width, bool slopes) { return width > 128 ? 1 : slopes ? 2 : groups_per_cu(fmt, width, 1); }

template <int FMT, int C, bool SLOPES, bool CAPPED>
__global__ void __launch_bounds__(256, list_groups_per_cu(FMT, 64 * C, SLOPES)) k_attend_selected(Attend a, u32 units, u32 tiles) {
    __shared__ __align__(16) Exchange<C, SPLIT_WAVES> sh;
    __shared__ __align__(16) Entries<FMT, C> sh_entries[SPLIT_WAVES][2];
    const u32 cost = units + PIECE;
    const u64 total = (u64)a.s.tokens * a.id_heads * tiles * cost;
    const u32 parts = (u32)min((u64)gridDim.x, total);
    if (blockIdx.x >= parts) return;
    u64 at = share(total, parts, blockIdx.x);
    const u64 end = share(total, parts, blockIdx.x + 1);
    attend_lists<FMT, C, SPLIT_WAVES, false, SLOPES, CAPPED>(a, sh, sh_entries, units, [&](ListPiece& p) -> bool {
        while (at < end) {
            const u64 part = divide(at, cost), list = divide(part, tiles);
            const u32 c0 = (u32)(at - part * cost), c1 = (u32)min((u64)cost, c0 + (end - at));
            at += c1 - c0;
            p.u0 = max(c0, PIECE) - PIECE;
            p.u1 = max(c1, PIECE) - PIECE;
            if (p.u0 == p.u1) continue;
            p.last = p.u0 == 0 && p.u1 < units ? (int)divide((part + 1) * cost * parts - 1, total) : -1;
            place_list(a, p, list, (u32)(part - list * tiles));
            return true;
        }
        return false;
    });
}

template <int FMT, int C, int NW, bool SLOPES, bool CAPPED>
__global__ void __launch_bounds__(64 * NW, C <= 2 ? 2 : 1) k_attend_selected_whole(Attend a, u32 tiles) {
    __shared__ __align__(16) Exchange<C, NW> sh;
    __shared__ __align__(16) Entries<FMT, C> sh_entries[NW][2];
    const u32 units = max((a.k + a.window + NW * TILE - 1) / (NW * TILE), 1u);
    bool first = true;
    attend_lists<FMT, C, NW, true, SLOPES, CAPPED>(a, sh, sh_entries, units, [&](ListPiece& p) -> bool {
        if (!first) return false;
        first = false;
        p.u0 = 0;
        p.u1 = units;
        p.last = -1;
        place_list(a, p, blockIdx.x / tiles, blockIdx.x % tiles);
        return true;
    });
}

template <int FMT, int C, int NW, bool CAPPED>
void run_whole(hipStream_t st, const Attend& a) {
    if (a.listed) {
        const u32 tiles = (a.group + ROWS - 1) / ROWS;
        if (a.slopes) k_attend_selected_whole<FMT, C, NW, true, CAPPED><<<a.s.tokens * a.id_heads * tiles, 64 * NW, 0, st>>>(a, tiles);
        else k_attend_selected_whole<FMT, C, NW, false, CAPPED><<<a.s.tokens * a.id_heads * tiles, 64 * NW, 0, st>>>(a, tiles);
    } else {
        k_attend_whole<FMT, C, 1, NW, CAPPED><<<a.s.requests * a.c.kv_heads, 64 * NW, 0, st>>>(a);
    }
}

template <int FMT, int C, bool CAPPED>
void run_narrow(hipStream_t st, const Attend& a, int num_cu, bool whole) {
    if (whole) {
        if constexpr (C <= 3) {
            if (!a.listed && a.row_tiles == 2) {
                k_attend_whole<FMT, C, 2, 4, CAPPED><<<a.s.requests * a.c.kv_heads, 256, 0, st>>>(a);
                return;
            }
        }
        // Eight waves where there are CUs enough, four where workgroups queue (and where registers last for no more).  Four and eight, in us: one request of
        // 777 tokens 9.7, 8.3; 16 of 500 tokens 10.7, 9.9; 64 lists of 1,064 keys 17.2, 14.4; 64 requests of 10 to 100 tokens 8.7, 12.9; 96 of 300 to 1,000
        // tokens 32, 37; 1,536 lists of 164 keys 27, 44
        if constexpr (C <= 2) {
            if (narrow_groups(a) <= (u64)num_cu) return run_whole<FMT, C, 8, CAPPED>(st, a);
        }
        return run_whole<FMT, C, 4, CAPPED>(st, a);
    }
    const u32 grid = (u32)num_cu * groups_per_cu(FMT, 64 * C, a.row_tiles);
    if (a.listed) {
        const u32 units = std::max<u32>((a.k + a.window + UNIT - 1) / UNIT, 1), tiles = (a.group + ROWS - 1) / ROWS;
        if (a.slopes) return k_attend_selected<FMT, C, true, CAPPED><<<(u32)num_cu * list_groups_per_cu(FMT, 64 * C, true), 256, 0, st>>>(a, units, tiles);
        return k_attend_selected<FMT, C, false, CAPPED><<<(u32)num_cu * list_groups_per_cu(FMT, 64 * C, false), 256, 0, st>>>(a, units, tiles);
    }
    if constexpr (C <= 3) {
        if (a.row_tiles == 2) return k_attend<FMT, C, 2, CAPPED><<<grid, 256, 0, st>>>(a);
    }
    k_attend<FMT, C, 1, CAPPED><<<grid, 256, 0, st>>>(a);
}

}  // namespace

template <int FMT, int C>
void launch_narrow(hipStream_t st, const Attend& a, int num_cu, bool whole) {
    if (a.softcap > NEAR_CAP) run_narrow<FMT, C, true>(st, a, num_cu, whole);
    else run_narrow<FMT, C, false>(st, a, num_cu, whole);
}

}  // namespace pagkv
