// Attention over the 8-bit cache: pag_kv_attend and pag_kv_attend_selected.
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
#include "pag_kv_attend.h"

namespace pagkv {
namespace {

constexpr u32 ROWS = 16;                  // query rows of a tile
constexpr u32 TILE = 32;                  // keys of a tile
constexpr u32 WAVES = 4;
constexpr u32 UNIT = WAVES * TILE;        // keys of the smallest share

// a lane's part of 32 keys: of row lane % 16 of both halves the 16-byte pieces lane / 16 + 4 h, and of tokens 4 (lane / 16) + 0 .. 3
// of both halves the values' numbers 4 C (lane % 16) + 0 .. 4 C - 1
template <int C>
struct Tile {
    uint4 k[2][C];
    u32 v[8][C];
};

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

// what a wave knows of its 16 rows and has summed up
template <int C>
struct Rows {
    half8_t q[2 * C];          // row lane % 16, numbers 64 h + 16 (lane / 16) + 8 s + 0 .. 7 in q[2 h + s]
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

template <int C>
__device__ __forceinline__ void load_rows(const Attend& a, const Where& w, int first_position, Rows<C>& r) {
    const u32 lane = threadIdx.x & 63, row = w.row0 + (lane & 15), g = lane >> 4;
    const u32 i = row / a.group, head = w.head0 + row % a.group;
    const bool real = row < w.rows;
    r.position = real ? first_position + (int)i : -1;
    r.slope = real && a.slopes ? a.slopes[head] * LOG2E : 0.f;
    float x[2 * C][8];
    float most = 0.f;
#pragma unroll
    for (int n = 0; n < 2 * C; ++n) {
        const u32 at = (n >> 1) * 64 + g * 16 + (n & 1) * 8;
#pragma unroll
        for (int j = 0; j < 8; ++j) x[n][j] = 0.f;
        if (real && at < a.c.dim) load8(a.q, (u64)(w.t0 + i) * (u64)a.q_ts + head * (u64)a.q_hs + at, a.dtype, x[n]);
#pragma unroll
        for (int j = 0; j < 8; ++j) most = fmaxf(most, fabsf(x[n][j]));
    }
    most = fmaxf(most, __shfl_xor(most, 16));
    most = fmaxf(most, __shfl_xor(most, 32));
    // the largest number of the row comes to lie between 2^7 and 2^8
    int e = (int)(__float_as_uint(most) >> 23) - 127 - 7;
    e = min(max(e, -100), 100);
    const float down = power(-e);
#pragma unroll
    for (int n = 0; n < 2 * C; ++n) {
#pragma unroll
        for (int j = 0; j < 8; ++j) r.q[n][j] = (_Float16)(x[n][j] * down);
    }
    r.factor = a.scale * power(e);
    r.M = LOWEST;
    r.sum = 0.f;
#pragma unroll
    for (int c = 0; c < 4 * C; ++c) r.acc[c] = float4_t{ 0.f, 0.f, 0.f, 0.f };
}

// ek, ev: this lane's 8 keys' scales as 2^e (keys) and e (values); position of its key j; keep: bit j set if the row may read key j.
// LISTED: the keys have their own exponents and positions; otherwise keys 0 .. 3 and 4 .. 7 share theirs, and have position at, at + 1, ..
template <int FMT, int C, bool LISTED>
__device__ __forceinline__ void add_tile(const Attend& a, Tile<C>& tile, Rows<C>& r, const float* ek, const float* ev, const int* at, bool masked, u32 keep) {
    float4_t s[2] = { { 0.f, 0.f, 0.f, 0.f }, { 0.f, 0.f, 0.f, 0.f } };
#pragma unroll
    for (int h = 0; h < C; ++h) {
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            s[b] = __builtin_amdgcn_mfma_f32_16x16x32_f16(widen8<FMT>(tile.k[b][h].x, tile.k[b][h].y), r.q[2 * h], s[b], 0, 0, 0);
            s[b] = __builtin_amdgcn_mfma_f32_16x16x32_f16(widen8<FMT>(tile.k[b][h].z, tile.k[b][h].w), r.q[2 * h + 1], s[b], 0, 0, 0);
        }
    }
    float t[8];
    if (a.softcap > 0.f) {
        // tanh(y) = 1 - 2 / (1 + e^(2 y))
        const float in = 2.f * LOG2E * r.factor / a.softcap, cap = a.softcap * LOG2E;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float z = __builtin_amdgcn_exp2f(s[j >> 2][j & 3] * (in * ek[LISTED ? j : j >> 2]));
            t[j] = cap - 2.f * cap * __builtin_amdgcn_rcpf(1.f + z);
        }
    } else {
        const float f = r.factor * LOG2E;
#pragma unroll
        for (int j = 0; j < 8; ++j) t[j] = s[j >> 2][j & 3] * (f * ek[LISTED ? j : j >> 2]);
    }
    if (a.slopes) {
#pragma unroll
        for (int j = 0; j < 8; ++j) t[j] -= r.slope * (float)(r.position - (LISTED ? at[j] : at[j >> 2] + (j & 3)));
    }
    float most = -INFINITY;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        t[j] += ev[LISTED ? j : j >> 2];
        if (masked && !(keep >> j & 1u)) t[j] = -INFINITY;
        most = fmaxf(most, t[j]);
    }
    if (__ballot(most > r.M + HEADROOM)) {
        most = fmaxf(most, __shfl_xor(most, 16));
        most = fmaxf(most, __shfl_xor(most, 32));
        // rows that need not move stay as they are: a row's result does not depend on its neighbours in the tile
        const float M = most > r.M + HEADROOM ? most - START : r.M, alpha = __builtin_amdgcn_exp2f(r.M - M);
        r.sum *= alpha;
#pragma unroll
        for (int c = 0; c < 4 * C; ++c) r.acc[c] *= alpha;
        r.M = M;
    }
    half8_t p;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float x = __builtin_amdgcn_exp2f(t[j] - r.M);
        r.sum = __builtin_fmaf(x, power(-(int)ev[LISTED ? j : j >> 2]), r.sum);
        p[j] = (_Float16)x;
    }
#pragma unroll
    for (int w = 0; w < C; ++w) {
        u32 words[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) words[j] = tile.v[j][w];
        half8_t v[4];
        columns<FMT>(words, v);
#pragma unroll
        for (int c = 0; c < 4; ++c) r.acc[4 * w + c] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v[c], p, r.acc[4 * w + c], 0, 0, 0);
    }
}

// Adds up the four waves' sums and writes the rows' results, or the piece's sums for the second kernel.  partial: null, or
// [16] offsets, [16] sums, [16][width]
template <int C>
__device__ __forceinline__ void finish(const Attend& a, const Where& w, Rows<C>& r, float* lds, float* partial) {
    constexpr u32 W = 64 * C, STRIDE = W + 4;
    const u32 lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 15, g = lane >> 4;
    float* sh_m = lds;                           // [waves][16]
    float* sh_s = lds + WAVES * ROWS;
    float* sh_acc = lds + 2 * WAVES * ROWS;      // [waves][16][STRIDE]
    float sum = r.sum;
    sum += __shfl_xor(sum, 16);
    sum += __shfl_xor(sum, 32);
    if (g == 0) {
        sh_m[wave * ROWS + col] = r.M;
        sh_s[wave * ROWS + col] = sum;
    }
    __syncthreads();
    float M = sh_m[col];
#pragma unroll
    for (u32 x = 1; x < WAVES; ++x) M = fmaxf(M, sh_m[x * ROWS + col]);
    const float alpha = __builtin_amdgcn_exp2f(r.M - M);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
#pragma unroll
        for (int q = 0; q < C; ++q) {
            float4 x;
            x.x = r.acc[4 * q][i] * alpha; x.y = r.acc[4 * q + 1][i] * alpha; x.z = r.acc[4 * q + 2][i] * alpha; x.w = r.acc[4 * q + 3][i] * alpha;
            *(float4*)(sh_acc + (wave * ROWS + col) * STRIDE + (4 * g + i) * 4 * C + 4 * q) = x;
        }
    }
    __syncthreads();
    // 16 threads a row, 4 C numbers each
    const u32 row = threadIdx.x >> 4, first = (threadIdx.x & 15) * 4 * C;
    M = sh_m[row];
#pragma unroll
    for (u32 x = 1; x < WAVES; ++x) M = fmaxf(M, sh_m[x * ROWS + row]);
    sum = 0.f;
#pragma unroll
    for (u32 x = 0; x < WAVES; ++x) sum += sh_s[x * ROWS + row] * __builtin_amdgcn_exp2f(sh_m[x * ROWS + row] - M);
    float o[4 * C];
#pragma unroll
    for (int n = 0; n < 4 * C; ++n) o[n] = 0.f;
#pragma unroll
    for (u32 x = 0; x < WAVES; ++x) {
#pragma unroll
        for (int q = 0; q < C; ++q) {
            const float4 y = *(const float4*)(sh_acc + (x * ROWS + row) * STRIDE + first + 4 * q);
            o[4 * q] += y.x; o[4 * q + 1] += y.y; o[4 * q + 2] += y.z; o[4 * q + 3] += y.w;
        }
    }
    if (partial) {
        if (first == 0) { partial[row] = M; partial[ROWS + row] = sum; }
#pragma unroll
        for (int q = 0; q < C; ++q)
            *(float4*)(partial + 2 * ROWS + row * W + first + 4 * q) = make_float4(o[4 * q], o[4 * q + 1], o[4 * q + 2], o[4 * q + 3]);
    } else if (w.row0 + row < w.rows) {
        const u32 t = w.t0 + (w.row0 + row) / a.group, head = w.head0 + (w.row0 + row) % a.group;
        const float f = sum != 0.f ? 1.f / sum : 0.f;
        uint16_t* out = (uint16_t*)a.out + (int64_t)t * a.o_ts + (int64_t)head * a.o_hs + first;
#pragma unroll
        for (int q = 0; q < C; ++q) {
            if (first + 4 * q < a.c.dim)
                *(uint2*)(out + 4 * q) = make_uint2(pack2(o[4 * q] * f, o[4 * q + 1] * f, a.dtype), pack2(o[4 * q + 2] * f, o[4 * q + 3] * f, a.dtype));
        }
        if (a.lse && first == 0) a.lse[(u64)t * a.heads + head] = sum != 0.f ? LN2 * (M + __builtin_amdgcn_logf(sum)) : -INFINITY;
    }
    __syncthreads();
}

// ---- attention over all tokens --------------------------------------------------------------------------------------

struct Request {
    Span s;
    u32 tiles, units;      // units of one row tile
};

__device__ __forceinline__ Request request_of(const Attend& a, u32 b) {
    Request r;
    r.s = span_of(a, b);
    r.tiles = (r.s.tokens * a.group + ROWS - 1) / ROWS;
    // with a window a tile's first token begins `window` before itself, at the edge of a block
    const u32 span = a.window ? (u32)min((u64)r.s.context, (u64)a.window + (ROWS - 1) / a.group + 1 + BLOCK - 1) : (u32)r.s.context;
    r.units = r.s.tokens ? (span + UNIT - 1) / UNIT : 0;
    return r;
}

__device__ __forceinline__ u64 units_of(const Attend& a, const Request& r) { return (u64)r.tiles * r.units * a.c.kv_heads; }

__device__ __forceinline__ void write_joined(const Attend& a, const Where& w, int2 j) {
    if (threadIdx.x < ROWS && w.row0 + threadIdx.x < w.rows) {
        const u32 row = w.row0 + threadIdx.x;
        a.joined[(u64)(w.t0 + row / a.group) * a.heads + w.head0 + row % a.group] = j;
    }
}

template <int C>
constexpr u32 lds_floats() { return 2 * WAVES * ROWS + WAVES * ROWS * (64 * C + 4); }

template <int FMT, int C>
__global__ void __launch_bounds__(256) k_attend(Attend a) {
    __shared__ __align__(16) float lds[lds_floats<C>()];
    __shared__ u64 sh_sum[256 / 64];
    __shared__ u64 sh_begin;
    __shared__ u32 sh_b;
    const u32 lane = threadIdx.x & 63, wave = threadIdx.x >> 6;

    // this workgroup's share of all units
    const u32 per = (a.s.requests + 255) / 256, b0 = min(threadIdx.x * per, a.s.requests), b1 = min(b0 + per, a.s.requests);
    u64 mine = 0;
    for (u32 b = b0; b < b1; ++b) mine += units_of(a, request_of(a, b));
    u64 upto = mine;
#pragma unroll
    for (u32 o = 1; o < 64; o <<= 1) {
        const u64 y = __shfl_up(upto, o);
        if (lane >= o) upto += y;
    }
    if (lane == 63) sh_sum[wave] = upto;
    __syncthreads();
    u64 total = 0;
    for (u32 x = 0; x < 256 / 64; ++x) {
        if (x < wave) upto += sh_sum[x];
        total += sh_sum[x];
    }
    const u32 parts = (u32)min((u64)gridDim.x, total);
    const u64 begin = blockIdx.x < parts ? share(total, parts, blockIdx.x) : total, end = blockIdx.x < parts ? share(total, parts, blockIdx.x + 1) : total;
    if (begin < end && begin >= upto - mine && begin < upto) {
        u64 before = upto - mine;
        u32 b = b0;
        for (;; ++b) {
            const u64 n = units_of(a, request_of(a, b));
            if (begin < before + n) break;
            before += n;
        }
        sh_b = b;
        sh_begin = before;
    }
    // tokens that have nothing to read, and padding
    for (u32 b = blockIdx.x; b < a.s.requests; b += gridDim.x) {
        const Request r = request_of(a, b);
        if (r.s.tokens && !r.units) write_empty(a, r.s.t0, r.s.t0 + r.s.tokens);
    }
    write_padding(a);
    if (begin >= end) return;
    __syncthreads();
    u32 b = sh_b;
    u64 before = sh_begin, at = begin;

    while (at < end) {
        Request q = request_of(a, b);
        u64 n = units_of(a, q);
        while (at >= before + n) {
            before += n;
            ++b;
            q = request_of(a, b);
            n = units_of(a, q);
        }
        const u64 in = at - before;
        const u32 u0 = (u32)(in % q.units), u1 = (u32)min((u64)q.units, u0 + (end - at));
        Where w;
        w.t0 = q.s.t0;
        w.rows = q.s.tokens * a.group;
        w.row0 = (u32)(in / q.units % q.tiles) * ROWS;
        w.kv_head = (u32)(in / q.units / q.tiles);
        w.head0 = w.kv_head * a.group;
        const int p0 = q.s.first + (int)(w.row0 / a.group), p1 = q.s.first + (int)(min(w.row0 + ROWS - 1, w.rows - 1) / a.group);
        const int low = a.window ? max(0, p0 - (int)min(a.window, 0x7FFFFFFFu) + 1) : 0;
        const int start = (low & ~(int)(BLOCK - 1)) + (int)(u0 * UNIT), stop = min(p1 + 1, start + (int)((u1 - u0) * UNIT));

        Rows<C> rows;
        load_rows<C>(a, w, q.s.first, rows);
        const u32 col = lane & 15, g = lane >> 4;
        const int32_t* table = a.s.table + b * a.s.table_stride;
        // 64 blocks of this wave's tiles at a time: lane 2 i + s has block s of tile i
        for (int from = start + (int)(wave * TILE); from < stop; from += 32 * (int)UNIT) {
            const int mine_at = from + (int)(lane >> 1) * (int)UNIT + (int)(lane & 1) * (int)BLOCK;
            u32 block_row = 0;
            int ek_mine = 0, ev_mine = 0;
            bool ok = false;
            if (mine_at < stop) {
                const u32 blk = (u32)mine_at / BLOCK, page = (u32)table[blk / a.c.page_blocks];
                if (page < a.c.num_pages) {
                    ok = true;
                    block_row = row_of(a.c, page, w.kv_head, blk % a.c.page_blocks * BLOCK);
                    const int8_t* e = a.c.exponents + (u64)(block_row / BLOCK) * 2;
                    ek_mine = e[0];
                    ev_mine = e[1];
                }
            }
            const u64 there = __ballot(ok);
            const int count = min(32, (stop - from + (int)UNIT - 1) / (int)UNIT);
            for (int i = 0; i < count; ++i) {
                const int pos = from + i * (int)UNIT;
                Tile<C> tile;
                float ek[2], ev[2];
                int where[2];
#pragma unroll
                for (int s = 0; s < 2; ++s) {
                    const uint8_t* rows_at = a.c.data + (u64)(u32)__builtin_amdgcn_readlane((int)block_row, 2 * i + s) * (2 * a.c.width);
                    ek[s] = power(__builtin_amdgcn_readlane(ek_mine, 2 * i + s));
                    ev[s] = (float)__builtin_amdgcn_readlane(ev_mine, 2 * i + s);
                    where[s] = pos + s * (int)BLOCK + 4 * (int)g;
#pragma unroll
                    for (int h = 0; h < C; ++h) tile.k[s][h] = *(const uint4*)(rows_at + col * (128 * C) + h * 64 + g * 16);
#pragma unroll
                    for (int j = 0; j < 4; ++j) load_words<C>(rows_at + (4 * g + j) * (128 * C) + 64 * C + col * (4 * C), tile.v[4 * s + j]);
                }
                const u32 two = (u32)(there >> (2 * i)) & 3u;
                const bool masked = two != 3u || pos + (int)TILE > p0 + 1 || pos <= p1 - (int)min(a.window - 1, 0x7FFFFFFEu) - 1;
                u32 keep = 0xFF;
                if (masked) {
                    keep = 0;
                    const int oldest = a.window ? max(0, rows.position - (int)min(a.window, 0x7FFFFFFFu) + 1) : 0;
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const int p = where[j >> 2] + (j & 3);
                        const bool exists = (two >> (j >> 2) & 1u) && p < stop;
                        if (exists && p <= rows.position && p >= oldest) keep |= 1u << j;
                        if (!exists) {
#pragma unroll
                            for (int x = 0; x < C; ++x) tile.v[j][x] = 0;      // the memory behind the last token may hold anything
                        }
                    }
                }
                add_tile<FMT, C, false>(a, tile, rows, ek, ev, where, masked, keep);
            }
        }
        const bool begun = u0 == 0, ended = u1 == q.units;
        float* partial = nullptr;
        if (!begun || !ended) partial = a.partial + (2 * (u64)blockIdx.x + (begun ? 1 : 0)) * (ROWS * (64 * C + 2));
        if (begun) {
            int2 j = make_int2(-1, -1);
            if (!ended) j = make_int2((int)blockIdx.x, (int)(((at + q.units) * parts - 1) / total));     // the workgroup of unit at + q.units - 1
            write_joined(a, w, j);
        }
        finish<C>(a, w, rows, lds, partial);
        at += u1 - u0;
    }
}

// ---- attention over listed tokens -----------------------------------------------------------------------------------

template <int FMT, int C>
__global__ void __launch_bounds__(256) k_attend_selected(Attend a, u32 units, u32 tiles) {
    __shared__ __align__(16) float lds[lds_floats<C>()];
    __shared__ uint4 sh_entry[WAVES][64];        // row, exponents of key and value, position, found
    const u32 lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const u64 total = (u64)a.s.tokens * a.id_heads * tiles * units;
    const u32 parts = (u32)min((u64)gridDim.x, total);
    if (blockIdx.x >= parts) return;
    u64 at = share(total, parts, blockIdx.x);
    const u64 end = share(total, parts, blockIdx.x + 1);
    const u32 entries = a.k + a.window;

    while (at < end) {
        const u32 u0 = (u32)(at % units), u1 = (u32)min((u64)units, u0 + (end - at));
        const u64 list = at / units / tiles;
        const u32 t = (u32)(list / a.id_heads), id_head = (u32)(list % a.id_heads);
        Where w;
        w.t0 = t;
        w.rows = a.group;
        w.row0 = (u32)(at / units % tiles) * ROWS;
        w.head0 = id_head * a.group;
        w.kv_head = (u32)((u64)id_head * a.c.kv_heads / a.id_heads);
        const int request = a.s.request[t];
        int position = a.s.positions[t];
        if (request < 0 || (u32)request >= a.s.requests || (u64)(u32)max(position, 0) >= (u64)a.s.max_pages * a.c.page_tokens) position = -1;
        const int32_t* table = a.s.table + (u64)(u32)max(position < 0 ? 0 : request, 0) * a.s.table_stride;
        const int64_t* ids = a.ids + (int64_t)t * a.ids_ts + (int64_t)id_head * a.ids_hs;
        Rows<C> rows;
        load_rows<C>(a, w, position, rows);
        const u32 col = lane & 15, g = lane >> 4;
        const u32 start = u0 * UNIT, stop = min(entries, u1 * UNIT);
        for (u32 from = start + wave * TILE; from < stop; from += 2 * UNIT) {
            // 64 entries, two tiles
            const u32 n = from + (lane & 31) + (lane >> 5) * UNIT;
            uint4 entry = make_uint4(0, 0, 0, 0);
            if (n < stop && position >= 0) {
                int64_t p = n < a.k ? ids[n] : (int64_t)position - (int64_t)(n - a.k);
                if (n < a.k && p > (int64_t)position - (int64_t)a.window) p = -1;
                if (p >= 0) {
                    const u32 blk = (u32)p / BLOCK, page = (u32)table[blk / a.c.page_blocks];
                    if (page < a.c.num_pages) {
                        entry.x = row_of(a.c, page, w.kv_head, blk % a.c.page_blocks * BLOCK + ((u32)p & (BLOCK - 1)));
                        const int8_t* e = a.c.exponents + (u64)(entry.x / BLOCK) * 2;
                        entry.y = (u32)(uint8_t)e[0] | (u32)(uint8_t)e[1] << 8;
                        entry.z = (u32)p;
                        entry.w = 1;
                    }
                }
            }
            const u64 there = __ballot(entry.w != 0);
            sh_entry[wave][lane] = entry;
            __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
            __builtin_amdgcn_wave_barrier();
            __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const u32 found = (u32)(there >> (32 * i));
                if (!found) continue;
                Tile<C> tile;
                float ek[8], ev[8];
                int where[8];
                u32 keep = 0;
#pragma unroll
                for (int s = 0; s < 2; ++s) {
                    const u32 row = sh_entry[wave][32 * i + 16 * s + col].x;
                    const uint8_t* p = a.c.data + (u64)row * (2 * a.c.width) + g * 16;
#pragma unroll
                    for (int h = 0; h < C; ++h) tile.k[s][h] = *(const uint4*)(p + h * 64);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const uint4 x = sh_entry[wave][32 * i + 16 * s + 4 * g + j];
                        load_words<C>(a.c.data + (u64)x.x * (2 * a.c.width) + 64 * C + col * (4 * C), tile.v[4 * s + j]);
                        ek[4 * s + j] = power((int8_t)x.y);
                        ev[4 * s + j] = (float)(int8_t)(x.y >> 8);
                        where[4 * s + j] = (int)x.z;
                        keep |= x.w << (4 * s + j);
                    }
                }
                const bool masked = found != 0xFFFFFFFFu;
                if (masked) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        if (!(keep >> j & 1u)) {
#pragma unroll
                            for (int x = 0; x < C; ++x) tile.v[j][x] = 0;
                        }
                    }
                }
                add_tile<FMT, C, true>(a, tile, rows, ek, ev, where, masked, keep);
            }
            __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
            __builtin_amdgcn_wave_barrier();
        }
        const bool begun = u0 == 0, ended = u1 == units;
        float* partial = nullptr;
        if (!begun || !ended) partial = a.partial + (2 * (u64)blockIdx.x + (begun ? 1 : 0)) * (ROWS * (64 * C + 2));
        if (begun) {
            int2 j = make_int2(-1, -1);
            if (!ended) j = make_int2((int)blockIdx.x, (int)(((at + units) * parts - 1) / total));
            write_joined(a, w, j);
        }
        finish<C>(a, w, rows, lds, partial);
        at += u1 - u0;
    }
}

// ---- joining --------------------------------------------------------------------------------------------------------

// A workgroup for each token and head; if its keys went to several workgroups, its waves take every fourth of their pieces.
template <int C>
__global__ void __launch_bounds__(256) k_join(Attend a, bool listed, int groups) {
    __shared__ float sh_m[4], sh_s[4];
    __shared__ float sh_acc[4][64 * C];
    const u32 t = blockIdx.x / a.heads, head = blockIdx.x % a.heads, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int2 j = a.joined[(u64)t * a.heads + head];
    if (j.x < 0 || j.y < j.x || j.y >= groups) return;
    u32 row = head % a.group;
    if (!listed) {
        // number of the token in its request
        u32 lo = 0, hi = a.s.requests;
        while (hi - lo > 1) {
            const u32 mid = (lo + hi) / 2;
            if ((u32)max(a.s.offsets[mid], 0) <= t) lo = mid; else hi = mid;
        }
        row += (t - (u32)max(a.s.offsets[lo], 0)) * a.group;
    }
    row %= ROWS;
    constexpr u32 SLOT = ROWS * (64 * C + 2);
    float M = LOWEST, sum = 0.f, acc[C];
#pragma unroll
    for (int c = 0; c < C; ++c) acc[c] = 0.f;
    for (int wg = j.x + (int)wave; wg <= j.y; wg += 4) {
        const float* p = a.partial + (2 * (u64)wg + (wg == j.x ? 1 : 0)) * SLOT;
        const float m = p[row], s = p[ROWS + row], top = fmaxf(M, m);
        const float was = __builtin_amdgcn_exp2f(M - top), is = __builtin_amdgcn_exp2f(m - top);
        sum = sum * was + s * is;
#pragma unroll
        for (int c = 0; c < C; ++c) acc[c] = acc[c] * was + p[2 * ROWS + row * (64 * C) + c * 64 + lane] * is;
        M = top;
    }
    if (lane == 0) { sh_m[wave] = M; sh_s[wave] = sum; }
#pragma unroll
    for (int c = 0; c < C; ++c) sh_acc[wave][c * 64 + lane] = acc[c];
    __syncthreads();
    const float top = fmaxf(fmaxf(sh_m[0], sh_m[1]), fmaxf(sh_m[2], sh_m[3]));
    float f[4], all = 0.f;
#pragma unroll
    for (int x = 0; x < 4; ++x) {
        f[x] = __builtin_amdgcn_exp2f(sh_m[x] - top);
        all += sh_s[x] * f[x];
    }
    const u32 d = threadIdx.x * 2;
    if (d < a.c.dim) {
        float o[2] = { 0.f, 0.f };
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            o[0] += sh_acc[x][d] * f[x];
            o[1] += sh_acc[x][d + 1] * f[x];
        }
        const float by = all != 0.f ? 1.f / all : 0.f;
        *(u32*)((uint16_t*)a.out + (int64_t)t * a.o_ts + (int64_t)head * a.o_hs + d) = pack2(o[0] * by, o[1] * by, a.dtype);
    }
    if (a.lse && threadIdx.x == 0) a.lse[(u64)t * a.heads + head] = all != 0.f ? LN2 * (top + __builtin_amdgcn_logf(all)) : -INFINITY;
}

constexpr u32 groups_per_cu(u32 width) { return width <= 128 ? 3 : 2; }
u64 partial_floats(u32 width, int num_cu) { return 2ull * (u32)num_cu * groups_per_cu(width) * ROWS * (width + 2); }

template <int FMT, int C>
void run_attend(hipStream_t st, const Attend& a, int num_cu) {
    const u32 grid = (u32)num_cu * groups_per_cu(64 * C);
    if (a.listed) {
        const u32 units = max((a.k + a.window + UNIT - 1) / UNIT, 1u), tiles = (a.group + ROWS - 1) / ROWS;
        k_attend_selected<FMT, C><<<grid, 256, 0, st>>>(a, units, tiles);
    } else {
        k_attend<FMT, C><<<grid, 256, 0, st>>>(a);
    }
    k_join<C><<<a.s.tokens * a.heads, 256, 0, st>>>(a, a.listed != 0, (int)grid);
}

}  // namespace

u64 narrow_workspace(u32 width, u64 rows, int num_cu) { return 4 * partial_floats(width, num_cu) + 8 * rows; }

int launch_attend(hipStream_t st, const Attend& args, int num_cu) {
    Attend a = args;
    a.joined = (int2*)(a.partial + partial_floats(a.c.width, num_cu));
    const u32 n = a.c.width / 64;
    if (a.c.fmt == PAG_KV_INT8) {
        if (n == 1) run_attend<PAG_KV_INT8, 1>(st, a, num_cu);
        else if (n == 2) run_attend<PAG_KV_INT8, 2>(st, a, num_cu);
        else if (n == 3) run_attend<PAG_KV_INT8, 3>(st, a, num_cu);
        else run_attend<PAG_KV_INT8, 4>(st, a, num_cu);
    } else {
        if (n == 1) run_attend<PAG_KV_FP8, 1>(st, a, num_cu);
        else if (n == 2) run_attend<PAG_KV_FP8, 2>(st, a, num_cu);
        else if (n == 3) run_attend<PAG_KV_FP8, 3>(st, a, num_cu);
        else run_attend<PAG_KV_FP8, 4>(st, a, num_cu);
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) { pag_set_error(std::string("pag_kv_attend: ") + hipGetErrorString(e)); return PAG_EHIP; }
    return PAG_OK;
}

}  // namespace pagkv
