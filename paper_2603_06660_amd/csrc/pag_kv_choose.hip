// Blocks of tokens: their summaries, and which of them a query reads.
//
// A block's summary is, for each number of its keys, the largest and the smallest of them, as integers of 8 bits with one power of two, rounded outwards.  With q as
// integers of 8 bits the sum of hi * max(q, 0) + lo * min(q, 0) bounds what any of the block's keys scores (but for q's rounding), and is a product of
// matrices: 16 summaries by 16 rows of q, hi by what is positive of q and lo by what is negative, on the integer matrix unit.  Integers add up exactly in any
// order, and a float holds the sum (2 * 256 * 127^2 < 2^23) times a power of two exactly, so which blocks are chosen depends on nothing but the inputs.
#include <algorithm>

#include "pag_kv_attend.h"

namespace pagkv {
namespace {

typedef int int4_t __attribute__((ext_vector_type(4)));

constexpr u32 CHUNK = 256;                  // blocks that a workgroup scores where a list goes to several
constexpr u32 MOST_SHORT = 1024;            // keys of a list that a wave holds in registers
constexpr u32 QUEUE = 1024;                 // workgroups that are too many to run at once

// ---- summaries ------------------------------------------------------------------------------------------------------

// The largest and smallest of 16 numbers of a lane over rows r0 to r1 - 1 of a block, and then over the lanes that have the same numbers: lanes 0 .. 4 C - 1 end up with
// all of them.  16 / C rows a turn, TURNS turns asked for together.
template <int FMT, int C, int TURNS>
__device__ __forceinline__ void extremes_of(const Cache& c, u32 row0, u32 r0, u32 r1, float* hi, float* lo) {
    constexpr u32 LANES = 4 * C, ROWS_A_TURN = 64 / LANES;          // of a row; 12 lanes a row leave four without one
    const u32 lane = threadIdx.x & 63, row = lane / LANES, at = lane % LANES * 16;
#pragma unroll
    for (int j = 0; j < 16; ++j) { hi[j] = -INFINITY; lo[j] = INFINITY; }
    for (; r0 < r1; r0 += TURNS * ROWS_A_TURN) {
        uint4 w[TURNS];
        int e[TURNS];
#pragma unroll
        for (u32 n = 0; n < TURNS; ++n) {                  // behind the last row the last one again
            const u32 r = row0 + min(r0 + n * ROWS_A_TURN + (row < ROWS_A_TURN ? row : 0), r1 - 1);
            if constexpr (FMT == PAG_KV_FP4) {
                const uint2 x = *(const uint2*)(c.data + (u64)r * (64 * C) + at / 2);
                w[n] = make_uint4(x.x, x.y, 0, 0);
                e[n] = parts_of<C>(c, r / BLOCK, 0)[at / PART * BLOCK + r % BLOCK];
            } else {
                w[n] = *(const uint4*)(c.data + (u64)r * (128 * C) + at);
                e[n] = c.exponents[(u64)(r / BLOCK) * 2];
            }
        }
#pragma unroll
        for (u32 n = 0; n < TURNS; ++n) {
            const float up = power(e[n]);
            float x[16];
            if constexpr (FMT == PAG_KV_FP4) {
#pragma unroll
                for (int j = 0; j < 4; ++j) decode4_fp4((j < 2 ? w[n].x : w[n].y) >> (16 * (j & 1)), 1.f, x + 4 * j);
            } else {
                decode4<FMT>(w[n].x, x);
                decode4<FMT>(w[n].y, x + 4);
                decode4<FMT>(w[n].z, x + 8);
                decode4<FMT>(w[n].w, x + 12);
            }
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                const float y = x[j] * up;
                hi[j] = fmaxf(hi[j], y);
                lo[j] = fminf(lo[j], y);
            }
        }
    }
    // rows LANES apart, whatever their number
#pragma unroll
    for (u32 o = 1; o < ROWS_A_TURN; o *= 2) {
        const u32 from = lane + o * LANES < ROWS_A_TURN * LANES ? lane + o * LANES : lane;
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            hi[j] = fmaxf(hi[j], __shfl(hi[j], (int)from));
            lo[j] = fminf(lo[j], __shfl(lo[j], (int)from));
        }
    }
}

// the summary of block `block` of all pages, from what lanes 0 .. 4 C - 1 of a wave have
template <int C>
__device__ __forceinline__ void write_summary(const Cache& c, const Blocks& blocks, u32 block, u32 head, float* hi, float* lo) {
    constexpr u32 LANES = 4 * C;
    const u32 lane = threadIdx.x & 63, at = lane % LANES * 16;
    float most = 0.f;
#pragma unroll
    for (int j = 0; j < 16; ++j) {                  // as the numbers that the cache is read as
        hi[j] = finite(hi[j]);
        lo[j] = finite(lo[j]);
        most = fmaxf(most, fmaxf(fabsf(hi[j]), fabsf(lo[j])));
    }
    most = wave_max(lane < LANES ? most : 0.f);
    const int e = least_exponent<PAG_KV_INT8>(most);
    const float down = power(-e);
    if (lane < LANES) {
        u32 up[4], low[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float x[4], y[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) { x[j] = ceilf(hi[4 * i + j] * down); y[j] = floorf(lo[4 * i + j] * down); }
            up[i] = encode4<PAG_KV_INT8>(x);
            low[i] = encode4<PAG_KV_INT8>(y);
        }
        const u64 to = (u64)(block / blocks.page_blocks * c.kv_heads + head) * blocks.page_blocks + block % blocks.page_blocks;
        int8_t* codes = blocks.codes + to * (128 * C) + at;
        *(uint4*)codes = make_uint4(up[0], up[1], up[2], up[3]);
        *(uint4*)(codes + 64 * C) = make_uint4(low[0], low[1], low[2], low[3]);
        if (lane == 0) blocks.exponents[to] = (int8_t)e;
    }
}

__device__ __forceinline__ u32 row0_of(const Cache& c, const Blocks& blocks, u32 block, u32 head) {
    return row_of(c, block / blocks.page_blocks, head, block % blocks.page_blocks * blocks.tokens);
}

// A wave has a window of new tokens and a head, and writes the summaries of the blocks whose last new token lies in its window: that token is the last one that
// the block holds.  4 requests' 16,384 tokens each, 8 heads, blocks of 64 in int8: 38 us, where reading their keys is 11; widening, comparing and the shuffles at the end do not overlap
// with it enough.
template <int FMT, int C>
__global__ void __launch_bounds__(256) k_summarise(Cache c, Blocks blocks, const int64_t* __restrict__ slots, u64 tokens, u32 window) {
    const u32 lane = threadIdx.x & 63;
    const u64 wave = (u64)blockIdx.x * 4 + (threadIdx.x >> 6), t0 = wave / c.kv_heads * window;
    if (t0 >= tokens) return;
    const u32 head = (u32)(wave % c.kv_heads);
    // lanes 0 .. window: the window and the token behind it
    int64_t slot = -1;
    if (lane <= window && t0 + lane < tokens) slot = slots[t0 + lane];
    if (slot >= (int64_t)c.num_pages * c.page_tokens || slot < 0) slot = -1;
    const int block = slot < 0 ? -1 : (int)((u64)slot / blocks.tokens), place = slot < 0 ? 0 : (int)((u64)slot % blocks.tokens);
    const int right = __shfl_down(block, 1);
    u64 lasts = __ballot(lane < window && block >= 0 && block != right);
    for (; lasts; lasts &= lasts - 1) {
        const int l = __builtin_ctzll(lasts);
        const u32 mine = (u32)__builtin_amdgcn_readlane(block, l);
        float hi[16], lo[16];
        extremes_of<FMT, C, 8>(c, row0_of(c, blocks, mine, head), 0, (u32)__builtin_amdgcn_readlane(place, l) + 1, hi, lo);
        write_summary<C>(c, blocks, mine, head, hi, lo);
    }
}

// A workgroup for a token and head, whose waves share the block's rows, where there are few: one token of each of 48 requests, blocks of 32, 7.4 -> 6.7 us.
template <int FMT, int C>
__global__ void __launch_bounds__(256) k_summarise_one(Cache c, Blocks blocks, const int64_t* __restrict__ slots, u64 tokens) {
    __shared__ float sh[4][32][4 * C + 1];
    const u32 lane = threadIdx.x & 63, wave = wave_of(), head = blockIdx.x % c.kv_heads;
    const u64 t = blockIdx.x / c.kv_heads;
    const int64_t all = (int64_t)c.num_pages * c.page_tokens, slot = slots[t], next = t + 1 < tokens ? slots[t + 1] : -1;
    if (slot < 0 || slot >= all) return;
    const u32 block = (u32)((u64)slot / blocks.tokens), count = (u32)((u64)slot % blocks.tokens) + 1;
    if (next >= 0 && next < all && (u32)((u64)next / blocks.tokens) == block) return;
    const u32 each = (count + 3) / 4, r0 = min(wave * each, count), r1 = min(r0 + each, count);
    float hi[16], lo[16];
    extremes_of<FMT, C, 2>(c, row0_of(c, blocks, block, head), r0, r1, hi, lo);
    if (lane < 4 * C) {
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            sh[wave][j][lane] = hi[j];
            sh[wave][16 + j][lane] = lo[j];
        }
    }
    __syncthreads();
    if (wave) return;
    if (lane < 4 * C) {
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            hi[j] = fmaxf(fmaxf(sh[0][j][lane], sh[1][j][lane]), fmaxf(sh[2][j][lane], sh[3][j][lane]));
            lo[j] = fminf(fminf(sh[0][16 + j][lane], sh[1][16 + j][lane]), fminf(sh[2][16 + j][lane], sh[3][16 + j][lane]));
        }
    }
    write_summary<C>(c, blocks, block, head, hi, lo);
}

// ---- scores ---------------------------------------------------------------------------------------------------------

// Rows of q that a wave scores together: the heads of whole lists where a list has up to 16 heads, 16 of a list's heads otherwise.
struct Columns {
    u32 lists, heads;          // lists of a tile, 0 if a list takes several tiles; heads of a list
    u32 tiles, per_list;       // tiles of a key/value head, tiles of a list
};

__host__ __device__ inline Columns columns_of(u32 group, u32 list_heads) {
    Columns x;
    x.heads = list_heads;
    x.lists = list_heads <= 16 ? 16 / list_heads : 0;
    x.per_list = list_heads <= 16 ? 1 : (list_heads + 15) / 16;
    const u32 all = group / list_heads;
    x.tiles = x.lists ? (all + x.lists - 1) / x.lists : all * x.per_list;
    return x;
}

template <int C>
struct Queries {
    int4_t positive[C], negative[C];
    int e;
};

// Row lane % 16 of a tile: numbers 64 h + 16 (lane / 16) + 0 .. 15 are this lane's; as they come, and as integers
template <int C>
struct RawQueries { uint4 x[2 * C]; };

template <int C>
__device__ __forceinline__ void fetch_queries(const Choose& a, u32 t, u32 head, bool real, RawQueries<C>& raw) {
    const u32 g = (threadIdx.x & 63) >> 4;
    const u64 from = (u64)t * (u64)a.q_ts + (u64)head * (u64)a.q_hs;
#pragma unroll
    for (int n = 0; n < 2 * C; ++n) {
        const u32 at = (n >> 1) * 64 + g * 16 + (n & 1) * 8;
        raw.x[n] = make_uint4(0, 0, 0, 0);
        if (real && at < a.c.dim) raw.x[n] = *(const uint4*)((const uint16_t*)a.q + from + at);
    }
}

template <int C>
__device__ __forceinline__ void encode_queries(const Choose& a, const RawQueries<C>& raw, Queries<C>& q) {
    float most = 0.f, x[8];
#pragma unroll
    for (int n = 0; n < 2 * C; ++n) {
        widen_row8(raw.x[n], a.dtype, x);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float y = fabsf(x[j]);
            if (y <= 3.402823466e38f) most = fmaxf(most, y);
        }
    }
    most = fmaxf(most, __shfl_xor(most, 16));
    most = fmaxf(most, __shfl_xor(most, 32));
    q.e = least_exponent<PAG_KV_INT8>(most);
    const float down = power(-q.e);
#pragma unroll
    for (int n = 0; n < 2 * C; ++n) {
        widen_row8(raw.x[n], a.dtype, x);
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] *= down;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const u32 w = encode4<PAG_KV_INT8>(x + 4 * i), minus = (w >> 7 & 0x01010101u) * 255u;
            q.positive[n >> 1][2 * (n & 1) + i] = (int)(w & ~minus);
            q.negative[n >> 1][2 * (n & 1) + i] = (int)(w & minus);
        }
    }
}

// One tile of columns as integers, by the whole workgroup: 8 numbers a thread (every wave for itself: 450 instructions each, of 1,600), LANES threads a row.
template <int C>
struct SharedQueries {
    static constexpr u32 STRIDE = 128 * C + 16;          // rows that lanes read together begin in different banks
    __align__(16) int8_t codes[16 * STRIDE];
    int e[16];
};

template <int C>
__device__ __forceinline__ void share_queries(const Choose& a, u32 t, u32 head0, u32 rows, SharedQueries<C>& sh) {
    constexpr u32 LANES = C == 3 ? 32 : 8 * C;
    for (u32 i = threadIdx.x; i < 16 * LANES; i += blockDim.x) {
        const u32 row = i / LANES, at = i % LANES * 8;
        uint4 raw = make_uint4(0, 0, 0, 0);
        if (row < rows && at < a.c.dim) raw = *(const uint4*)((const uint16_t*)a.q + (u64)t * (u64)a.q_ts + (u64)(head0 + row) * (u64)a.q_hs + at);
        float x[8], most = 0.f;
        widen_row8(raw, a.dtype, x);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float y = fabsf(x[j]);
            if (y <= 3.402823466e38f) most = fmaxf(most, y);
        }
#pragma unroll
        for (u32 o = 1; o < LANES; o *= 2) most = fmaxf(most, __shfl_xor(most, (int)o));
        const int e = least_exponent<PAG_KV_INT8>(most);
        const float down = power(-e);
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] *= down;
        u32 positive[2], negative[2];
#pragma unroll
        for (int n = 0; n < 2; ++n) {
            const u32 w = encode4<PAG_KV_INT8>(x + 4 * n), minus = (w >> 7 & 0x01010101u) * 255u;
            positive[n] = w & ~minus;
            negative[n] = w & minus;
        }
        if (at < 64 * C) {
            int8_t* to = sh.codes + row * SharedQueries<C>::STRIDE + at;
            *(uint2*)to = make_uint2(positive[0], positive[1]);
            *(uint2*)(to + 64 * C) = make_uint2(negative[0], negative[1]);
        }
        if (at == 0) sh.e[row] = e;
    }
}

template <int C>
__device__ __forceinline__ void take_queries(const SharedQueries<C>& sh, Queries<C>& q) {
    const u32 lane = threadIdx.x & 63, row = lane & 15;
    const int8_t* from = sh.codes + row * SharedQueries<C>::STRIDE + (lane >> 4) * 16;
#pragma unroll
    for (int h = 0; h < C; ++h) {
        q.positive[h] = *(const int4_t*)(from + 64 * h);
        q.negative[h] = *(const int4_t*)(from + 64 * C + 64 * h);
    }
    q.e = sh.e[row];
}

// the query head of this lane's column in a tile of columns, and whether there is one
__device__ __forceinline__ u32 head_of(const Choose& a, const Columns& columns, u32 kv_head, u32 tile, bool& real) {
    const u32 col = threadIdx.x & 15;
    const u32 list0 = columns.lists ? tile * columns.lists : tile / columns.per_list, lists = a.group / columns.heads;
    const u32 head = columns.lists ? list0 * columns.heads + col : list0 * columns.heads + tile % columns.per_list * 16 + col;
    real = head < (columns.lists ? min(lists, list0 + columns.lists) * columns.heads : (list0 + 1) * columns.heads);
    return kv_head * a.group + head;
}

// a token's request, position, and blocks that begin before its window
struct Token {
    u32 request;
    int position;
    u32 blocks;
};

__device__ __forceinline__ Token token_of(const Choose& a, u32 t) {
    Token x;
    // the same for all lanes, and in scalar registers
    const int request = __builtin_amdgcn_readfirstlane(a.s.request[t]);
    x.position = __builtin_amdgcn_readfirstlane(a.s.positions[t]);
    if (request < 0 || (u32)request >= a.s.requests || (u64)(u32)max(x.position, 0) >= (u64)a.s.max_pages * a.c.page_tokens) x.position = -1;
    x.request = x.position >= 0 ? (u32)request : 0;
    x.blocks = x.position >= 0 && (u32)x.position >= a.window ? ((u32)x.position - a.window) / a.b.tokens + 1 : 0;
    return x;
}

// order of floats as that of unsigned numbers; 0 is no float's but a NaN's
__device__ __forceinline__ u32 key_of(float x) {
    const u32 u = __float_as_uint(x);
    return u ^ ((u >> 31) ? 0xFFFFFFFFu : 0x80000000u);
}

// where a lane's block of 64 lies
struct Found {
    u32 at;                    // of its summary
    int e;
    u64 there;                 // which of the 64 are blocks
};

__device__ __forceinline__ Found find_blocks(const Choose& a, const Token& x, u32 kv_head, u32 first) {
    const u32 block = first + (threadIdx.x & 63);
    u32 page = 0xFFFFFFFFu;
    if (block < x.blocks) page = (u32)a.s.table[x.request * a.s.table_stride + block / a.b.page_blocks];
    const bool ok = page < a.c.num_pages;
    Found f;
    f.at = ok ? (page * a.c.kv_heads + kv_head) * a.b.page_blocks + block % a.b.page_blocks : 0;
    f.there = __ballot(ok);
    f.e = a.b.exponents[f.at];
    return f;
}

// a lane's part of 16 summaries: of that of block lane % 16 the 16-byte pieces lane / 16 + 4 h of either row
template <int C>
struct Summaries { int4_t hi[C], lo[C]; };

template <int C>
__device__ __forceinline__ void load_summaries(const Choose& a, const Found& f, u32 tile, Summaries<C>& s) {
    const u32 lane = threadIdx.x & 63;
    const int8_t* codes = a.b.codes + (u64)(u32)__shfl((int)f.at, (int)(16 * tile + (lane & 15))) * (128 * C) + (lane >> 4) * 16;
#pragma unroll
    for (int h = 0; h < C; ++h) {
        s.hi[h] = *(const int4_t*)(codes + 64 * h);
        s.lo[h] = *(const int4_t*)(codes + 64 * C + 64 * h);
    }
}

// Scores of 16 blocks and a tile of columns: y[i] is that of block 4 (lane / 16) + i, of all heads of a list that are in the tile, in the list's first column.
template <int C>
__device__ __forceinline__ void score_tile(const Found& f, u32 tile, const Summaries<C>& s, const Queries<C>& q, const Columns& columns, bool real, float* y) {
    const u32 lane = threadIdx.x & 63, col = lane & 15, g = lane >> 4;
    int4_t sum = { 0, 0, 0, 0 };
#pragma unroll
    for (int h = 0; h < C; ++h) {
        sum = __builtin_amdgcn_mfma_i32_16x16x64_i8(s.hi[h], q.positive[h], sum, 0, 0, 0);
        sum = __builtin_amdgcn_mfma_i32_16x16x64_i8(s.lo[h], q.negative[h], sum, 0, 0, 0);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int e = __shfl(f.e, (int)(16 * tile + 4 * g) + i);
        y[i] = real ? __builtin_ldexpf((float)sum[i], q.e + e) : -INFINITY;
    }
    const u32 width = columns.lists ? columns.heads : 16, last = columns.lists ? min(15u, col / width * width + width - 1) : 15;
    for (u32 o = 1; o < width; o *= 2) {
        const int from = (int)(16 * g + min(col + o, last));
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = fmaxf(y[i], __shfl(y[i], from));
    }
}

// 64 blocks, from block first on, of a token and key/value head: their scores as keys, 0 for blocks that are none, to out(block, key) in each list's first column.  One tile of columns: a
// tile of 16 summaries is on its way while another one is multiplied.  ready: called when the first two have been asked for.
template <int C, typename Ready, typename Out>
__device__ __forceinline__ void score_blocks(const Choose& a, const Token& x, u32 kv_head, u32 first, const Columns& columns, bool real, const Queries<C>& q, Ready&& ready,
                                             Out&& out) {      // real: this lane's column is one
    const u32 lane = threadIdx.x & 63, col = lane & 15, g = lane >> 4, width = columns.lists ? columns.heads : 16;
    const bool writes = real && col % width == 0;
    const Found f = find_blocks(a, x, kv_head, first);
    Summaries<C> s[2];
    load_summaries<C>(a, f, 0, s[0]);
    load_summaries<C>(a, f, 1, s[1]);
    ready();
#pragma unroll
    for (int tile = 0; tile < 4; ++tile) {
        if (first + tile * 16 >= x.blocks) break;
        float y[4];
        score_tile<C>(f, tile, s[tile & 1], q, columns, real, y);
        if (tile < 2) load_summaries<C>(a, f, tile + 2, s[tile & 1]);
        if (writes) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const u32 b = tile * 16 + 4 * g + i;
                if (first + b < x.blocks) out(first + b, (f.there >> b & 1u) ? key_of(y[i]) : 0u);
            }
        }
    }
}

// The same of several tiles of columns, to out(list, block, key); queries are looked at anew for each 64 blocks.
template <int C, typename Out>
__device__ __forceinline__ void score_columns(const Choose& a, const Token& x, u32 kv_head, u32 first, const Columns& columns, u32 t, Out&& out) {
    const u32 lane = threadIdx.x & 63, col = lane & 15, g = lane >> 4;
    const Found f = find_blocks(a, x, kv_head, first);
    float best[4][4];
#pragma unroll 1
    for (u32 tile = 0; tile < columns.tiles; ++tile) {
        const u32 list0 = columns.lists ? tile * columns.lists : tile / columns.per_list, width = columns.lists ? columns.heads : 16;
        bool real;
        const u32 head = head_of(a, columns, kv_head, tile, real);
        RawQueries<C> raw;
        Queries<C> q;
        fetch_queries<C>(a, t, head, real, raw);
        encode_queries<C>(a, raw, q);
        const bool begins = columns.lists || tile % columns.per_list == 0, ends = columns.lists || tile % columns.per_list + 1 == columns.per_list;
#pragma unroll
        for (int n = 0; n < 4; ++n) {
            if (first + n * 16 >= x.blocks) break;
            Summaries<C> s;
            load_summaries<C>(a, f, n, s);
            float y[4];
            score_tile<C>(f, n, s, q, columns, real, y);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                best[n][i] = begins ? y[i] : fmaxf(best[n][i], y[i]);
                const u32 b = n * 16 + 4 * g + i;
                if (ends && real && col % width == 0 && first + b < x.blocks) out(list0 + (columns.lists ? col / width : 0), first + b, (f.there >> b & 1u) ? key_of(best[n][i]) : 0u);
            }
        }
    }
}

// ---- the best ones --------------------------------------------------------------------------------------------------

// bits of a mask below this lane's
__device__ __forceinline__ u32 below(u64 mask) { return __builtin_amdgcn_mbcnt_hi((u32)(mask >> 32), __builtin_amdgcn_mbcnt_lo((u32)mask, 0u)); }

// Writes the numbers of the keys above the cut, and of the first ones equal to it while there are ties left, in their order.  to: how many came before, equal: how many of
// those equal to the cut.
__device__ __forceinline__ void write_chosen(u32 key, u32 number, u32 cut, u32 ties, int32_t* ids, u32& to, u32& equal) {
    const u64 may = __ballot(ties ? key >= cut && key != 0 : key > cut);
    if (!may) return;
    u64 all = may;
    if (ties) {
        const u64 same = __ballot(key == cut && key != 0);
        all = __ballot(key > cut || (key == cut && key != 0 && equal + below(same) < ties));
        equal += (u32)__popcll(same);
    }
    if (all >> (threadIdx.x & 63) & 1u) ids[to + below(all)] = (int32_t)number;
    to += (u32)__popcll(all);
}

// ids that a list has no block for
__device__ __forceinline__ void write_none(int32_t* ids, u32 from, u32 k, u32 thread, u32 threads) {
    for (u32 i = from + thread; i < k; i += threads) ids[i] = -1;
}

// The k largest of up to 64 R keys, the first ones of those that are equal, in their order, by a wave: the k-th largest key is found bit by bit, by counting,
// from the first bit in which keys differ on; once exactly k keys reach what is found, the rest of the bits does not matter.  Registers without a key hold 0 and
// are counted like the others: a branch around each costs more than its comparison.  Once the k-th is among 64 keys or fewer these go into one register,
// by way of the keys' own place in LDS.
template <int R>
__device__ __forceinline__ void pick_short(u32* keys, u32 n, u32 k, int32_t* ids) {
    const u32 lane = threadIdx.x & 63;
    u32 x[R], most = 0, least = 0xFFFFFFFFu, valid = 0;
#pragma unroll
    for (int r = 0; r < R; ++r) {
        x[r] = r * 64 + lane < n ? keys[r * 64 + lane] : 0u;
        most = max(most, x[r]);
        least = min(least, x[r] ? x[r] : 0xFFFFFFFFu);
        valid += (u32)__popcll(__ballot(x[r] != 0));
    }
#pragma unroll
    for (int o = 32; o; o >>= 1) {
        most = max(most, (u32)__shfl_xor((int)most, o));
        least = min(least, (u32)__shfl_xor((int)least, o));
    }
    u32 cut = 0, ties = 0;                   // keys above the cut, and the first `ties` that are equal to it
    if (valid > k) {
        const u32 differ = (u32)__builtin_amdgcn_readfirstlane((int)(most ^ least));
        int bit = differ ? 31 - __builtin_clz(differ) : -1;
        u32 at = bit < 0 ? most : most & ~((2u << bit) - 1);
        at = (u32)__builtin_amdgcn_readfirstlane((int)at);
        u32 above = 0, upto = valid;             // keys of at + 2^(bit + 1) and more, and of `at` and more
        const auto step = [&](u32 count) {
            if (count >= k) {
                at |= 1u << bit;
                upto = count;
            } else {
                above = count;
            }
            --bit;
            return count == k;
        };
        bool done = false;
        while (!done && bit >= 0 && upto - above > 64) {
            u32 count = 0;
#pragma unroll
            for (int r = 0; r < R; ++r) count += (u32)__popcll(__ballot(x[r] >= (at | 1u << bit)));
            done = step(count);
        }
        if (!done && bit >= 0) {
            u32 found = 0;
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const bool in = x[r] != 0 && x[r] >= at && (x[r] - at) >> bit < 2;
                const u64 mask = __ballot(in);
                if (in) keys[found + below(mask)] = x[r];
                found += (u32)__popcll(mask);
            }
            __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
            __builtin_amdgcn_wave_barrier();
            __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
            const u32 y = lane < found ? keys[lane] : 0u;
            const u32 more = above;
            while (!done && bit >= 0) done = step(more + (u32)__popcll(__ballot(y >= (at | 1u << bit))));
        }
        cut = done ? at - 1 : at;
        ties = done ? 0 : k - above;
    }
    u32 to = 0, equal = 0;
#pragma unroll
    for (int r = 0; r < R; ++r) write_chosen(x[r], r * 64 + lane, cut, ties, ids, to, equal);
    write_none(ids, to, k, lane, 64);
}

// The same by a workgroup of WAVES waves, each of which has a run of the keys: in HELD registers a lane, if they last.  Counting by all of them costs a
// barrier a bit, so keys are counted once in BINS parts of their range, which leaves a few keys around the k-th.
constexpr int LOG_BINS = 10;
constexpr u32 BINS = 1u << LOG_BINS;

__device__ __forceinline__ u32 place_of(u32 bin) {
    const u32 from_top = BINS - 1 - bin;
    return from_top % (BINS / 64) * 64 + from_top / (BINS / 64);
}

template <int WAVES, int HELD>
__device__ __forceinline__ void pick_long(const u32* keys, u32 n, u32 k, int32_t* ids) {
    constexpr int R = HELD ? HELD : 1;
    __shared__ u32 sh_count[32], sh_bins[BINS], sh_found[64];
    __shared__ u32 sh_most[WAVES], sh_least[WAVES], sh_above[WAVES], sh_same[WAVES];
    const u32 lane = threadIdx.x & 63, wave = wave_of();
    const u32 run = (n + 64 * WAVES - 1) / (64 * WAVES) * 64, r0 = min(wave * run, n), r1 = min(r0 + run, n), turns = (r1 - r0 + 63) / 64;
    u32 x[R];
    const auto key = [&](u32 r) -> u32 { return r0 + r * 64 + lane < r1 ? keys[r0 + r * 64 + lane] : 0u; };
    // f(key, its number) of all of the wave's keys in their order
    const auto each = [&](auto&& f) {
        if constexpr (HELD) {
#pragma unroll
            for (int r = 0; r < R; ++r) f(x[r], (u32)r);
        } else {
            for (u32 r = 0; r < turns; ++r) f(key(r), r);
        }
    };
    if constexpr (HELD) {
#pragma unroll
        for (int r = 0; r < R; ++r) x[r] = key((u32)r);
    }
    if (threadIdx.x < 32) sh_count[threadIdx.x] = 0;
    for (u32 i = threadIdx.x; i < BINS; i += 64 * WAVES) sh_bins[i] = 0;
    u32 most = 0, least = 0xFFFFFFFFu;               // less 1: 0 is no key
    each([&](u32 y, u32) {
        most = max(most, y);
        least = min(least, y - 1);
    });
#pragma unroll
    for (int o = 32; o; o >>= 1) {
        most = max(most, (u32)__shfl_xor((int)most, o));
        least = min(least, (u32)__shfl_xor((int)least, o));
    }
    __syncthreads();
    if (lane == 0) {
        sh_most[wave] = most;
        sh_least[wave] = least;
    }
    __syncthreads();
#pragma unroll
    for (u32 w = 0; w < WAVES; ++w) {
        most = max(most, sh_most[w]);
        least = min(least, sh_least[w]);
    }
    most = (u32)__builtin_amdgcn_readfirstlane((int)most);
    least = (u32)__builtin_amdgcn_readfirstlane((int)least) + 1;
    u32 cut = 0, ties = 0;
    if (most && n > k) {
        // which of BINS equal parts of the keys' range has the k-th largest, and how many are above that part
        const u32 range = most - least;
        const int shift = max(32 - __builtin_clz(range | 1u) - LOG_BINS, 0);
        each([&](u32 y, u32) { if (y) atomicAdd(&sh_bins[place_of((y - least) >> shift)], 1u); });
        lds_barrier();
        u32 above = 0, bin = 0, valid;
        {
            // every wave adds up all parts, from the top: lane l has 16 of them, the topmost ones lane 0; side by side in LDS lie those that lanes read together
            constexpr u32 EACH = BINS / 64;
            u32 c[EACH], sum = 0;
#pragma unroll
            for (u32 i = 0; i < EACH; ++i) { c[i] = sh_bins[i * 64 + lane]; sum += c[i]; }
            u32 upto = sum;
#pragma unroll
            for (u32 o = 1; o < 64; o <<= 1) {
                const u32 y = (u32)__shfl_up((int)upto, o);
                if (lane >= o) upto += y;
            }
            const u64 reach = __ballot(upto >= k);
            const int l = reach ? __builtin_ctzll(reach) : 63;
            valid = (u32)__builtin_amdgcn_readlane((int)upto, 63);
            u32 before = upto - sum;
            u32 mine = 0;
#pragma unroll
            for (u32 i = 0; i < EACH; ++i) {
                if (before < k) { mine = i; above = before; }
                before += c[i];
            }
            bin = BINS - 1 - ((u32)l * EACH + (u32)__builtin_amdgcn_readlane((int)mine, l));
            above = (u32)__builtin_amdgcn_readlane((int)above, l);
        }
        // that part's keys, bit by bit: by each wave for itself where a register of them is enough, by all waves otherwise
        if (valid > k) {
            const u32 low = least + (bin << shift), need = k - above, inside = (u32)__builtin_amdgcn_readfirstlane((int)sh_bins[place_of(bin)]);
            int bit = shift - 1;
            u32 at = 0, over = 0;                    // counted from low
            bool done = inside == need;
            const auto step = [&](u32 count, u32 to) {
                if (count >= need) at = to;
                else over = count;
                done = count == need;
            };
            if (!done && inside <= 64) {
                each([&](u32 y, u32) { if (y >= low && (y - low) >> shift == 0) sh_found[atomicAdd(&sh_count[0], 1u)] = y - low; });
                lds_barrier();
                const u32 y = lane < inside ? sh_found[lane] : 0u;
                for (; bit >= 0 && !done; --bit) step((u32)__popcll(__ballot(lane < inside && y >= (at | 1u << bit))), at | 1u << bit);
            } else if (!done) {
                for (; bit >= 0 && !done; --bit) {
                    const u32 to = at | 1u << bit;
                    u32 count = 0;
                    each([&](u32 y, u32) { count += (u32)__popcll(__ballot(y >= low && (y - low) >> shift == 0 && y - low >= to)); });
                    if (lane == 0 && count) atomicAdd(&sh_count[bit], count);
                    lds_barrier();
                    step((u32)__builtin_amdgcn_readfirstlane((int)sh_count[bit]), to);
                }
            }
            cut = low + at - (done ? 1 : 0);
            ties = done ? 0 : need - over;
        }
    }
    // where this wave's keys go
    u32 over = 0, same = 0;
    each([&](u32 y, u32) { over += (u32)__popcll(__ballot(y > cut)); });
    if (ties) each([&](u32 y, u32) { same += (u32)__popcll(__ballot(y == cut)); });          // the cut is a key then
    if (lane == 0) { sh_above[wave] = over; sh_same[wave] = same; }
    lds_barrier();
    u32 to = 0, equal = 0, all = 0, all_same = 0;
#pragma unroll
    for (u32 w = 0; w < WAVES; ++w) {
        if (w < wave) { to += sh_above[w]; equal += sh_same[w]; }
        all += sh_above[w];
        all_same += sh_same[w];
    }
    to += min(equal, ties);
    each([&](u32 y, u32 r) { write_chosen(y, r0 + r * 64 + lane, cut, ties, ids, to, equal); });
    write_none(ids, all + min(all_same, ties), k, threadIdx.x, 64 * WAVES);
}

// A workgroup for a token and key/value head: scores into LDS, then a wave a list.  MANY: several tiles of columns, whose rows of q need registers for two waves a SIMD only (64 heads
// over 2 for 48 requests of up to 625 blocks 43 us with four waves and 43 spilled registers, 36 this way).  48 requests, 32 lists each of up to 625 blocks: 19 us, of which 6 for
// choosing, by four waves of eight; the 33 MB of summaries are 6 at the memory's rate.
template <int C, int NW, bool MANY>
__global__ void __launch_bounds__(64 * NW, C <= 2 && !MANY ? 4 : 2) k_choose(Choose a, Columns columns, u32 room) {
    extern __shared__ u32 sh_keys[];
    const u32 t = blockIdx.x / a.c.kv_heads, kv_head = blockIdx.x % a.c.kv_heads, wave = wave_of(), lists = a.group / columns.heads;
    u32 blocks;
    if constexpr (MANY) {
        const auto out = [&](u32 list, u32 block, u32 key) { sh_keys[list * room + block] = key; };
        const Token x = token_of(a, t);
        blocks = x.blocks;
        for (u32 first = wave * 64; first < x.blocks; first += 64 * NW) score_columns<C>(a, x, kv_head, first, columns, t, out);
    } else {
        __shared__ SharedQueries<C> sh;
        const u32 col = threadIdx.x & 15, width = columns.lists ? columns.heads : 16;
        share_queries<C>(a, t, kv_head * a.group, a.group, sh);
        const Token x = token_of(a, t);
        blocks = x.blocks;
        u32* keys = sh_keys + col / width * room;
        Queries<C> q;
        bool waits = true;
        const auto ready = [&]() {
            if (waits) {
                __syncthreads();
                take_queries<C>(sh, q);
            }
            waits = false;
        };
        for (u32 first = wave * 64; first < x.blocks; first += 64 * NW)
            score_blocks<C>(a, x, kv_head, first, columns, col < a.group, q, ready, [&](u32 block, u32 key) { keys[block] = key; });
        if (waits) __syncthreads();
    }
    __syncthreads();
    for (u32 list = wave; list < lists; list += NW) {
        u32* keys = sh_keys + list * room;
        int32_t* ids = a.ids + (int64_t)t * a.ids_ts + (int64_t)(kv_head * lists + list) * a.ids_hs;
        if (blocks <= 64 * 4) pick_short<4>(keys, blocks, a.k, ids);
        else if (blocks <= 64 * 8) pick_short<8>(keys, blocks, a.k, ids);
        else pick_short<MOST_SHORT / 64>(keys, blocks, a.k, ids);
    }
}

// Scores of a long list's part, 64 blocks a wave.  Bound by waits for table, exponents and summaries, one after the other: 8 lists of 6,250 blocks 7.7 us, and 7.9 for k_pick.
template <int C, bool MANY>
__global__ void __launch_bounds__(256) k_score(Choose a, Columns columns, u32 chunks) {
    const u32 part = blockIdx.x % chunks, list0 = blockIdx.x / chunks, t = list0 / a.c.kv_heads, kv_head = list0 % a.c.kv_heads, lists = a.group / columns.heads;
    const u32 first = (part * 4 + wave_of()) * 64;
    if constexpr (MANY) {
        const auto out = [&](u32 list, u32 block, u32 key) { a.keys[((u64)t * a.id_heads + kv_head * lists + list) * a.most_blocks + block] = key; };
        const Token x = token_of(a, t);
        if (first < x.blocks) score_columns<C>(a, x, kv_head, first, columns, t, out);
    } else {
        __shared__ SharedQueries<C> sh;
        const u32 col = threadIdx.x & 15, width = columns.lists ? columns.heads : 16;
        share_queries<C>(a, t, kv_head * a.group, a.group, sh);
        const Token x = token_of(a, t);
        u32* keys = a.keys + ((u64)t * a.id_heads + kv_head * lists + col / width) * a.most_blocks;
        Queries<C> q;
        if (first < x.blocks) {
            score_blocks<C>(a, x, kv_head, first, columns, col < a.group, q, [&]() { __syncthreads(); take_queries<C>(sh, q); }, [&](u32 block, u32 key) { keys[block] = key; });
        } else {
            __syncthreads();
        }
    }
}

template <int WAVES, int HELD>
__global__ void __launch_bounds__(64 * WAVES) k_pick(Choose a) {
    const u32 t = blockIdx.x / a.id_heads, list = blockIdx.x % a.id_heads;
    const Token x = token_of(a, t);
    pick_long<WAVES, HELD>(a.keys + (u64)blockIdx.x * a.most_blocks, x.blocks, a.k, a.ids + (int64_t)t * a.ids_ts + (int64_t)list * a.ids_hs);
}

// One workgroup for all lists of a head, or parts of them and a second kernel, where a wave's registers do not last for a list's keys, or LDS for all lists'
// (64 KB, of which the queries take up to 8.5).
bool choose_whole(const Choose& a) {
    static_assert(sizeof(SharedQueries<4>) <= 9 * 1024, "queries and keys share 64 KB");
    return a.most_blocks <= MOST_SHORT && (u64)(a.id_heads / a.c.kv_heads) * a.most_blocks * 4 <= 55 * 1024;
}

// Tokens of a launch, where scores go through the workspace: as many as have room in ROOM bytes, one at least, in launches of about as many tokens each.  A launch has
// fewer than 2^32 threads, 256 for CHUNK blocks of a key/value head (one token's are fewer, the host has looked) and up to 1024 for a list.
// What several launches cost (32 lists of 8,192 blocks for 4,096 tokens, 10,810 us in one launch and 4.3 GB): 10,950 to 11,010 in 8 launches, 11,120 in 16 of 256 MB, 12,190 in 64 of 64 MB, whose
// last workgroups leave the chip idle more often.
constexpr u64 ROOM = 512ull << 20;

u32 tokens_of_launch(const Choose& a) {
    const u64 each = 4 * (u64)a.id_heads * a.most_blocks, groups = (u64)a.c.kv_heads * ((a.most_blocks + CHUNK - 1) / CHUNK);
    const u64 most = std::max<u64>(std::min({ ROOM / each, ((1ull << 24) - 1) / groups, ((1ull << 22) - 1) / a.id_heads }), 1);
    const u64 launches = std::max<u64>((a.s.tokens + most - 1) / most, 1);
    return (u32)((a.s.tokens + launches - 1) / launches);
}

template <int C, bool MANY>
void launch(hipStream_t st, const Choose& a, const Columns& columns) {
    const u32 lists = a.id_heads / a.c.kv_heads;
    if (choose_whole(a)) {
        // As many waves as have 64 blocks to score or a list to choose from; where workgroups queue, a wave for 256 blocks, in us: 1,024 tokens of 4 requests and
        // 8 heads, 129 blocks 52, 41, 257 blocks 115, 68, 938 blocks 258, 224; 512 requests and 4 heads of up to 313 blocks 40, 32
        const u32 grid = a.s.tokens * a.c.kv_heads, each = grid >= QUEUE ? 256 : 64, waves = std::max((a.most_blocks + each - 1) / each, lists), room = lists * a.most_blocks * 4;
        if (!MANY && waves <= 2) k_choose<C, 2, false><<<grid, 128, room, st>>>(a, columns, a.most_blocks);
        else if (!MANY && waves <= 4) k_choose<C, 4, false><<<grid, 256, room, st>>>(a, columns, a.most_blocks);
        else k_choose<C, 8, MANY><<<grid, 512, room, st>>>(a, columns, a.most_blocks);
        return;
    }
    const u32 chunks = (a.most_blocks + CHUNK - 1) / CHUNK, each = tokens_of_launch(a);
    for (u32 t0 = 0; t0 < a.s.tokens; t0 += each) {
        Choose x = a;
        x.s.tokens = std::min(each, a.s.tokens - t0);
        x.s.request += t0;
        x.s.positions += t0;
        x.q = (const uint16_t*)a.q + (int64_t)t0 * a.q_ts;
        x.ids += (int64_t)t0 * a.ids_ts;
        const u32 grid = x.s.tokens * a.id_heads;
        k_score<C, MANY><<<x.s.tokens * a.c.kv_heads * chunks, 256, 0, st>>>(x, columns, chunks);
        if (a.most_blocks <= 8 * 64 * 8) k_pick<8, 8><<<grid, 512, 0, st>>>(x);
        else if (a.most_blocks <= 8 * 64 * 16) k_pick<8, 16><<<grid, 512, 0, st>>>(x);
        else if (a.most_blocks <= 8 * 64 * 32) k_pick<8, 32><<<grid, 512, 0, st>>>(x);
        else k_pick<16, 0><<<grid, 1024, 0, st>>>(x);
    }
}

template <int C>
void run(hipStream_t st, const Choose& a) {
    const Columns columns = columns_of(a.group, a.heads / a.id_heads);
    if (columns.tiles > 1) launch<C, true>(st, a, columns);
    else launch<C, false>(st, a, columns);
}

template <int FMT, int C>
void summarise(hipStream_t st, const Cache& c, const Blocks& b, const int64_t* slots, u64 tokens) {
    // a decoding step's blocks are spread over as many waves as there are; prompts' waves look at 32 tokens, most of which are not the last of a block
    if (tokens * c.kv_heads <= 4096) {
        k_summarise_one<FMT, C><<<(u32)(tokens * c.kv_heads), 256, 0, st>>>(c, b, slots, tokens);
        return;
    }
    const u32 window = 32;
    k_summarise<FMT, C><<<(u32)(((tokens + window - 1) / window * c.kv_heads + 3) / 4), 256, 0, st>>>(c, b, slots, tokens, window);
}

template <int FMT>
void summarise_width(hipStream_t st, const Cache& c, const Blocks& b, const int64_t* slots, u64 tokens) {
    const u32 n = c.width / 64;
    if (n == 1) summarise<FMT, 1>(st, c, b, slots, tokens);
    else if (n == 2) summarise<FMT, 2>(st, c, b, slots, tokens);
    else if (n == 3) summarise<FMT, 3>(st, c, b, slots, tokens);
    else summarise<FMT, 4>(st, c, b, slots, tokens);
}

int launched(const char* what) {
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) { pag_set_error(std::string(what) + ": " + hipGetErrorString(e)); return PAG_EHIP; }
    return PAG_OK;
}

}  // namespace

u64 choose_workspace(const Choose& a) { return choose_whole(a) ? 0 : 4 * (u64)tokens_of_launch(a) * a.id_heads * a.most_blocks; }

u64 choose_groups(const Choose& a) { return (u64)a.c.kv_heads * ((a.most_blocks + CHUNK - 1) / CHUNK); }

int launch_summarise(hipStream_t st, const Cache& c, const Blocks& b, const int64_t* slots, u64 tokens) {
    if (c.fmt == PAG_KV_INT8) summarise_width<PAG_KV_INT8>(st, c, b, slots, tokens);
    else if (c.fmt == PAG_KV_FP8) summarise_width<PAG_KV_FP8>(st, c, b, slots, tokens);
    else summarise_width<PAG_KV_FP4>(st, c, b, slots, tokens);
    return launched("pag_kv_blocks_update");
}

int launch_choose(hipStream_t st, const Choose& a) {
    const u32 n = a.c.width / 64;
    if (n == 1) run<1>(st, a);
    else if (n == 2) run<2>(st, a);
    else if (n == 3) run<3>(st, a);
    else run<4>(st, a);
    return launched("pag_kv_blocks_select");
}

}  // namespace pagkv
