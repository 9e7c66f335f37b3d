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

constexpr u32 SPLIT_TILES = 2;              // tiles of 16 blocks that a wave scores where a list goes to several workgroups
constexpr u32 MOST_SHORT = 1024;            // blocks of a list that one wave picks from, held in registers
constexpr u32 PICK_THREADS = 1024;
constexpr u32 LDS_KEYS = 16384;             // of a list that a workgroup picks from

// ---- summaries ------------------------------------------------------------------------------------------------------

// A wave has a window of new tokens and a head, and writes the summaries of the blocks whose last new token lies in its window: that token is the last one that
// the block holds.  16 numbers of a row are a lane's, 16 / C rows a turn.
template <int FMT, int C>
__global__ void __launch_bounds__(256) k_summarise(Cache c, Blocks blocks, const int64_t* __restrict__ slots, u64 tokens, u32 window) {
    constexpr u32 LANES = 4 * C, ROWS_A_TURN = 64 / LANES;          // of a row; 3 C = 192 numbers leave four lanes without one
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
    u64 lasts = __ballot(lane < window && block >= 0 && (lane == 63 || block != right));
    const u32 row = lane / LANES, at = lane % LANES * 16;
    const bool busy = row < ROWS_A_TURN;
    for (; lasts; lasts &= lasts - 1) {
        const int l = __builtin_ctzll(lasts);
        const u32 mine = (u32)__builtin_amdgcn_readlane(block, l), count = (u32)__builtin_amdgcn_readlane(place, l) + 1;
        const u32 page = mine / blocks.page_blocks, first = mine % blocks.page_blocks * blocks.tokens, row0 = row_of(c, page, head, first);
        float hi[16], lo[16];
#pragma unroll
        for (int j = 0; j < 16; ++j) { hi[j] = -INFINITY; lo[j] = INFINITY; }
        for (u32 r0 = 0; r0 < count; r0 += 4 * ROWS_A_TURN) {
            uint4 w[4];
            int e[4];
#pragma unroll
            for (u32 n = 0; n < 4; ++n) {                  // behind the last row the last one again
                const u32 r = row0 + min(r0 + n * ROWS_A_TURN + (busy ? row : 0), count - 1);
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
            for (u32 n = 0; n < 4; ++n) {
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
                    const float y = finite(x[j] * up);
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
        float most = 0.f;
#pragma unroll
        for (int j = 0; j < 16; ++j) most = fmaxf(most, fmaxf(fabsf(hi[j]), fabsf(lo[j])));
        most = lane < LANES ? most : 0.f;
        most = wave_max(most);
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
            const u64 to = (u64)(page * c.kv_heads + head) * blocks.page_blocks + mine % blocks.page_blocks;
            int8_t* codes = blocks.codes + to * (128 * C) + at;
            *(uint4*)codes = make_uint4(up[0], up[1], up[2], up[3]);
            *(uint4*)(codes + 64 * C) = make_uint4(low[0], low[1], low[2], low[3]);
            if (lane == 0) blocks.exponents[to] = (int8_t)e;
        }
    }
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

// Row lane % 16 of a tile as integers: numbers 64 h + 16 (lane / 16) + 0 .. 15 are this lane's.
template <int C>
__device__ __forceinline__ void load_queries(const Choose& a, u32 t, u32 head, bool real, Queries<C>& q) {
    const u32 g = (threadIdx.x & 63) >> 4;
    const u64 from = (u64)t * (u64)a.q_ts + (u64)head * (u64)a.q_hs;
    uint4 raw[2 * C];
#pragma unroll
    for (int n = 0; n < 2 * C; ++n) {
        const u32 at = (n >> 1) * 64 + g * 16 + (n & 1) * 8;
        raw[n] = make_uint4(0, 0, 0, 0);
        if (real && at < a.c.dim) raw[n] = *(const uint4*)((const uint16_t*)a.q + from + at);
    }
    float most = 0.f, x[8];
#pragma unroll
    for (int n = 0; n < 2 * C; ++n) {
        widen_row8(raw[n], a.dtype, x);
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
        widen_row8(raw[n], a.dtype, x);
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

// a token's request, position, and blocks that begin before its window
struct Token {
    u32 request;
    int position;
    u32 blocks;
};

__device__ __forceinline__ Token token_of(const Choose& a, u32 t) {
    Token x;
    const int request = a.s.request[t];
    x.position = a.s.positions[t];
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

// A tile of 16 blocks, from block first on, of a token and key/value head: their scores as keys, 0 for blocks that are none, to out(list, block, key).
template <int C, typename Out>
__device__ __forceinline__ void score_tile(const Choose& a, const Token& x, u32 kv_head, u32 first, const Columns& columns, u32 t, Queries<C>& q, u32& loaded, Out&& out) {
    const u32 lane = threadIdx.x & 63, col = lane & 15, g = lane >> 4;
    const u32 block = first + col;
    u32 page = 0xFFFFFFFFu;
    if (block < x.blocks) page = (u32)a.s.table[x.request * a.s.table_stride + block / a.b.page_blocks];
    const bool ok = page < a.c.num_pages;
    const u64 at = ok ? (u64)(page * a.c.kv_heads + kv_head) * a.b.page_blocks + block % a.b.page_blocks : 0;
    const int8_t* codes = a.b.codes + at * (128 * C) + g * 16;
    int4_t hi[C], lo[C];
#pragma unroll
    for (int h = 0; h < C; ++h) {
        hi[h] = *(const int4_t*)(codes + 64 * h);
        lo[h] = *(const int4_t*)(codes + 64 * C + 64 * h);
    }
    const int e_mine = a.b.exponents[at];
    const u32 there = (u32)__ballot(ok) & 0xFFFFu;
    int e[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) e[i] = __shfl(e_mine, (int)(4 * g) + i);
    float best[4];
    for (u32 tile = 0; tile < columns.tiles; ++tile) {
        const u32 list0 = columns.lists ? tile * columns.lists : tile / columns.per_list, lists = a.group / columns.heads;
        const u32 head = columns.lists ? list0 * columns.heads + col : list0 * columns.heads + tile % columns.per_list * 16 + col;
        const u32 end = columns.lists ? min(lists, list0 + columns.lists) * columns.heads : (list0 + 1) * columns.heads;
        const bool real = head < end;
        if (loaded != tile) {
            load_queries<C>(a, t, kv_head * a.group + head, real, q);
            loaded = tile;
        }
        int4_t s = { 0, 0, 0, 0 };
#pragma unroll
        for (int h = 0; h < C; ++h) {
            s = __builtin_amdgcn_mfma_i32_16x16x64_i8(hi[h], q.positive[h], s, 0, 0, 0);
            s = __builtin_amdgcn_mfma_i32_16x16x64_i8(lo[h], q.negative[h], s, 0, 0, 0);
        }
        float y[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = real ? __builtin_ldexpf((float)s[i], q.e + e[i]) : -INFINITY;
        // the largest of a list's heads, in its first column
        const u32 width = columns.lists ? columns.heads : 16, last = columns.lists ? min(15u, col / width * width + width - 1) : 15;
        for (u32 o = 1; o < width; o *= 2) {
            const int from = (int)(16 * g + min(col + o, last));
#pragma unroll
            for (int i = 0; i < 4; ++i) y[i] = fmaxf(y[i], __shfl(y[i], from));
        }
        if (!columns.lists) {
            const bool begins = tile % columns.per_list == 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) best[i] = begins ? y[i] : fmaxf(best[i], y[i]);
            if (tile % columns.per_list + 1 < columns.per_list) continue;
#pragma unroll
            for (int i = 0; i < 4; ++i) y[i] = best[i];
        }
        if (real && (columns.lists ? col % width == 0 : col == 0)) {
            const u32 list = columns.lists ? list0 + col / width : list0;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const u32 b = 4 * g + i;
                if (first + b < x.blocks) out(list, first + b, (there >> b & 1u) ? key_of(y[i]) : 0u);
            }
        }
    }
}

// ---- the best ones --------------------------------------------------------------------------------------------------

// ids that a list has no block for
__device__ __forceinline__ void write_none(int32_t* ids, u32 from, u32 k, u32 thread, u32 threads) {
    for (u32 i = from + thread; i < k; i += threads) ids[i] = -1;
}

// The k largest of up to MOST_SHORT keys, the first ones of those that are equal, in their order, by a wave: the k-th largest key is found bit by bit, by counting,
// from the first bit in which keys differ on; once exactly k keys reach what is found, the rest of the bits does not matter.
__device__ __forceinline__ void pick_short(const u32* keys, u32 n, u32 k, int32_t* ids) {
    constexpr int R = MOST_SHORT / 64;
    const u32 lane = threadIdx.x & 63;
    u32 x[R], most = 0, least = 0xFFFFFFFFu, valid = 0;
    const int turns = (int)(n + 63) / 64;
#pragma unroll
    for (int r = 0; r < R; ++r) {
        x[r] = 0;
        if (r < turns) {
            if (r * 64 + lane < n) x[r] = keys[r * 64 + lane];
            most = max(most, x[r]);
            least = min(least, x[r] ? x[r] : 0xFFFFFFFFu);
            valid += (u32)__popcll(__ballot(x[r] != 0));
        }
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
        u32 above = 0;
        bool done = false;
        for (; bit >= 0; --bit) {
            const u32 to = at | 1u << bit;
            u32 count = 0;
#pragma unroll
            for (int r = 0; r < R; ++r)
                if (r < turns) count += (u32)__popcll(__ballot(x[r] >= to));
            if (count >= k) at = to;
            else above = count;
            if (count == k) { done = true; break; }
        }
        cut = done ? at - 1 : at;
        ties = done ? 0 : k - above;
    }
    u32 to = 0, equal = 0;
#pragma unroll
    for (int r = 0; r < R; ++r) {
        if (r < turns) {
            const u64 same = __ballot(x[r] == cut && x[r] != 0), before = (1ull << lane) - 1;
            const bool mine = x[r] > cut || (x[r] == cut && x[r] != 0 && equal + (u32)__popcll(same & before) < ties);
            const u64 all = __ballot(mine);
            if (mine) ids[to + (u32)__popcll(all & before)] = r * 64 + (int)lane;
            to += (u32)__popcll(all);
            equal += (u32)__popcll(same);
        }
    }
    write_none(ids, to, k, lane, 64);
}

// The same by a workgroup, of any number of keys: each wave has a run of them.
template <typename Keys>
__device__ __forceinline__ void pick_long(Keys keys, u32 n, u32 k, int32_t* ids) {
    constexpr u32 WAVES = PICK_THREADS / 64;
    __shared__ u32 sh_count[34];
    __shared__ u32 sh_most[WAVES], sh_least[WAVES], sh_above[WAVES], sh_same[WAVES];
    const u32 lane = threadIdx.x & 63, wave = wave_of();
    const u32 run = (n + 64 * WAVES - 1) / (64 * WAVES) * 64, r0 = min(wave * run, n), r1 = min(r0 + run, n);
    if (threadIdx.x < 34) sh_count[threadIdx.x] = 0;
    u32 most = 0, least = 0xFFFFFFFFu, valid = 0;
    for (u32 i = r0; i < r1; i += 64) {
        const u32 x = i + lane < r1 ? keys(i + lane) : 0;
        most = max(most, x);
        least = min(least, x ? x : 0xFFFFFFFFu);
        valid += (u32)__popcll(__ballot(x != 0));
    }
#pragma unroll
    for (int o = 32; o; o >>= 1) {
        most = max(most, (u32)__shfl_xor((int)most, o));
        least = min(least, (u32)__shfl_xor((int)least, o));
    }
    __syncthreads();
    if (lane == 0) {
        sh_most[wave] = most;
        sh_least[wave] = least;
        atomicAdd(&sh_count[32], valid);
    }
    __syncthreads();
    for (u32 w = 0; w < WAVES; ++w) {
        most = max(most, sh_most[w]);
        least = min(least, sh_least[w]);
    }
    u32 cut = 0, ties = 0;
    if (sh_count[32] > k) {
        const u32 differ = most ^ least;
        int bit = differ ? 31 - __builtin_clz(differ) : -1;
        u32 at = bit < 0 ? most : most & ~((2u << bit) - 1), above = 0;
        bool done = false;
        for (; bit >= 0; --bit) {
            const u32 to = at | 1u << bit;
            u32 count = 0;
            for (u32 i = r0; i < r1; i += 64) count += (u32)__popcll(__ballot(i + lane < r1 && keys(i + lane) >= to));
            if (lane == 0 && count) atomicAdd(&sh_count[bit], count);
            __syncthreads();
            count = sh_count[bit];
            if (count >= k) at = to;
            else above = count;
            if (count == k) { done = true; break; }
        }
        cut = done ? at - 1 : at;
        ties = done ? 0 : k - above;
    }
    // where this wave's keys go
    u32 over = 0, same = 0;
    for (u32 i = r0; i < r1; i += 64) {
        const u32 x = i + lane < r1 ? keys(i + lane) : 0;
        over += (u32)__popcll(__ballot(x > cut));
        same += (u32)__popcll(__ballot(x == cut && x != 0));
    }
    if (lane == 0) { sh_above[wave] = over; sh_same[wave] = same; }
    __syncthreads();
    u32 to = 0, equal = 0, all = 0, all_same = 0;
    for (u32 w = 0; w < WAVES; ++w) {
        if (w < wave) { to += sh_above[w]; equal += sh_same[w]; }
        all += sh_above[w];
        all_same += sh_same[w];
    }
    to += min(equal, ties);
    for (u32 i = r0; i < r1; i += 64) {
        const u32 x = i + lane < r1 ? keys(i + lane) : 0;
        const u64 alike = __ballot(x == cut && x != 0), before = (1ull << lane) - 1;
        const bool mine = x > cut || (x == cut && x != 0 && equal + (u32)__popcll(alike & before) < ties);
        const u64 these = __ballot(mine);
        if (mine) ids[to + (u32)__popcll(these & before)] = (int32_t)(i + lane);
        to += (u32)__popcll(these);
        equal += (u32)__popcll(alike);
    }
    write_none(ids, all + min(all_same, ties), k, threadIdx.x, PICK_THREADS);
}

// A workgroup for a token and key/value head: scores into LDS, then a wave a list.
template <int C, int NW>
__global__ void __launch_bounds__(64 * NW) k_choose(Choose a, Columns columns, u32 room) {
    extern __shared__ u32 sh_keys[];
    const u32 t = blockIdx.x / a.c.kv_heads, kv_head = blockIdx.x % a.c.kv_heads, wave = wave_of(), lists = a.group / columns.heads;
    const Token x = token_of(a, t);
    Queries<C> q;
    u32 loaded = 0xFFFFFFFFu;
    for (u32 first = wave * 16; first < x.blocks; first += 16 * NW)
        score_tile<C>(a, x, kv_head, first, columns, t, q, loaded, [&](u32 list, u32 block, u32 key) { sh_keys[list * room + block] = key; });
    __syncthreads();
    for (u32 list = wave; list < lists; list += NW)
        pick_short(sh_keys + list * room, x.blocks, a.k, a.ids + (int64_t)t * a.ids_ts + (int64_t)(kv_head * lists + list) * a.ids_hs);
}

// Scores of a long list's part: a workgroup has `chunk` blocks.
template <int C>
__global__ void __launch_bounds__(256) k_score(Choose a, Columns columns, u32 chunks) {
    const u32 part = blockIdx.x % chunks, list0 = blockIdx.x / chunks, t = list0 / a.c.kv_heads, kv_head = list0 % a.c.kv_heads, lists = a.group / columns.heads;
    const Token x = token_of(a, t);
    Queries<C> q;
    u32 loaded = 0xFFFFFFFFu;
    for (u32 n = 0; n < SPLIT_TILES; ++n) {
        const u32 first = ((part * 4 + wave_of()) * SPLIT_TILES + n) * 16;
        if (first >= x.blocks) break;
        score_tile<C>(a, x, kv_head, first, columns, t, q, loaded,
                      [&](u32 list, u32 block, u32 key) { a.keys[((u64)t * a.id_heads + kv_head * lists + list) * a.most_blocks + block] = key; });
    }
}

template <bool LDS>
__global__ void __launch_bounds__(PICK_THREADS) k_pick(Choose a) {
    extern __shared__ u32 sh_keys[];
    const u32 t = blockIdx.x / a.id_heads, list = blockIdx.x % a.id_heads;
    const Token x = token_of(a, t);
    const u32* keys = a.keys + (u64)blockIdx.x * a.most_blocks;
    int32_t* ids = a.ids + (int64_t)t * a.ids_ts + (int64_t)list * a.ids_hs;
    if constexpr (LDS) {
        for (u32 i = threadIdx.x; i < x.blocks; i += PICK_THREADS) sh_keys[i] = keys[i];
        __syncthreads();
        pick_long([&](u32 i) { return sh_keys[i]; }, x.blocks, a.k, ids);
    } else {
        pick_long([&](u32 i) { return keys[i]; }, x.blocks, a.k, ids);
    }
}

// One workgroup for all of a list, or parts of it and a second kernel.
bool choose_whole(const Choose& a) { return a.most_blocks <= MOST_SHORT && (u64)(a.id_heads / a.c.kv_heads) * a.most_blocks * 4 <= 61440; }

template <int C>
int run(hipStream_t st, const Choose& a) {
    const Columns columns = columns_of(a.group, a.heads / a.id_heads);
    const u32 lists = a.id_heads / a.c.kv_heads;
    if (choose_whole(a)) {
        k_choose<C, 4><<<a.s.tokens * a.c.kv_heads, 256, lists * a.most_blocks * 4, st>>>(a, columns, a.most_blocks);
        return PAG_OK;
    }
    const u32 chunk = 4 * SPLIT_TILES * 16, chunks = (a.most_blocks + chunk - 1) / chunk;
    k_score<C><<<a.s.tokens * a.c.kv_heads * chunks, 256, 0, st>>>(a, columns, chunks);
    if (a.most_blocks <= LDS_KEYS) {
        const u32 bytes = a.most_blocks * 4;
        if (bytes > 61440) {
            const hipError_t e = hipFuncSetAttribute((const void*)k_pick<true>, hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
            if (e != hipSuccess) { pag_set_error(std::string("hipFuncSetAttribute: ") + hipGetErrorString(e)); return PAG_EHIP; }
        }
        k_pick<true><<<a.s.tokens * a.id_heads, PICK_THREADS, bytes, st>>>(a);
    } else {
        k_pick<false><<<a.s.tokens * a.id_heads, PICK_THREADS, 0, st>>>(a);
    }
    return PAG_OK;
}

template <int FMT, int C>
void summarise(hipStream_t st, const Cache& c, const Blocks& b, const int64_t* slots, u64 tokens) {
    // a window of one token spreads a decoding step over as many waves as there are; prompts' waves look at more
    const u32 window = tokens * c.kv_heads <= 8192 ? 1 : 32;
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

u64 choose_workspace(const Choose& a) { return choose_whole(a) ? 0 : 4 * (u64)a.s.tokens * a.id_heads * a.most_blocks; }

u64 choose_groups(const Choose& a) {
    if (choose_whole(a)) return (u64)a.s.tokens * a.c.kv_heads;
    const u64 chunk = 4 * SPLIT_TILES * 16;
    return std::max((u64)a.s.tokens * a.c.kv_heads * ((a.most_blocks + chunk - 1) / chunk), (u64)a.s.tokens * a.id_heads * (PICK_THREADS / 256));
}

int launch_summarise(hipStream_t st, const Cache& c, const Blocks& b, const int64_t* slots, u64 tokens) {
    if (c.fmt == PAG_KV_INT8) summarise_width<PAG_KV_INT8>(st, c, b, slots, tokens);
    else if (c.fmt == PAG_KV_FP8) summarise_width<PAG_KV_FP8>(st, c, b, slots, tokens);
    else summarise_width<PAG_KV_FP4>(st, c, b, slots, tokens);
    return launched("pag_kv_blocks_update");
}

int launch_choose(hipStream_t st, const Choose& a) {
    const u32 n = a.c.width / 64;
    const int rc = n == 1 ? run<1>(st, a) : n == 2 ? run<2>(st, a) : n == 3 ? run<3>(st, a) : run<4>(st, a);
    return rc ? rc : launched("pag_kv_blocks_select");
}

}  // namespace pagkv
