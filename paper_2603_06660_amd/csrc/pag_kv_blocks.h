// Attention over listed blocks of tokens and a window (pag_kv_attend_blocks): the pieces of pag_kv_narrow.h, whose keys are numbered through the list's blocks and
// then the window's.  Blocks lie in one piece in a page, so that 16 tokens are read as one stretch, as where everything is read, and a list costs
// one number for `block` keys.  A row block is one token's heads that share a list.  Bound by memory where there are many lists (48 requests, 8 lists of 32 blocks of 64 and
// windows of 256 in int8: 48 us, 4.8 TB/s, whole; blocks of 16 as fast), by list, table, exponents and rows one after the other where there are few (8 lists of 128 blocks of 64 in
// 4 bits: 12.5 us in shares, and 4 for joining).
#pragma once

#include "pag_kv_narrow.h"

namespace pagkv {
namespace {

// rows, request and keys of a list; every lane reads the same
__device__ __forceinline__ void place_blocks(const Attend& a, Piece& p, u64 list, u32 tile, u32 unit) {
    ListPiece w;
    place_list(a, w, list, tile);
    p.w = w;
    const int request = __builtin_amdgcn_readfirstlane(a.s.request[w.t0]);
    int position = __builtin_amdgcn_readfirstlane(a.s.positions[w.t0]);
    if (request < 0 || (u32)request >= a.s.requests || (u64)(u32)max(position, 0) >= (u64)a.s.max_pages * a.c.page_tokens) position = -1;
    p.b = position >= 0 ? (u32)request : 0;
    p.s = Span{ w.t0, 1, position + 1, position };
    p.p0 = p.p1 = position;
    p.ids = a.blocks + (int64_t)w.t0 * a.ids_ts + (int64_t)w.id_head * a.ids_hs;
    p.listed = a.k * a.block;
    p.near = max(position - (int)a.window + 1, 0) & ~(int)(BLOCK - 1);
    const int near = a.window ? position + 1 - p.near : 0;
    const int all = position >= 0 ? (int)p.listed + near : 0;
    p.start = min((u64)p.u0 * unit, (u64)0x7FFFFFFF);
    p.stop = (int)min((u64)all, (u64)p.u1 * unit);
}

template <int FMT, int C, bool SLOPES, bool CAPPED>
__global__ void __launch_bounds__(256, groups_per_cu(FMT, 64 * C, 1)) k_attend_blocks(Attend a, u32 units, u32 tiles) {
    __shared__ __align__(16) Exchange<C, SPLIT_WAVES> sh;
    const u32 cost = units + PIECE;
    const u64 total = (u64)a.s.tokens * a.id_heads * tiles * cost;
    const u32 parts = (u32)min((u64)gridDim.x, total);
    if (blockIdx.x >= parts) return;
    u64 at = share(total, parts, blockIdx.x);
    const u64 end = share(total, parts, blockIdx.x + 1);
    attend_pieces<FMT, C, 1, SPLIT_WAVES, false, CAPPED, true, SLOPES>(a, sh, [&](Piece& p) -> bool {
        while (at < end) {
            const u64 part = divide(at, cost), list = divide(part, tiles);
            const u32 c0 = (u32)(at - part * cost), c1 = (u32)min((u64)cost, c0 + (end - at));
            at += c1 - c0;
            p.u0 = max(c0, PIECE) - PIECE;
            p.u1 = max(c1, PIECE) - PIECE;
            if (p.u0 == p.u1) continue;
            p.units = units;
            p.last = p.u0 == 0 && p.u1 < units ? (int)divide((part + 1) * cost * parts - 1, total) : -1;
            place_blocks(a, p, list, (u32)(part - list * tiles), UNIT);
            return true;
        }
        return false;
    });
}

template <int FMT, int C, int NW, bool SLOPES, bool CAPPED>
__global__ void __launch_bounds__(64 * NW, C <= 2 ? 2 : 1) k_attend_blocks_whole(Attend a, u32 tiles) {
    __shared__ __align__(16) Exchange<C, NW> sh;
    bool first = true;
    attend_pieces<FMT, C, 1, NW, true, CAPPED, true, SLOPES>(a, sh, [&](Piece& p) -> bool {
        if (!first) return false;
        first = false;
        p.u0 = 0;
        p.u1 = p.units = 1;
        p.last = -1;
        place_blocks(a, p, blockIdx.x / tiles, blockIdx.x % tiles, 0x7FFFFFFFu);
        return true;
    });
}

template <int FMT, int C, int NW, bool CAPPED>
void run_blocks_whole(hipStream_t st, const Attend& a, u32 tiles) {
    const u32 grid = a.s.tokens * a.id_heads * tiles;
    if (a.slopes) k_attend_blocks_whole<FMT, C, NW, true, CAPPED><<<grid, 64 * NW, 0, st>>>(a, tiles);
    else k_attend_blocks_whole<FMT, C, NW, false, CAPPED><<<grid, 64 * NW, 0, st>>>(a, tiles);
}

template <int FMT, int C, bool CAPPED>
void run_blocks(hipStream_t st, const Attend& a, int num_cu, bool whole) {
    const u32 tiles = (a.group + ROWS - 1) / ROWS;
    if (whole) {
        if constexpr (C <= 2) {
            if (narrow_groups(a) <= (u64)num_cu) return run_blocks_whole<FMT, C, 8, CAPPED>(st, a, tiles);
        }
        return run_blocks_whole<FMT, C, 4, CAPPED>(st, a, tiles);
    }
    // the window may begin anywhere in a block of 16
    const u32 keys = a.k * a.block + (a.window ? a.window + BLOCK - 1 : 0), units = std::max<u32>((keys + UNIT - 1) / UNIT, 1);
    const u32 grid = (u32)num_cu * groups_per_cu(FMT, 64 * C, 1);
    if (a.slopes) k_attend_blocks<FMT, C, true, CAPPED><<<grid, 256, 0, st>>>(a, units, tiles);
    else k_attend_blocks<FMT, C, false, CAPPED><<<grid, 256, 0, st>>>(a, units, tiles);
}

}  // namespace

template <int FMT, int C>
void launch_blocks(hipStream_t st, const Attend& a, int num_cu, bool whole) {
    if (a.softcap > NEAR_CAP) run_blocks<FMT, C, true>(st, a, num_cu, whole);
    else run_blocks<FMT, C, false>(st, a, num_cu, whole);
}

}  // namespace pagkv
