// Attention over the 8-bit cache: which kernels a call runs, and the joining of rows whose keys went to several workgroups.
#include <algorithm>

#include "pag_kv_attend.h"

namespace pagkv {

u64 narrow_groups(const Attend& a) { return a.listed ? (u64)a.s.tokens * a.id_heads * ((a.group + ROWS - 1) / ROWS) : (u64)a.s.requests * a.c.kv_heads; }

namespace {

// A workgroup for each token and head; if its keys went to several workgroups, its threads look at their pieces' offsets first, and then
// each wave adds up every fourth piece, eight of them asked for at a time.
template <int C>
__global__ void __launch_bounds__(256) k_join(Attend a, int groups) {
    __shared__ float sh_max[4], sh_by[256], sh_sum[4];
    __shared__ float sh_acc[4][64 * C];
    const u32 t = blockIdx.x / a.heads, head = blockIdx.x % a.heads, lane = threadIdx.x & 63, wave = wave_of();
    const int2 j = a.joined[(u64)t * a.heads + head];
    if (j.x < 0 || j.y < j.x || j.y >= groups) return;
    u32 row = head % a.group;
    if (!a.listed) {
        // number of the token in its request
        u32 lo = 0, hi = a.s.requests;
        while (hi - lo > 1) {
            const u32 mid = (lo + hi) / 2;
            if ((u32)max(a.s.offsets[mid], 0) <= t) lo = mid; else hi = mid;
        }
        row += (t - (u32)max(a.s.offsets[lo], 0)) * a.group;
    }
    constexpr u32 TILE_SLOT = ROWS * (64 * C + 2);
    const u32 slot = TILE_SLOT * a.row_tiles, first_row = row % (ROWS * a.row_tiles) / ROWS * TILE_SLOT;
    row %= ROWS;
    const int pieces = j.y - j.x + 1;
    const auto piece = [&](int i) { return a.partial + (2 * (u64)(j.x + i) + (i == 0 ? 1 : 0)) * slot + first_row; };
    float top = LOWEST;
    for (int i = (int)threadIdx.x; i < pieces; i += 256) top = fmaxf(top, piece(i)[row]);
#pragma unroll
    for (int o = 32; o; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
    if (lane == 0) sh_max[wave] = top;
    __syncthreads();
    top = fmaxf(fmaxf(sh_max[0], sh_max[1]), fmaxf(sh_max[2], sh_max[3]));
    float sum = 0.f, acc[C];
#pragma unroll
    for (int c = 0; c < C; ++c) acc[c] = 0.f;
    for (int first = 0; first < pieces; first += 256) {
        const int n = min(256, pieces - first);
        __syncthreads();
        if ((int)threadIdx.x < n) {
            const float* p = piece(first + (int)threadIdx.x);
            const float by = __builtin_amdgcn_exp2f(p[row] - top);
            sh_by[threadIdx.x] = by;
            sum = add_scaled(sum, p[ROWS + row], p[row] - top);
        }
        __syncthreads();
        for (int i = (int)wave; i < n; i += 32) {
            float x[8][C];
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const float* p = piece(first + min(i + 4 * u, n - 1)) + 2 * ROWS + row * (64 * C) + lane * C;
#pragma unroll
                for (int c = 0; c < C; ++c) x[u][c] = p[c];
            }
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const float by = i + 4 * u < n ? sh_by[i + 4 * u] : 0.f;
#pragma unroll
                for (int c = 0; c < C; ++c) acc[c] = i + 4 * u < n ? __builtin_fmaf(x[u][c], by, acc[c]) : acc[c];
            }
        }
    }
#pragma unroll
    for (int o = 32; o; o >>= 1) sum += __shfl_xor(sum, o);
    if (lane == 0) sh_sum[wave] = sum;
#pragma unroll
    for (int c = 0; c < C; ++c) sh_acc[wave][lane * C + c] = acc[c];
    __syncthreads();
    const float all = sh_sum[0] + sh_sum[1] + sh_sum[2] + sh_sum[3];
    const u32 d = threadIdx.x * 2;
    if (d < a.c.dim) {
        const float by = all != 0.f ? 1.f / all : 0.f;
        const float x = sh_acc[0][d] + sh_acc[1][d] + sh_acc[2][d] + sh_acc[3][d], y = sh_acc[0][d + 1] + sh_acc[1][d + 1] + sh_acc[2][d + 1] + sh_acc[3][d + 1];
        *(u32*)((uint16_t*)a.out + (int64_t)t * a.o_ts + (int64_t)head * a.o_hs + d) = pack2(finite(x * by), finite(y * by), a.dtype);
    }
    if (a.lse && threadIdx.x == 0) a.lse[(u64)t * a.heads + head] = all != 0.f ? LN2 * (top + __builtin_amdgcn_logf(all)) : -INFINITY;
}

// Whether a workgroup reads all keys of its rows, without shares to find and a second kernel to join them.  Split and whole, in us, heads of 128:
//   tables and windows: one request of 777 tokens 12.3, 8.8; 16 of 100 to 2,000 tokens 17.9, 16.2; 32 of 2,000 tokens 34.9, 27; 96 of 300 to 2,000 tokens
//   51.8, 47.8; one of 2,000 tokens 14.0, 18.3, whose 8 workgroups leave the chip idle
//   lists: 384 of 1,256 keys 38.6, 29.6; 1,536 of 164 keys 36, 27; 64 of 1,064 keys 19, 15; 32 of 1,064 keys 13.3, 14.3
bool narrow_whole(const Attend& a, int num_cu) {
    const u64 keys = a.listed ? (u64)a.k + a.window : std::min<u64>((u64)a.s.max_pages * a.c.page_tokens, a.window ? (u64)a.window + 2 * ROWS : ~0ull);
    const u64 groups = narrow_groups(a);
    if (keys <= 1024) return true;
    if (!a.listed) return keys <= 2048 && groups >= (u64)num_cu / 2;
    return (keys <= 2048 && groups >= (u64)num_cu / 4) || (keys <= 4096 && groups >= (u64)num_cu);
}

u64 partial_floats(const Attend& a, int num_cu) {
    return 2ull * (u32)num_cu * groups_per_cu(a.c.width, (int)a.row_tiles) * a.row_tiles * ROWS * (a.c.width + 2);
}

template <int C>
void run(hipStream_t st, const Attend& a, int num_cu) {
    const bool whole = narrow_whole(a, num_cu);
    if (a.c.fmt == PAG_KV_INT8) launch_narrow<PAG_KV_INT8, C>(st, a, num_cu, whole);
    else launch_narrow<PAG_KV_FP8, C>(st, a, num_cu, whole);
    if (!whole) k_join<C><<<a.s.tokens * a.heads, 256, 0, st>>>(a, num_cu * (int)groups_per_cu(64 * C, (int)a.row_tiles));
}

}  // namespace

u64 attend_workspace(const Attend& a, int num_cu) {
    if (a.row_tiles == 0) return wide_workspace(a.c.width, num_cu);
    return narrow_whole(a, num_cu) ? 0 : 4 * partial_floats(a, num_cu) + 8 * (u64)a.s.tokens * a.heads;
}

int launch_attend(hipStream_t st, const Attend& args, int num_cu) {
    if (args.row_tiles == 0) return launch_attend_wide(st, args, num_cu);
    Attend a = args;
    a.joined = narrow_whole(a, num_cu) ? nullptr : (int2*)(a.partial + partial_floats(a, num_cu));
    const u32 n = a.c.width / 64;
    if (n == 1) run<1>(st, a, num_cu);
    else if (n == 2) run<2>(st, a, num_cu);
    else if (n == 3) run<3>(st, a, num_cu);
    else run<4>(st, a, num_cu);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) { pag_set_error(std::string("pag_kv_attend: ") + hipGetErrorString(e)); return PAG_EHIP; }
    return PAG_OK;
}

}  // namespace pagkv
