// Block tables and slots of a step, and what goes into the cache and comes out of it.
#include "pag_kv.h"

namespace pagkv {
namespace {

constexpr u32 PLAN_THREADS = 1024;

// inclusive sum over the workgroup; sh: an entry a wave
__device__ __forceinline__ u64 scan1024(u64 x, u64* sh) {
    const u32 lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (u32 o = 1; o < 64; o <<= 1) {
        const u64 y = __shfl_up(x, o);
        if (lane >= o) x += y;
    }
    if (lane == 63) sh[wave] = x;
    __syncthreads();
    u64 before = 0;
    for (u32 w = 0; w < wave; ++w) before += sh[w];
    __syncthreads();
    return x + before;
}

struct Extend {
    const int32_t *add, *lengths, *free_pages, *free_count;
    int32_t* table;
    u64 table_stride, tokens;
    u32 requests, max_pages, page_tokens, num_pages;
    int32_t *offsets, *context, *granted, *out_lengths, *out_free_count, *scratch, *request, *positions;
    int64_t* slots;
};

struct Want { u64 have, need, add, length; bool fits; };

__device__ __forceinline__ Want want_of(const Extend& e, u32 r) {
    Want w;
    const int32_t n = e.lengths[r], a = e.add[r];
    w.length = n < 0 ? 0 : (u64)n;
    w.add = a < 0 ? 0 : (u64)a;
    w.have = (w.length + e.page_tokens - 1) / e.page_tokens;
    w.need = (w.length + w.add + e.page_tokens - 1) / e.page_tokens - w.have;
    w.fits = w.have + w.need <= e.max_pages;
    return w;
}

// Slot of new token t, and the entry of the table if the token is the first of a page.  offsets, granted, out_lengths and scratch
// (pages that were taken before the request's; behind the requests the count of free pages before the step) are written.
__device__ __forceinline__ void fill_token(const Extend& e, u64 t, u64 free_before) {
    int32_t request = -1, position = -1;
    int64_t slot = -1;
    if (t < (u64)(u32)e.offsets[e.requests]) {
        u32 lo = 0, hi = e.requests;               // the last request whose tokens begin at t or before, with tokens of its own
        while (hi - lo > 1) {
            const u32 mid = (lo + hi) / 2;
            if ((u64)(u32)e.offsets[mid] <= t) lo = mid; else hi = mid;
        }
        request = (int32_t)lo;
        if (e.granted[lo]) {
            const u64 i = t - (u32)e.offsets[lo], add = (u32)(e.offsets[lo + 1] - e.offsets[lo]);
            const u64 length = (u32)e.out_lengths[lo] - add, p = length + i;
            const u64 have = (length + e.page_tokens - 1) / e.page_tokens, at = p / e.page_tokens, place = p % e.page_tokens;
            int32_t page;
            int32_t* entry = e.table + lo * e.table_stride + at;
            if (at >= have) {
                page = e.free_pages[free_before - 1 - (u32)e.scratch[lo] - (at - have)];
                if (place == 0) *entry = page;
            } else {
                page = *entry;
            }
            position = (int32_t)p;
            if (page >= 0) slot = (int64_t)page * e.page_tokens + (int64_t)place;
        }
    }
    e.request[t] = request;
    e.positions[t] = position;
    e.slots[t] = slot;
}

// One workgroup: who gets pages, and from where.  A thread has a run of consecutive requests; the sums over all of them come from one scan
// of the threads' sums.  Up to `fill` tokens get their slots here as well.
__global__ void __launch_bounds__(PLAN_THREADS) k_extend(Extend e, u64 fill) {
    __shared__ u64 sh[PLAN_THREADS / 64];
    __shared__ u64 sh_taken;
    const u32 per = (e.requests + PLAN_THREADS - 1) / PLAN_THREADS, r0 = min(threadIdx.x * per, e.requests), r1 = min(r0 + per, e.requests);
    int32_t count = *e.free_count;
    const u64 avail = count < 0 ? 0 : min((u32)count, e.num_pages);
    if (threadIdx.x == 0) sh_taken = 0;
    u64 need = 0, add = 0;
    for (u32 r = r0; r < r1; ++r) {
        const Want w = want_of(e, r);
        if (w.fits) need += w.need;
        add += w.add;
    }
    u64 upto = scan1024(need, sh) - need, first = scan1024(add, sh) - add, taken = 0;
    for (u32 r = r0; r < r1; ++r) {
        const Want w = want_of(e, r);
        const u64 before = upto;
        if (w.fits) upto += w.need;
        // all of its new tokens need rows in the step: the token that begins a page writes the table's entry and one without a row would leave
        // there what an earlier holder of the row's place wrote.  After a request without rows only those that want none are served, so upto stands
        const bool rows = w.add == 0 || first + w.add <= e.tokens;
        const bool granted = w.fits && rows && (w.need == 0 || upto <= avail);
        if (granted && w.need) taken = upto;
        e.offsets[r] = (int32_t)min(first, (u64)0x7FFFFFFF);
        first += w.add;
        e.granted[r] = granted ? 1 : 0;
        e.scratch[r] = (int32_t)min(before, (u64)0x7FFFFFFF);
        const int32_t length = (int32_t)(granted ? w.length + w.add : w.length);
        e.context[r] = granted ? length : 0;
        e.out_lengths[r] = length;
        if (r + 1 == e.requests) e.offsets[e.requests] = (int32_t)min(first, (u64)0x7FFFFFFF);
    }
    if (taken) atomicMax((unsigned long long*)&sh_taken, (unsigned long long)taken);
    __syncthreads();
    if (threadIdx.x == 0) {
        *e.out_free_count = (int32_t)(avail - sh_taken);
        e.scratch[e.requests] = (int32_t)avail;
    }
    // what this workgroup has written, its threads read
    __threadfence_block();
    __syncthreads();
    for (u64 t = threadIdx.x; t < fill; t += PLAN_THREADS) fill_token(e, t, avail);
}

__global__ void __launch_bounds__(256) k_extend_tokens(Extend e) {
    const u64 t = (u64)blockIdx.x * 256 + threadIdx.x;
    if (t < e.tokens) fill_token(e, t, (u64)(u32)e.scratch[e.requests]);
}

__global__ void __launch_bounds__(PLAN_THREADS) k_release(pag_kv_tables t, const int32_t* __restrict__ done) {
    __shared__ u64 sh[PLAN_THREADS / 64];
    __shared__ u64 sh_end;
    const u32 per = (t.requests + PLAN_THREADS - 1) / PLAN_THREADS, r0 = min(threadIdx.x * per, t.requests), r1 = min(r0 + per, t.requests);
    const int32_t count = *t.free_count;
    const u64 have = count < 0 ? 0 : min((u64)count, t.num_pages);
    const auto pages_of = [&](u32 r) -> u64 {
        const int32_t n = t.lengths[r];
        return done[r] && n > 0 ? min(((u64)n + t.page_tokens - 1) / t.page_tokens, (u64)t.max_pages) : 0;
    };
    u64 back = 0;
    for (u32 r = r0; r < r1; ++r) back += pages_of(r);
    u64 upto = scan1024(back, sh);
    if (threadIdx.x == PLAN_THREADS - 1) sh_end = min(have + upto, t.num_pages);
    u64 at = have + upto - back;
    for (u32 r = r0; r < r1; ++r) {
        const u64 n = pages_of(r);
        for (u64 i = 0; i < n; ++i, ++at)
            if (at < t.num_pages) t.free_pages[at] = t.table[r * t.table_stride + i];
        if (done[r]) t.lengths[r] = 0;
    }
    __syncthreads();
    if (threadIdx.x == 0) *t.free_count = (int32_t)sh_end;
}

// ---- rotation ---------------------------------------------------------------------------------------------------------

// cos and sin of an angle below 2^31 or so, to 2^-50: the nearest multiple of pi / 2 is taken off in two parts, which leave out less than 2^-77 of it; r, |r| <= pi / 4, is
// rounded to 53 bits, 2^-54 at most, and of r Taylor's series, whose first terms left out, r^17 / 17! and r^18 / 18!, are below 2^-54.
__device__ __forceinline__ double2 spin_of(double angle) {
    const double n = __builtin_rint(angle * 0.63661977236758134308);
    double r = __builtin_fma(n, -1.57079632679489655800, angle);
    r = __builtin_fma(n, -6.12323399573676603587e-17, r);
    const double u = r * r;
    double s = -1.0 / 1307674368000.0, c = 1.0 / 20922789888000.0;
    s = __builtin_fma(s, u, 1.0 / 6227020800.0);
    c = __builtin_fma(c, u, -1.0 / 87178291200.0);
    s = __builtin_fma(s, u, -1.0 / 39916800.0);
    c = __builtin_fma(c, u, 1.0 / 479001600.0);
    s = __builtin_fma(s, u, 1.0 / 362880.0);
    c = __builtin_fma(c, u, -1.0 / 3628800.0);
    s = __builtin_fma(s, u, -1.0 / 5040.0);
    c = __builtin_fma(c, u, 1.0 / 40320.0);
    s = __builtin_fma(s, u, 1.0 / 120.0);
    c = __builtin_fma(c, u, -1.0 / 720.0);
    s = __builtin_fma(s, u, -1.0 / 6.0);
    c = __builtin_fma(c, u, 1.0 / 24.0);
    s = __builtin_fma(s * u, r, r);
    c = __builtin_fma(c, u, -0.5);
    c = __builtin_fma(c, u, 1.0);
    const int q = (int)(n - 4.0 * __builtin_floor(n * 0.25));
    const double x = q & 1 ? s : c, y = q & 1 ? c : s;
    return make_double2(q == 1 || q == 2 ? -x : x, q >= 2 ? -y : y);
}

// A number of 64 bits on its way to fewer than 24: rounded to 32 bits towards zero, and the last bit set if that took anything off, so that rounding
// it again gives what rounding once would have given.
__device__ __forceinline__ float odd(double x) {
    const float f = (float)x;
    const double y = (double)f;
    const u32 bits = __float_as_uint(f);
    if (y == x || x != x) return f;
    return __uint_as_float((bits - (fabs(y) > fabs(x) ? 1u : 0u)) | 1u);
}

// the angles of tokens t0 to t0 + n - 1, into LDS, by the workgroup; for keys in 64 bits, for queries in 32
__device__ __forceinline__ void spin_tokens(const Store& a, u64 t0, u32 n, double2* spin) {
    const u32 half = a.turned / 2;
    for (u32 i = threadIdx.x; i < n * half; i += blockDim.x) spin[i] = spin_of((double)a.positions[t0 + i / half] * (double)a.frequencies[i % half]);
}

__device__ __forceinline__ void spin_queries(const Store& a, u64 t0, u32 n, float2* spin) {
    const u32 half = a.turned / 2;
    for (u32 i = threadIdx.x; i < n * half; i += blockDim.x) {
        const double2 x = spin_of((double)a.positions[t0 + i / half] * (double)a.frequencies[i % half]);
        spin[i] = make_float2((float)x.x, (float)x.y);
    }
}

// Numbers at to at + 7 of a row, which x holds as they came, turned.  row: the element that the row begins with.
__device__ __forceinline__ void turn8(const Store& a, const void* p, u64 row, u32 at, const double2* spin, float* x) {
    if (at >= a.turned) return;
    if (a.pairs == PAG_KV_NEIGHBOURS) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const double2 by = spin[at / 2 + j];
            const double u = x[2 * j], v = x[2 * j + 1];
            x[2 * j] = odd(__builtin_fma(u, by.x, -v * by.y));
            x[2 * j + 1] = odd(__builtin_fma(v, by.x, u * by.y));
        }
        return;
    }
    // four at a time lie on one side of the middle, and so do their partners
    const u32 half = a.turned / 2;
#pragma unroll
    for (int z = 0; z < 2; ++z) {
        const u32 first = at + 4 * z;
        const bool low = first < half;
        float y[4];
        load4(p, row + (low ? first + half : first - half), a.dtype, y);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const double2 by = spin[(low ? first : first - half) + j];
            x[4 * z + j] = odd(__builtin_fma((double)x[4 * z + j], by.x, (double)(low ? -y[j] : y[j]) * by.y));
        }
    }
}

constexpr u32 QUERY_TOKENS = 4;       // of a workgroup that turns queries, where there are many
constexpr u32 QUERY_TURNS = 4;

__device__ __forceinline__ void store_past(uint8_t* to, const uint4& x) {
    typedef u32 word4 __attribute__((ext_vector_type(4)));
    __builtin_nontemporal_store(word4{ x.x, x.y, x.z, x.w }, (word4*)to);
}

// 16 bytes of a row as they come, and as they go
template <bool WIDE>
__device__ __forceinline__ void numbers_of(const uint4& r, u32 dtype, float* x) {
    if constexpr (WIDE) {
        x[0] = __uint_as_float(r.x); x[1] = __uint_as_float(r.y); x[2] = __uint_as_float(r.z); x[3] = __uint_as_float(r.w);
    } else {
        widen_row8(r, dtype, x);
    }
}

template <bool WIDE>
__device__ __forceinline__ uint4 bytes_of(const float* x, u32 dtype) {
    if constexpr (WIDE) return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
    else return make_uint4(pack2(x[0], x[1], dtype), pack2(x[2], x[3], dtype), pack2(x[4], x[5], dtype), pack2(x[6], x[7], dtype));
}

// q's rows of tokens t0 to t0 + n - 1, n <= QUERY_TOKENS, by the workgroup, in 32 bits.  A pair is one thread's, so that rows may be turned in place.  N numbers, 16 bytes, are
// a thread's piece; of halves it has the N numbers half a turn on as well, and QUERY_TURNS rows' pieces are asked for before the first is turned.  Rows whose
// halves do not begin at a multiple of N go in pieces of 4 numbers of 16 bits, 8 bytes.
template <bool WIDE>
__device__ __forceinline__ void turn_queries(const Store& a, u64 t0, u32 n, const float2* spin) {
    constexpr u32 N = WIDE ? 4 : 8, SIZE = WIDE ? 4 : 2;
    const u32 half = a.turned / 2;
    const bool neighbours = a.pairs == PAG_KV_NEIGHBOURS;
    if (!neighbours && half % N) {
        const u32 pairs = half / 4, pieces = pairs + (a.c.dim - a.turned) / 8;
        for (u32 i = threadIdx.x; i < n * a.heads * pieces; i += blockDim.x) {
            const u32 piece = i % pieces, head = i / pieces % a.heads, token = i / pieces / a.heads;
            const u64 from = (t0 + token) * (u64)a.q_ts + head * (u64)a.q_hs, to = (t0 + token) * (u64)a.o_ts + head * (u64)a.o_hs;
            if (piece >= pairs) {
                const u32 at = a.turned + (piece - pairs) * 8;
                *(uint4*)((uint16_t*)a.out + to + at) = *(const uint4*)((const uint16_t*)a.q + from + at);
            } else {
                float x[4], y[4], u[4], v[4];
                load4(a.q, from + piece * 4, a.dtype, x);
                load4(a.q, from + half + piece * 4, a.dtype, y);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float2 by = spin[token * half + piece * 4 + j];
                    u[j] = __builtin_fmaf(x[j], by.x, -(y[j] * by.y));
                    v[j] = __builtin_fmaf(y[j], by.x, x[j] * by.y);
                }
                *(uint2*)((uint16_t*)a.out + to + piece * 4) = make_uint2(pack2(u[0], u[1], a.dtype), pack2(u[2], u[3], a.dtype));
                *(uint2*)((uint16_t*)a.out + to + half + piece * 4) = make_uint2(pack2(v[0], v[1], a.dtype), pack2(v[2], v[3], a.dtype));
            }
        }
        return;
    }
    // A wave has 64 / pieces rows at a time; a lane keeps its piece, so that nothing is divided on the way.
    const u32 pairs = neighbours ? a.turned / N : half / N, pieces = pairs + (a.c.dim - a.turned) / N, per_wave = 64 / pieces;
    const u32 lane = threadIdx.x & 63, piece = lane % pieces, sub = lane / pieces, rows = n * a.heads, step = per_wave * (blockDim.x / 64);
    if (sub >= per_wave) return;
    const bool turns = piece < pairs, two = turns && !neighbours;
    const u32 at = turns ? piece * N : a.turned + (piece - pairs) * N, other = two ? half : 0;
    const float2* by = spin + (turns ? (neighbours ? piece * (N / 2) : at) : 0);
    for (u32 row0 = wave_of() * per_wave + sub; row0 < rows; row0 += QUERY_TURNS * step) {
        uint4 r[QUERY_TURNS][2];
        u32 token[QUERY_TURNS];
        u64 to[QUERY_TURNS];
#pragma unroll
        for (u32 i = 0; i < QUERY_TURNS; ++i) {
            const u32 row = min(row0 + i * step, rows - 1);
            token[i] = (row >= a.heads) + (row >= 2 * a.heads) + (row >= 3 * a.heads);
            const u32 head = row - token[i] * a.heads;
            const uint8_t* from = (const uint8_t*)a.q + ((t0 + token[i]) * (u64)a.q_ts + head * (u64)a.q_hs + at) * SIZE;
            to[i] = (t0 + token[i]) * (u64)a.o_ts + head * (u64)a.o_hs + at;
            r[i][0] = *(const uint4*)from;
            if (two) r[i][1] = *(const uint4*)(from + other * SIZE);
        }
#pragma unroll
        for (u32 i = 0; i < QUERY_TURNS; ++i) {
            if (row0 + i * step >= rows) break;
            uint8_t* out = (uint8_t*)a.out + to[i] * SIZE;
            const float2* spins = by + token[i] * half;
            if (two) {
                float x[N], y[N], u[N], v[N];
                numbers_of<WIDE>(r[i][0], a.dtype, x);
                numbers_of<WIDE>(r[i][1], a.dtype, y);
#pragma unroll
                for (u32 j = 0; j < N; ++j) {
                    const float2 s = spins[j];
                    u[j] = __builtin_fmaf(x[j], s.x, -(y[j] * s.y));
                    v[j] = __builtin_fmaf(y[j], s.x, x[j] * s.y);
                }
                store_past(out, bytes_of<WIDE>(u, a.dtype));
                store_past(out + other * SIZE, bytes_of<WIDE>(v, a.dtype));
            } else if (turns) {
                float x[N], u[N];
                numbers_of<WIDE>(r[i][0], a.dtype, x);
#pragma unroll
                for (u32 j = 0; j < N / 2; ++j) {
                    const float2 s = spins[j];
                    u[2 * j] = __builtin_fmaf(x[2 * j], s.x, -(x[2 * j + 1] * s.y));
                    u[2 * j + 1] = __builtin_fmaf(x[2 * j + 1], s.x, x[2 * j] * s.y);
                }
                store_past(out, bytes_of<WIDE>(u, a.dtype));
            } else {
                store_past(out, r[i][0]);
            }
        }
    }
}

__device__ __forceinline__ void turn_queries(const Store& a, u64 t0, u32 n, const float2* spin) {
    if (a.dtype == PAG_F32) turn_queries<true>(a, t0, n, spin);
    else turn_queries<false>(a, t0, n, spin);
}

// A wave has a window of new tokens, one head and one kind.  It writes the blocks whose first new token lies in its window, with all
// their new tokens, one block after the other.  8 numbers of a row are a lane's; a block of 16 rows is 2 C of these pieces a lane.
// A window of one token spreads a decoding step's blocks over as many waves as there are; the more tokens, the more of the waves of
// prompts start only to find that their token is not the first of its block.  Windows of 1, 4 and 16 tokens, 8 heads of 128, in us:
// one token each: 256 requests 6.0, 9.3, 28; 512 requests 9.1, 10.5, 28; 2,048 requests 29, 25, 35; 4,096 requests 53, 44, 47;
// prompts: 256 tokens 8.5, 5.9, 5.9; 512 tokens 9.8, 6.5, 5.9; 2,048 tokens 18, 12.5, 11; 4,096 tokens 35, 20, 14; 15,000 tokens 139, 53, 36.
// Bound by memory where there are many tokens (60,000: 370 MB in 124 us), by the waits for a slot, an exponent and a row where there are few.
// TURN: keys are turned.  The four waves of a workgroup then have one window and kind, and four heads, and share their tokens' angles; the workgroups from
// number `writers` on turn queries.  18,596 tokens, 8 heads of 128: 44 us as they are, 86 with keys turned, 128 with 32 heads of queries (419 MB, 81 as a copy); one token of each of
// 192 requests 9 on the GPU.  144 registers, three waves a SIMD, whose waits for rows, angles and partners do not overlap enough.
template <int FMT, int C, bool TURN>
__global__ void __launch_bounds__(256) k_append(Store a, u32 window, u32 writers, u32 each) {
    extern __shared__ double2 spin[];
    const u32 lane = threadIdx.x & 63, kinds = 2 * a.c.kv_heads;
    u64 t0;
    u32 head, kind;
    if constexpr (TURN) {
        if (blockIdx.x >= writers) {
            const u64 first = (u64)(blockIdx.x - writers) * each;
            const u32 n = (u32)min((u64)each, a.tokens - first);
            spin_queries(a, first, n, (float2*)spin);
            __syncthreads();
            turn_queries(a, first, n, (const float2*)spin);
            return;
        }
        const u32 fours = (a.c.kv_heads + 3) / 4, part = blockIdx.x % (2 * fours);
        t0 = (u64)(blockIdx.x / (2 * fours)) * window;
        head = (part >> 1) * 4 + (threadIdx.x >> 6);
        kind = part & 1;
    } else {
        const u64 wave = (u64)blockIdx.x * 4 + (threadIdx.x >> 6);
        t0 = wave / kinds * window;
        if (t0 >= a.tokens) return;
        head = (u32)(wave % kinds) >> 1;
        kind = (u32)(wave % kinds) & 1;
    }
    // lane 0: the token before, lanes 1 .. window: the window, and the next 15
    int64_t slot = -1;
    if (lane < window + BLOCK && t0 + lane >= 1 && t0 + lane - 1 < a.tokens) slot = a.slots[t0 + lane - 1];
    if (slot >= (int64_t)a.c.num_pages * a.c.page_tokens || slot < 0) slot = -1;
    const int block = slot < 0 ? -1 : (int)(slot / BLOCK), place = (int)(slot & (BLOCK - 1));
    const int left = __shfl_up(block, 1);
    u64 firsts = __ballot(lane >= 1 && lane <= window && block >= 0 && block != left);
    for (; firsts; firsts &= firsts - 1) {
        const u32 at_lane = (u32)__builtin_ctzll(firsts);
        const u64 t = t0 + at_lane - 1;
        const int mine = __builtin_amdgcn_readlane(block, (int)at_lane);
        const u64 same = __ballot(block == mine && lane >= at_lane && lane < at_lane + BLOCK) >> at_lane;
        const u32 run = (u32)__builtin_ctzll(~same);
        u32 present = 0;
        for (u32 i = 0; i < run; ++i) present |= 1u << __builtin_amdgcn_readlane(place, (int)(at_lane + i));
        if constexpr (TURN) {
            if (kind == 0) {                     // the whole workgroup comes here: its waves see the same slots
                __syncthreads();
                spin_tokens(a, t, run, spin);
                __syncthreads();
            }
            if (head >= a.c.kv_heads) continue;
        }
        const bool begins = present & 1u;
        const u32 page = (u32)mine / a.c.page_blocks, first = (u32)mine % a.c.page_blocks * BLOCK;
        uint8_t* rows = a.c.data + (u64)row_of(a.c, page, head, first) * (2 * a.c.width) + kind * a.c.width;
        int8_t* exponent = a.c.exponents + ((u64)(page * a.c.kv_heads + head) * a.c.page_blocks + first / BLOCK) * 2 + kind;
        const int held = *exponent;

        float x[2 * C][8];
        float most = 0.f;
#pragma unroll
        for (int n = 0; n < 2 * C; ++n) {
            const u32 i = lane + 64 * n, row = i / (8 * C), at = i % (8 * C) * 8;
#pragma unroll
            for (int j = 0; j < 8; ++j) x[n][j] = 0.f;
            if (row < run && at < a.c.dim) {
                const u64 from = (t + row) * (u64)a.ts[kind] + head * (u64)a.hs[kind];
                load8(a.x[kind], from + at, a.dtype, x[n]);
                if constexpr (TURN) {
                    if (kind == 0) turn8(a, a.x[0], from, at, spin + row * (a.turned / 2), x[n]);
                }
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float y = fabsf(x[n][j]);
                if (y <= 3.402823466e38f) most = fmaxf(most, y);
            }
        }
        const int least = least_exponent<FMT>(wave_max(most));
        const int e = begins ? least : max(least, held);
        const float down = power(-e);
#pragma unroll
        for (int n = 0; n < 2 * C; ++n) {
            const u32 i = lane + 64 * n, row = i / (8 * C), at = i % (8 * C) * 8;
            const int to = __shfl(place, (int)(row + at_lane));
            if (row < run) {
#pragma unroll
                for (int j = 0; j < 8; ++j) x[n][j] *= down;
                *(uint2*)(rows + (u64)to * (2 * a.c.width) + at) = make_uint2(encode4<FMT>(x[n]), encode4<FMT>(x[n] + 4));
            }
        }
        if (begins || e > held) {
            const float again = begins ? 0.f : power(max(held - e, -126));
#pragma unroll
            for (int n = 0; n < 2 * C; ++n) {
                const u32 i = lane + 64 * n, row = i / (8 * C), at = i % (8 * C) * 8;
                if (!(present >> row & 1u)) {
                    uint2* p = (uint2*)(rows + (u64)row * (2 * a.c.width) + at);
                    uint2 w = make_uint2(0, 0);
                    if (!begins) {
                        w = *p;
                        float y[8];
                        decode4<FMT>(w.x, y);
                        decode4<FMT>(w.y, y + 4);
#pragma unroll
                        for (int j = 0; j < 8; ++j) y[j] *= again;
                        w = make_uint2(encode4<FMT>(y), encode4<FMT>(y + 4));
                    }
                    *p = w;
                }
            }
        }
        if (lane == 0) *exponent = (int8_t)e;
    }
}

// 4-bit codes: a row's parts have their exponents to themselves, so that 8 numbers of a row are a thread's, whatever else the call writes, and four
// threads share a part.  A workgroup has `each` tokens, all their heads, keys and values; the workgroups from number `writers` on turn queries.  A lane keeps its
// piece of a row, and FP4_TURNS rows' pieces are asked for before the first is encoded.  18,596 tokens, 8 heads of 128: 30 us as they are, 50 with keys turned, 99 with 32 heads of
// queries (400 MB, 77 as a copy).
constexpr u32 FP4_TURNS = 4;

template <int C, bool TURN>
__global__ void __launch_bounds__(256) k_append_fp4(Store a, u32 writers, u32 each) {
    extern __shared__ double2 spin[];
    const bool writes = !TURN || blockIdx.x < writers;
    const u64 first = (u64)(writes ? blockIdx.x : blockIdx.x - writers) * each;
    const u32 n = (u32)min((u64)each, a.tokens - first);
    if constexpr (TURN) {
        if (!writes) {
            spin_queries(a, first, n, (float2*)spin);
            __syncthreads();
            turn_queries(a, first, n, (const float2*)spin);
            return;
        }
        spin_tokens(a, first, n, spin);
        __syncthreads();
    }
    // rows: token and head, all keys before all values, so that a wave has one kind and what turns keys stays out of the values' way
    constexpr u32 PIECES = 8 * C, PER_WAVE = 64 / PIECES;
    const u32 lane = threadIdx.x & 63, at = lane % PIECES * 8, sub = lane / PIECES, kv = a.c.kv_heads, rows = 2 * n * kv, step = PER_WAVE * 4;
    if (sub >= PER_WAVE) return;
    for (u32 row0 = wave_of() * PER_WAVE + sub; row0 < rows; row0 += FP4_TURNS * step) {
        float x[FP4_TURNS][8];
        int64_t slot[FP4_TURNS];
        u32 token[FP4_TURNS], head[FP4_TURNS];
        u64 from[FP4_TURNS];
#pragma unroll
        for (u32 i = 0; i < FP4_TURNS; ++i) {
            const u32 both = min(row0 + i * step, rows - 1), kind = both >= n * kv, row = both - kind * n * kv;
            token[i] = (row >= kv) + (row >= 2 * kv) + (row >= 3 * kv);
            head[i] = row - token[i] * kv;
            slot[i] = a.slots[first + token[i]];
            from[i] = (first + token[i]) * (u64)(kind ? a.ts[1] : a.ts[0]) + head[i] * (u64)(kind ? a.hs[1] : a.hs[0]);
#pragma unroll
            for (int j = 0; j < 8; ++j) x[i][j] = 0.f;
            if (at < a.c.dim) load8(kind ? a.x[1] : a.x[0], from[i] + at, a.dtype, x[i]);
        }
#pragma unroll
        for (u32 i = 0; i < FP4_TURNS; ++i) {
            const u32 row = row0 + i * step, kind = row >= n * kv;
            if (row >= rows || slot[i] < 0 || slot[i] >= (int64_t)a.c.num_pages * a.c.page_tokens) continue;          // the same for a part's four lanes
            if constexpr (TURN) {
                if (kind == 0 && at < a.c.dim) turn8(a, a.x[0], from[i], at, spin + token[i] * (a.turned / 2), x[i]);
            }
            float most = 0.f;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float y = fabsf(x[i][j]);
                if (y <= 3.402823466e38f) most = fmaxf(most, y);
            }
            most = fmaxf(most, __shfl_xor(most, 1));
            most = fmaxf(most, __shfl_xor(most, 2));
            const int e = least_exponent<PAG_KV_FP4>(most);
            const float down = power(-e);
#pragma unroll
            for (int j = 0; j < 8; ++j) x[i][j] *= down;
            const u32 page = (u32)((u64)slot[i] / a.c.page_tokens), place = row_of(a.c, page, head[i], (u32)((u64)slot[i] % a.c.page_tokens));
            *(u32*)(a.c.data + (u64)place * (64 * C) + kind * (32 * C) + at / 2) = encode8_fp4(x[i]);
            if (at % PART == 0) a.c.exponents[((u64)(place / BLOCK) * 2 + kind) * (2 * C * BLOCK) + at / PART * BLOCK + place % BLOCK] = (int8_t)e;
        }
    }
}

struct Load {
    Cache c;
    void* x[2];
    int64_t ts[2], hs[2];
    const int64_t* slots;
    u64 tokens;
    u32 dtype;
};

// A workgroup has 16 tokens of a head, keys and values, 16 bytes of output a thread and turn: all that a thread reads is asked for before the
// first of it is used.  Tokens that follow each other in a page are one stretch of 16 rows to read (16 rows of any heads and tokens:
// 128 us for 50,001 tokens, 8 heads of 128, to 16-bit floats; this way 126).  What is written goes past the caches, which
// keep the rows that were read (read again: 128 us through them, 74 past them).  Bound by memory: 105 MB in and 410 MB out, 4.1 TB/s where a copy reaches 5.2.
template <int FMT, int C, typename T>
__global__ void __launch_bounds__(256) k_read(Load a) {
    constexpr u32 EACH = 16 / sizeof(T), PIECES = 128 * C / EACH, TURNS = 16 * PIECES / 256;      // numbers, pieces of a row, turns
    __shared__ u32 sh_row[16];
    __shared__ float sh_up[16][2];
    const u32 head = blockIdx.x % a.c.kv_heads;
    const u64 token0 = (u64)(blockIdx.x / a.c.kv_heads) * 16;
    if (threadIdx.x < 16) {
        const int64_t slot = a.slots[min(token0 + threadIdx.x, a.tokens - 1)];
        u32 row = 0;
        float k = 0.f, v = 0.f;                  // zeros for slots that are none
        if (slot >= 0 && slot < (int64_t)a.c.num_pages * a.c.page_tokens) {
            row = row_of(a.c, (u32)((u64)slot / a.c.page_tokens), head, (u32)((u64)slot % a.c.page_tokens));
            const int8_t* e = a.c.exponents + (u64)(row / BLOCK) * 2;
            k = power(e[0]);
            v = power(e[1]);
        }
        sh_row[threadIdx.x] = row;
        sh_up[threadIdx.x][0] = k;
        sh_up[threadIdx.x][1] = v;
    }
    __syncthreads();
    u32 w[TURNS][EACH / 4];
#pragma unroll
    for (u32 n = 0; n < TURNS; ++n) {
        const u32 i = threadIdx.x + 256 * n, r = i / PIECES, at = i % PIECES * EACH;
#pragma unroll
        for (u32 x = 0; x < EACH / 4; ++x) w[n][x] = *(const u32*)(a.c.data + (u64)sh_row[r] * (128 * C) + at + 4 * x);
    }
#pragma unroll
    for (u32 n = 0; n < TURNS; ++n) {
        const u32 i = threadIdx.x + 256 * n, r = i / PIECES, both = i % PIECES * EACH, kind = both / (64 * C), at = both % (64 * C);
        if (token0 + r < a.tokens && at < a.c.dim && a.x[kind]) {
            const float up = sh_up[r][kind];
            float x[EACH];
#pragma unroll
            for (u32 y = 0; y < EACH / 4; ++y) decode4<FMT>(w[n][y], x + 4 * y);
            // a slot that is none has no numbers, whatever the row that was read instead holds
#pragma unroll
            for (u32 y = 0; y < EACH; ++y) x[y] = up != 0.f ? finite(x[y] * up) : 0.f;
            T* to = (T*)a.x[kind] + (int64_t)(token0 + r) * a.ts[kind] + (int64_t)head * a.hs[kind] + at;
            typedef u32 word4 __attribute__((ext_vector_type(4)));
            word4 y;
            if constexpr (sizeof(T) == 4) y = word4{ __float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]) };
            else y = word4{ pack2(x[0], x[1], a.dtype), pack2(x[2], x[3], a.dtype), pack2(x[4], x[5], a.dtype), pack2(x[6], x[7], a.dtype) };
            __builtin_nontemporal_store(y, (word4*)to);
        }
    }
}

// The same of 4-bit codes; every 16 bytes of output are numbers of one part.
template <int C, typename T>
__global__ void __launch_bounds__(256) k_read_fp4(Load a) {
    constexpr u32 EACH = 16 / sizeof(T), PIECES = 128 * C / EACH, TURNS = 16 * PIECES / 256;
    __shared__ u32 sh_row[16];
    __shared__ u32 sh_there[16];
    const u32 head = blockIdx.x % a.c.kv_heads;
    const u64 token0 = (u64)(blockIdx.x / a.c.kv_heads) * 16;
    if (threadIdx.x < 16) {
        const int64_t slot = a.slots[min(token0 + threadIdx.x, a.tokens - 1)];
        const bool there = slot >= 0 && slot < (int64_t)a.c.num_pages * a.c.page_tokens;
        sh_row[threadIdx.x] = there ? row_of(a.c, (u32)((u64)slot / a.c.page_tokens), head, (u32)((u64)slot % a.c.page_tokens)) : 0;
        sh_there[threadIdx.x] = there;
    }
    __syncthreads();
    u32 w[TURNS];
    int8_t e[TURNS];
#pragma unroll
    for (u32 n = 0; n < TURNS; ++n) {
        const u32 i = threadIdx.x + 256 * n, r = i / PIECES, both = i % PIECES * EACH, row = sh_row[r];
        const uint8_t* p = a.c.data + (u64)row * (64 * C) + both / 2;
        if constexpr (EACH == 4) w[n] = *(const uint16_t*)p;
        else w[n] = *(const u32*)p;
        e[n] = parts_of<C>(a.c, row / BLOCK, both / (64 * C))[both % (64 * C) / PART * BLOCK + row % BLOCK];
    }
#pragma unroll
    for (u32 n = 0; n < TURNS; ++n) {
        const u32 i = threadIdx.x + 256 * n, r = i / PIECES, both = i % PIECES * EACH, kind = both / (64 * C), at = both % (64 * C);
        if (token0 + r < a.tokens && at < a.c.dim && a.x[kind]) {
            const float up = power(e[n]);
            float x[EACH];
#pragma unroll
            for (u32 y = 0; y < EACH / 4; ++y) decode4_fp4(w[n] >> (16 * y), 1.f, x + 4 * y);
#pragma unroll
            for (u32 y = 0; y < EACH; ++y) x[y] = sh_there[r] ? finite(x[y] * up) : 0.f;
            T* to = (T*)a.x[kind] + (int64_t)(token0 + r) * a.ts[kind] + (int64_t)head * a.hs[kind] + at;
            typedef u32 word4 __attribute__((ext_vector_type(4)));
            word4 y;
            if constexpr (sizeof(T) == 4) y = word4{ __float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]) };
            else y = word4{ pack2(x[0], x[1], a.dtype), pack2(x[2], x[3], a.dtype), pack2(x[4], x[5], a.dtype), pack2(x[6], x[7], a.dtype) };
            __builtin_nontemporal_store(y, (word4*)to);
        }
    }
}

// f<FMT, C>() for the cache's format and row width
template <template <int, int> class F, int FMT, typename... A>
void for_width(const Cache& c, A&&... args) {
    const u32 n = c.width / 64;
    if (n == 1) F<FMT, 1>::run(args...);
    else if (n == 2) F<FMT, 2>::run(args...);
    else if (n == 3) F<FMT, 3>::run(args...);
    else F<FMT, 4>::run(args...);
}

template <template <int, int> class F, typename... A>
void for_cache(const Cache& c, A&&... args) {
    if (c.fmt == PAG_KV_INT8) for_width<F, PAG_KV_INT8>(c, args...);
    else if (c.fmt == PAG_KV_FP8) for_width<F, PAG_KV_FP8>(c, args...);
    else for_width<F, PAG_KV_FP4>(c, args...);
}

template <int FMT, int C>
struct RunAppend {
    static void run(hipStream_t st, const Store& a) {
        const u64 waves = a.tokens * 2 * a.c.kv_heads;
        const u32 spins = (u32)sizeof(double2) * (a.turned / 2);
        const u32 each = a.tokens <= 1024 ? 1 : QUERY_TOKENS;
        if constexpr (FMT == PAG_KV_FP4) {
            const u32 grid = (u32)((a.tokens + each - 1) / each);
            if (a.turned) k_append_fp4<C, true><<<a.heads ? 2 * grid : grid, 256, each * spins, st>>>(a, grid, each);
            else k_append_fp4<C, false><<<grid, 256, 0, st>>>(a, grid, each);
        } else {
            const u32 window = waves <= 4096 ? 1 : waves <= 32768 ? 4 : 16;
            const u64 windows = (a.tokens + window - 1) / window;
            if (a.turned) {
                const u32 writers = (u32)(windows * 2 * ((a.c.kv_heads + 3) / 4)), turners = a.heads ? (u32)((a.tokens + each - 1) / each) : 0;
                k_append<FMT, C, true><<<writers + turners, 256, BLOCK * spins, st>>>(a, window, writers, each);
            } else {
                k_append<FMT, C, false><<<(u32)((windows * 2 * a.c.kv_heads + 3) / 4), 256, 0, st>>>(a, window, 0, 0);
            }
        }
    }
};
template <int FMT, int C>
struct RunRead {
    static void run(hipStream_t st, u32 grid, const Load& a) {
        if constexpr (FMT == PAG_KV_FP4) {
            if (a.dtype == PAG_F32) k_read_fp4<C, float><<<grid, 256, 0, st>>>(a);
            else k_read_fp4<C, uint16_t><<<grid, 256, 0, st>>>(a);
        } else {
            if (a.dtype == PAG_F32) k_read<FMT, C, float><<<grid, 256, 0, st>>>(a);
            else k_read<FMT, C, uint16_t><<<grid, 256, 0, st>>>(a);
        }
    }
};

int launched(const char* what) {
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) { pag_set_error(std::string(what) + ": " + hipGetErrorString(e)); return PAG_EHIP; }
    return PAG_OK;
}

}  // namespace

int launch_extend(hipStream_t st, const pag_kv_tables& t, const int32_t* add, const pag_kv_step& s) {
    const Extend e{ add, t.lengths, t.free_pages, t.free_count, t.table, t.table_stride, s.tokens, t.requests, t.max_pages, t.page_tokens,
                    (u32)t.num_pages, s.offsets, s.context, s.granted, s.lengths, s.free_count, s.scratch, s.request, s.positions, s.slots };
    // one launch or two: 1,024 tokens 7.6 and 8.7 us, 2,048 tokens 9.0 and 9.2, 4,096 tokens 12.3 and 9.5
    const bool alone = s.tokens <= 2 * PLAN_THREADS;
    k_extend<<<1, PLAN_THREADS, 0, st>>>(e, alone ? s.tokens : 0);
    if (!alone) k_extend_tokens<<<(u32)((s.tokens + 255) / 256), 256, 0, st>>>(e);
    return launched("pag_kv_extend");
}

int launch_release(hipStream_t st, const pag_kv_tables& t, const int32_t* done) {
    k_release<<<1, PLAN_THREADS, 0, st>>>(t, done);
    return launched("pag_kv_release");
}

int launch_append(hipStream_t st, const Store& a) {
    for_cache<RunAppend>(a.c, st, a);
    return launched("pag_kv_append");
}

int launch_read(hipStream_t st, const Cache& c, const int64_t* slots, u64 tokens, u32 dtype, void* k, int64_t k_ts, int64_t k_hs, void* v,
                int64_t v_ts, int64_t v_hs) {
    const Load a{ c, { k, v }, { k_ts, v_ts }, { k_hs, v_hs }, slots, tokens, dtype };
    for_cache<RunRead>(c, st, (u32)((tokens + 15) / 16 * c.kv_heads), a);
    return launched("pag_kv_read");
}

}  // namespace pagkv
