// The 8-bit key/value cache: what its kernels share.
#pragma once

#include "pag_internal.h"

namespace pagkv {

constexpr int LOWEST_EXPONENT = -64;   // blocks of zeros, and what is too small to matter beside them
constexpr u32 BLOCK = 16;              // tokens that share an exponent

typedef _Float16 half2_t __attribute__((ext_vector_type(2)));
typedef _Float16 half8_t __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef float float2_t __attribute__((ext_vector_type(2)));
typedef float float4_t __attribute__((ext_vector_type(4)));

struct Cache {
    uint8_t* data;
    int8_t* exponents;
    u32 kv_heads, dim, width, page_tokens, page_blocks, num_pages, fmt;
};

struct Step {
    const int32_t* table;
    const int32_t* offsets;
    const int32_t* context;
    const int32_t* request;
    const int32_t* positions;
    u64 table_stride;
    u32 requests, max_pages, tokens;
};

// the wave's number in its workgroup, in a scalar register: what follows from it takes none of the lanes'
__device__ __forceinline__ u32 wave_of() { return (u32)__builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)); }

// 2^e in 32 bits, -126 <= e <= 127
__device__ __forceinline__ float power(int e) { return __uint_as_float((u32)(e + 127) << 23); }

// row of a token of a page and head; fits 32 bits (checked by the host)
__device__ __forceinline__ u32 row_of(const Cache& c, u32 page, u32 head, u32 place) { return (page * c.kv_heads + head) * c.page_tokens + place; }

// four codes of a word as numbers without their exponent
template <int FMT>
__device__ __forceinline__ void decode4(u32 w, float* x) {
    if constexpr (FMT == PAG_KV_INT8) {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = (float)(int8_t)(w >> (8 * i));
    } else {
        const float2_t lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
        x[0] = lo.x; x[1] = lo.y; x[2] = hi.x; x[3] = hi.y;
    }
}

// x: already divided by the power of two.  NaN is held as 0, what is beyond the largest code as that code.
template <int FMT>
__device__ __forceinline__ u32 encode4(const float* x) {
    constexpr float MOST = FMT == PAG_KV_INT8 ? 127.f : 448.f;
    float y[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = x[i] == x[i] ? fminf(fmaxf(x[i], -MOST), MOST) : 0.f;
    if constexpr (FMT == PAG_KV_INT8) {
        u32 w = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) w |= ((u32)(int)rintf(y[i]) & 255u) << (8 * i);
        return w;
    } else {
        int w = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
        return (u32)__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], w, true);
    }
}

// the smallest exponent at which the largest code reaches `most` (127 = 1.984375 * 2^6, 448 = 1.75 * 2^8)
template <int FMT>
__device__ __forceinline__ int least_exponent(float most) {
    const u32 bits = __float_as_uint(most);
    constexpr u32 FRACTION = FMT == PAG_KV_INT8 ? 0x7E0000u : 0x600000u;
    const int e = (int)(bits >> 23) - 127 - (FMT == PAG_KV_INT8 ? 6 : 8) + ((bits & 0x7FFFFFu) > FRACTION ? 1 : 0);
    return e < LOWEST_EXPONENT ? LOWEST_EXPONENT : e;
}

__device__ __forceinline__ void widen_row8(const uint4& r, u32 dtype, float* x) {      // PAG_F16 or PAG_BF16
    const u32 w[4] = { r.x, r.y, r.z, r.w };
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (dtype == PAG_BF16) {
            x[2 * i] = __uint_as_float(w[i] << 16);
            x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
        } else {
            const half2_t h = __builtin_bit_cast(half2_t, w[i]);
            x[2 * i] = (float)h.x;
            x[2 * i + 1] = (float)h.y;
        }
    }
}

// eight numbers of an input row in 32 bits
__device__ __forceinline__ void load8(const void* p, u64 at, u32 dtype, float* x) {
    if (dtype == PAG_F32) {
        const float4 a = *(const float4*)((const float*)p + at), b = *(const float4*)((const float*)p + at + 4);
        x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
        return;
    }
    widen_row8(*(const uint4*)((const uint16_t*)p + at), dtype, x);
}

// Blocks near the end of 32 bits hold their largest numbers rounded up to 2^128 (255.99 * 2^120 at 2^122 is 64 of these); what comes out, and means
// of such numbers, ends at the largest that bf16 holds.  NaN stays what it is.
__device__ __forceinline__ float finite(float x) {
    constexpr float MOST = 0x1.fep127f;
    return fabsf(x) > MOST ? copysignf(MOST, x) : x;
}

__device__ __forceinline__ u32 pack2(float a, float b, u32 dtype) {       // to nearest even
    const float2_t x = { a, b };
    if (dtype == PAG_BF16) return __builtin_bit_cast(u32, __builtin_convertvector(x, bf16x2_t));
    return __builtin_bit_cast(u32, __builtin_convertvector(x, half2_t));
}

struct Attend {
    Cache c;
    Step s;
    const void* q;
    void* out;
    float* lse;
    const float* slopes;
    const int64_t* ids;
    int64_t q_ts, q_hs, o_ts, o_hs, ids_ts, ids_hs;
    u32 heads, group, dtype, window, id_heads, k;
    u32 listed;                           // attention over ids and a window
    u32 row_tiles;                        // tiles of 16 query rows that a wave has at most to a key/value head; 0: the wide kernel
    u32 many_rows;                        // the wide kernel: a request has more rows than four of its waves
    float scale, softcap;
    float* partial;                       // the workspace: two parts a workgroup, of the piece that another one began, and of the piece that it began and another one ends
    int2* joined;                         // narrow kernels: [tokens * heads] first and last workgroup of the row's pieces; first < 0: written whole
};

int launch_extend(hipStream_t st, const pag_kv_tables& t, const int32_t* add, const pag_kv_step& s);
int launch_release(hipStream_t st, const pag_kv_tables& t, const int32_t* done);
int launch_append(hipStream_t st, const Cache& c, u32 dtype, const void* k, int64_t k_ts, int64_t k_hs, const void* v, int64_t v_ts, int64_t v_hs,
                  const int64_t* slots, u64 tokens);
int launch_read(hipStream_t st, const Cache& c, const int64_t* slots, u64 tokens, u32 dtype, void* k, int64_t k_ts, int64_t k_hs, void* v,
                int64_t v_ts, int64_t v_hs);
int launch_attend(hipStream_t st, const Attend& a, int num_cu);

int launch_attend_wide(hipStream_t st, const Attend& a, int num_cu);

u64 attend_workspace(const Attend& a, int num_cu);      // bytes
u64 wide_workspace(u32 width, int num_cu);
int num_cu_of_current();                        // < 0: no GPU

}  // namespace pagkv
