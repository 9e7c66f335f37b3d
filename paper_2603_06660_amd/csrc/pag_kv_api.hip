// C ABI of the 8-bit key/value cache: argument checking; everything that computes runs in the kernels.
#include <algorithm>
#include <atomic>
#include <cmath>

#include "pag_kv.h"

namespace pagkv {

int num_cu_of_current() {
    static std::atomic<int> known[64];
    int device = -1, n = 0;
    if (hipGetDevice(&device) != hipSuccess || device < 0) return -1;
    if (device < 64 && (n = known[device].load(std::memory_order_relaxed)) > 0) return n;
    if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, device) != hipSuccess || n <= 0) return -1;
    if (device < 64) known[device].store(n, std::memory_order_relaxed);
    return n;
}

namespace {

bool aligned(const void* p, uintptr_t to) { return ((uintptr_t)p & (to - 1)) == 0; }

int cache_of(const pag_kv_cache* c, Cache* out) {
    PAG_CHECK(c != nullptr, PAG_EINVAL, "cache is null");
    PAG_CHECK(c->struct_size == sizeof(pag_kv_cache), PAG_EINVAL, "pag_kv_cache.struct_size does not match this library");
    PAG_CHECK(c->format <= PAG_KV_FP8, PAG_EINVAL, "unknown cache format");
    PAG_CHECK(c->kv_heads > 0 && c->head_dim > 0 && c->page_tokens > 0 && c->num_pages > 0, PAG_EINVAL,
              "kv_heads, head_dim, page_tokens and num_pages must be positive");
    PAG_CHECK(c->head_dim % 8 == 0 && c->head_dim <= 256, PAG_EUNSUPPORTED, "this build needs head_dim % 8 == 0 and head_dim <= 256");
    PAG_CHECK(c->page_tokens % BLOCK == 0 && c->page_tokens <= (1u << 20), PAG_EUNSUPPORTED, "this build needs page_tokens % 16 == 0 and page_tokens <= 2^20");
    PAG_CHECK(c->kv_heads <= 4096, PAG_EUNSUPPORTED, "kv_heads above 4096 is not built");
    PAG_CHECK(c->num_pages <= 0xFFFFFFFFull / c->page_tokens / c->kv_heads && c->num_pages < (1ull << 31), PAG_EUNSUPPORTED,
              "num_pages * kv_heads * page_tokens must be below 2^32");
    PAG_CHECK(c->data != nullptr && c->exponents != nullptr, PAG_EINVAL, "cache data or exponents is null");
    PAG_CHECK(aligned(c->data, 16) && aligned(c->exponents, 2), PAG_EINVAL, "cache data must be 16-byte aligned, exponents 2-byte");
    *out = Cache{ c->data, c->exponents, c->kv_heads, c->head_dim, (c->head_dim + 63) / 64 * 64, c->page_tokens, c->page_tokens / BLOCK,
                  (u32)c->num_pages, c->format };
    return PAG_OK;
}

int check_step(const pag_kv_step* s) {
    PAG_CHECK(s != nullptr, PAG_EINVAL, "step is null");
    PAG_CHECK(s->struct_size == sizeof(pag_kv_step), PAG_EINVAL, "pag_kv_step.struct_size does not match this library");
    PAG_CHECK(s->requests > 0 && s->requests < (1u << 24), PAG_EINVAL, "a step needs between 1 and 2^24 - 1 requests");
    PAG_CHECK(s->tokens < (1ull << 31), PAG_EUNSUPPORTED, "a step of 2^31 tokens or more is not built");
    PAG_CHECK(s->table != nullptr && s->max_pages > 0 && s->table_stride >= s->max_pages, PAG_EINVAL, "the step's table is null, empty, or its rows overlap");
    return PAG_OK;
}

int check_tables(const pag_kv_tables* t) {
    PAG_CHECK(t != nullptr, PAG_EINVAL, "tables is null");
    PAG_CHECK(t->struct_size == sizeof(pag_kv_tables), PAG_EINVAL, "pag_kv_tables.struct_size does not match this library");
    PAG_CHECK(t->requests > 0 && t->requests < (1u << 24), PAG_EINVAL, "tables need between 1 and 2^24 - 1 requests");
    PAG_CHECK(t->max_pages > 0 && t->table_stride >= t->max_pages, PAG_EINVAL, "the table is empty, or its rows overlap");
    PAG_CHECK(t->page_tokens > 0 && t->page_tokens % BLOCK == 0 && t->page_tokens <= (1u << 20), PAG_EUNSUPPORTED,
              "this build needs page_tokens % 16 == 0 and page_tokens <= 2^20");
    PAG_CHECK((u64)t->max_pages * t->page_tokens <= 0x7FFF0000ull, PAG_EUNSUPPORTED, "requests of more than 2^31 - 2^16 tokens are not built");
    PAG_CHECK(t->num_pages > 0 && t->num_pages < (1ull << 31), PAG_EINVAL, "num_pages must be between 1 and 2^31 - 1");
    PAG_CHECK(t->table && t->lengths && t->free_pages && t->free_count, PAG_EINVAL, "tables: null pointer");
    return PAG_OK;
}

int check_rows(const void* p, int64_t token_stride, int64_t head_stride, u32 bytes, u32 to, const char* message) {
    PAG_CHECK(aligned(p, to) && token_stride * (int64_t)bytes % (int64_t)to == 0 && head_stride * (int64_t)bytes % (int64_t)to == 0, PAG_EINVAL, message);
    return PAG_OK;
}

// What decides how a call is laid out: everything but its arrays.
int layout_of(const pag_kv_cache* cache, const pag_kv_step* step, const pag_kv_attention* args, bool selected, uint32_t id_heads, uint32_t k, Attend* a) {
    int rc;
    if ((rc = cache_of(cache, &a->c)) || (rc = check_step(step))) return rc;
    PAG_CHECK(args != nullptr, PAG_EINVAL, "args is null");
    PAG_CHECK(args->struct_size == sizeof(pag_kv_attention), PAG_EINVAL, "pag_kv_attention.struct_size does not match this library");
    PAG_CHECK(args->dtype == PAG_F16 || args->dtype == PAG_BF16, PAG_EUNSUPPORTED, "attention takes PAG_F16 or PAG_BF16");
    PAG_CHECK(args->heads > 0 && args->heads <= 65536 && args->heads % a->c.kv_heads == 0, PAG_EINVAL, "heads must be a multiple of kv_heads, at most 65536");
    PAG_CHECK((u64)step->max_pages * a->c.page_tokens <= 0x7FFF0000ull, PAG_EUNSUPPORTED, "requests of more than 2^31 - 2^16 tokens are not built");
    PAG_CHECK(step->tokens * args->heads < (1ull << 31) && (u64)step->requests * a->c.kv_heads < (1ull << 31), PAG_EUNSUPPORTED,
              "tokens * heads and requests * kv_heads must be below 2^31");
    a->s = Step{ step->table, step->offsets, step->context, step->request, step->positions, step->table_stride, step->requests, step->max_pages, (u32)step->tokens };
    a->heads = args->heads;
    a->dtype = args->dtype;
    a->window = args->window;
    a->group = a->heads / a->c.kv_heads;
    if (selected) {
        PAG_CHECK(id_heads > 0 && id_heads % a->c.kv_heads == 0 && args->heads % id_heads == 0, PAG_EINVAL, "id_heads must be a multiple of kv_heads that divides heads");
        PAG_CHECK((u64)k + args->window < (1ull << 30), PAG_EUNSUPPORTED, "k + window must be below 2^30");
        a->listed = 1;
        a->id_heads = id_heads;
        a->k = k;
        a->group = a->heads / id_heads;
    }
    // Query rows that a request's new tokens make for a key/value head, as far as the host can tell.  One or two tiles of 16 rows a wave, each
    // of which widens its own keys, or the wide kernel, whose waves share them; in us, 8 key/value heads of 128, as one, two, wide:
    //   32 requests of 300 to 12,000 tokens: 16 rows 50, 51, 114; 20 rows 79, 54, 114; 64 rows 143, 92, 126; 96 rows 203, 125, 128; 256 rows 483, 278, 223
    //   one of 30,000 tokens: 16 rows 23, 27, 45; 64 rows 39, 35, 49; 128 rows 60, 47, 52; 256 rows 102, 73, 64
    //   32 of 3,000 tokens: 64 rows 130, 74, 90; 96 rows 192, 119, 92.  With few keys the wide kernel is not better before some 500 rows (one request of
    //   3,000 tokens, 128 rows: 21, 24, 36), but those are the short calls.
    // Rows of more than 192 numbers leave no registers for two tiles, which spill: 32 requests of 4,000 tokens, 256 numbers a head: 32 rows 201, (225), 259;
    // 48 rows 288, (429), 265.
    const u64 rows = (step->max_new ? step->max_new : (step->tokens + step->requests - 1) / step->requests) * (u64)a->group;
    const bool two = a->c.width <= 192;
    a->row_tiles = selected || rows <= (two ? 16u : 32u) ? 1 : two && rows <= 64 ? 2 : 0;
    a->many_rows = rows > 128;
    // a launch has fewer than 2^32 threads: these kernels have up to 512 for a list, a request's head or a row to join; the wide kernel's grid is the chip's
    const bool fits = step->tokens * args->heads < (1ull << 23) && (u64)step->requests * a->c.kv_heads < (1ull << 23);
    PAG_CHECK(!selected || fits, PAG_EUNSUPPORTED, "attention over ids needs tokens * heads and requests * kv_heads below 2^23");
    if (!fits) a->row_tiles = 0;
    return PAG_OK;
}

int arrays_of(const pag_kv_step* step, const pag_kv_attention* args, Attend* a, int* num_cu) {
    PAG_CHECK(std::isfinite(args->scale) && std::isfinite(args->softcap) && args->softcap >= 0.f, PAG_EINVAL, "scale and softcap must be finite, softcap not negative");
    if (step->tokens == 0) return PAG_OK;
    int rc;
    PAG_CHECK(args->q != nullptr && args->out != nullptr, PAG_EINVAL, "q or out is null");
    if ((rc = check_rows(args->q, args->q_token_stride, args->q_head_stride, 2, 16, "q must be 16-byte aligned, its strides multiples of 8 elements"))) return rc;
    if ((rc = check_rows(args->out, args->out_token_stride, args->out_head_stride, 2, 16, "out must be 16-byte aligned, its strides multiples of 8 elements"))) return rc;
    PAG_CHECK((args->slopes == nullptr || aligned(args->slopes, 4)) && (args->lse == nullptr || aligned(args->lse, 4)), PAG_EINVAL, "slopes and lse must be 4-byte aligned");
    PAG_CHECK(aligned(args->workspace, 16) && (args->workspace != nullptr || args->workspace_bytes == 0), PAG_EINVAL,
              "workspace is null but has a size, or is not 16-byte aligned");
    *num_cu = num_cu_of_current();
    PAG_CHECK(*num_cu > 0, PAG_EHIP, "no current GPU");
    const u64 need = attend_workspace(*a, *num_cu);
    PAG_CHECK(need == 0 || (args->workspace != nullptr && args->workspace_bytes >= need), PAG_EINVAL, "workspace is null or smaller than pag_kv_workspace_bytes");
    a->q = args->q; a->q_ts = args->q_token_stride; a->q_hs = args->q_head_stride;
    a->out = args->out; a->o_ts = args->out_token_stride; a->o_hs = args->out_head_stride;
    a->lse = args->lse;
    a->slopes = args->slopes;
    a->scale = args->scale;
    // scores below 2^-64 are all the same to a weight of 32 bits, and the reciprocal of a smaller cap leaves them
    a->softcap = args->softcap > 0.f ? std::max(args->softcap, 0x1p-64f) : 0.f;
    a->partial = (float*)args->workspace;
    return PAG_OK;
}

}  // namespace
}  // namespace pagkv

using namespace pagkv;

extern "C" int pag_kv_extend(const pag_kv_tables* tables, const int32_t* add, const pag_kv_step* step, void* stream) {
    return guarded("pag_kv_extend", [&]() -> int {
        int rc;
        if ((rc = check_tables(tables)) || (rc = check_step(step))) return rc;
        PAG_CHECK(add != nullptr, PAG_EINVAL, "add is null");
        PAG_CHECK(step->requests == tables->requests && step->table == tables->table && step->table_stride == tables->table_stride && step->max_pages == tables->max_pages,
                  PAG_EINVAL, "the step belongs to other tables");
        PAG_CHECK(step->offsets && step->context && step->granted && step->lengths && step->free_count && step->scratch, PAG_EINVAL, "step: null pointer");
        PAG_CHECK(step->tokens == 0 || (step->request && step->positions && step->slots), PAG_EINVAL, "step: null pointer");
        return launch_extend((hipStream_t)stream, *tables, add, *step);
    });
}

extern "C" int pag_kv_release(const pag_kv_tables* tables, const int32_t* done, void* stream) {
    return guarded("pag_kv_release", [&]() -> int {
        const int rc = check_tables(tables);
        if (rc) return rc;
        PAG_CHECK(done != nullptr, PAG_EINVAL, "done is null");
        return launch_release((hipStream_t)stream, *tables, done);
    });
}

extern "C" int pag_kv_append(const pag_kv_cache* cache, uint32_t dtype, const void* k, int64_t k_token_stride, int64_t k_head_stride, const void* v,
                             int64_t v_token_stride, int64_t v_head_stride, const int64_t* slots, uint64_t tokens, void* stream) {
    return guarded("pag_kv_append", [&]() -> int {
        Cache c;
        int rc = cache_of(cache, &c);
        if (rc) return rc;
        PAG_CHECK(dtype <= PAG_BF16, PAG_EINVAL, "unknown dtype");
        PAG_CHECK(tokens < (1ull << 27) && tokens * c.kv_heads < (1ull << 27), PAG_EUNSUPPORTED, "tokens * kv_heads must be below 2^27");
        if (tokens == 0) return PAG_OK;
        PAG_CHECK(k && v && slots, PAG_EINVAL, "k, v or slots is null");
        const u32 bytes = dtype == PAG_F32 ? 4 : 2;
        if ((rc = check_rows(k, k_token_stride, k_head_stride, bytes, 16, "k and its strides must be multiples of 16 bytes"))) return rc;
        if ((rc = check_rows(v, v_token_stride, v_head_stride, bytes, 16, "v and its strides must be multiples of 16 bytes"))) return rc;
        return launch_append((hipStream_t)stream, c, dtype, k, k_token_stride, k_head_stride, v, v_token_stride, v_head_stride, slots, tokens);
    });
}

extern "C" int pag_kv_read(const pag_kv_cache* cache, const int64_t* slots, uint64_t tokens, uint32_t dtype, void* k, int64_t k_token_stride, int64_t k_head_stride,
                           void* v, int64_t v_token_stride, int64_t v_head_stride, void* stream) {
    return guarded("pag_kv_read", [&]() -> int {
        Cache c;
        int rc = cache_of(cache, &c);
        if (rc) return rc;
        PAG_CHECK(dtype <= PAG_BF16, PAG_EINVAL, "unknown dtype");
        PAG_CHECK(tokens < (1ull << 27) && tokens * c.kv_heads < (1ull << 27), PAG_EUNSUPPORTED, "tokens * kv_heads must be below 2^27");
        if (tokens == 0 || (!k && !v)) return PAG_OK;
        PAG_CHECK(slots != nullptr, PAG_EINVAL, "slots is null");
        const u32 bytes = dtype == PAG_F32 ? 4 : 2;
        if (k && (rc = check_rows(k, k_token_stride, k_head_stride, bytes, 16, "k and its strides must be multiples of 16 bytes"))) return rc;
        if (v && (rc = check_rows(v, v_token_stride, v_head_stride, bytes, 16, "v and its strides must be multiples of 16 bytes"))) return rc;
        return launch_read((hipStream_t)stream, c, slots, tokens, dtype, k, k_token_stride, k_head_stride, v, v_token_stride, v_head_stride);
    });
}

extern "C" int pag_kv_workspace_bytes(const pag_kv_cache* cache, const pag_kv_step* step, const pag_kv_attention* args, int selected, uint32_t id_heads, uint32_t k,
                                      uint64_t* bytes) {
    return guarded("pag_kv_workspace_bytes", [&]() -> int {
        Attend a = {};
        const int rc = layout_of(cache, step, args, selected != 0, id_heads, k, &a);
        if (rc) return rc;
        PAG_CHECK(bytes != nullptr, PAG_EINVAL, "bytes is null");
        const int num_cu = num_cu_of_current();
        PAG_CHECK(num_cu > 0, PAG_EHIP, "no current GPU");
        *bytes = attend_workspace(a, num_cu);
        return PAG_OK;
    });
}

extern "C" int pag_kv_attend(const pag_kv_cache* cache, const pag_kv_step* step, const pag_kv_attention* args, void* stream) {
    return guarded("pag_kv_attend", [&]() -> int {
        Attend a = {};
        int num_cu = 0, rc;
        if ((rc = layout_of(cache, step, args, false, 0, 0, &a)) || (rc = arrays_of(step, args, &a, &num_cu)) || step->tokens == 0) return rc;
        PAG_CHECK(step->offsets && step->context, PAG_EINVAL, "step: offsets or context is null");
        return launch_attend((hipStream_t)stream, a, num_cu);
    });
}

extern "C" int pag_kv_attend_selected(const pag_kv_cache* cache, const pag_kv_step* step, const pag_kv_attention* args, const int64_t* ids, int64_t ids_token_stride,
                                      int64_t ids_head_stride, uint32_t id_heads, uint32_t k, void* stream) {
    return guarded("pag_kv_attend_selected", [&]() -> int {
        Attend a = {};
        int num_cu = 0, rc;
        if ((rc = layout_of(cache, step, args, true, id_heads, k, &a)) || (rc = arrays_of(step, args, &a, &num_cu)) || step->tokens == 0) return rc;
        PAG_CHECK(step->request && step->positions, PAG_EINVAL, "step: request or positions is null");
        PAG_CHECK(k == 0 || (ids != nullptr && aligned(ids, 8)), PAG_EINVAL, "ids is null or not 8-byte aligned");
        a.ids = ids;
        a.ids_ts = ids_token_stride;
        a.ids_hs = ids_head_stride;
        return launch_attend((hipStream_t)stream, a, num_cu);
    });
}
