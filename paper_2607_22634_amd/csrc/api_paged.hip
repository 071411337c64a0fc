// Host side of the paged KV cache: argument validation, workspace sizing and
// dispatch.  Nothing here touches the GPU before every check has passed.
#include <math.h>

#include "common.hpp"
#include "paged.hpp"

namespace presto_host {

size_t pages_workspace_bytes(const presto_pages_desc* d, int64_t n);
presto_status launch_pages_reserve(const presto_pages_desc* d, int32_t* refs, int32_t* table, const int32_t* ctx,
                                   const int32_t* add, int32_t extra, int32_t* ctx_out, int32_t* flags, void* ws,
                                   hipStream_t stream);
presto_status launch_pages_fork(const presto_pages_desc* d, int32_t* refs, int32_t* table, int32_t* ctx,
                                const int32_t* parent, const int32_t* child, int32_t n, void* k, void* v,
                                int32_t* flags, void* ws, hipStream_t stream);
presto_status launch_pages_free(const presto_pages_desc* d, int32_t* refs, int32_t* table, int32_t* ctx,
                                const int32_t* rows, int32_t n, int32_t* flags, hipStream_t stream);
presto_status launch_pages_trim(const presto_pages_desc* d, int32_t* refs, int32_t* table, const int32_t* ctx,
                                int32_t window, int32_t sinks, int32_t* flags, hipStream_t stream);
presto_status launch_pages_compact(const presto_pages_desc* d, const int32_t* refs, int32_t* refs_out,
                                   const int32_t* table, int32_t* table_out, int32_t* n_live, int32_t* map_out,
                                   void* k, void* v, int32_t* flags, void* ws, hipStream_t stream);
presto_status launch_append_kv(const presto_pages_desc* d, const void* k_new, const void* v_new, int64_t new_stride,
                               int64_t new_rows, const int32_t* offsets, int32_t max_new, void* k, void* v,
                               const int32_t* table, const int32_t* ctx, const int32_t* ctx_new, int32_t* flags,
                               hipStream_t stream);

}  // namespace presto_host

using namespace presto_host;

#define REQUIRE(cond, ...)                                        \
    do {                                                          \
        if (!(cond)) return set_error(PRESTO_ERR_INVALID_ARG, __VA_ARGS__); \
    } while (0)

static presto_status check_ws(void* ws, size_t have, size_t need) {
    if (need > 0 && (ws == nullptr || have < need))
        return set_error(PRESTO_ERR_WORKSPACE, "workspace of %zu bytes needed, %zu given", need,
                         ws ? have : (size_t)0);
    return PRESTO_OK;
}

extern "C" {

// Checks a pool and fills in its default strides.
static presto_status check_pages(presto_pages_desc& p, const char* who) {
    REQUIRE(p.dt == PRESTO_DT_BF16 || p.dt == PRESTO_DT_F32, "%s: unknown dtype %d", who, (int)p.dt);
    REQUIRE(p.batch >= 0, "%s: batch < 0", who);
    REQUIRE(p.page_size >= 16 && p.page_size <= 1024 && (p.page_size & (p.page_size - 1)) == 0,
            "%s: page_size=%d is not a power of two in 16..1024", who, p.page_size);
    REQUIRE(p.hkv >= 1 && p.hkv <= 4096, "%s: hkv=%d outside 1..4096", who, p.hkv);
    REQUIRE(p.head_dim == 64 || p.head_dim == 128, "%s: head_dim %d", who, p.head_dim);
    REQUIRE(p.num_pages >= 1, "%s: num_pages < 1", who);
    REQUIRE(p.max_pages >= 1 && p.max_pages <= (1 << 20) &&
                (int64_t)p.max_pages * p.page_size < ((int64_t)1 << 30),
            "%s: max_pages=%d outside 1..2^20 or 2^30 positions or more", who, p.max_pages);
    REQUIRE(p.batch < (1 << 23) && (int64_t)p.batch * p.max_pages < ((int64_t)1 << 31),
            "%s: 2^23 sequences or 2^31 table entries, or more", who);
    REQUIRE(p.layers >= 1, "%s: layers < 1", who);
    const int64_t page = (int64_t)p.page_size * p.hkv * p.head_dim;
    const int64_t unit = p.dt == PRESTO_DT_BF16 ? 8 : 4;
    if (p.page_stride == 0) p.page_stride = page;
    REQUIRE(p.page_stride >= page && p.page_stride % unit == 0 &&
                p.page_stride <= ((int64_t)1 << 60) / p.num_pages,
            "%s: page_stride %lld", who, (long long)p.page_stride);
    if (p.layer_stride == 0) p.layer_stride = p.page_stride * p.num_pages;
    REQUIRE(p.layer_stride > 0 && p.layer_stride % unit == 0 && p.layer_stride <= ((int64_t)1 << 60) / p.layers,
            "%s: layer_stride %lld", who, (long long)p.layer_stride);
    return PRESTO_OK;
}

static bool aligned16(const void* a, const void* b, const void* c = nullptr, const void* d = nullptr) {
    return (((uintptr_t)a | (uintptr_t)b | (uintptr_t)c | (uintptr_t)d) & 15) == 0;
}

// Checks a call, fills in its default strides and plans it.
static presto_status check_paged_attn(presto_paged_attn_desc& d, PagedPlan& plan, bool decode, const char* who) {
    presto_status st = check_pages(d.pages, who);
    if (st != PRESTO_OK) return st;
    if (decode) {
        d.max_q = 1;
        d.total_q = d.pages.batch;
    }
    REQUIRE(d.hq >= 1 && d.hq % d.pages.hkv == 0, "%s: hq must be a positive multiple of hkv", who);
    REQUIRE(d.max_ctx >= 0 && d.max_ctx <= (int64_t)d.pages.max_pages * d.pages.page_size,
            "%s: max_ctx=%d outside 0..max_pages * page_size", who, d.max_ctx);
    REQUIRE(d.total_ctx >= 0, "%s: total_ctx < 0", who);
    REQUIRE(d.total_q >= 0 && d.total_q < ((int64_t)1 << 30), "%s: total_q outside 0..2^30", who);
    REQUIRE(d.max_q >= 0 && (int64_t)d.max_q * (d.hq / d.pages.hkv) < ((int64_t)1 << 30),
            "%s: max_q < 0 or too many query rows", who);
    REQUIRE(d.window >= 0 && d.window <= (1 << 30), "%s: window outside 0..2^30", who);
    REQUIRE(d.sinks >= 0 && d.sinks <= (1 << 30), "%s: sinks outside 0..2^30", who);
    REQUIRE(isfinite(d.scale) && d.scale > 0.f, "%s: scale must be positive", who);
    if (d.q_stride == 0) d.q_stride = (int64_t)d.hq * d.pages.head_dim;
    REQUIRE(d.q_stride >= (int64_t)d.hq * d.pages.head_dim && d.q_stride <= ((int64_t)1 << 31) &&
                d.q_stride % (d.pages.dt == PRESTO_DT_BF16 ? 8 : 4) == 0,
            "%s: q_stride %lld", who, (long long)d.q_stride);
    if (d.pages.batch > 0 && d.max_q > 0) {
        plan = paged_plan(&d);
        if (!plan.fits) return set_error(PRESTO_ERR_UNSUPPORTED, "%s: too many query rows for one call", who);
    }
    return PRESTO_OK;
}

static size_t paged_attn_ws(const presto_paged_attn_desc* desc, bool decode) {
    if (!desc) return 0;
    presto_paged_attn_desc d = *desc;
    PagedPlan plan{};
    return check_paged_attn(d, plan, decode, "workspace") == PRESTO_OK ? plan.bytes : 0;
}

static presto_status paged_attn(const presto_paged_attn_desc* desc, bool decode, const char* who, const void* q,
                                const int32_t* q_offsets, const void* k_pages, const void* v_pages,
                                const int32_t* page_table, const int32_t* ctx, void* out, int32_t* flags, void* ws,
                                size_t ws_bytes, hipStream_t stream) {
    set_error(PRESTO_OK, "%s", "");
    REQUIRE(desc, "%s: null descriptor", who);
    presto_paged_attn_desc d = *desc;
    PagedPlan plan{};
    presto_status st = check_paged_attn(d, plan, decode, who);
    if (st != PRESTO_OK) return st;
    if (d.pages.batch == 0 || d.max_q == 0 || d.total_q == 0) return PRESTO_OK;
    REQUIRE(q && (decode || q_offsets) && k_pages && v_pages && page_table && ctx && out, "%s: null pointer", who);
    REQUIRE(aligned16(q, k_pages, v_pages, out), "%s: tensors must be 16-byte aligned", who);
    st = check_ws(ws, ws_bytes, plan.bytes);
    if (st != PRESTO_OK) return st;
    REQUIRE(aligned16(ws, nullptr), "%s: the workspace must be 16-byte aligned", who);
    return launch_paged_attn(&d, plan, q, decode ? nullptr : q_offsets, k_pages, v_pages, page_table, ctx, out, flags, ws,
                             stream);
}

size_t presto_paged_attention_workspace(const presto_paged_attn_desc* desc) { return paged_attn_ws(desc, true); }
size_t presto_window_attention_workspace(const presto_paged_attn_desc* desc) { return paged_attn_ws(desc, false); }

presto_status presto_paged_attention(const presto_paged_attn_desc* desc, const void* q, const void* k_pages,
                                     const void* v_pages, const int32_t* page_table, const int32_t* ctx, void* out,
                                     int32_t* flags, void* ws, size_t ws_bytes, hipStream_t stream) {
    return paged_attn(desc, true, "presto_paged_attention", q, nullptr, k_pages, v_pages, page_table, ctx, out,
                      flags, ws, ws_bytes, stream);
}

presto_status presto_window_attention(const presto_paged_attn_desc* desc, const void* q, const int32_t* q_offsets,
                                      const void* k_pages, const void* v_pages, const int32_t* page_table,
                                      const int32_t* ctx, void* out, int32_t* flags, void* ws, size_t ws_bytes,
                                      hipStream_t stream) {
    return paged_attn(desc, false, "presto_window_attention", q, q_offsets, k_pages, v_pages, page_table, ctx, out,
                      flags, ws, ws_bytes, stream);
}

size_t presto_pages_workspace(const presto_pages_desc* desc) {
    if (!desc) return 0;
    presto_pages_desc d = *desc;
    if (check_pages(d, "presto_pages_workspace") != PRESTO_OK) return 0;
    return pages_workspace_bytes(&d, d.batch);
}

// what the calls on the books have in common
static presto_status check_books(const presto_pages_desc* desc, presto_pages_desc& d, const char* who) {
    set_error(PRESTO_OK, "%s", "");
    REQUIRE(desc, "%s: null descriptor", who);
    d = *desc;
    return check_pages(d, who);
}
static presto_status check_books_ws(const presto_pages_desc& d, const char* who, void* ws, size_t ws_bytes) {
    const presto_status st = check_ws(ws, ws_bytes, pages_workspace_bytes(&d, d.batch));
    if (st != PRESTO_OK) return st;
    REQUIRE(aligned16(ws, nullptr), "%s: the workspace must be 16-byte aligned", who);
    return PRESTO_OK;
}

presto_status presto_pages_reserve(const presto_pages_desc* desc, int32_t* refs, int32_t* page_table,
                                   const int32_t* ctx, const int32_t* add, int32_t extra, int32_t* ctx_out,
                                   int32_t* flags, void* ws, size_t ws_bytes, hipStream_t stream) {
    const char* who = "presto_pages_reserve";
    presto_pages_desc d;
    presto_status st = check_books(desc, d, who);
    if (st != PRESTO_OK) return st;
    REQUIRE(extra >= 0, "%s: extra < 0", who);
    if (d.batch == 0) return PRESTO_OK;
    REQUIRE(refs && page_table && ctx && ctx_out, "%s: null pointer", who);
    st = check_books_ws(d, who, ws, ws_bytes);
    if (st != PRESTO_OK) return st;
    return launch_pages_reserve(&d, refs, page_table, ctx, add, extra, ctx_out, flags, ws, stream);
}

presto_status presto_append_kv(const presto_pages_desc* desc, const void* k_new, const void* v_new,
                               int64_t new_rows, int64_t new_stride, const int32_t* offsets, int32_t max_new,
                               void* k_pages, void* v_pages, const int32_t* page_table, const int32_t* ctx,
                               const int32_t* ctx_new, int32_t* flags, hipStream_t stream) {
    const char* who = "presto_append_kv";
    presto_pages_desc d;
    presto_status st = check_books(desc, d, who);
    if (st != PRESTO_OK) return st;
    REQUIRE(new_rows >= 0 && new_rows < ((int64_t)1 << 31), "%s: new_rows outside 0..2^31", who);
    REQUIRE(max_new >= 0, "%s: max_new < 0", who);
    const int64_t row = (int64_t)d.hkv * d.head_dim;
    if (new_stride == 0) new_stride = row;
    REQUIRE(new_stride >= row && new_stride <= ((int64_t)1 << 31) &&
                new_stride % (d.dt == PRESTO_DT_BF16 ? 8 : 4) == 0,
            "%s: new_stride %lld", who, (long long)new_stride);
    REQUIRE((int64_t)d.batch * max_new < ((int64_t)1 << 24), "%s: batch * max_new is 2^24 or more", who);
    if (d.batch == 0 || max_new == 0 || new_rows == 0) return PRESTO_OK;
    REQUIRE(k_new && v_new && offsets && k_pages && v_pages && page_table && ctx && ctx_new, "%s: null pointer",
            who);
    REQUIRE(aligned16(k_new, v_new, k_pages, v_pages), "%s: K/V tensors must be 16-byte aligned", who);
    return launch_append_kv(&d, k_new, v_new, new_stride, new_rows, offsets, max_new, k_pages, v_pages, page_table,
                            ctx, ctx_new, flags, stream);
}

presto_status presto_pages_fork(const presto_pages_desc* desc, int32_t* refs, int32_t* page_table, int32_t* ctx,
                                const int32_t* parent, const int32_t* child, int32_t n, void* k_pages,
                                void* v_pages, int32_t* flags, void* ws, size_t ws_bytes, hipStream_t stream) {
    const char* who = "presto_pages_fork";
    presto_pages_desc d;
    presto_status st = check_books(desc, d, who);
    if (st != PRESTO_OK) return st;
    REQUIRE(n >= 0 && n <= d.batch, "%s: n=%d outside 0..batch", who, n);
    if (n == 0) return PRESTO_OK;
    REQUIRE(refs && page_table && ctx && parent && child && k_pages && v_pages, "%s: null pointer", who);
    REQUIRE(aligned16(k_pages, v_pages), "%s: K/V tensors must be 16-byte aligned", who);
    st = check_books_ws(d, who, ws, ws_bytes);
    if (st != PRESTO_OK) return st;
    return launch_pages_fork(&d, refs, page_table, ctx, parent, child, n, k_pages, v_pages, flags, ws, stream);
}

presto_status presto_pages_free(const presto_pages_desc* desc, int32_t* refs, int32_t* page_table, int32_t* ctx,
                                const int32_t* rows, int32_t n, int32_t* flags, hipStream_t stream) {
    const char* who = "presto_pages_free";
    presto_pages_desc d;
    presto_status st = check_books(desc, d, who);
    if (st != PRESTO_OK) return st;
    REQUIRE(n >= 0 && n <= d.batch, "%s: n=%d outside 0..batch", who, n);
    if (n == 0) return PRESTO_OK;
    REQUIRE(refs && page_table && ctx && rows, "%s: null pointer", who);
    return launch_pages_free(&d, refs, page_table, ctx, rows, n, flags, stream);
}

presto_status presto_pages_trim(const presto_pages_desc* desc, int32_t* refs, int32_t* page_table,
                                const int32_t* ctx, int32_t window, int32_t sinks, int32_t* flags,
                                hipStream_t stream) {
    const char* who = "presto_pages_trim";
    presto_pages_desc d;
    presto_status st = check_books(desc, d, who);
    if (st != PRESTO_OK) return st;
    REQUIRE(window >= 1 && window <= (1 << 30), "%s: window outside 1..2^30", who);
    REQUIRE(sinks >= 0 && sinks <= (1 << 30), "%s: sinks outside 0..2^30", who);
    if (d.batch == 0) return PRESTO_OK;
    REQUIRE(refs && page_table && ctx, "%s: null pointer", who);
    return launch_pages_trim(&d, refs, page_table, ctx, window, sinks, flags, stream);
}

presto_status presto_pages_compact(const presto_pages_desc* desc, const int32_t* refs, int32_t* refs_out,
                                   const int32_t* page_table, int32_t* table_out, int32_t* n_live,
                                   int32_t* page_map, void* k_pages, void* v_pages, int32_t* flags, void* ws,
                                   size_t ws_bytes, hipStream_t stream) {
    const char* who = "presto_pages_compact";
    presto_pages_desc d;
    presto_status st = check_books(desc, d, who);
    if (st != PRESTO_OK) return st;
    REQUIRE(refs && refs_out && n_live && k_pages && v_pages && (d.batch == 0 || (page_table && table_out)),
            "%s: null pointer", who);
    REQUIRE(aligned16(k_pages, v_pages), "%s: K/V tensors must be 16-byte aligned", who);
    st = check_books_ws(d, who, ws, ws_bytes);
    if (st != PRESTO_OK) return st;
    return launch_pages_compact(&d, refs, refs_out, page_table, table_out, n_live, page_map, k_pages, v_pages, flags,
                                ws, stream);
}

}  // extern "C"
