// Host side of the operators around a decoding step: rotary positions, the
// append that applies them, the 4-bit cache and its attention, sampling.
// Argument validation, workspace sizing and dispatch; nothing here touches the
// GPU before every check has passed.
#include <math.h>

#include "checks.hpp"
#include "common.hpp"
#include "step.hpp"

using namespace presto_host;

namespace {

bool value_type(presto_dtype dt) { return dt == PRESTO_DT_BF16 || dt == PRESTO_DT_F32; }
int64_t unit16(presto_dtype dt) { return dt == PRESTO_DT_BF16 ? 8 : 4; }  // elements of 16 bytes

// Whether `stride` (0: row) keeps rows of `row` elements apart and aligned.
bool row_stride(int64_t& stride, int64_t row, presto_dtype dt) {
    if (stride == 0) stride = row;
    return stride >= row && stride <= ((int64_t)1 << 31) && stride % unit16(dt) == 0;
}

presto_status check_rope(const presto_rope_desc* r, const uint64_t* steps, int32_t head_dim, const char* who) {
    REQUIRE(r->rot_dim >= 0 && r->rot_dim <= head_dim && r->rot_dim % 2 == 0,
            "%s: rot_dim=%d is not an even number up to the head's %d", who, r->rot_dim, head_dim);
    REQUIRE(r->interleaved == 0 || r->interleaved == 1, "%s: interleaved is 0 or 1", who);
    REQUIRE(isfinite(r->magnitude), "%s: magnitude must be finite", who);
    REQUIRE(r->rot_dim == 0 || steps, "%s: null steps", who);
    REQUIRE(((uintptr_t)steps & 7) == 0, "%s: steps must be 8-byte aligned", who);
    return PRESTO_OK;
}

// What the append and its way back have in common; fills in default strides.
presto_status check_append(const presto_append_desc* desc, presto_append_desc& d, const char* who) {
    set_error(PRESTO_OK, "%s", "");
    REQUIRE(desc, "%s: null descriptor", who);
    d = *desc;
    const presto_status st = check_pages(d.pages, who);
    if (st != PRESTO_OK) return st;
    REQUIRE(value_type(d.dt), "%s: unknown dtype %d", who, (int)d.dt);
    REQUIRE(d.pages.dt == d.dt || d.pages.dt == PRESTO_DT_FP4, "%s: rows and pool of different types", who);
    REQUIRE(d.new_rows >= 0 && d.new_rows < ((int64_t)1 << 31), "%s: new_rows outside 0..2^31", who);
    REQUIRE(d.max_new >= 0, "%s: max_new < 0", who);
    REQUIRE((int64_t)d.pages.batch * d.max_new < ((int64_t)1 << 24), "%s: batch * max_new is 2^24 or more", who);
    const int64_t row = (int64_t)d.pages.hkv * d.pages.head_dim;
    REQUIRE(row_stride(d.k_stride, row, d.dt), "%s: k_stride %lld", who, (long long)d.k_stride);
    REQUIRE(row_stride(d.v_stride, row, d.dt), "%s: v_stride %lld", who, (long long)d.v_stride);
    return PRESTO_OK;
}

}  // namespace

extern "C" {

presto_status presto_rope_steps(const presto_rope_freq_desc* d, const double* freq, uint64_t* steps) {
    const char* who = "presto_rope_steps";
    set_error(PRESTO_OK, "%s", "");
    REQUIRE(d && steps, "%s: null pointer", who);
    REQUIRE(d->rot_dim >= 2 && d->rot_dim <= 256 && d->rot_dim % 2 == 0, "%s: rot_dim=%d is not even in 2..256", who,
            d->rot_dim);
    const int n = d->rot_dim / 2;
    if (freq) {
        for (int i = 0; i < n; ++i)
            REQUIRE(isfinite(freq[i]) && fabs(freq[i]) < 0x1p20, "%s: frequency %d", who, i);
    } else {
        REQUIRE(isfinite(d->base) && d->base > 0, "%s: base must be positive", who);
        REQUIRE(isfinite(d->factor) && d->factor > 0, "%s: factor must be positive", who);
        REQUIRE(d->ramp >= PRESTO_ROPE_RAMP_NONE && d->ramp <= PRESTO_ROPE_RAMP_LOG, "%s: unknown ramp %d", who, d->ramp);
        if (d->ramp != PRESTO_ROPE_RAMP_NONE) {
            REQUIRE(isfinite(d->original) && d->original > 0, "%s: original must be positive", who);
            REQUIRE(isfinite(d->high) && d->low > 0 && d->low < d->high, "%s: the ramp needs 0 < low < high", who);
        }
    }
    const long double two_pi = 6.283185307179586476925286766559005768L;
    for (int i = 0; i < n; ++i) {
        double f;
        if (freq) {
            f = freq[i];
        } else {
            f = pow(d->base, -2.0 * i / d->rot_dim);
            if (d->ramp == PRESTO_ROPE_RAMP_NONE) {
                f /= d->factor;
            } else {
                const double r = d->original * f / (double)two_pi;
                double g = d->ramp == PRESTO_ROPE_RAMP_TURNS
                               ? (r - d->low) / (d->high - d->low)
                               : (log(r) - log(d->low)) / (log(d->high) - log(d->low));
                g = g > 0 ? (g < 1 ? g : 1) : 0;
                f *= g + (1 - g) / d->factor;
            }
            REQUIRE(isfinite(f) && f < 0x1p20, "%s: frequency %d is 2^20 or more", who, i);
        }
        long double turn = f / two_pi;
        turn -= floorl(turn);  // in 0 .. 1
        const long double at = roundl(turn * 0x1p64L);
        steps[i] = at >= 0x1p64L ? 0 : (uint64_t)at;
    }
    return PRESTO_OK;
}

presto_status presto_rope(const presto_rope_desc* rope, const uint64_t* steps, presto_dtype dt, const void* x,
                          int64_t x_stride, int64_t rows, int32_t heads, int32_t head_dim, const int32_t* positions,
                          void* out, int64_t out_stride, hipStream_t stream) {
    const char* who = "presto_rope";
    set_error(PRESTO_OK, "%s", "");
    REQUIRE(rope, "%s: null descriptor", who);
    REQUIRE(value_type(dt), "%s: unknown dtype %d", who, (int)dt);
    REQUIRE(rows >= 0 && rows < ((int64_t)1 << 31), "%s: rows outside 0..2^31", who);
    REQUIRE(heads >= 1 && heads <= 65536, "%s: heads=%d outside 1..65536", who, heads);
    REQUIRE(head_dim >= 8 && head_dim <= 256 && head_dim % 8 == 0, "%s: head_dim=%d is not a multiple of 8 in 8..256",
            who, head_dim);
    REQUIRE(row_stride(x_stride, (int64_t)heads * head_dim, dt), "%s: x_stride %lld", who, (long long)x_stride);
    REQUIRE(row_stride(out_stride, (int64_t)heads * head_dim, dt), "%s: out_stride %lld", who, (long long)out_stride);
    REQUIRE(x != out || rows < 2 || x_stride == out_stride, "%s: in place, with another stride", who);
    const presto_status st = check_rope(rope, rows == 0 ? reinterpret_cast<const uint64_t*>(8) : steps, head_dim, who);
    if (st != PRESTO_OK) return st;
    if (rows == 0) return PRESTO_OK;
    REQUIRE(x && positions && out, "%s: null pointer", who);
    REQUIRE(aligned16(x, out), "%s: tensors must be 16-byte aligned", who);
    return launch_rope(rope, steps, dt, x, x_stride, rows, heads, head_dim, positions, out, out_stride, stream);
}

presto_status presto_append_rope(const presto_append_desc* desc, const presto_rope_desc* rope, const uint64_t* steps,
                                 const void* q, const void* k_new, const void* v_new, const int32_t* offsets,
                                 void* q_out, void* k_pages, void* v_pages, const int32_t* page_table,
                                 const int32_t* ctx, const int32_t* ctx_new, int32_t* flags, hipStream_t stream) {
    const char* who = "presto_append_rope";
    presto_append_desc d;
    presto_status st = check_append(desc, d, who);
    if (st != PRESTO_OK) return st;
    const bool nothing = d.pages.batch == 0 || d.max_new == 0 || d.new_rows == 0;
    const presto_rope_desc none = {0, 0, 1.f};
    if (!rope) rope = &none;
    st = check_rope(rope, nothing ? reinterpret_cast<const uint64_t*>(8) : steps, d.pages.head_dim, who);
    if (st != PRESTO_OK) return st;
    if (q) {
        const int64_t row = (int64_t)d.hq * d.pages.head_dim;
        REQUIRE(d.hq >= 0 && d.hq <= 65536, "%s: hq=%d outside 0..65536", who, d.hq);
        REQUIRE(row_stride(d.q_stride, row, d.dt), "%s: q_stride %lld", who, (long long)d.q_stride);
        REQUIRE(row_stride(d.q_out_stride, row, d.dt), "%s: q_out_stride %lld", who, (long long)d.q_out_stride);
        REQUIRE(q != q_out || d.new_rows < 2 || d.q_stride == d.q_out_stride, "%s: in place, with another stride", who);
    }
    if (nothing) return PRESTO_OK;
    REQUIRE(k_new && v_new && offsets && k_pages && v_pages && page_table && ctx && ctx_new && (!q || q_out),
            "%s: null pointer", who);
    REQUIRE(aligned16(k_new, v_new, k_pages, v_pages) && (!q || aligned16(q, q_out)),
            "%s: tensors must be 16-byte aligned", who);
    return launch_append_rope(&d, rope, steps, q, k_new, v_new, offsets, q_out, k_pages, v_pages, page_table, ctx,
                              ctx_new, flags, stream);
}

presto_status presto_read_kv(const presto_append_desc* desc, const void* k_pages, const void* v_pages,
                             const int32_t* page_table, const int32_t* ctx, const int32_t* ctx_new,
                             const int32_t* offsets, void* k_out, void* v_out, int32_t* flags, hipStream_t stream) {
    const char* who = "presto_read_kv";
    presto_append_desc d;
    const presto_status st = check_append(desc, d, who);
    if (st != PRESTO_OK) return st;
    if (d.pages.batch == 0 || d.max_new == 0 || d.new_rows == 0 || (!k_out && !v_out)) return PRESTO_OK;
    REQUIRE(offsets && k_pages && v_pages && page_table && ctx && ctx_new, "%s: null pointer", who);
    REQUIRE(aligned16(k_out, v_out, k_pages, v_pages), "%s: tensors must be 16-byte aligned", who);
    return launch_read_kv(&d, k_pages, v_pages, page_table, ctx, ctx_new, offsets, k_out, v_out, flags, stream);
}

// Checks a call, fills in its default strides and plans it.
static presto_status check_quant_attn(presto_paged_attn_desc& d, presto_dtype dt, QuantPlan& plan, bool decode,
                                      const char* who) {
    REQUIRE(value_type(dt), "%s: unknown dtype %d", who, (int)dt);
    const presto_status st = check_pages(d.pages, who);
    if (st != PRESTO_OK) return st;
    REQUIRE(d.pages.dt == PRESTO_DT_FP4, "%s: not a 4-bit pool", who);
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
    REQUIRE(row_stride(d.q_stride, (int64_t)d.hq * d.pages.head_dim, dt), "%s: q_stride %lld", who,
            (long long)d.q_stride);
    if (d.pages.batch > 0 && d.max_q > 0) {
        plan = quant_plan(&d, dt);
        if (!plan.fits) return set_error(PRESTO_ERR_UNSUPPORTED, "%s: too many query rows for one call", who);
    }
    return PRESTO_OK;
}

size_t presto_quant_attention_workspace(const presto_paged_attn_desc* desc, presto_dtype dt, int32_t ragged) {
    if (!desc) return 0;
    presto_paged_attn_desc d = *desc;
    QuantPlan plan{};
    return check_quant_attn(d, dt, plan, !ragged, "workspace") == PRESTO_OK ? plan.bytes : 0;
}

presto_status presto_quant_attention(const presto_paged_attn_desc* desc, presto_dtype dt, const void* q,
                                     const int32_t* q_offsets, const void* k_pages, const void* v_pages,
                                     const int32_t* page_table, const int32_t* ctx, void* out, int32_t* flags, void* ws,
                                     size_t ws_bytes, hipStream_t stream) {
    const char* who = "presto_quant_attention";
    set_error(PRESTO_OK, "%s", "");
    REQUIRE(desc, "%s: null descriptor", who);
    presto_paged_attn_desc d = *desc;
    QuantPlan plan{};
    presto_status st = check_quant_attn(d, dt, plan, !q_offsets, who);
    if (st != PRESTO_OK) return st;
    if (d.pages.batch == 0 || d.max_q == 0 || d.total_q == 0) return PRESTO_OK;
    REQUIRE(q && k_pages && v_pages && page_table && ctx && out, "%s: null pointer", who);
    REQUIRE(aligned16(q, k_pages, v_pages, out), "%s: tensors must be 16-byte aligned", who);
    st = check_ws(ws, ws_bytes, plan.bytes);
    if (st != PRESTO_OK) return st;
    REQUIRE(aligned16(ws, nullptr), "%s: the workspace must be 16-byte aligned", who);
    return launch_quant_attn(&d, dt, plan, q, q_offsets, k_pages, v_pages, page_table, ctx, out, flags, ws, stream);
}

static presto_status check_sample(presto_dtype dt, int64_t rows, int32_t vocab, const char* who) {
    REQUIRE(value_type(dt), "%s: unknown dtype %d", who, (int)dt);
    REQUIRE(rows >= 0 && rows <= (1 << 21), "%s: rows outside 0..2^21", who);
    REQUIRE(vocab >= 1 && vocab <= (1 << 20), "%s: vocab=%d outside 1..2^20", who, vocab);
    return PRESTO_OK;
}

size_t presto_sample_workspace(presto_dtype dt, int64_t rows, int32_t vocab) {
    if (check_sample(dt, rows, vocab, "presto_sample_workspace") != PRESTO_OK) return 0;
    return sample_plan(dt, rows, vocab).bytes;
}

presto_status presto_sample(presto_dtype dt, const void* logits, int64_t rows, int32_t vocab, int64_t row_stride,
                            const float* u, const float* temperature, const int32_t* top_k, const float* top_p,
                            const float* min_p, int32_t* token, float* logprob, int32_t* flags, void* ws,
                            size_t ws_bytes, hipStream_t stream) {
    const char* who = "presto_sample";
    set_error(PRESTO_OK, "%s", "");
    presto_status st = check_sample(dt, rows, vocab, who);
    if (st != PRESTO_OK) return st;
    REQUIRE(row_stride >= vocab && row_stride <= ((int64_t)1 << 40), "%s: row_stride=%lld below vocab", who,
            (long long)row_stride);
    if (rows == 0) return PRESTO_OK;
    REQUIRE(logits && u && token, "%s: null pointer", who);
    REQUIRE(((uintptr_t)logits & (dt == PRESTO_DT_BF16 ? 1 : 3)) == 0, "%s: misaligned logits", who);
    st = check_ws(ws, ws_bytes, sample_plan(dt, rows, vocab).bytes);
    if (st != PRESTO_OK) return st;
    REQUIRE(aligned16(ws, nullptr), "%s: the workspace must be 16-byte aligned", who);
    return launch_sample(dt, logits, rows, vocab, row_stride, u, temperature, top_k, top_p, min_p, token, logprob,
                         flags, ws, stream);
}

}  // extern "C"
