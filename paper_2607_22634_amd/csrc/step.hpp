// Launchers of the operators around a decoding step.
#pragma once

#include <stddef.h>
#include <stdint.h>

#include "presto.h"

namespace presto_host {

presto_status launch_rope(const presto_rope_desc* r, const uint64_t* steps, presto_dtype dt, const void* x,
                          int64_t x_stride, int64_t rows, int32_t heads, int32_t dim, const int32_t* positions,
                          void* out, int64_t out_stride, hipStream_t stream);
presto_status launch_append_rope(const presto_append_desc* d, const presto_rope_desc* r, const uint64_t* steps,
                                 const void* q, const void* k_new, const void* v_new, const int32_t* offsets,
                                 void* q_out, void* k_pages, void* v_pages, const int32_t* table, const int32_t* ctx,
                                 const int32_t* ctx_new, int32_t* flags, hipStream_t stream);
presto_status launch_read_kv(const presto_append_desc* d, const void* k_pages, const void* v_pages,
                             const int32_t* table, const int32_t* ctx, const int32_t* ctx_new, const int32_t* offsets,
                             void* k_out, void* v_out, int32_t* flags, hipStream_t stream);

struct QuantPlan {
    bool fits;  // false: more workgroups than a grid holds
    bool own;   // waves have rows of their own, and do not share the tiles of the same ones
    int r;      // 16-row blocks of a wave
    int64_t row_blocks, splits, split_tiles, blocks, merge_blocks;
    size_t o_bytes, bytes;  // workspace
};
QuantPlan quant_plan(const presto_paged_attn_desc* d, presto_dtype dt);
presto_status launch_quant_attn(const presto_paged_attn_desc* d, presto_dtype dt, const QuantPlan& p, const void* q,
                                const int32_t* q_off, const void* k, const void* v, const int32_t* table,
                                const int32_t* ctx, void* out, int32_t* flags, void* ws, hipStream_t stream);

struct SamplePlan {
    int64_t rows;  // of a round
    int slices, slice;  // of a row, and their length
    size_t bytes;  // workspace
};
SamplePlan sample_plan(presto_dtype dt, int64_t rows, int32_t vocab);
presto_status launch_sample(presto_dtype dt, const void* logits, int64_t rows, int32_t vocab, int64_t row_stride,
                            const float* u, const float* temperature, const int32_t* top_k, const float* top_p,
                            const float* min_p, int32_t* token, float* logprob, int32_t* flags, void* ws,
                            hipStream_t stream);

}  // namespace presto_host
