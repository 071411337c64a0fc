// The paged attention's launch plan, shared by the argument checks and the
// launcher.
#pragma once

#include <stddef.h>
#include <stdint.h>

#include "presto.h"

namespace presto_host {

struct PagedPlan {
    bool fits;         // false: more workgroups than a grid holds
    bool tiles;        // the kernel that shares tiles in LDS
    int order;         // of the row blocks
    int nb;            // (rows) 16-row blocks per workgroup
    int block_rows, row_blocks;
    int splits, split_tiles;
    int pieces, n_slots;  // (rows) pieces > 0: pieces of one length in the place of splits
    int64_t blocks, merge_blocks;
    int merge_parts;
    size_t o_bytes, ml_bytes, bytes;  // workspace
};

PagedPlan paged_plan(const presto_paged_attn_desc* d);
presto_status launch_paged_attn(const presto_paged_attn_desc* d, const PagedPlan& p, const void* q, const int32_t* q_off,
                                const void* kp, const void* vp, const int32_t* table, const int32_t* ctx, void* out,
                                int32_t* flags, void* ws, hipStream_t stream);

}  // namespace presto_host
