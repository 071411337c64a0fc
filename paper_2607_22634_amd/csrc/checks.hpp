// Argument checks that the entry points of the paged caches share.
#pragma once

#include <stddef.h>
#include <stdint.h>

#include "common.hpp"

#define REQUIRE(cond, ...)                                        \
    do {                                                          \
        if (!(cond)) return set_error(PRESTO_ERR_INVALID_ARG, __VA_ARGS__); \
    } while (0)

namespace presto_host {

inline presto_status check_ws(void* ws, size_t have, size_t need) {
    if (need > 0 && (ws == nullptr || have < need))
        return set_error(PRESTO_ERR_WORKSPACE, "workspace of %zu bytes needed, %zu given", need,
                         ws ? have : (size_t)0);
    return PRESTO_OK;
}

// Checks a pool and fills in its default strides.
inline presto_status check_pages(presto_pages_desc& p, const char* who) {
    REQUIRE(p.dt == PRESTO_DT_BF16 || p.dt == PRESTO_DT_F32 || p.dt == PRESTO_DT_FP4, "%s: unknown dtype %d", who,
            (int)p.dt);
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
    const bool fp4 = p.dt == PRESTO_DT_FP4;  // (whose strides are bytes)
    const int64_t page = (int64_t)p.page_size * p.hkv * p.head_dim * (fp4 ? 17 : 32) / 32;
    const int64_t unit = fp4 ? 16 : p.dt == PRESTO_DT_BF16 ? 8 : 4;
    if (p.page_stride == 0) p.page_stride = page;
    REQUIRE(p.page_stride >= page && p.page_stride % unit == 0 &&
                p.page_stride <= ((int64_t)1 << 60) / p.num_pages,
            "%s: page_stride %lld", who, (long long)p.page_stride);
    if (p.layer_stride == 0) p.layer_stride = p.page_stride * p.num_pages;
    REQUIRE(p.layer_stride > 0 && p.layer_stride % unit == 0 && p.layer_stride <= ((int64_t)1 << 60) / p.layers,
            "%s: layer_stride %lld", who, (long long)p.layer_stride);
    return PRESTO_OK;
}

inline bool aligned16(const void* a, const void* b, const void* c = nullptr, const void* d = nullptr) {
    return (((uintptr_t)a | (uintptr_t)b | (uintptr_t)c | (uintptr_t)d) & 15) == 0;
}

}  // namespace presto_host
