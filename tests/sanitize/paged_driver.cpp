// Sanitizer driver for the host side of the paged cache: built like
// api_driver.cpp (host code under AddressSanitizer and
// UndefinedBehaviorSanitizer, nothing launched), it calls the paged entry
// points with arguments that the host rejects or that launch nothing, and asks
// for workspaces over the whole range of shapes, which runs every plan.
#include <stdint.h>
#include <stdio.h>
#include <string.h>

#include "presto.h"

static int failures = 0;

static void expect(presto_status got, presto_status want, const char* what) {
    const char* msg = presto_last_error();
    if (got != want || strlen(msg) >= 512) {
        fprintf(stderr, "%s: status %d, expected %d (%s)\n", what, (int)got, (int)want, msg);
        ++failures;
    }
}

int main() {
    void* fake = reinterpret_cast<void*>(0x1000);  // never dereferenced: the checks fail first
    int32_t* fi = static_cast<int32_t*>(fake);
    const size_t room = (size_t)1 << 60;
    const presto_pages_desc p = {4, 64, 300, 16, 8, 128, PRESTO_DT_BF16, 2, 0, 0};

    presto_pages_desc bad[18];
    for (auto& b : bad) b = p;
    bad[0].page_size = 24; bad[1].page_size = INT32_MIN; bad[2].head_dim = 96; bad[3].hkv = INT32_MAX;
    bad[4].num_pages = 0; bad[5].num_pages = INT32_MIN; bad[6].max_pages = INT32_MAX; bad[7].layers = INT32_MIN;
    bad[8].dt = (presto_dtype)9; bad[9].batch = INT32_MAX; bad[10].page_stride = INT64_MAX;
    bad[11].page_stride = INT64_MIN; bad[12].layer_stride = INT64_MAX; bad[13].layer_stride = INT64_MIN;
    bad[14].batch = -1; bad[15].max_pages = 0; bad[16].page_stride = 4; bad[17].hkv = -1;
    for (auto& b : bad) {
        const presto_status e = PRESTO_ERR_INVALID_ARG;
        const presto_paged_attn_desc a = {b, 32, 8, 900, 0, 0, 0.1f, 32, 0, 0};
        expect(presto_paged_attention(&a, fake, fake, fake, fi, fi, fake, 0, fake, room, 0), e, "decode pool");
        expect(presto_window_attention(&a, fake, fi, fake, fake, fi, fi, fake, 0, fake, room, 0), e, "window pool");
        expect(presto_pages_reserve(&b, fi, fi, fi, fi, 1, fi, 0, fake, room, 0), e, "reserve pool");
        expect(presto_append_kv(&b, fake, fake, 4, 0, fi, 4, fake, fake, fi, fi, fi, 0, 0), e, "append pool");
        expect(presto_pages_fork(&b, fi, fi, fi, fi, fi, 1, fake, fake, 0, fake, room, 0), e, "fork pool");
        expect(presto_pages_free(&b, fi, fi, fi, fi, 1, 0, 0), e, "free pool");
        expect(presto_pages_trim(&b, fi, fi, fi, 1, 0, 0, 0), e, "trim pool");
        expect(presto_pages_compact(&b, fi, fi, fi, fi, fi, 0, fake, fake, 0, fake, room, 0), e, "compact pool");
        if (presto_pages_workspace(&b) || presto_paged_attention_workspace(&a) || presto_window_attention_workspace(&a)) {
            fprintf(stderr, "workspace of a bad pool\n");
            ++failures;
        }
    }
    expect(presto_paged_attention(nullptr, fake, fake, fake, fi, fi, fake, 0, fake, room, 0), PRESTO_ERR_INVALID_ARG,
           "null descriptor");
    expect(presto_pages_free(nullptr, fi, fi, fi, fi, 1, 0, 0), PRESTO_ERR_INVALID_ARG, "null descriptor");
    if (presto_pages_workspace(nullptr) || presto_paged_attention_workspace(nullptr)) ++failures;

    // every plan: the smallest, odd and largest shapes
    const int32_t batches[] = {1, 2, 7, 64, 65, 300, 2048, 2049, 70000, (1 << 23) - 1};
    const int32_t lens[] = {0, 1, 33, 384, 4097, 131073, 1 << 20, (1 << 30) - 1024};
    const int32_t news[] = {1, 2, 9, 64, 1000, 65536, (1 << 26)};
    const int32_t windows[] = {0, 1, 500, 1 << 30};
    for (int32_t batch : batches)
        for (int32_t len : lens)
            for (int32_t n : news)
                for (int32_t w : windows)
                    for (int32_t hkv : {1, 8, 4096})
                        for (int32_t g : {1, 5, 17, 64}) {
                            presto_pages_desc q = p;
                            q.batch = batch;
                            q.hkv = hkv;
                            q.page_size = 1024;
                            q.max_pages = (1 << 20) - 1;
                            while ((int64_t)q.max_pages * batch >= ((int64_t)1 << 31)) q.max_pages /= 2;
                            if (q.max_pages < 1) q.max_pages = 1;
                            q.dt = n % 2 ? PRESTO_DT_F32 : PRESTO_DT_BF16;
                            q.head_dim = g % 2 ? 64 : 128;
                            presto_paged_attn_desc a = {q, hkv * g, n, len, w, w ? 4 : 0, 0.1f, 0, 0, len};
                            if (len > (int64_t)q.max_pages * q.page_size) continue;
                            a.total_q = (int64_t)batch * n < ((int64_t)1 << 30) ? (int64_t)batch * n : (1 << 30) - 1;
                            if (w == 1) a.sinks = 1 << 30;
                            presto_paged_attention_workspace(&a);
                            presto_window_attention_workspace(&a);
                            presto_pages_workspace(&q);
                        }

    // nothing to do, small workspaces, grids too large
    presto_paged_attn_desc a = {p, 32, 8, 900, 0, 0, 0.1f, 32, 0, 0};
    a.pages.batch = 0;
    expect(presto_paged_attention(&a, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0), PRESTO_OK, "batch 0");
    a.pages = p;
    a.max_q = 0;
    expect(presto_window_attention(&a, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0), PRESTO_OK, "max_q 0");
    a.max_q = 1;
    a.pages.batch = 1;
    a.pages.max_pages = 60000;
    a.max_ctx = 900000;
    expect(presto_window_attention(&a, fake, fi, fake, fake, fi, fi, fake, 0, fake, 16, 0), PRESTO_ERR_WORKSPACE,
           "small workspace");
    expect(presto_pages_reserve(&p, fi, fi, fi, fi, 1, fi, 0, fake, 16, 0), PRESTO_ERR_WORKSPACE, "small workspace");
    expect(presto_pages_reserve(&p, fi, fi, fi, fi, INT32_MIN, fi, 0, fake, room, 0), PRESTO_ERR_INVALID_ARG, "extra");
    expect(presto_append_kv(&p, fake, fake, INT64_MAX, INT64_MAX, fi, INT32_MAX, fake, fake, fi, fi, fi, 0, 0),
           PRESTO_ERR_INVALID_ARG, "append rows");
    expect(presto_append_kv(&p, fake, fake, 4, 0, fi, INT32_MAX, fake, fake, fi, fi, fi, 0, 0), PRESTO_ERR_INVALID_ARG,
           "append grid");

    if (failures) {
        fprintf(stderr, "%d failure(s)\n", failures);
        return 1;
    }
    printf("paged driver: ok\n");
    return 0;
}
