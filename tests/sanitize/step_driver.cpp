// Sanitizer driver for the host side of the operators around a decoding step
// (rotary positions, append, 4-bit cache, its attention, sampling): built like
// paged_driver.cpp, nothing is launched.  Arguments that the host rejects or
// that launch nothing, and workspaces over the whole range of shapes, which runs
// every plan.
#include <math.h>
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
    float* ff = static_cast<float*>(fake);
    const uint64_t* fs = static_cast<const uint64_t*>(fake);
    const size_t room = (size_t)1 << 60;
    const presto_status bad_arg = PRESTO_ERR_INVALID_ARG;

    // ---- frequencies
    uint64_t steps[128];
    double freq[128];
    for (int i = 0; i < 128; ++i) freq[i] = i % 2 ? -0x1.fffffp19 + i : 1e-300 * i;
    for (int32_t rot = 2; rot <= 256; rot += 2)
        for (int32_t ramp = 0; ramp <= 2; ++ramp)
            for (double base : {1e-30, 0.5, 10000.0, 1e300})
                for (double factor : {1e-300, 1.0, 40.0, 1e300}) {
                    const presto_rope_freq_desc d = {rot, ramp, base, factor, factor > 1 ? 1e300 : 4096.0, 1e-300, 1e308};
                    const presto_status st = presto_rope_steps(&d, nullptr, steps);
                    if (st != PRESTO_OK && st != bad_arg) ++failures;
                    expect(presto_rope_steps(&d, freq, steps), PRESTO_OK, "frequencies one by one");
                }
    const presto_rope_freq_desc fine = {64, PRESTO_ROPE_RAMP_TURNS, 10000.0, 4.0, 4096.0, 1.0, 32.0};
    presto_rope_freq_desc odd[12];
    for (auto& d : odd) d = fine;
    odd[0].rot_dim = 0; odd[1].rot_dim = 3; odd[2].rot_dim = INT32_MAX; odd[3].rot_dim = INT32_MIN; odd[4].base = NAN;
    odd[5].base = 0; odd[6].factor = -1; odd[7].ramp = 3; odd[8].ramp = INT32_MIN; odd[9].original = INFINITY;
    odd[10].low = 32; odd[11].high = NAN;
    for (auto& d : odd) expect(presto_rope_steps(&d, nullptr, steps), bad_arg, "frequencies");
    expect(presto_rope_steps(nullptr, nullptr, steps), bad_arg, "null descriptor");
    expect(presto_rope_steps(&fine, nullptr, nullptr), bad_arg, "null steps");
    freq[7] = NAN;
    expect(presto_rope_steps(&fine, freq, steps), bad_arg, "frequency");

    // ---- rotation
    const presto_rope_desc rope = {128, 0, 1.f};
    const presto_dtype bf = PRESTO_DT_BF16;
    struct { presto_rope_desc r; int64_t xs, rows; int32_t heads, dim; int64_t os; } r[] = {
        {{130, 0, 1.f}, 0, 4, 8, 128, 0},   {{-2, 0, 1.f}, 0, 4, 8, 128, 0},    {{128, 2, 1.f}, 0, 4, 8, 128, 0},
        {{128, 0, NAN}, 0, 4, 8, 128, 0},   {rope, 0, -1, 8, 128, 0},           {rope, 0, INT64_MAX, 8, 128, 0},
        {rope, 0, 4, 0, 128, 0},            {rope, 0, 4, INT32_MAX, 128, 0},    {rope, 0, 4, 8, 260, 0},
        {rope, 0, 4, 8, INT32_MIN, 0},      {rope, INT64_MAX, 4, 8, 128, 0},    {rope, INT64_MIN, 4, 8, 128, 0},
        {rope, 0, 4, 8, 128, INT64_MIN},    {rope, 0, 4, 8, 128, 1025},         {rope, 1016, 4, 8, 128, 0}};
    for (auto& c : r)
        expect(presto_rope(&c.r, fs, bf, fake, c.xs, c.rows, c.heads, c.dim, fi, fake, c.os, 0), bad_arg, "rope");
    expect(presto_rope(nullptr, fs, bf, fake, 0, 4, 8, 128, fi, fake, 0, 0), bad_arg, "rope descriptor");
    expect(presto_rope(&rope, fs, PRESTO_DT_FP4, fake, 0, 4, 8, 128, fi, fake, 0, 0), bad_arg, "rope type");
    expect(presto_rope(&rope, nullptr, bf, nullptr, 0, 0, 8, 128, nullptr, nullptr, 0, 0), PRESTO_OK, "rope, no rows");

    // ---- pools
    const presto_pages_desc p = {4, 64, 300, 16, 8, 128, PRESTO_DT_FP4, 1, 0, 0};
    presto_pages_desc bad[16];
    for (auto& b : bad) b = p;
    bad[0].page_size = 24; bad[1].page_size = INT32_MIN; bad[2].head_dim = 96; bad[3].hkv = INT32_MAX;
    bad[4].num_pages = 0; bad[5].num_pages = INT32_MIN; bad[6].max_pages = INT32_MAX; bad[7].layers = INT32_MIN;
    bad[8].dt = (presto_dtype)9; bad[9].batch = INT32_MAX; bad[10].page_stride = INT64_MAX;
    bad[11].page_stride = INT64_MIN; bad[12].batch = -1; bad[13].max_pages = 0; bad[14].page_stride = 4; bad[15].hkv = -1;
    for (auto& b : bad) {
        const presto_append_desc d = {b, bf, 32, 8, 16, 0, 0, 0, 0};
        expect(presto_append_rope(&d, &rope, fs, fake, fake, fake, fi, fake, fake, fake, fi, fi, fi, 0, 0), bad_arg,
               "append pool");
        expect(presto_read_kv(&d, fake, fake, fi, fi, fi, fi, fake, fake, 0, 0), bad_arg, "read pool");
        const presto_paged_attn_desc a = {b, 32, 8, 900, 0, 0, 0.1f, 32, 0, 0};
        expect(presto_quant_attention(&a, bf, fake, fi, fake, fake, fi, fi, fake, 0, fake, room, 0), bad_arg, "pool");
        if (presto_quant_attention_workspace(&a, bf, 1)) ++failures;
    }
    const presto_append_desc d0 = {p, bf, 32, 8, 16, 0, 0, 0, 0};
    presto_append_desc ds[12];
    for (auto& d : ds) d = d0;
    ds[0].dt = PRESTO_DT_FP4; ds[1].dt = (presto_dtype)3; ds[2].new_rows = -1; ds[3].new_rows = INT64_MAX;
    ds[4].max_new = INT32_MAX; ds[5].max_new = INT32_MIN; ds[6].k_stride = INT64_MIN; ds[7].v_stride = INT64_MAX;
    ds[8].q_stride = 8; ds[9].q_out_stride = INT64_MIN; ds[10].hq = INT32_MAX; ds[11].hq = -1;
    for (auto& d : ds)
        expect(presto_append_rope(&d, &rope, fs, fake, fake, fake, fi, fake, fake, fake, fi, fi, fi, 0, 0), bad_arg,
               "append");
    expect(presto_append_rope(nullptr, &rope, fs, fake, fake, fake, fi, fake, fake, fake, fi, fi, fi, 0, 0), bad_arg,
           "append descriptor");
    expect(presto_read_kv(nullptr, fake, fake, fi, fi, fi, fi, fake, fake, 0, 0), bad_arg, "read descriptor");
    presto_append_desc none = d0;
    none.max_new = 0;
    expect(presto_append_rope(&none, nullptr, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0), PRESTO_OK, "append of nothing");
    expect(presto_read_kv(&none, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0), PRESTO_OK, "read of nothing");

    // ---- attention: every plan, the smallest, odd and largest shapes
    presto_paged_attn_desc a = {p, 32, 8, 900, 0, 0, 0.1f, 32, 0, 0};
    for (int32_t batch : {1, 2, 7, 64, 65, 300, 2048, 70000, (1 << 23) - 1, INT32_MAX})
        for (int32_t len : {0, 1, 33, 384, 4097, 131073, 1 << 20, (1 << 30) - 1024})
            for (int32_t n : {0, 1, 2, 9, 64, 1000, 65536, 1 << 26, (1 << 30) - 1})
                for (int32_t w : {0, 1, 500, 1 << 30})
                    for (int32_t hkv : {1, 8, 4096})
                        for (int32_t g : {1, 5, 17, 64})
                            for (int64_t total : {(int64_t)0, (int64_t)1, (int64_t)len, INT64_MAX}) {
                                presto_paged_attn_desc x = a;
                                x.pages.batch = batch;
                                x.pages.hkv = hkv;
                                x.pages.page_size = 1024;
                                x.pages.max_pages = (1 << 20) - 1;
                                while ((int64_t)x.pages.max_pages * batch >= ((int64_t)1 << 31)) x.pages.max_pages /= 2;
                                if (x.pages.max_pages < 1) x.pages.max_pages = 1;
                                x.pages.head_dim = g % 2 ? 64 : 128;
                                x.hq = hkv * g;
                                x.max_q = n;
                                x.max_ctx = len;
                                x.window = w;
                                x.sinks = w == 1 ? 1 << 30 : w ? 4 : 0;
                                x.total_q = (int64_t)batch * n < ((int64_t)1 << 30) ? (int64_t)batch * n : (1 << 30) - 1;
                                x.total_ctx = total;
                                for (int ragged : {0, 1})
                                    for (presto_dtype dt : {PRESTO_DT_BF16, PRESTO_DT_F32})
                                        presto_quant_attention_workspace(&x, dt, ragged);
                            }
    presto_paged_attn_desc as[13];
    for (auto& x : as) x = a;
    as[0].hq = 12; as[1].hq = INT32_MIN; as[2].max_ctx = 1025; as[3].max_ctx = -1; as[4].total_ctx = -1;
    as[5].total_q = INT64_MAX; as[6].max_q = INT32_MAX; as[7].window = -1; as[8].sinks = INT32_MAX; as[9].scale = NAN;
    as[10].scale = 0.f; as[11].q_stride = INT64_MIN; as[12].pages.dt = PRESTO_DT_BF16;
    for (auto& x : as)
        expect(presto_quant_attention(&x, bf, fake, fi, fake, fake, fi, fi, fake, 0, fake, room, 0), bad_arg, "attention");
    expect(presto_quant_attention(&a, PRESTO_DT_FP4, fake, fi, fake, fake, fi, fi, fake, 0, fake, room, 0), bad_arg, "type");
    expect(presto_quant_attention(nullptr, bf, fake, fi, fake, fake, fi, fi, fake, 0, fake, room, 0), bad_arg,
           "attention descriptor");
    a.pages.max_pages = 60000;
    a.max_ctx = 900000;
    expect(presto_quant_attention(&a, bf, fake, fi, fake, fake, fi, fi, fake, 0, fake, 16, 0), PRESTO_ERR_WORKSPACE,
           "small workspace");
    a.max_q = 0;
    expect(presto_quant_attention(&a, bf, 0, fi, 0, 0, 0, 0, 0, 0, 0, 0, 0), PRESTO_OK, "max_q 0");
    if (presto_quant_attention_workspace(nullptr, bf, 0)) ++failures;

    // ---- sampling
    for (int64_t rows : {(int64_t)0, (int64_t)1, (int64_t)63, (int64_t)2048, (int64_t)2049, (int64_t)1 << 21})
        for (int32_t vocab : {1, 2, 1024, 1025, 4095, 32768, 32769, 151936, (1 << 20) - 1, 1 << 20})
            for (presto_dtype dt : {PRESTO_DT_BF16, PRESTO_DT_F32}) {
                const size_t need = presto_sample_workspace(dt, rows, vocab);
                if ((need == 0) != (rows == 0 || vocab <= 1024) || need % 16) ++failures;
            }
    struct { int64_t rows; int32_t vocab; int64_t stride; } s[] = {
        {-1, 100, 100}, {(1 << 21) + 1, 100, 100}, {INT64_MAX, 100, 100}, {4, 0, 100}, {4, INT32_MIN, 100},
        {4, (1 << 20) + 1, INT64_MAX}, {4, 100, 99}, {4, 100, INT64_MAX}, {4, 100, INT64_MIN}};
    for (auto& c : s) {
        expect(presto_sample(bf, fake, c.rows, c.vocab, c.stride, ff, 0, 0, 0, 0, fi, 0, 0, fake, room, 0), bad_arg,
               "sample");
    }
    expect(presto_sample(PRESTO_DT_FP4, fake, 4, 100, 100, ff, 0, 0, 0, 0, fi, 0, 0, fake, room, 0), bad_arg, "type");
    expect(presto_sample(bf, fake, 4, 5000, 5000, ff, 0, 0, 0, 0, fi, 0, 0, fake, 16, 0), PRESTO_ERR_WORKSPACE,
           "small workspace");
    expect(presto_sample(bf, 0, 0, 100, 100, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0), PRESTO_OK, "no rows");

    if (failures) {
        fprintf(stderr, "%d failure(s)\n", failures);
        return 1;
    }
    printf("step driver: ok\n");
    return 0;
}
