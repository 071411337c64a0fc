// Attention over a paged KV cache: one new token per sequence (decoding) or a
// ragged batch of new tokens (prompts, chunks, drafted chains), causal, with
// an optional sliding window and sinks.
//
//   O[i, h] = sum_j e^{s_j - m} v_j / sum_j e^{s_j - m},  s_j = scale q[i, h] . k_j
//
// over the keys j that the query at position p = ctx - n + i sees: j <= p and,
// with a window, j > p - window or j < sinks.  Position j of sequence b is row
// j mod page of page table[b, j / page].
//
// Rows are packed per KV head: row rho = i * G + (h - g * G), so that the G
// query heads of a KV head share every key that is read.  The keys that the
// rows of a workgroup see are a list of tiles: those that hold sinks, then
// those from the window's start to the last row's position; what lies between
// is never touched, so its pages may have been given back.
#include <math.h>

#include <type_traits>

#include "common.hpp"

namespace presto {
namespace paged {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float floatx2 __attribute__((ext_vector_type(2)));
typedef float floatx4 __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.4426950408889634f;

// Two fp32 -> two bf16 (round to nearest even) in one instruction.
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((floatx2){lo, hi}, bf16x2));
}

__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

// Maximum and sum over the four lanes l, l ^ 16, l ^ 32, l ^ 48.
__device__ __forceinline__ float quad_max(float v) {
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float quad_sum(float v) {
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

struct Args {
    const char* q;
    const char* kp;
    const char* vp;
    const int32_t* table;
    const int32_t* ctx;
    const int32_t* q_off;  // null: one row per sequence
    char* out;
    float* part_o;    // [b, g, split, rho, D] fp32, normalised by the split's own sum
    float2* part_ml;  // [b, g, rho, split] (reference in log2 units, sum)
    int32_t* flags;
    int64_t q_stride, page_stride;  // elements
    int64_t total_q;
    int32_t batch, hq, hkv, G, max_q, max_ctx, num_pages, max_pages, page_shift;
    int32_t window, sinks;
    int32_t row_blocks, splits, split_tiles;
    float scale_log2;  // scale * log2(e)
};

// Sequence b: its new tokens are rows r0 .. r0 + n - 1 of q at positions
// pos0 ...  Lengths and offsets outside their ranges are cut to them.
struct Seq {
    int64_t r0;
    int n, pos0;
    bool bad;
};
__device__ __forceinline__ Seq seq_of(const Args& a, int b) {
    const int c = a.ctx[b], ctx = min(max(c, 0), a.max_ctx);
    if (a.q_off == nullptr) return {b, 1, ctx - 1, c != ctx};
    const int o0 = a.q_off[b], o1 = a.q_off[b + 1];
    if (o0 < 0 || o1 < o0 || o1 > a.total_q) return {0, 0, 0, true};
    const int n = o1 - o0;
    return {o0, min(n, a.max_q), ctx - n, c != ctx || n > a.max_q};
}

// Keys that rows at positions p_lo .. p_hi see: [0, sinks) and [lo, hi), as
// tiles of T keys: sink_tiles of them from key 0 up to key `sink`, the others
// from `start` (a multiple of 16, so that sixteen keys from a tile's 16-key
// step lie in one page) up to `hi`.
struct Span {
    int lo, hi, start, sink, sink_tiles, tiles;
};
template <int T>
__device__ __forceinline__ Span span_of(const Args& a, int p_lo, int p_hi) {
    Span s;
    s.hi = max(p_hi + 1, 0);
    s.lo = a.window > 0 ? max(max(p_lo, 0) - a.window + 1, 0) : 0;
    s.start = s.lo & ~15;
    s.sink = min(a.sinks, s.start);
    s.sink_tiles = (s.sink + T - 1) / T;
    if (s.sink_tiles * T >= s.start) s.start = s.sink = s.sink_tiles = 0;
    s.tiles = s.sink_tiles + (s.hi - s.start + T - 1) / T;
    return s;
}

__device__ __forceinline__ bool sees(const Args& a, int pos, int key) {
    return key <= pos && (a.window == 0 || key > pos - a.window || key < a.sinks);
}

// One row on its own, key by key: what the matrix instructions cannot do when
// a row does not see a key whose V is not finite (0 * inf).  Tiles t0 .. t1 - 1
// of the span; O normalised into s_acc[D], (reference, sum) returned.
template <bool BF16, int D, int T>
__device__ float2 row_alone(const Args& a, const Span& sp, int b, int g, int64_t qrow, int head, int pos, int t0,
                            int t1, float* s_q, float* s_p, float* s_red, float* s_acc) {
    constexpr int E = BF16 ? 2 : 4;
    const int tid = threadIdx.x, NT = blockDim.x;
    const int keys = (t1 - t0) * T;
    auto value = [](const char* p) {
        if constexpr (BF16)
            return bf16_to_f(*reinterpret_cast<const uint16_t*>(p));
        else
            return *reinterpret_cast<const float*>(p);
    };
    __syncthreads();
    for (int d = tid; d < D; d += NT) {
        s_q[d] = value(a.q + (qrow * a.q_stride + (int64_t)head * D + d) * E);
        s_acc[d] = 0.f;
    }
    __syncthreads();
    auto key_at = [&](int i) {
        const int t = t0 + i / T, r = i % T;
        const bool sink = t < sp.sink_tiles;
        const int key = (sink ? t * T : sp.start + (t - sp.sink_tiles) * T) + r;
        return key < (sink ? sp.sink : sp.hi) && sees(a, pos, key) ? key : -1;
    };
    auto row_at = [&](const char* pool, int key) -> const char* {
        const int page = a.table[(int64_t)b * a.max_pages + (key >> a.page_shift)];
        if (page < 0 || page >= a.num_pages) return nullptr;
        return pool + (page * a.page_stride + ((int64_t)(key & ((1 << a.page_shift) - 1)) * a.hkv + g) * D) * E;
    };
    auto score = [&](int i) {
        const int key = key_at(i);
        const char* k = key < 0 ? nullptr : row_at(a.kp, key);
        if (k == nullptr) return -INFINITY;
        float s = 0.f;
        for (int d = 0; d < D; ++d) s = fmaf(s_q[d], value(k + d * E), s);
        return s * a.scale_log2;
    };
    float m = -INFINITY;
    for (int i = tid; i < keys; i += NT) m = fmaxf(m, score(i));
    s_red[tid] = m;
    __syncthreads();
    m = -INFINITY;
    for (int i = 0; i < NT; ++i) m = fmaxf(m, s_red[i]);
    float l = 0.f;
    for (int i0 = 0; i0 < keys; i0 += NT) {
        __syncthreads();
        const float s = i0 + tid < keys ? score(i0 + tid) : -INFINITY;
        s_p[tid] = s == -INFINITY ? -1.f : __builtin_amdgcn_exp2f(s - m);  // -1: no part in the sums
        __syncthreads();
        for (int i = 0; i < min(NT, keys - i0); ++i) {
            const float p = s_p[i];
            if (p == -1.f) continue;
            l += p;
            const char* v = row_at(a.vp, key_at(i0 + i));
            for (int d = tid; d < D; d += NT) s_acc[d] = fmaf(p, value(v + d * E), s_acc[d]);
        }
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
    for (int d = tid; d < D; d += NT) s_acc[d] *= inv;
    __syncthreads();
    return make_float2(m, l);
}

// The keys straight from memory into the registers of the matrix
// instructions: nothing is shared between waves, so there is no LDS and no
// barrier in the key loop.  A workgroup's four waves take every fourth tile of
// its keys (32 in bf16, 16 in fp32) and its 16 NB rows, and their states
// (reference, sum, O) are joined through LDS at the end.
//
// Scores are computed transposed, S^T = K Q^T with 16x16 instructions: lane
// (t16, tq) takes key t16 of sixteen and 16 bytes of its row per step, and
// holds row t16's scores of keys 4 tq .. 4 tq + 3.  O^T = V^T P^T contracts
// over keys in the order the scores are in: lane (t16, tq) reads the rows of
// just those keys, D / 16 neighbouring dims of each (so sixteen lanes read a
// whole row), and the dims of an instruction are t16 * (D / 16) + t.  In fp32
// that is the operand; in bf16 it takes one v_perm per pair of keys and dim.
//
// The reference m of a row moves only when a score exceeds it by 8 (in log2
// units), so that the common tile needs no reduction across lanes.
constexpr int kWaves = 4;

template <bool BF16, int D, int NB>
__global__ __launch_bounds__(kWaves * kWave, 2) void paged_attn_rows_kernel(Args a) {
    constexpr int E = BF16 ? 2 : 4;
    constexpr int KB = BF16 ? 2 : 1;  // 16-key groups per tile
    constexpr int T = 16 * KB;
    constexpr int KC = D * E / 64;        // 16-byte chunks of a K row per lane
    constexpr int VD = D / 16;            // dims of a V row per lane
    constexpr int VW = VD * E / 4;        // the same in words
    constexpr int R = 16 * NB;            // rows of the workgroup
    constexpr int SD = D + 4;             // row stride of the states in LDS
    constexpr int NT = kWaves * kWave;
    __shared__ __align__(16) float s_o[kWaves * R * SD];
    __shared__ float s_ml[2 * kWaves * R];
    __shared__ int s_bad[R];

    // blocks: the last row block (the longest key range) first, neighbours
    // differ in the KV head
    int id = blockIdx.x;
    const int g = id % a.hkv;
    id /= a.hkv;
    const int split = id % a.splits;
    id /= a.splits;
    const int b = id % a.batch;
    const int rev = id / a.batch;
    const Seq sq = seq_of(a, b);
    const int rows = sq.n * a.G;
    const int rb = (rows + R - 1) / R - 1 - rev;
    const int tid = threadIdx.x, lane = lane_id();
    const int wave = uniform(tid / kWave);
    if (rev == 0 && g == 0 && split == 0 && tid == 0 && sq.bad) raise_flag(a.flags, PRESTO_FLAG_BAD_SEQ);
    if (rb < 0) return;
    const int row0 = rb * R;
    const int p_lo = sq.pos0 + row0 / a.G, p_hi = sq.pos0 + (min(row0 + R, rows) - 1) / a.G;
    const Span sp = span_of<T>(a, p_lo, p_hi);
    const int t_begin = split * a.split_tiles, t_end = min(t_begin + a.split_tiles, sp.tiles);
    if (split > 0 && t_begin >= t_end) return;  // the merge knows

    const int t16 = lane & 15, tq = lane >> 4;
    const int RS = a.hkv * D * E;  // bytes from a cache row to the next

    // ---- queries, as the second operand: row t16, chunk i at byte 64 i + 16 tq
    uint4 qf[NB][KC];
    int pos[NB];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
        const int rho = min(row0 + nb * 16 + t16, rows - 1);
        const int tok = rho / a.G, h = rho - tok * a.G;
        pos[nb] = sq.pos0 + tok;
        const char* qp = a.q + ((sq.r0 + tok) * a.q_stride + (int64_t)(g * a.G + h) * D) * E + tq * 16;
#pragma unroll
        for (int i = 0; i < KC; ++i) qf[nb][i] = *reinterpret_cast<const uint4*>(qp + i * 64);
    }

    // ---- where a tile lies; all of it is the same for the whole wave
    struct Tile {
        int key0, limit;
        int page[KB];  // -1: nothing to read
    };
    bool bad_page = false;
    const int32_t* trow = a.table + (int64_t)b * a.max_pages;
    auto locate = [&](int t) {
        Tile x;
        const bool sink = t < sp.sink_tiles;
        x.key0 = uniform(sink ? t * T : sp.start + (t - sp.sink_tiles) * T);
        x.limit = sink ? sp.sink : sp.hi;
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) {
            // (sixteen keys that no row sees may be without a page)
            const int k0 = x.key0 + 16 * kb;
            const bool wanted = k0 < x.limit && (k0 + 16 > sp.lo || k0 < a.sinks);
            x.page[kb] = wanted ? trow[k0 >> a.page_shift] : -1;
            if (wanted && (uint32_t)x.page[kb] >= (uint32_t)a.num_pages) {
                bad_page = true;
                x.page[kb] = -1;
            }
        }
        return x;
    };
    auto group = [&](const char* pool, const Tile& x, int kb) {
        const int r = (x.key0 + 16 * kb) & ((1 << a.page_shift) - 1);
        const int64_t at = x.page[kb] < 0 ? 0 : x.page[kb] * a.page_stride + (int64_t)r * a.hkv * D;
        return pool + (at + g * D) * E;  // (page 0 stands for one that is not there)
    };
    uint4 kf[KB][KC];
    uint32_t vf[4 * KB][VW];
    auto load_k = [&](const Tile& x) {
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) {
            const char* p = group(a.kp, x, kb);
#pragma unroll
            for (int i = 0; i < KC; ++i)
                kf[kb][i] = *reinterpret_cast<const uint4*>(p + (uint32_t)(t16 * RS + tq * 16 + i * 64));
        }
    };
    auto load_v = [&](const Tile& x) {
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) {
            const char* p = group(a.vp, x, kb);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const char* pr = p + (uint32_t)((4 * tq + r) * RS + t16 * VW * 4);
                if constexpr (VW == 2) {
                    const uint2 u = *reinterpret_cast<const uint2*>(pr);
                    vf[4 * kb + r][0] = u.x;
                    vf[4 * kb + r][1] = u.y;
                } else {
#pragma unroll
                    for (int w = 0; w < VW; w += 4) {
                        const uint4 u = *reinterpret_cast<const uint4*>(pr + w * 4);
                        vf[4 * kb + r][w] = u.x;
                        vf[4 * kb + r][w + 1] = u.y;
                        vf[4 * kb + r][w + 2] = u.z;
                        vf[4 * kb + r][w + 3] = u.w;
                    }
                }
            }
        }
    };

    floatx4 o[NB][VD];
    float m[NB], l[NB];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
        m[nb] = -INFINITY;
        l[nb] = 0.f;
#pragma unroll
        for (int t = 0; t < VD; ++t) o[nb][t] = (floatx4){0.f, 0.f, 0.f, 0.f};
    }

    int t = t_begin + wave;
    Tile cur, nxt;
    if (t < t_end) {
        cur = locate(t);
        load_k(cur);
        load_v(cur);
        if (t + kWaves < t_end) nxt = locate(t + kWaves);
    }
    for (; t < t_end; t += kWaves) {
        const bool more = t + kWaves < t_end;
        // ---- scores
        floatx4 S[NB][KB];
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int kb = 0; kb < KB; ++kb) {
                S[nb][kb] = (floatx4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int i = 0; i < KC; ++i) {
                    if constexpr (BF16) {
                        S[nb][kb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                            __builtin_bit_cast(bf16x8, kf[kb][i]), __builtin_bit_cast(bf16x8, qf[nb][i]), S[nb][kb],
                            0, 0, 0);
                    } else {
                        const floatx4 kv = __builtin_bit_cast(floatx4, kf[kb][i]);
                        const floatx4 qv = __builtin_bit_cast(floatx4, qf[nb][i]);
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            S[nb][kb] = __builtin_amdgcn_mfma_f32_16x16x4f32(kv[e], qv[e], S[nb][kb], 0, 0, 0);
                    }
                }
            }
        if (more) load_k(nxt);

        // ---- masks, on the tiles that need them
        bool edge = cur.key0 + T > min(cur.limit, p_lo + 1) ||
                    (a.window > 0 && cur.key0 <= p_hi - a.window && cur.key0 + T > a.sinks);
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) edge |= cur.page[kb] < 0;
        if (edge) {
#pragma unroll
            for (int kb = 0; kb < KB; ++kb)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int key = cur.key0 + 16 * kb + 4 * tq + r;
                    const bool here = cur.page[kb] >= 0 && key < cur.limit;
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb)
                        S[nb][kb][r] = here && sees(a, pos[nb], key) ? S[nb][kb][r] : -INFINITY;
                    // rows that nobody sees may hold anything
                    const bool any = here && (key >= sp.lo || key < a.sinks);
#pragma unroll
                    for (int w = 0; w < VW; ++w) vf[4 * kb + r][w] = any ? vf[4 * kb + r][w] : 0u;
                }
        }

        // ---- probabilities
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            float mx = -INFINITY;
#pragma unroll
            for (int kb = 0; kb < KB; ++kb)
#pragma unroll
                for (int r = 0; r < 4; ++r) mx = fmaxf(mx, S[nb][kb][r]);
            mx *= a.scale_log2;
            if (__ballot(mx > m[nb] + 8.f)) {
                const float mn = fmaxf(m[nb], quad_max(mx));
                const float al = m[nb] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m[nb] - mn);
                m[nb] = mn;
                l[nb] *= al;
#pragma unroll
                for (int i = 0; i < VD; ++i) o[nb][i] *= al;
            }
            const float mr = m[nb] == -INFINITY ? 0.f : m[nb];  // no key seen yet: every term is 0
#pragma unroll
            for (int kb = 0; kb < KB; ++kb)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    S[nb][kb][r] = __builtin_amdgcn_exp2f(fmaf(S[nb][kb][r], a.scale_log2, -mr));
        }

        // ---- O^T += V^T P^T
        if constexpr (BF16) {
            const bf16x2 ones = {(__bf16)1.0f, (__bf16)1.0f};
            bf16x8 pb[NB];
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
                uint32_t w[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    // (rounded to the product's bf16; the sum takes the rounded values)
                    w[i] = pack2(S[nb][i / 2][2 * (i % 2)], S[nb][i / 2][2 * (i % 2) + 1]);
                    l[nb] = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, w[i]), ones, l[nb], false);
                }
                pb[nb] = __builtin_bit_cast(bf16x8, make_uint4(w[0], w[1], w[2], w[3]));
            }
#pragma unroll
            for (int i = 0; i < VD; ++i) {
                uint32_t w[4];
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    w[j] = __builtin_amdgcn_perm(vf[2 * j + 1][i / 2], vf[2 * j][i / 2],
                                                 i % 2 ? 0x07060302u : 0x05040100u);
                const bf16x8 va = __builtin_bit_cast(bf16x8, make_uint4(w[0], w[1], w[2], w[3]));
#pragma unroll
                for (int nb = 0; nb < NB; ++nb)
                    o[nb][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va, pb[nb], o[nb][i], 0, 0, 0);
            }
        } else {
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    l[nb] += S[nb][0][r];
#pragma unroll
                    for (int i = 0; i < VD; ++i)
                        o[nb][i] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(vf[r][i]), S[nb][0][r],
                                                                        o[nb][i], 0, 0, 0);
                }
        }
        if (more) {
            load_v(nxt);
            cur = nxt;
            if (t + 2 * kWaves < t_end) nxt = locate(t + 2 * kWaves);
        }
    }
    if (bad_page && lane == 0) raise_flag(a.flags, PRESTO_FLAG_BAD_PAGE);

    // ---- join the waves
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
        const float ls = quad_sum(l[nb]);
        const int r = wave * R + nb * 16 + t16;
        if (tq == 0) {
            s_ml[r] = m[nb];
            s_ml[kWaves * R + r] = ls;
        }
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int i = 0; i < VD; i += 4)
                *reinterpret_cast<floatx4*>(&s_o[r * SD + (4 * tq + e) * VD + i]) =
                    (floatx4){o[nb][i][e], o[nb][i + 1][e], o[nb][i + 2][e], o[nb][i + 3][e]};
    }
    if (tid < R) s_bad[tid] = 0;
    __syncthreads();

    const int64_t bg = (int64_t)b * a.hkv + g, all = (int64_t)a.G * a.max_q;
    auto put = [&](int rho, int d, floatx4 v) {
        if (a.splits > 1) {
            *reinterpret_cast<floatx4*>(a.part_o + ((bg * a.splits + split) * all + rho) * D + d) = v;
            return;
        }
        const int tok = rho / a.G, h = rho - tok * a.G;
        char* p = a.out + (((sq.r0 + tok) * a.hq + g * a.G + h) * D + d) * E;
        if constexpr (BF16)
            *reinterpret_cast<uint2*>(p) = make_uint2(pack2(v[0], v[1]), pack2(v[2], v[3]));
        else
            *reinterpret_cast<floatx4*>(p) = v;
    };
    auto put_ml = [&](int rho, float M, float L) {
        if (a.splits > 1) a.part_ml[(bg * all + rho) * a.splits + split] = make_float2(M, L);
    };
    for (int i = tid; i < R * (D / 4); i += NT) {
        const int r = i / (D / 4), d = i % (D / 4) * 4;
        const int rho = row0 + r;
        if (rho >= rows) break;
        float M = -INFINITY, L = 0.f;
        floatx4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < kWaves; ++w) M = fmaxf(M, s_ml[w * R + r]);
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            const float mw = s_ml[w * R + r];
            const float f = mw == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mw - M);
            L = fmaf(f, s_ml[kWaves * R + w * R + r], L);
            const floatx4 ow = *reinterpret_cast<const floatx4*>(&s_o[(w * R + r) * SD + d]);
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[e] = fmaf(f, ow[e], acc[e]);
        }
        // (a sum that is not a number stays one)
        const float inv = L == 0.f ? 0.f : 1.f / L;
        bool fine = true;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            acc[e] *= inv;
            fine &= fabsf(acc[e]) < INFINITY;
        }
        if (!fine) s_bad[r] = 1;
        put(rho, d, acc);
        if (d == 0) put_ml(rho, M, L);
    }
    // ---- rows of several positions whose sums are not all finite: a key that
    // only others see may be the cause
    if (p_lo == p_hi) return;
    __syncthreads();
    for (int r = 0; r < R; ++r) {
        if (!s_bad[r]) continue;
        const int rho = row0 + r, tok = rho / a.G;
        float* const s_acc = s_o;
        const float2 ml = row_alone<BF16, D, T>(a, sp, b, g, sq.r0 + tok, g * a.G + rho - tok * a.G, sq.pos0 + tok,
                                                t_begin, t_end, s_o + D, s_o + 2 * D, s_o + 2 * D + NT, s_acc);
        for (int d = tid * 4; d < D; d += NT * 4) put(rho, d, *reinterpret_cast<const floatx4*>(&s_acc[d]));
        if (tid == 0) put_ml(rho, ml.x, ml.y);
    }
}

// Joins the splits of a row: D / 4 lanes per row.  Splits past a sequence's
// keys have written nothing.
template <bool BF16, int D, int T>
__global__ __launch_bounds__(256) void paged_attn_merge_kernel(Args a, int rows_per_block) {
    constexpr int E = BF16 ? 2 : 4;
    constexpr int LR = D / 4;  // lanes per row: 16 or 32
    const int per_seq = a.max_q * a.hq;
    const int64_t idx = (int64_t)blockIdx.x * (256 / LR) + threadIdx.x / LR;
    const int ln = threadIdx.x % LR;
    const int b = (int)(idx / per_seq), rest = (int)(idx % per_seq);
    if (b >= a.batch) return;
    const Seq sq = seq_of(a, b);
    const int tok = rest / a.hq, head = rest - tok * a.hq;
    if (tok >= sq.n) return;
    const int g = head / a.G, rho = tok * a.G + head - g * a.G;
    const int row0 = rho / rows_per_block * rows_per_block;
    const Span sp = span_of<T>(a, sq.pos0 + row0 / a.G,
                               sq.pos0 + (min(row0 + rows_per_block, sq.n * a.G) - 1) / a.G);
    const int live = max(min((sp.tiles + a.split_tiles - 1) / a.split_tiles, a.splits), 1);
    const int64_t bg = (int64_t)b * a.hkv + g, all = (int64_t)a.G * a.max_q;
    const float2* ml = a.part_ml + (bg * all + rho) * a.splits;
    const float* po = a.part_o + (bg * a.splits * all + rho) * D + ln * 4;
    float M = -INFINITY;
    for (int s = ln; s < live; s += LR) M = fmaxf(M, ml[s].x);
#pragma unroll
    for (int o = LR / 2; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor(M, o, LR));
    float L = 0.f;
    floatx4 acc = {0.f, 0.f, 0.f, 0.f};
    for (int s0 = 0; s0 < live; s0 += 8) {
        floatx4 v[8];
        float w[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int s = min(s0 + j, live - 1);
            v[j] = *reinterpret_cast<const floatx4*>(po + (int64_t)s * all * D);
            const float2 x = ml[s];
            // a split in which the row sees nothing has sum 0
            const bool part = s0 + j < live && x.y != 0.f;
            w[j] = part ? x.y * __builtin_amdgcn_exp2f(x.x - M) : 0.f;
            if (!part) v[j] = (floatx4){0.f, 0.f, 0.f, 0.f};
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            L += w[j];
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[e] = fmaf(w[j], v[j][e], acc[e]);
        }
    }
    const float inv = L == 0.f ? 0.f : 1.f / L;
    char* p = a.out + (((sq.r0 + tok) * a.hq + head) * D + ln * 4) * E;
    if constexpr (BF16)
        *reinterpret_cast<uint2*>(p) =
            make_uint2(pack2(acc[0] * inv, acc[1] * inv), pack2(acc[2] * inv, acc[3] * inv));
    else
        *reinterpret_cast<floatx4*>(p) = acc * inv;
}

}  // namespace paged
}  // namespace presto

namespace presto_host {

using namespace presto;
using namespace presto::paged;

namespace {

struct PagedPlan {
    int nb;          // 16-row blocks per workgroup
    int rows_per_block, row_blocks, splits, split_tiles;
    int64_t blocks;
    size_t o_bytes, bytes;
};

int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }

PagedPlan paged_plan(const presto_paged_attn_desc* d) {
    PagedPlan p{};
    const bool bf16 = d->pages.dt == PRESTO_DT_BF16;
    const int G = d->hq / d->pages.hkv;
    const int64_t rows = (int64_t)G * d->max_q;
    const int T = bf16 ? 32 : 16;
    p.nb = rows > 16 ? 2 : 1;
    p.rows_per_block = 16 * p.nb;
    p.row_blocks = (int)cdiv(rows, p.rows_per_block);
    // keys of one row block: all of the context, or the sinks and the window
    // of its first to its last row
    int64_t longest = d->max_ctx > 0 ? d->max_ctx : 1;
    if (d->window > 0) {
        const int64_t span = (int64_t)d->window + p.rows_per_block / G + 1 + d->sinks + 16 + T;
        if (span < longest) longest = span;
    }
    const int64_t all = (int64_t)d->pages.batch * d->pages.hkv * p.row_blocks;
    int64_t mean = longest;
    if (d->total_ctx > 0 && d->total_ctx / d->pages.batch < mean) mean = d->total_ctx / d->pages.batch + 1;
    const int64_t tiles = cdiv(longest, T);
    // enough workgroups to fill the chip twice, of at least one tile per wave
    int64_t per = cdiv(all * cdiv(mean, T), 1536);
    per = cdiv(per, kWaves) * kWaves;
    if (per >= tiles) per = tiles;
    p.splits = (int)cdiv(tiles, per);
    p.split_tiles = (int)per;
    p.blocks = all * p.splits;
    if (p.splits > 1) {
        const int64_t parts = (int64_t)d->pages.batch * d->pages.hkv * p.splits * rows;
        p.o_bytes = (size_t)parts * d->pages.head_dim * sizeof(float);
        p.bytes = p.o_bytes + (size_t)parts * sizeof(float2);
    }
    return p;
}

template <bool BF16, int D>
void launch_rows(const PagedPlan& p, const Args& a, hipStream_t stream) {
    if (p.nb == 1)
        paged_attn_rows_kernel<BF16, D, 1><<<(unsigned)p.blocks, kWaves * kWave, 0, stream>>>(a);
    else
        paged_attn_rows_kernel<BF16, D, 2><<<(unsigned)p.blocks, kWaves * kWave, 0, stream>>>(a);
    if (p.splits > 1) {
        constexpr int T = BF16 ? 32 : 16;
        const int64_t rows = (int64_t)a.batch * a.max_q * a.hq;
        paged_attn_merge_kernel<BF16, D, T>
            <<<(unsigned)cdiv(rows, 256 / (D / 4)), 256, 0, stream>>>(a, p.rows_per_block);
    }
}

}  // namespace

size_t paged_attn_workspace_bytes(const presto_paged_attn_desc* d) { return paged_plan(d).bytes; }

// false: more workgroups than a grid holds
bool paged_attn_fits(const presto_paged_attn_desc* d) {
    const PagedPlan p = paged_plan(d);
    const int64_t rows = (int64_t)d->pages.batch * d->max_q * d->hq;
    return p.blocks < ((int64_t)1 << 31) && rows < ((int64_t)1 << 31);
}

presto_status launch_paged_attn(const presto_paged_attn_desc* d, const void* q, const int32_t* q_off,
                                const void* kp, const void* vp, const int32_t* table, const int32_t* ctx, void* out,
                                int32_t* flags, void* ws, hipStream_t stream) {
    const PagedPlan p = paged_plan(d);
    Args a{};
    a.q = static_cast<const char*>(q);
    a.kp = static_cast<const char*>(kp);
    a.vp = static_cast<const char*>(vp);
    a.table = table;
    a.ctx = ctx;
    a.q_off = q_off;
    a.out = static_cast<char*>(out);
    a.part_o = static_cast<float*>(ws);
    a.part_ml = reinterpret_cast<float2*>(static_cast<char*>(ws) + p.o_bytes);
    a.flags = flags;
    a.q_stride = d->q_stride;
    a.page_stride = d->pages.page_stride;
    a.total_q = d->total_q;
    a.batch = d->pages.batch;
    a.hq = d->hq;
    a.hkv = d->pages.hkv;
    a.G = d->hq / d->pages.hkv;
    a.max_q = d->max_q;
    a.max_ctx = d->max_ctx;
    a.num_pages = d->pages.num_pages;
    a.max_pages = d->pages.max_pages;
    a.page_shift = __builtin_ctz((unsigned)d->pages.page_size);
    a.window = d->window;
    a.sinks = d->window > 0 ? d->sinks : 0;
    a.row_blocks = p.row_blocks;
    a.splits = p.splits;
    a.split_tiles = p.split_tiles;
    a.scale_log2 = d->scale * kLog2e;
    const bool bf16 = d->pages.dt == PRESTO_DT_BF16;
    if (d->pages.head_dim == 128)
        bf16 ? launch_rows<true, 128>(p, a, stream) : launch_rows<false, 128>(p, a, stream);
    else
        bf16 ? launch_rows<true, 64>(p, a, stream) : launch_rows<false, 64>(p, a, stream);
    return check_launch("paged_attn_rows_kernel");
}

}  // namespace presto_host
