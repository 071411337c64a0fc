// Attention over a paged cache in 4 bits.
//
// A wave takes 32 keys at a time and 16 query rows of one KV head (its heads
// and tokens) on 16 x 16 x 32 matrix instructions, scores transposed: S^T = K
// Q^T.  A lane (n = lane % 16, g = lane / 16) loads of two blocks of 16 keys
//   K: key n, a quarter of its dims (g): its own words are, converted, the A
//      operands of the contraction over dims, whose order is free;
//   V: keys 4 g .. 4 g + 3, dims PER n .. PER n + PER - 1 (as the block lays
//      them out): the A operands of O^T = V^T P^T, M index n of instruction t
//      being dim PER n + t, its contraction slots the lane's own 8 keys.
// S^T leaves a lane with row n and the same 8 keys, so the probabilities are the
// B operand as they stand, and O^T leaves it with row n again: no value crosses
// lanes but in the row maximum, and the cache goes from memory to the matrix
// cores through registers only.
#include <algorithm>
#include <type_traits>

#include "common.hpp"
#include "quant.hpp"
#include "step.hpp"

namespace presto {
namespace qattn {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kTile = 32;  // keys
constexpr int kWaves = 4;
constexpr int kThreads = kWaves * kWave;
constexpr float kSlack = 16.f;  // a row's reference may lie this far (log2) below its largest score

struct Args {
    const void* q;
    const char *k, *v;
    const int32_t *table, *ctx, *q_off;  // q_off null: one token per sequence
    void* out;
    float* part_o;
    float2* part_ml;
    int32_t* flags;
    int64_t page_bytes, q_stride, total_q;
    int32_t batch, hkv, group, max_q, max_ctx, window, sinks, max_pages, num_pages, shift;
    int32_t row_blocks, splits, split_tiles;
    float scale;  // times log2 e
};

// What a sequence asks for.
struct Seq {
    int64_t row;   // of q: its first token
    int n, first;  // tokens that are computed, the first one's position
    bool odd;      // something about it is wrong
};
__device__ __forceinline__ Seq sequence(const Args& a, int b) {
    Seq s;
    int64_t o0 = b, o1 = b + 1;
    if (a.q_off) {
        o0 = a.q_off[b];
        o1 = a.q_off[b + 1];
    }
    const int c = a.ctx[b], cut = min(max(c, 0), a.max_ctx);
    s.odd = c != cut;
    if (o0 < 0 || o1 < o0 || o1 > a.total_q) {
        s.odd = true;
        o1 = o0 = 0;
    }
    s.odd |= o1 - o0 > a.max_q;
    s.row = o0;
    s.n = (int)min(o1 - o0, (int64_t)a.max_q);
    s.first = (int)(cut - (o1 - o0));
    return s;
}

// The keys that rows at positions pmin .. pmax see between them, as a list of
// tiles: those of the sinks, then those of the window.
struct Tiles {
    int lo, pmin, pmax, sink, t0, count;
};
__device__ __forceinline__ Tiles tiles_of(const Args& a, int pmin, int pmax) {
    Tiles t;
    t.pmin = pmin;
    t.pmax = pmax;
    t.lo = a.window ? max(0, pmin - a.window + 1) : 0;
    t.sink = (min(a.sinks, t.lo) + kTile - 1) / kTile;
    t.t0 = max(t.lo / kTile, t.sink);
    t.count = pmax < 0 ? 0 : t.sink + max(0, pmax / kTile - t.t0 + 1);
    return t;
}
__device__ __forceinline__ int tile_at(const Tiles& t, int u) { return u < t.sink ? u : t.t0 + u - t.sink; }

// Whether some row needs a key of the block at j0.
__device__ __forceinline__ bool needed(const Args& a, const Tiles& t, int j0) {
    return j0 <= t.pmax && (j0 + 15 >= t.lo || j0 < a.sinks);
}

__device__ __forceinline__ bool sees(const Args& a, int p, int j) {
    return j <= p && (a.window == 0 || j > p - a.window || j < a.sinks);
}

// A tile as a lane holds it.
template <int D>
struct Tile {
    static constexpr int W = D / 32;  // words
    uint32_t kc[2][W], vc[2][W], ve[2];
    uint32_t ke[2];
};

template <int D>
__device__ __forceinline__ void load_words(uint32_t (&w)[D / 32], const char* p) {
    if constexpr (D == 128) {
        const uint4 x = *reinterpret_cast<const uint4*>(p);
        w[0] = x.x;
        w[1] = x.y;
        w[2] = x.z;
        w[3] = x.w;
    } else {
        const uint2 x = *reinterpret_cast<const uint2*>(p);
        w[0] = x.x;
        w[1] = x.y;
    }
}

template <int D>
__device__ __forceinline__ void load_tile(Tile<D>& t, const char* k0, const char* v0, const char* k1, const char* v1) {
    const int n = lane_id() & 15, g = lane_id() >> 4;
    const int kc = n * (D / 2) + g * (D / 8), ke = 8 * D + n * (D / 32) + g * (D / 4) / 32;
    const int vc = lane_id() * (D / 8), ve = 8 * D + (g * (D / 32) + n * (D / 16) / 32) * 4;
    load_words<D>(t.kc[0], k0 + kc);
    load_words<D>(t.kc[1], k1 + kc);
    t.ke[0] = (uint8_t)k0[ke];
    t.ke[1] = (uint8_t)k1[ke];
    load_words<D>(t.vc[0], v0 + vc);
    load_words<D>(t.vc[1], v1 + vc);
    t.ve[0] = *reinterpret_cast<const uint32_t*>(v0 + ve);
    t.ve[1] = *reinterpret_cast<const uint32_t*>(v1 + ve);
}

__device__ __forceinline__ bf16x8 eight(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    const u32x4 w = {a, b, c, d};
    return __builtin_bit_cast(bf16x8, w);
}
__device__ __forceinline__ uint32_t pack2(float a, float b) {
    const quant::bf16x2 p = {(__bf16)a, (__bf16)b};
    return __builtin_bit_cast(uint32_t, p);
}

// Eight values as N bf16 each, each holding what the ones before left.
template <int N>
__device__ __forceinline__ void split8(float v[8], bf16x8 (&p)[N]) {
#pragma unroll
    for (int k = 0; k < N; ++k) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            w[i] = pack2(v[2 * i], v[2 * i + 1]);
            if (k + 1 < N) {
                v[2 * i] -= bf16lo(w[i]);
                v[2 * i + 1] -= bf16hi(w[i]);
            }
        }
        p[k] = eight(w[0], w[1], w[2], w[3]);
    }
}

__device__ __forceinline__ f32x4 mma(const bf16x8& a, const bf16x8& b, const f32x4& c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// Exponents of groups that are not finite (above kMostExp): the top bits of
// their bytes, and the others with those bytes 0.
__device__ __forceinline__ uint32_t odd_exps(uint32_t w) {
    static_assert(quant::kMostExp == 252, "255 - 3");
    return ((w & 0x7f7f7f7fu) + 0x03030303u) & w & 0x80808080u;
}
__device__ __forceinline__ uint32_t without(uint32_t w, uint32_t odd) { return w & ~((odd >> 7) * 255u); }

// R blocks of 16 query rows per wave; the waves of a workgroup take its tiles
// in turn.
template <bool F32, int D, int R>
__global__ __launch_bounds__(kThreads) void quant_attn_kernel(Args a) {
    constexpr int NQ = F32 ? 3 : 1, NP = F32 ? 3 : 2;  // bf16 per query value and per probability
    constexpr int STEPS = D / 32, PER = D / 16, ROWS = 16 * R;
    using T = std::conditional_t<F32, float, uint16_t>;
    __shared__ float s_o[kWaves][ROWS][D + 4];
    __shared__ float s_m[kWaves][ROWS], s_l[kWaves][ROWS];

    const int lane = lane_id(), n = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    int x = blockIdx.x;
    const int head = x % a.hkv;
    x /= a.hkv;
    const int split = x % a.splits;
    x /= a.splits;
    const int rb = x % a.row_blocks, b = x / a.row_blocks;

    const Seq s = sequence(a, b);
    if (s.odd && rb == 0 && split == 0 && head == 0 && threadIdx.x == 0) raise_flag(a.flags, PRESTO_FLAG_BAD_SEQ);
    const int r0 = rb * ROWS;  // of the sequence's rows (token, head of the group)
    const int i0 = r0 / a.group;
    if (i0 >= s.n) return;
    const int i1 = min((r0 + ROWS - 1) / a.group, s.n - 1);
    const Tiles t = tiles_of(a, s.first + i0, s.first + i1);
    const int u0 = split * a.split_tiles, u1 = min(u0 + a.split_tiles, t.count);

    // this lane's rows: positions (-1: none) and queries
    int pos[R];
    bf16x8 qf[R][NQ][STEPS];
#pragma unroll
    for (int j = 0; j < R; ++j) {
        const int r = r0 + 16 * j + n, i = r / a.group;
        pos[j] = i < s.n ? s.first + i : -1;
        const T* q = static_cast<const T*>(a.q) + (s.row + min(i, s.n - 1)) * a.q_stride +
                     ((int64_t)head * a.group + r % a.group) * D + g * (D / 4);
#pragma unroll
        for (int st = 0; st < STEPS; ++st) {
            if constexpr (F32) {
                const float4 x0 = *reinterpret_cast<const float4*>(q + 8 * st),
                             x1 = *reinterpret_cast<const float4*>(q + 8 * st + 4);
                float v[8] = {x0.x, x0.y, x0.z, x0.w, x1.x, x1.y, x1.z, x1.w};
                bf16x8 p[NQ];
                split8<NQ>(v, p);
#pragma unroll
                for (int k = 0; k < NQ; ++k) qf[j][k][st] = p[k];
            } else {
                qf[j][0][st] = *reinterpret_cast<const bf16x8*>(q + 8 * st);
            }
        }
    }

    float m[R], l[R];
    f32x4 o[R][PER];
#pragma unroll
    for (int j = 0; j < R; ++j) {
        m[j] = -INFINITY;  // no key yet
        l[j] = 0.f;
#pragma unroll
        for (int d = 0; d < PER; ++d) o[j][d] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    bool odd_v = false;  // a group of V that is not finite

    // the pages of this wave's next 32 tiles, one block of 16 keys per lane
    int pages = -1;
    auto look_up = [&](int first) {
        const int u = u0 + wave + (first + (lane >> 1)) * kWaves;
        pages = -1;
        if (u < u1) {
            const int j0 = tile_at(t, u) * kTile + (lane & 1) * 16;
            if (needed(a, t, j0)) {
                const int e = a.table[(int64_t)b * a.max_pages + (j0 >> a.shift)];
                if (e >= 0 && e < a.num_pages)
                    pages = e;
                else
                    raise_flag(a.flags, PRESTO_FLAG_BAD_PAGE);
            }
        }
    };
    const int blocks = 1 << (a.shift - 4);  // of a page
    auto offset = [&](int page, int tile, int half) -> int64_t {
        const int in_page = ((tile * kTile + half * 16) & ((1 << a.shift) - 1)) >> 4;
        return max(page, 0) * a.page_bytes + ((int64_t)head * blocks + in_page) * quant::block_bytes(D);
    };
    struct Where {
        int tile, p0, p1;
    };
    auto where = [&](int it) {
        Where w;
        w.tile = tile_at(t, u0 + wave + it * kWaves);
        w.p0 = __builtin_amdgcn_readlane(pages, 2 * (it & 31));
        w.p1 = __builtin_amdgcn_readlane(pages, 2 * (it & 31) + 1);
        return w;
    };
    auto fetch = [&](Tile<D>& tl, const Where& w) {
        const int64_t f0 = offset(w.p0, w.tile, 0), f1 = offset(w.p1, w.tile, 1);
        load_tile<D>(tl, a.k + f0, a.v + f0, a.k + f1, a.v + f1);
    };

    const int mine = u1 > u0 + wave ? (u1 - u0 - wave + kWaves - 1) / kWaves : 0;
    Tile<D> next;
    Where w_next;
    if (mine > 0) {
        look_up(0);
        w_next = where(0);
        fetch(next, w_next);
    }
    for (int it = 0; it < mine; ++it) {
        const Tile<D> cur = next;
        const Where w = w_next;
        if (it + 1 < mine) {
            if (((it + 1) & 31) == 0) look_up(it + 1);
            w_next = where(it + 1);
            fetch(next, w_next);
        }
        const int j0 = w.tile * kTile;
        const bool whole = j0 + kTile - 1 <= t.pmin &&
                           (a.window == 0 || j0 > t.pmax - a.window || j0 + kTile - 1 < a.sinks) && w.p0 >= 0 &&
                           w.p1 >= 0;

        // scores
        f32x4 sc[R][2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const float ks = quant::exp_scale(cur.ke[h]);
#pragma unroll
            for (int j = 0; j < R; ++j) sc[j][h] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int st = 0; st < STEPS; ++st) {
                const uint32_t c = cur.kc[h][st];
                const bf16x8 kf = eight(quant::decode2<0>(c, ks), quant::decode2<1>(c, ks), quant::decode2<2>(c, ks),
                                        quant::decode2<3>(c, ks));
#pragma unroll
                for (int k = NQ - 1; k >= 0; --k)
#pragma unroll
                    for (int j = 0; j < R; ++j) sc[j][h] = mma(kf, qf[j][k][st], sc[j][h]);
            }
        }

        // probabilities: x = s c - m
        bf16x8 p[R][NP];
#pragma unroll
        for (int j = 0; j < R; ++j) {
            float z[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) z[i] = sc[j][i >> 2][i & 3] * a.scale;
            if (!whole) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int key = j0 + (i >> 2) * 16 + 4 * g + (i & 3);
                    if (!(sees(a, pos[j], key) && (i < 4 ? w.p0 : w.p1) >= 0)) z[i] = -INFINITY;
                }
            }
            float top = z[0];
#pragma unroll
            for (int i = 1; i < 8; ++i) top = fmaxf(top, z[i]);
            // (NaN scores take no part in the maximum and reach l through exp2)
            const bool unset = m[j] == -INFINITY;
            if (__any(unset ? top > -INFINITY : top > m[j] + kSlack)) {
                top = fmaxf(top, __shfl_xor(top, 16));
                top = fmaxf(top, __shfl_xor(top, 32));
                if (top > m[j]) {
                    const float f = unset ? 0.f : __builtin_amdgcn_exp2f(m[j] - top);
                    m[j] = top;
                    l[j] *= f;
#pragma unroll
                    for (int d = 0; d < PER; ++d) o[j][d] *= f;
                }
            }
            const float ref = m[j] == -INFINITY ? 0.f : m[j];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                z[i] = __builtin_amdgcn_exp2f(z[i] - ref);
                l[j] += z[i];
            }
            split8<NP>(z, p[j]);
        }

        // values
        uint32_t ve[2] = {cur.ve[0], cur.ve[1]};
        if (!whole) {  // keys that no row sees may be anything
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int key = j0 + (i >> 2) * 16 + 4 * g + (i & 3);
                const bool seen = key <= t.pmax && (key >= t.lo || key < a.sinks) && (i < 4 ? w.p0 : w.p1) >= 0;
                if (!seen) ve[i >> 2] &= ~(255u << (8 * (i & 3)));
            }
        }
        if (__any(odd_exps(ve[0]) | odd_exps(ve[1]))) {
            odd_v = true;
            ve[0] = without(ve[0], odd_exps(ve[0]));
            ve[1] = without(ve[1], odd_exps(ve[1]));
        }
        float vs[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) vs[i] = quant::exp_scale((ve[i >> 2] >> (8 * (i & 3))) & 255);
        auto pv = [&](auto B) {  // dims 2 B and 2 B + 1 of the lane's
            uint32_t c[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if constexpr (D == 128) {
                    c[i] = quant::decode2<B()>(cur.vc[i >> 2][i & 3], vs[i]);
                } else {
                    const uint32_t word = cur.vc[i >> 2][(i & 3) >> 1];
                    c[i] = (i & 1) ? quant::decode2<2 + B()>(word, vs[i]) : quant::decode2<B()>(word, vs[i]);
                }
            }
            uint32_t w0[4], w1[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                w0[i] = __builtin_amdgcn_perm(c[2 * i + 1], c[2 * i], 0x05040100u);
                w1[i] = __builtin_amdgcn_perm(c[2 * i + 1], c[2 * i], 0x07060302u);
            }
            const bf16x8 v0 = eight(w0[0], w0[1], w0[2], w0[3]), v1 = eight(w1[0], w1[1], w1[2], w1[3]);
#pragma unroll
            for (int k = NP - 1; k >= 0; --k)
#pragma unroll
                for (int j = 0; j < R; ++j) {
                    o[j][2 * B()] = mma(v0, p[j][k], o[j][2 * B()]);
                    o[j][2 * B() + 1] = mma(v1, p[j][k], o[j][2 * B() + 1]);
                }
        };
        pv(std::integral_constant<int, 0>{});
        pv(std::integral_constant<int, 1>{});
        if constexpr (D == 128) {
            pv(std::integral_constant<int, 2>{});
            pv(std::integral_constant<int, 3>{});
        }
    }

    // A group of V that is not finite took part as zeros: now the rows that see
    // its key lose the group's dims (a lane's are all of one group).
    if (odd_v) {
        const int grp = D == 128 ? g : g >> 1;
        bool lost[R] = {};
        for (int it = 0; it < mine; ++it) {
            if ((it & 31) == 0) look_up(it);
            const Where w = where(it);
            for (int h = 0; h < 2; ++h) {
                const int page = h ? w.p1 : w.p0;
                if (page < 0) continue;
                const char* e = a.v + offset(page, w.tile, h) + 8 * D + grp * 4;
                for (int r = 0; r < 16; ++r) {
                    if ((uint8_t)e[(r >> 2) * (D / 8) + (r & 3)] <= quant::kMostExp) continue;
#pragma unroll
                    for (int j = 0; j < R; ++j) lost[j] |= sees(a, pos[j], w.tile * kTile + h * 16 + r);
                }
            }
        }
#pragma unroll
        for (int j = 0; j < R; ++j)
            if (lost[j]) {
#pragma unroll
                for (int d = 0; d < PER; ++d) o[j][d] = f32x4{NAN, NAN, NAN, NAN};
            }
    }

    // the waves' states, joined
#pragma unroll
    for (int j = 0; j < R; ++j) {
        l[j] += __shfl_xor(l[j], 16);
        l[j] += __shfl_xor(l[j], 32);
        if (g == 0) {
            s_m[wave][16 * j + n] = m[j];
            s_l[wave][16 * j + n] = l[j];
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int d = 0; d < PER; d += 4)
                *reinterpret_cast<float4*>(&s_o[wave][16 * j + n][PER * (4 * g + i) + d]) =
                    make_float4(o[j][d][i], o[j][d + 1][i], o[j][d + 2][i], o[j][d + 3][i]);
    }
    __syncthreads();
    constexpr int PIECES = D / 8;
    for (int e = threadIdx.x; e < ROWS * PIECES; e += kThreads) {
        const int r = e / PIECES, x0 = e % PIECES * 8, i = (r0 + r) / a.group;
        if (i >= s.n) continue;
        float top = -INFINITY, sum = 0.f, v[8] = {};
        for (int w = 0; w < kWaves; ++w) top = fmaxf(top, s_m[w][r]);
        for (int w = 0; w < kWaves; ++w) {
            if (s_m[w][r] == -INFINITY && s_l[w][r] == 0.f) continue;  // (no key)
            const float f = __builtin_amdgcn_exp2f(s_m[w][r] - (top == -INFINITY ? 0.f : top));
            sum += f * s_l[w][r];
            for (int d = 0; d < 8; ++d) v[d] += f * s_o[w][r][x0 + d];
        }
        const int64_t row = (s.row + i) * a.hkv * a.group + (int64_t)head * a.group + (r0 + r) % a.group;
        if (a.splits > 1) {
            const int64_t at = row * a.splits + split;
            if (x0 == 0) a.part_ml[at] = make_float2(top, sum);
            float4* to = reinterpret_cast<float4*>(a.part_o + at * D + x0);
            to[0] = make_float4(v[0], v[1], v[2], v[3]);
            to[1] = make_float4(v[4], v[5], v[6], v[7]);
        } else {
            const float f = sum == 0.f ? 0.f : 1.f / sum;
            if constexpr (F32) {
                float4* to = reinterpret_cast<float4*>(static_cast<float*>(a.out) + row * D + x0);
                to[0] = make_float4(v[0] * f, v[1] * f, v[2] * f, v[3] * f);
                to[1] = make_float4(v[4] * f, v[5] * f, v[6] * f, v[7] * f);
            } else {
                *reinterpret_cast<uint4*>(static_cast<uint16_t*>(a.out) + row * D + x0) =
                    make_uint4(pack2(v[0] * f, v[1] * f), pack2(v[2] * f, v[3] * f), pack2(v[4] * f, v[5] * f),
                               pack2(v[6] * f, v[7] * f));
            }
        }
    }
}

// Joins the splits of a row: a wave per row.
template <bool F32, int D>
__global__ __launch_bounds__(kThreads) void quant_merge_kernel(Args a) {
    const int lane = lane_id();
    const int hq = a.hkv * a.group;
    const int64_t u = (int64_t)blockIdx.x * kWaves + threadIdx.x / kWave;
    const int64_t token = u / hq;
    const int h = (int)(u - token * hq);
    const int b = (int)(token / a.max_q), i = (int)(token - (int64_t)b * a.max_q);
    if (b >= a.batch) return;
    const Seq s = sequence(a, b);
    if (i >= s.n) return;
    const int64_t row = (s.row + i) * hq + h;
    const float2* ml = a.part_ml + row * a.splits;
    float top = -INFINITY;
    for (int k = lane; k < a.splits; k += kWave) top = fmaxf(top, ml[k].x);
    top = wave_max_f32_dpp(top);
    const float ref = top == -INFINITY ? 0.f : top;
    constexpr int N = D / kWave;
    float sum = 0.f, v[N] = {};
    for (int k = 0; k < a.splits; ++k) {
        const float2 x = ml[k];
        if (x.y == 0.f) continue;  // (no key)
        const float f = __builtin_amdgcn_exp2f((x.x == -INFINITY ? 0.f : x.x) - ref);
        sum += f * x.y;
        const float* o = a.part_o + (row * a.splits + k) * D + lane * N;
#pragma unroll
        for (int d = 0; d < N; ++d) v[d] += f * o[d];
    }
    const float f = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
    for (int d = 0; d < N; ++d) {
        if constexpr (F32)
            static_cast<float*>(a.out)[row * D + lane * N + d] = v[d] * f;
        else
            static_cast<__bf16*>(a.out)[row * D + lane * N + d] = (__bf16)(v[d] * f);
    }
}

}  // namespace qattn
}  // namespace presto

namespace presto_host {

using namespace presto;
using namespace presto::qattn;

QuantPlan quant_plan(const presto_paged_attn_desc* d, presto_dtype dt) {
    QuantPlan p{};
    const int64_t group = d->hq / d->pages.hkv, rows = (int64_t)d->max_q * group;
    p.r = rows > 16 && dt == PRESTO_DT_BF16 ? 2 : 1;
    p.row_blocks = (rows + 16 * p.r - 1) / (16 * p.r);
    // the tiles of a row block: the longest, and on average
    int64_t most = ((int64_t)d->max_ctx + kTile - 1) / kTile;
    const int64_t span = 16 * p.r / group + 2;  // tokens of a row block
    if (d->window)
        most = std::min(most, ((int64_t)d->window + span) / kTile + 2 + ((int64_t)d->sinks + kTile - 1) / kTile);
    most = std::max<int64_t>(most, 1);
    const int64_t blocks = (int64_t)d->pages.batch * p.row_blocks * d->pages.hkv;
    int64_t mean = most;
    if (d->total_ctx > 0) mean = std::min(most, d->total_ctx / d->pages.batch / kTile + 1);
    constexpr int64_t kTarget = 1024, kLeast = 16, kMostSplits = 256;
    int64_t tiles = std::max(kLeast, (blocks * mean + kTarget - 1) / kTarget);
    tiles = std::max(tiles, (most + kMostSplits - 1) / kMostSplits);
    p.splits = (most + tiles - 1) / tiles;
    p.split_tiles = (most + p.splits - 1) / p.splits;
    p.blocks = blocks * p.splits;
    const int64_t out_rows = d->total_q * d->hq, merge_rows = (int64_t)d->pages.batch * d->max_q * d->hq;
    p.merge_blocks = (merge_rows + kWaves - 1) / kWaves;
    p.fits = p.blocks <= (1 << 23) && merge_rows < ((int64_t)1 << 31) && p.merge_blocks <= (1 << 23);
    if (p.splits > 1) {
        p.o_bytes = (size_t)(out_rows * p.splits * d->pages.head_dim) * 4;
        p.bytes = p.o_bytes + (size_t)(out_rows * p.splits) * 8;
    }
    return p;
}

presto_status launch_quant_attn(const presto_paged_attn_desc* d, presto_dtype dt, const QuantPlan& p, const void* q,
                                const int32_t* q_off, const void* k, const void* v, const int32_t* table,
                                const int32_t* ctx, void* out, int32_t* flags, void* ws, hipStream_t stream) {
    const presto_pages_desc& g = d->pages;
    Args a{};
    a.q = q;
    a.k = static_cast<const char*>(k);
    a.v = static_cast<const char*>(v);
    a.table = table;
    a.ctx = ctx;
    a.q_off = q_off;
    a.out = out;
    a.part_o = static_cast<float*>(ws);
    a.part_ml = reinterpret_cast<float2*>(static_cast<char*>(ws) + p.o_bytes);
    a.flags = flags;
    a.page_bytes = g.page_stride;
    a.q_stride = d->q_stride;
    a.total_q = d->total_q;
    a.batch = g.batch;
    a.hkv = g.hkv;
    a.group = d->hq / g.hkv;
    a.max_q = d->max_q;
    a.max_ctx = d->max_ctx;
    a.window = d->window;
    a.sinks = d->window ? d->sinks : 0;
    a.max_pages = g.max_pages;
    a.num_pages = g.num_pages;
    a.shift = __builtin_ctz((unsigned)g.page_size);
    a.row_blocks = (int)p.row_blocks;
    a.splits = (int)p.splits;
    a.split_tiles = (int)p.split_tiles;
    a.scale = d->scale * 1.4426950408889634f;
    auto run = [&](auto f32, auto dim) {
        if (p.r == 2)
            quant_attn_kernel<f32(), dim(), f32() ? 1 : 2><<<(unsigned)p.blocks, kThreads, 0, stream>>>(a);
        else
            quant_attn_kernel<f32(), dim(), 1><<<(unsigned)p.blocks, kThreads, 0, stream>>>(a);
        if (p.splits > 1) quant_merge_kernel<f32(), dim()><<<(unsigned)p.merge_blocks, kThreads, 0, stream>>>(a);
    };
    auto with = [&](auto f32) {
        if (g.head_dim == 64)
            run(f32, std::integral_constant<int, 64>{});
        else
            run(f32, std::integral_constant<int, 128>{});
    };
    if (dt == PRESTO_DT_F32)
        with(std::true_type{});
    else
        with(std::false_type{});
    return check_launch("quant_attn_kernel");
}

}  // namespace presto_host
