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
// lanes but in the row maximum, and nothing is turned through LDS.
//
// What bounds it.  Decoding: the cache read once.  16 x 32768 keys of 8 heads of
// 128 (571 MB) take 98 us and 4.8 of the merge, 5.5 TB/s; the conversions and
// products of those tiles alone about 78, so tiles come through an LDS ring while
// the ones before are in work.  16 ragged sequences (75 MB) 21 and 4.7: the
// workgroups' starts, about 5 us, and their first tiles.  Long prompts: the matrix
// cores and the vector ALU of two waves per SIMD.  A tile of a wave's 64 rows is 68
// products (1088 cycles) and some 260 vector instructions (about 1400), of which
// half convert keys and values, a quarter are exponentials at a quarter of the
// rate; 4 x 332..448 new tokens on 11000 take 375 us, 770 TFLOP/s, on 392
// workgroups, two to a CU.  There a probability is one bf16: two, as everywhere
// else, take the registers of 49 values and half as many products again, 671 us.
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
// A row's reference lies this far (log2) above its largest score when it is
// chosen, and at most one below its largest score later on.  (Its probabilities
// then begin at 2^-4, and their products with the least values that a cache holds,
// 2^-121, are still normal numbers.)
constexpr float kAbove = 4.f;
constexpr float kNoKey = -3.402823466e38f;  // reference of a row without keys (so that masked scores weigh 0)

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
    int32_t row_blocks, splits, split_tiles, own;  // own: rows of a wave
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

// A lane's offsets in a block.
template <int D>
struct Lane {
    uint32_t kc, ke, vc, ve;
    __device__ __forceinline__ Lane() {
        const uint32_t n = lane_id() & 15, g = lane_id() >> 4;
        kc = n * (D / 2) + g * (D / 8);
        ke = 8 * D + n * (D / 32) + g * (D / 4) / 32;
        vc = lane_id() * (D / 8);
        ve = 8 * D + (g * (D / 32) + n * (D / 16) / 32) * 4;
    }
};

// Loads from global memory to LDS: lane l's bytes land at lds + 16 l (or 4 l),
// lds the same for the wave (in m0).  From inline assembly, so that the compiler
// does not put a wait for all of them in front of every LDS read; the kernel
// waits for a tile itself.  The hardware wants a wait state between m0's write
// and the load, which the compiler does not put in front of assembly (nor the
// five that an address in scalar registers would need after a v_readfirstlane:
// the addresses here are in vector registers).
// ONCE: past the caches.
template <bool ONCE>
__device__ __forceinline__ void to_lds16(const char* at, uint32_t lds) {
    if constexpr (ONCE)
        asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %0, off nt" ::"v"(at), "{m0}"(lds) : "memory");
    else
        asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(at), "{m0}"(lds) : "memory");
}
template <bool ONCE>
__device__ __forceinline__ void to_lds4(const char* at, uint32_t lds) {
    if constexpr (ONCE)
        asm volatile("s_nop 0\n\tglobal_load_lds_dword %0, off nt" ::"v"(at), "{m0}"(lds) : "memory");
    else
        asm volatile("s_nop 0\n\tglobal_load_lds_dword %0, off" ::"v"(at), "{m0}"(lds) : "memory");
}
template <int N>
__device__ __forceinline__ void wait_loads() {  // all but the N last ones
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
__device__ __forceinline__ void wait_lds_reads() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

// A tile in LDS: K codes of its blocks, V codes, then the exponents of K's two
// blocks and of V's.
template <int D>
struct Slot {
    static constexpr int kCodes = 2 * quant::code_bytes(D), kBytes = 2 * kCodes + 256;
    static constexpr int kLoads = (D == 128 ? 4 : 2) + 1;
};

// The unit-th (sequence, piece).  Pieces behind a sequence's end are left out
// where batches are small enough to count the others: they would take the places
// of those that work.
__device__ __forceinline__ bool piece_at(const Args& a, int unit, int& b, int& split) {
    if (a.splits == 1 || a.batch > 4 * kWave) {
        split = unit / a.batch;
        b = unit % a.batch;
        return split < a.splits;
    }
    int before = 0;
    for (int b0 = 0; b0 < a.batch; b0 += kWave) {
        const int i = b0 + lane_id();
        const int tiles = i < a.batch ? (min(max(a.ctx[i], 0), a.max_ctx) + kTile - 1) / kTile : 0;
        const int pieces = i < a.batch ? max(1, min((tiles + a.split_tiles - 1) / a.split_tiles, a.splits)) : 0;
        const int run = before + (int)wave_scan_dpp((uint32_t)pieces);
        const uint64_t past = __ballot(run > unit);
        if (past) {
            const int k = __ffsll((unsigned long long)past) - 1;
            b = b0 + k;
            split = unit - (__builtin_amdgcn_readlane(run, k) - __builtin_amdgcn_readlane(pieces, k));
            return true;
        }
        before = __builtin_amdgcn_readlane(run, kWave - 1);
    }
    return false;
}

// What a lane holds of a tile's K, or of its V: of two blocks the codes, and
// exponents.
template <int D>
struct Half {
    uint32_t code[2][D / 32], exp[2];
    __device__ __forceinline__ void load_k(const Lane<D>& at, const char* k0, const char* k1) {
        load_words<D>(code[0], k0 + at.kc);
        load_words<D>(code[1], k1 + at.kc);
        exp[0] = (uint8_t)k0[at.ke];
        exp[1] = (uint8_t)k1[at.ke];
    }
    __device__ __forceinline__ void load_v(const Lane<D>& at, const char* v0, const char* v1) {
        load_words<D>(code[0], v0 + at.vc);
        load_words<D>(code[1], v1 + at.vc);
        exp[0] = *reinterpret_cast<const uint32_t*>(v0 + at.ve);
        exp[1] = *reinterpret_cast<const uint32_t*>(v1 + at.ve);
    }
};

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

// The larger one of two below the largest number, as one instruction: fmaxf
// first makes NaN operands quiet.  (Of a number and a NaN the number.)
__device__ __forceinline__ float larger(float x, float y) { return __builtin_amdgcn_fmed3f(x, y, 3.402823466e38f); }

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

// The same of one exponent of K, whose group then is NaN in every product.
__device__ __forceinline__ uint32_t odd_as_nan(uint32_t e) { return e > (uint32_t)quant::kMostExp ? 255u : e; }

// The scale of byte B of w: the conversions read bits 23 .. 30 of it only.
template <int B>
__device__ __forceinline__ float scale_of(uint32_t w) {
    return __uint_as_float(B == 3 ? w >> 1 : w << (23 - 8 * B));
}

// Whether queries are kept in LDS, as they do not fit registers.
template <bool F32, int R>
constexpr bool queries_in_lds() {
    return !F32 && R > 2;
}

// R blocks of 16 query rows per wave.  The waves of a workgroup share their rows
// and take the tiles in turn; ROWS: two by two of them, on two sets of rows.
template <bool F32, int D, int R, bool ROWS>
__global__ __launch_bounds__(kThreads, F32 || R > 1 ? 2 : 4) void quant_attn_kernel(Args a) {
    constexpr int NQ = F32 ? 3 : 1, NP = F32 ? 3 : ROWS ? 1 : 2;  // bf16 per query value and per probability
    constexpr int STEPS = D / 32, PER = D / 16, OWN = 16 * R;     // rows of a wave
    constexpr int SETS = ROWS ? 2 : 1, STRIDE = kWaves / SETS;    // of rows; waves on each
    constexpr bool LDS_Q = queries_in_lds<F32, R>();
    using T = std::conditional_t<F32, float, uint16_t>;
    constexpr int RING = 2;       // tiles on their way per wave (four workgroups fill a CU's LDS)
    constexpr bool ONCE = R == 1;  // (with one row block nobody else reads them)
    constexpr int LDS = std::max(ROWS ? SETS * R * STEPS * kWave * 16 : kWaves * RING * Slot<D>::kBytes,
                                 kWaves * 16 * (D + 4) * 4);
    __shared__ __align__(16) char s_mem[LDS];
    __shared__ float s_m[kWaves][16], s_l[kWaves][16];
    __shared__ int s_pos[SETS][OWN];

    const int lane = lane_id(), n = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int set = wave % SETS;
    // blocks go round the eight XCDs.  ROWS: those of one head, which share its
    // keys, to one of them where there are eight heads, and first pieces, which are
    // whole, before last ones; else the heads of a stretch of positions, which lie
    // side by side in the pool
    int x = blockIdx.x, head, split, rb, b;
    if constexpr (ROWS) {
        head = x % a.hkv;
        x /= a.hkv;
        rb = x % a.row_blocks;
        x /= a.row_blocks;
        b = x % a.batch;
        split = x / a.batch;
    } else {
        const int xcd = x % 8;
        x /= 8;
        rb = x % a.row_blocks;
        x /= a.row_blocks;
        head = x % a.hkv;
        const int unit = x / a.hkv * 8 + xcd;
        if (!piece_at(a, unit, b, split)) return;
    }

    const Seq s = sequence(a, b);
    if (s.odd && rb == 0 && split == 0 && head == 0 && threadIdx.x == 0) raise_flag(a.flags, PRESTO_FLAG_BAD_SEQ);
    const int r0 = (rb * SETS + set) * OWN;  // of the sequence's rows (token, head of the group)
    if (rb * SETS * OWN / a.group >= s.n) return;
    const int i0 = r0 / a.group, i1 = min((r0 + OWN - 1) / a.group, s.n - 1);  // (i0 > i1: a set without rows)
    const Tiles t = tiles_of(a, s.first + i0, s.first + i1);
    const int u0 = split * a.split_tiles, u1 = i0 > i1 ? 0 : min(u0 + a.split_tiles, t.count);
    if (SETS == 1 && split > 0 && u0 >= u1) return;  // (the merge knows)
    const int u_wave = u0 + wave / SETS;

    // this lane's rows: positions (-1: none; by every wave of the set) and queries
    bf16x8* s_q = reinterpret_cast<bf16x8*>(s_mem) + set * R * STEPS * kWave;
    bf16x8 qf[LDS_Q ? 1 : R][NQ][STEPS];
#pragma unroll
    for (int j = 0; j < R; ++j) {
        const int r = r0 + 16 * j + n, i = r / a.group;
        s_pos[set][16 * j + n] = i < s.n ? s.first + i : -1;
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
            } else if constexpr (LDS_Q) {  // (by every wave of the set: the same)
                s_q[(j * STEPS + st) * kWave + lane] = *reinterpret_cast<const bf16x8*>(q + 8 * st);
            } else {
                qf[j][0][st] = *reinterpret_cast<const bf16x8*>(q + 8 * st);
            }
        }
    }

    float m[R];
    f32x4 l[R], o[R][PER];  // (l: the same four times, from a product with ones)
    bool chosen = false;    // every row of the wave has a reference
#pragma unroll
    for (int j = 0; j < R; ++j) {
        m[j] = kNoKey;
        l[j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int d = 0; d < PER; ++d) o[j][d] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    bool odd_v = false;  // a group of V that is not finite

    // the pages of this wave's next 32 tiles, one block of 16 keys per lane
    int pages = -1;
    auto look_up = [&](int first) {
        const int u = u_wave + (first + (lane >> 1)) * STRIDE;
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
    const int in_page = (1 << a.shift) - 1;
    const int64_t head_at = (int64_t)head * ((1 << a.shift) >> 4) * quant::block_bytes(D);
    auto offset = [&](int page, int tile, int half) -> int64_t {
        return max(page, 0) * a.page_bytes + head_at +
               (((tile * kTile + half * 16) & in_page) >> 4) * quant::block_bytes(D);
    };
    struct Where {
        int tile, p0, p1;
    };
    auto where = [&](int it) {
        Where w;
        w.tile = tile_at(t, u_wave + it * STRIDE);
        w.p0 = __builtin_amdgcn_readlane(pages, 2 * (it & 31));
        w.p1 = __builtin_amdgcn_readlane(pages, 2 * (it & 31) + 1);
        return w;
    };
    const Lane<D> at;
    const int mine = u1 > u_wave ? (u1 - u_wave + STRIDE - 1) / STRIDE : 0;

    // ROWS: the next tile's K is asked for when this one's is used up, its V
    // likewise: one set of registers, and what is on its way has the rest of the
    // step (the last tile asks for itself again: a load that might not be made
    // costs a wait for those that are).  Else, where memory is what counts, tiles come through LDS, two ahead:
    // a lane's registers could not hold as much.
    Half<D> tk, tv;
    Where w, w_next, w_then;
    int64_t f0 = 0, f1 = 0;
    auto next = [&](int it) {
        if ((it & 31) == 0) look_up(it);
        w_next = where(it);
        f0 = offset(w_next.p0, w_next.tile, 0);
        f1 = offset(w_next.p1, w_next.tile, 1);
        tk.load_k(at, a.k + f0, a.k + f1);
    };
    char* ring = s_mem + wave * RING * Slot<D>::kBytes;
    const uint32_t ring_at = (uint32_t)__builtin_amdgcn_readfirstlane(
        (int)(uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)ring);
    auto send = [&](int it) {  // tile `it` on its way
        if ((it & 31) == 0) look_up(it);
        w_then = where(it);
        const char *k0 = a.k, *v0 = a.v, *k1 = a.k, *v1 = a.v;
        const int64_t o0 = offset(w_then.p0, w_then.tile, 0), o1 = offset(w_then.p1, w_then.tile, 1);
        k0 += o0, v0 += o0, k1 += o1, v1 += o1;
        const uint32_t lds = ring_at + (it & 1) * Slot<D>::kBytes;
        constexpr int CODES = quant::code_bytes(D);
        if constexpr (D == 128) {
            // (the four pieces of a K row in an order that turns with the row, so
            // that the lanes' reads spread over the banks)
            const int piece = (lane ^ (lane >> 4)) & 3 | (lane & ~3);
            to_lds16<ONCE>(k0 + piece * 16, lds);
            to_lds16<ONCE>(k1 + piece * 16, lds + CODES);
            to_lds16<ONCE>(v0 + at.vc, lds + 2 * CODES);
            to_lds16<ONCE>(v1 + at.vc, lds + 3 * CODES);
        } else {
            const char *k = lane < 32 ? k0 : k1, *v = lane < 32 ? v0 : v1;
            to_lds16<ONCE>(k + (lane & 31) * 16, lds);
            to_lds16<ONCE>(v + (lane & 31) * 16, lds + 2 * CODES);
        }
        const char *e0 = lane < 16 ? k0 : k1, *e1 = lane < 48 ? v0 : v1;
        to_lds4<ONCE>((lane < 32 ? e0 : e1) + CODES + (lane & (D / 8 - 1)) * 4, lds + 4 * CODES);
    };
    auto take = [&](int it) {
        const char* p = ring + (it & 1) * Slot<D>::kBytes;
        constexpr int CODES = quant::code_bytes(D);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            load_words<D>(tk.code[h], p + h * CODES + (D == 128 ? n * 64 + (g ^ (n >> 2)) * 16 : at.kc));
            load_words<D>(tv.code[h], p + (2 + h) * CODES + at.vc);
            tk.exp[h] = (uint8_t)p[4 * CODES + h * 64 + at.ke - 8 * D];
            tv.exp[h] = *reinterpret_cast<const uint32_t*>(p + 4 * CODES + 128 + h * 64 + at.ve - 8 * D);
        }
    };
    if constexpr (ROWS) {
        if (mine > 0) {
            next(0);
            tv.load_v(at, a.v + f0, a.v + f1);
        }
    } else {
        if (mine > 0) send(0);
        w_next = w_then;
        if (mine > 1) send(1);
    }
    for (int it = 0; it < mine; ++it) {
        w = w_next;
        if constexpr (!ROWS) {
            w_next = w_then;
            if (it + 1 < mine)
                wait_loads<Slot<D>::kLoads>();
            else
                wait_loads<0>();
            take(it);
            wait_lds_reads();
            if (it + 2 < mine) send(it + 2);
        }
        const int j0 = w.tile * kTile;
        const bool whole = j0 + kTile - 1 <= t.pmin &&
                           (a.window == 0 || j0 > t.pmax - a.window || j0 + kTile - 1 < a.sinks) && w.p0 >= 0 &&
                           w.p1 >= 0;
        // scores
        f32x4 sc[R][2];
#pragma unroll
        for (int j = 0; j < R; ++j) sc[j][0] = sc[j][1] = f32x4{0.f, 0.f, 0.f, 0.f};
        const float ks[2] = {scale_of<0>(odd_as_nan(tk.exp[0])), scale_of<0>(odd_as_nan(tk.exp[1]))};
        constexpr int AHEAD = 2;  // reads of queries on their way (more, and registers spill)
        bf16x8 ql[LDS_Q ? AHEAD : 1];
        auto read_q = [&](int i) { return s_q[(i % R * STEPS + i / R) * kWave + lane]; };
        if constexpr (LDS_Q) ql[0] = read_q(0);
#pragma unroll
        for (int st = 0; st < STEPS; ++st) {
            bf16x8 kf[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint32_t c = tk.code[h][st];
                kf[h] = eight(quant::decode2<0>(c, ks[h]), quant::decode2<1>(c, ks[h]), quant::decode2<2>(c, ks[h]),
                              quant::decode2<3>(c, ks[h]));
            }
#pragma unroll
            for (int j = 0; j < R; ++j)
#pragma unroll
                for (int k = NQ - 1; k >= 0; --k) {
                    bf16x8 q;
                    if constexpr (LDS_Q) {
                        const int i = st * R + j;
                        if (i + 1 < STEPS * R) ql[(i + 1) % AHEAD] = read_q(i + 1);
                        __builtin_amdgcn_sched_barrier(0x6);  // (the read stays in front of the products)
                        q = ql[i % AHEAD];
                    } else {
                        q = qf[j][k][st];
                    }
                    sc[j][0] = mma(kf[0], q, sc[j][0]);
                    sc[j][1] = mma(kf[1], q, sc[j][1]);
                }
        }

        __builtin_amdgcn_sched_barrier(0);
        if constexpr (ROWS) next(min(it + 1, mine - 1));

        if (!whole) {
#pragma unroll
            for (int j = 0; j < R; ++j) {
                const int pos = s_pos[set][16 * j + n];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int key = j0 + (i >> 2) * 16 + 4 * g + (i & 3);
                    if (!(sees(a, pos, key) && (i < 4 ? w.p0 : w.p1) >= 0)) sc[j][i >> 2][i & 3] = -INFINITY;
                }
            }
        }
        // probabilities 2^x, x = s c - m.  The largest score is looked for only
        // where one of them reaches 2, which a bit of its exponent tells (or is
        // not finite), or where a row has had no key: rarely after the first
        // tiles.  (A NaN score reaches l, whatever m is.)
        bf16x8 p[R][NP];
        for (bool choose = !chosen;;) {
            if (choose) {
                bool all = true;
#pragma unroll
                for (int j = 0; j < R; ++j) {
                    float top = larger(larger(larger(sc[j][0][0], sc[j][0][1]), larger(sc[j][0][2], sc[j][0][3])),
                                       larger(larger(sc[j][1][0], sc[j][1][1]), larger(sc[j][1][2], sc[j][1][3])));
                    top = fmaxf(top, __shfl_xor(top, 16));
                    top = fmaxf(top, __shfl_xor(top, 32));
                    top = fmaf(top, a.scale, kAbove);
                    if (top > m[j]) {
                        const float f = __builtin_amdgcn_exp2f(m[j] - top);  // (0 where there was no key)
                        m[j] = top;
                        l[j] *= f;
#pragma unroll
                        for (int d = 0; d < PER; ++d) o[j][d] *= f;
                    }
                    all &= m[j] > kNoKey || s_pos[set][16 * j + n] < 0;
                }
                chosen = __all(all);
            }
            u32x4 bits = {0, 0, 0, 0};
#pragma unroll
            for (int j = 0; j < R; ++j) {
                float z[8];
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    z[i] = __builtin_amdgcn_exp2f(fmaf(sc[j][i >> 2][i & 3], a.scale, -m[j]));
                split8<NP>(z, p[j]);
                bits |= __builtin_bit_cast(u32x4, p[j][0]);
            }
            if (choose || !__any((bits[0] | bits[1] | bits[2] | bits[3]) & 0x40004000u)) break;
            choose = true;
        }
        // (the sum is that of the rounded probabilities, as the values' is)
#pragma unroll
        for (int j = 0; j < R; ++j)
#pragma unroll
            for (int k = NP - 1; k >= 0; --k)
                l[j] = mma(eight(0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u), p[j][k], l[j]);

        // values
        uint32_t ve[2] = {tv.exp[0], tv.exp[1]};
        if (!whole) {  // keys that no row sees may be anything
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int key = j0 + (i >> 2) * 16 + 4 * g + (i & 3);
                const bool seen = key <= t.pmax && (key >= t.lo || key < a.sinks) && (i < 4 ? w.p0 : w.p1) >= 0;
                if (!seen) ve[i >> 2] &= ~(255u << (8 * (i & 3)));
            }
        }
        // (bytes above kMostExp are above 127, which few are)
        if (__any((ve[0] | ve[1]) & 0x80808080u) && __any(odd_exps(ve[0]) | odd_exps(ve[1]))) {
            odd_v = true;
            ve[0] = without(ve[0], odd_exps(ve[0]));
            ve[1] = without(ve[1], odd_exps(ve[1]));
        }
        const float vs[8] = {scale_of<0>(ve[0]), scale_of<1>(ve[0]), scale_of<2>(ve[0]), scale_of<3>(ve[0]),
                             scale_of<0>(ve[1]), scale_of<1>(ve[1]), scale_of<2>(ve[1]), scale_of<3>(ve[1])};
        auto pv = [&](auto B) {  // dims 2 B and 2 B + 1 of the lane's
            uint32_t c[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if constexpr (D == 128) {
                    c[i] = quant::decode2<B()>(tv.code[i >> 2][i & 3], vs[i]);
                } else {
                    const uint32_t word = tv.code[i >> 2][(i & 3) >> 1];
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
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (ROWS) tv.load_v(at, a.v + f0, a.v + f1);
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
                    for (int j = 0; j < R; ++j) lost[j] |= sees(a, s_pos[set][16 * j + n], w.tile * kTile + h * 16 + r);
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
    // Eight values of a row (of the sequence's) from dim x0 on: as part of the
    // row, or as its output.
    auto put = [&](int r, int x0, const float (&v)[8], float top, float sum) {
        const int64_t row = (s.row + r / a.group) * a.hkv * a.group + (int64_t)head * a.group + r % a.group;
        if (a.splits > 1) {
            const int64_t part = row * a.splits + split;
            if (x0 == 0) a.part_ml[part] = make_float2(top, sum);
            float4* to = reinterpret_cast<float4*>(a.part_o + part * D + x0);
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
    };

    // the states of the waves on the same rows, joined, 16 rows at a time (in the
    // place of what the loop had in LDS)
    float(*s_o)[16][D + 4] = reinterpret_cast<float(*)[16][D + 4]>(s_mem);
    constexpr int PIECES = D / 8;
#pragma unroll
    for (int j = 0; j < R; ++j) {
        __syncthreads();
        if (g == 0) {
            s_m[wave][n] = m[j];
            s_l[wave][n] = l[j][0];
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int d = 0; d < PER; d += 4)
                *reinterpret_cast<float4*>(&s_o[wave][n][PER * (4 * g + i) + d]) =
                    make_float4(o[j][d][i], o[j][d + 1][i], o[j][d + 2][i], o[j][d + 3][i]);
        __syncthreads();
        for (int e = threadIdx.x; e < SETS * 16 * PIECES; e += kThreads) {
            const int of = e / (16 * PIECES), r = e / PIECES % 16, x0 = e % PIECES * 8;
            const int row = (rb * SETS + of) * OWN + 16 * j + r;
            if (row / a.group >= s.n) continue;
            float most = kNoKey, sum = 0.f, v[8] = {};
#pragma unroll
            for (int k = 0; k < STRIDE; ++k) most = fmaxf(most, s_m[k * SETS + of][r]);
#pragma unroll
            for (int k = 0; k < STRIDE; ++k) {
                const int from = k * SETS + of;
                const float f = __builtin_amdgcn_exp2f(s_m[from][r] - most);
                sum += f * s_l[from][r];
#pragma unroll
                for (int d = 0; d < 8; ++d) v[d] += f * s_o[from][r][x0 + d];
            }
            put(row, x0, v, most, sum);
        }
    }
}

// Joins the splits of a row: a wave per row, a lane per split for the weights and
// per D / 64 dims for the sums, the parts of eight splits on their way at a time.
template <bool F32, int D>
__global__ __launch_bounds__(kThreads) void quant_merge_kernel(Args a) {
    const int lane = lane_id();
    const int hq = a.hkv * a.group;
    const int64_t u = (int64_t)blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int64_t token = u / hq;
    const int h = (int)(u - token * hq);
    const int b = (int)(token / a.max_q), i = (int)(token - (int64_t)b * a.max_q);
    if (b >= a.batch) return;
    const Seq s = sequence(a, b);
    if (i >= s.n) return;
    const int64_t row = (s.row + i) * hq + h;
    // the pieces that the tiles of this row's block make (the first one always is
    // one)
    const int r0 = (i * a.group + h % a.group) / a.own * a.own;
    const Tiles t = tiles_of(a, s.first + r0 / a.group, s.first + min((r0 + a.own - 1) / a.group, s.n - 1));
    const int splits = min(max((t.count + a.split_tiles - 1) / a.split_tiles, 1), a.splits);
    constexpr int N = D / kWave;
    float top = -INFINITY, sum = 0.f, v[N] = {};
    for (int k0 = 0; k0 < splits; k0 += kWave) {
        const int k = k0 + lane;
        const float2 ml = k < splits ? a.part_ml[row * a.splits + k] : make_float2(-INFINITY, 0.f);
        // (a part without keys has no mass, and undefined sums)
        const uint64_t some = __ballot(ml.y != 0.f);
        if (some == 0) continue;
        const float most = fmaxf(top, wave_max_f32_dpp(ml.y != 0.f ? ml.x : -INFINITY));
        const float ref = most == -INFINITY ? 0.f : most;
        const float f = ml.y != 0.f ? __builtin_amdgcn_exp2f(ml.x - ref) : 0.f;
        const float old = top == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(top - ref);
        top = most;
        sum = sum * old + wave_sum_f32_dpp(ml.y != 0.f ? f * ml.y : 0.f);
#pragma unroll
        for (int d = 0; d < N; ++d) v[d] *= old;
        const int end = min(splits - k0, 64 - __clzll((long long)some));
        const float* o = a.part_o + (row * a.splits + k0) * D + lane * N;
        for (int j0 = 0; j0 < end; j0 += 8) {
            float x[8][N];
#pragma unroll
            for (int j = 0; j < 8; ++j)
                __builtin_memcpy(x[j], o + (int64_t)min(j0 + j, end - 1) * D, sizeof(x[j]));
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int at = min(j0 + j, end - 1);
                const bool on = j0 + j < end && (some >> at & 1);
                const float w = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(f), at));
#pragma unroll
                for (int d = 0; d < N; ++d) v[d] += on ? w * x[j][d] : 0.f;
            }
        }
    }
    const float f = sum == 0.f ? 0.f : 1.f / sum;
    if constexpr (F32) {
#pragma unroll
        for (int d = 0; d < N; ++d) static_cast<float*>(a.out)[row * D + lane * N + d] = v[d] * f;
    } else if constexpr (N == 2) {
        static_cast<uint32_t*>(a.out)[(row * D) / 2 + lane] = pack2(v[0] * f, v[1] * f);
    } else {
        static_cast<__bf16*>(a.out)[row * D + lane] = (__bf16)(v[0] * f);
    }
}

}  // namespace qattn
}  // namespace presto

namespace presto_host {

using namespace presto;
using namespace presto::qattn;

QuantPlan quant_plan(const presto_paged_attn_desc* d, presto_dtype dt) {
    QuantPlan p{};
    const int64_t group = d->hq / d->pages.hkv, rows = (int64_t)d->max_q * group, batch = d->pages.batch;
    const bool f32 = dt == PRESTO_DT_F32;
    // (sizes whose products below would not fit 64 bits are more than a launch)
    if (batch * d->max_q >= ((int64_t)1 << 31) || batch * d->max_q * d->hq >= ((int64_t)1 << 31) ||
        d->total_q * d->hq >= ((int64_t)1 << 40))
        return p;
    // Waves on rows of their own from 128 rows on (4 x 32 new tokens on 8192 with 4
    // heads per KV head 41 us, shared 43; 4 x 64 of them 57 and 73; 4 x 16 31 and
    // 28), and 32 rows of a wave from 17 on (4 x 16 28, on 16 rows each 34; 4 x 8
    // 23.2 and 22.6).  fp32 operands take three times the registers.
    p.own = !f32 && rows >= 128;
    p.r = f32 ? 1 : p.own ? 4 : rows > 16 ? 2 : 1;
    const int64_t of_group = (p.own ? 2 : 1) * 16 * p.r;
    p.row_blocks = (rows + of_group - 1) / of_group;
    // the tiles of a row block: the longest, and on average
    int64_t most = ((int64_t)d->max_ctx + kTile - 1) / kTile;
    const int64_t span = 16 * p.r / group + 2;  // tokens of a wave
    if (d->window)
        most = std::min(most, ((int64_t)d->window + span) / kTile + 2 + ((int64_t)d->sinks + kTile - 1) / kTile);
    most = std::max<int64_t>(most, 1);
    // Contexts are cut into pieces of one length, so many that they make one round
    // of workgroups, as many as run at once (half as many decoding 16 x 8192 keys
    // 35.4 us, these 34.6, twice as many 38.2); ragged ones so that there are about
    // that many.
    const int64_t room = (p.own ? 512 : p.r == 1 && !f32 ? 1024 : 512) / (p.row_blocks * d->pages.hkv);
    // No piece is shorter than 16 tiles, or, where those would be less than 256
    // workgroups, so short that they are that many, but of 4 tiles and not more
    // than 16 of them (a sequence of 1024 keys 8.8 us, in pieces of 16 tiles 11.5;
    // of 4096 10.6 and 11.7; of 32768 19.6, in pieces of 8 26); up to 20 tiles are
    // not cut (300 keys 7.1 us, in pieces of 4 9.1; 16 x 600 10.0, of 10 11.4).
    constexpr int64_t kMostSplits = 256;  // (parts that one wave joins)
    const int64_t even = most * batch * p.row_blocks * d->pages.hkv / 256;
    const int64_t least = most <= 20 ? most : std::min<int64_t>(std::max({(int64_t)4, (most + 15) / 16, even}), 16);
    int64_t tiles = most;
    if (room > batch) {
        tiles = (most + room / batch - 1) / (room / batch);
        const int64_t all = d->total_ctx / kTile + batch;
        if (d->total_ctx > 0 && !d->window && all < batch * most) {
            const int64_t pieces = std::max<int64_t>(room - batch / 2, 1);
            tiles = std::min(tiles, (all + pieces - 1) / pieces);
        }
    }
    tiles = std::max(tiles, std::max(least, (most + kMostSplits - 1) / kMostSplits));
    p.splits = (most + tiles - 1) / tiles;
    p.split_tiles = (most + p.splits - 1) / p.splits;
    const int64_t blocks = batch * p.row_blocks * d->pages.hkv;
    p.blocks = p.own ? blocks * p.splits
                     : ((int64_t)d->pages.batch * p.splits + 7) / 8 * 8 * p.row_blocks * d->pages.hkv;
    const int64_t out_rows = d->total_q * d->hq, merge_rows = (int64_t)d->pages.batch * d->max_q * d->hq;
    p.merge_blocks = (merge_rows + kWaves - 1) / kWaves;
    p.fits = p.blocks <= (1 << 23) && p.merge_blocks <= (1 << 23);
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
    a.own = 16 * p.r;
    a.scale = d->scale * 1.4426950408889634f;
    auto run = [&](auto f32, auto dim) {
        const unsigned grid = (unsigned)p.blocks;
        if (p.own)
            quant_attn_kernel<f32(), dim(), f32() ? 1 : 4, !f32()><<<grid, kThreads, 0, stream>>>(a);
        else if (p.r == 2)
            quant_attn_kernel<f32(), dim(), f32() ? 1 : 2, false><<<grid, kThreads, 0, stream>>>(a);
        else
            quant_attn_kernel<f32(), dim(), 1, false><<<grid, kThreads, 0, stream>>>(a);
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
