// Rotary positions, the append that applies them on the way into a paged cache
// (bf16, fp32 or 4 bits), and the way back out of it.
//
// All are bound by memory: a token's rows are read once and written once.  A
// lane takes eight values of a head, x0 = 8 c .. x0 + 7, and makes their
// outputs: own * cos +- partner * sin, the partner half a rotation away (a
// second load, out of L1) or the neighbour.  Its eight cosines and sines depend
// on the token only and serve all heads that the wave takes, so they cost
// little, and no table of them is read.  A head lies in one wave, which reads
// all of it before it writes: rows may be rotated in place.
//
// Measured: 16384 rows of 40 heads of 128 bf16 values, half of them turning, 66 us,
// 5.1 TB/s, what a large copy moves; 528 rows 5.5 us as a call, the kernel's start
// and one round of loads.  Halves of a rot_dim that is no multiple of 16, whose
// partners are read value by value, take 115 us where others take 69.  23627 new tokens (32 + 2 x 8 heads of 128) into a 4-bit
// cache and back out of it 157 us, 4 TB/s: keys and values of a token go through 16
// lanes each with few loads in flight (both in one pass took 182 registers, and a
// fifth longer), and keys are coded three times (below).
#include <algorithm>
#include <type_traits>

#include "common.hpp"
#include "quant.hpp"
#include "step.hpp"

namespace presto {
namespace rope {

// How partners are found: the neighbour; half a rotation away, in whole pieces of
// eight; the same, value by value.
enum Pairs { kNext = 0, kHalf = 1, kHalfOdd = 2 };

struct Turn {
    int32_t rot;  // values of a head that rotate
    float magnitude;
    const uint64_t* steps;
};

// sin and cos of a 64-bit fraction of a turn.  The quarter turn next to it is
// taken out exactly; what is left, at most an eighth, enters the Taylor series:
// to x^9 and x^10 they are off by 2e-9 and less.
__device__ __forceinline__ void turn_sincos(uint64_t a, float& s, float& c) {
    const uint64_t r64 = a + (1ull << 61);
    const uint32_t quarter = (uint32_t)(r64 >> 62);
    const int64_t rest = (int64_t)(r64 & ((1ull << 62) - 1)) - (1ll << 61);
    const float hi = (float)(int32_t)(rest >> 32), lo = (float)(uint32_t)rest;
    const float x = fmaf(hi, 0x1p32f, lo) * 0x1.921fb6p-62f;  // 2 pi / 2^64
    const float y = x * x;
    const float sx = x * fmaf(y, fmaf(y, fmaf(y, fmaf(y, 1.f / 362880, -1.f / 5040), 1.f / 120), -1.f / 6), 1.f);
    const float cx =
        fmaf(y, fmaf(y, fmaf(y, fmaf(y, fmaf(y, -1.f / 3628800, 1.f / 40320), -1.f / 720), 1.f / 24), -0.5f), 1.f);
    const bool odd = quarter & 1;
    s = odd ? cx : sx;
    c = odd ? sx : cx;
    s = quarter & 2 ? -s : s;
    c = (quarter + 1) & 2 ? -c : c;
}

// The largest error of a rotation in 32 bits, relative to its terms |a| and |b|:
// x is off by 1.5e-7 of at most 0.79, sine and cosine with their roundings by less
// than 3e-7, the products, their sum and the magnitude by 2e-7 more.
constexpr float kTurnError = 0x1p-20f;

// The same in 64 bits, to x^15 and x^16 off by 1e-16 and less.
__device__ __forceinline__ void turn_sincos(uint64_t a, double& s, double& c) {
    const uint64_t r64 = a + (1ull << 61);
    const uint32_t quarter = (uint32_t)(r64 >> 62);
    const int64_t rest = (int64_t)(r64 & ((1ull << 62) - 1)) - (1ll << 61);
    const double x = (double)rest * 0x1.921fb54442d18p-62;  // 2 pi / 2^64
    const double y = x * x;
    double u = -1.0 / 1307674368000, v = 1.0 / 20922789888000;
    u = fma(u, y, 1.0 / 6227020800);
    v = fma(v, y, -1.0 / 87178291200);
    u = fma(u, y, -1.0 / 39916800);
    v = fma(v, y, 1.0 / 479001600);
    u = fma(u, y, 1.0 / 362880);
    v = fma(v, y, -1.0 / 3628800);
    u = fma(u, y, -1.0 / 5040);
    v = fma(v, y, 1.0 / 40320);
    u = fma(u, y, 1.0 / 120);
    v = fma(v, y, -1.0 / 720);
    u = fma(u, y, -1.0 / 6);
    v = fma(v, y, 1.0 / 24);
    v = fma(v, y, -0.5);
    const double sx = fma(u * y, x, x), cx = fma(v, y, 1.0);
    const bool odd = quarter & 1;
    s = odd ? cx : sx;
    c = odd ? sx : cx;
    s = quarter & 2 ? -s : s;
    c = (quarter + 1) & 2 ? -c : c;
}

// Eight consecutive values.
template <typename T>
struct Eight;
template <>
struct Eight<uint16_t> {
    uint4 a;
    __device__ __forceinline__ void load(const uint16_t* p) { a = *reinterpret_cast<const uint4*>(p); }
    __device__ __forceinline__ void stream(const uint16_t* p) { a = load_stream16(p); }
    __device__ __forceinline__ void store(uint16_t* p) const { *reinterpret_cast<uint4*>(p) = a; }
    __device__ __forceinline__ void get(float v[8]) const {
        const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = bf16lo(w[i]);
            v[2 * i + 1] = bf16hi(w[i]);
        }
    }
    __device__ __forceinline__ void set(const float v[8]) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const quant::bf16x2 p = {(__bf16)v[2 * i], (__bf16)v[2 * i + 1]};
            w[i] = __builtin_bit_cast(uint32_t, p);
        }
        a = make_uint4(w[0], w[1], w[2], w[3]);
    }
};
template <>
struct Eight<float> {
    uint4 a, b;
    __device__ __forceinline__ void load(const float* p) {
        a = *reinterpret_cast<const uint4*>(p);
        b = *reinterpret_cast<const uint4*>(p + 4);
    }
    __device__ __forceinline__ void stream(const float* p) {
        a = load_stream16(p);
        b = load_stream16(p + 4);
    }
    __device__ __forceinline__ void store(float* p) const {
        *reinterpret_cast<uint4*>(p) = a;
        *reinterpret_cast<uint4*>(p + 4) = b;
    }
    __device__ __forceinline__ void get(float v[8]) const {
        const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(w[i]);
    }
    __device__ __forceinline__ void set(const float v[8]) {
        a = make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
        b = make_uint4(__float_as_uint(v[4]), __float_as_uint(v[5]), __float_as_uint(v[6]), __float_as_uint(v[7]));
    }
};

__device__ __forceinline__ float value(const uint16_t* p) { return bf16_to_f(*p); }
__device__ __forceinline__ float value(const float* p) { return *p; }

// What a lane's eight outputs take of their own values and of their partners.
template <int PAIRS, bool PART, typename F = float>
struct Angles {
    F cs[8], sn[8];
    int rot, x0;

    // (x0 is below the head's length; values from rot on keep their own)
    __device__ __forceinline__ void make(const Turn& t, int64_t pos, int at) {
        rot = t.rot;
        x0 = at;
        constexpr int N = PAIRS == kNext ? 4 : 8;
        F s[N], c[N];
#pragma unroll
        for (int j = 0; j < N; ++j) {
            int i;  // the pair
            if constexpr (PAIRS == kNext) {
                i = x0 / 2 + j;
            } else {
                i = x0 + j;
                if (i >= rot / 2) i -= rot / 2;
            }
            uint64_t step = 0;
            if (!PART || i < rot / 2) step = t.steps[i];
            turn_sincos((uint64_t)pos * step, s[j], c[j]);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int k = PAIRS == kNext ? j / 2 : j;
            const bool first = PAIRS == kNext ? j % 2 == 0 : x0 + j < rot / 2;
            cs[j] = c[k] * t.magnitude;
            sn[j] = (first ? -s[k] : s[k]) * t.magnitude;
        }
    }

    // offset of the lane's partner piece (kHalf)
    __device__ __forceinline__ int partner() const {
        if (PART && x0 >= rot) return 0;
        return x0 < rot / 2 ? rot / 2 : -(rot / 2);
    }

    // (PART: a value from rot on takes itself, whatever its partner holds)
    __device__ __forceinline__ void turned(const float own[8], const float other[8], F out[8]) const {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const F a = own[j], b = PAIRS == kNext ? own[j ^ 1] : other[j];
            const F r = fma(a, cs[j], b * sn[j]);
            out[j] = PART && x0 + j >= rot ? a : r;
        }
    }
    // (2^-140: where the products' own roundings are of the least numbers)
    __device__ __forceinline__ void off(const float own[8], const float other[8], float eps, float out[8]) const {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float b = PAIRS == kNext ? own[j ^ 1] : other[j];
            const float r = fmaf(fabsf(own[j]) + fabsf(b), eps, 0x1p-140f);
            out[j] = PART && x0 + j >= rot ? 0.f : r;
        }
    }
};

// A lane's piece of a head and its partners.
template <typename T, int PAIRS>
struct Piece {
    Eight<T> own, other;
    float odd[PAIRS == kHalfOdd ? 8 : 1];

    template <typename A>
    __device__ __forceinline__ void load(const T* head, const A& a) {
        own.load(head + a.x0);
        if constexpr (PAIRS == kHalf) other.load(head + a.x0 + a.partner());
        if constexpr (PAIRS == kHalfOdd) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int x = a.x0 + j, h = a.rot / 2;
                odd[j] = value(head + (x >= a.rot ? x : x < h ? x + h : x - h));
            }
        }
    }
    template <typename F, typename A>
    __device__ __forceinline__ void turned(const A& a, F out[8]) const {
        float mine[8], theirs[8];
        values(mine, theirs);
        a.turned(mine, theirs, out);
    }
    // and how far the outputs may be off, by eps of their terms
    template <typename A>
    __device__ __forceinline__ void turned(const A& a, float out[8], float eps, float off[8]) const {
        float mine[8], theirs[8];
        values(mine, theirs);
        a.turned(mine, theirs, out);
        a.off(mine, theirs, eps, off);
    }
    __device__ __forceinline__ void values(float mine[8], float theirs[8]) const {
        own.get(mine);
        if constexpr (PAIRS == kHalf) other.get(theirs);
        if constexpr (PAIRS == kHalfOdd) {
#pragma unroll
            for (int j = 0; j < 8; ++j) theirs[j] = odd[j];
        }
    }
};

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;
constexpr int kFlight = 4;  // heads of a lane whose loads are in flight together

// Heads from .. to of one row, src to dst: head h of a row is dim values at
// h * dim.  The wave takes `per` heads at a time, this lane one of them (`mine`;
// lanes past the last whole head are idle).
template <typename T, int PAIRS, bool PART>
__device__ __forceinline__ void rotate_heads(const T* src, T* dst, int dim, int from, int to, int per, int mine,
                                             const Angles<PAIRS, PART>& a) {
    for (int h0 = from; h0 < to; h0 += kFlight * per) {
        Piece<T, PAIRS> p[kFlight];
        if (mine < per) {
#pragma unroll
            for (int j = 0; j < kFlight; ++j) {  // (past the end the last head is read again)
                const int h = min(h0 + j * per + mine, to - 1);
                p[j].load(src + (int64_t)h * dim, a);
            }
#pragma unroll
            for (int j = 0; j < kFlight; ++j) {
                const int h = h0 + j * per + mine;
                if (h >= to) break;
                float v[8];
                p[j].turned(a, v);
                Eight<T> o;
                o.set(v);
                o.store(dst + (int64_t)h * dim + a.x0);
            }
        }
    }
}

// A wave takes heads of one row: `segs` waves share a row.
template <typename T, int PAIRS, bool PART>
__global__ __launch_bounds__(kThreads) void rope_kernel(Turn turn, const T* x, int64_t x_stride, int64_t rows,
                                                        int32_t heads, int32_t dim, const int32_t* __restrict__ positions,
                                                        T* out, int64_t out_stride, int32_t segs, int32_t seg_heads) {
    const int lanes = dim / 8, per = kWave / lanes, mine = lane_id() / lanes, x0 = lane_id() % lanes * 8;
    const int64_t waves = (int64_t)gridDim.x * kWaves;
    for (int64_t u = (int64_t)blockIdx.x * kWaves + threadIdx.x / kWave; u < rows * segs; u += waves) {
        const int64_t row = u / segs;
        const int from = (int)(u - row * segs) * seg_heads, to = min(from + seg_heads, heads);
        Angles<PAIRS, PART> a;
        a.make(turn, positions[row], x0);
        rotate_heads<T, PAIRS, PART>(x + row * x_stride, out + row * out_stride, dim, from, to, per, mine, a);
    }
}

// ---------------------------------------------------------------------------
// the paged cache

struct Cache {
    char *k, *v;
    const int32_t *table, *ctx, *ctx_new, *offsets;
    int32_t* flags;
    int64_t page_bytes, new_rows;
    int32_t batch, max_new, max_pages, num_pages, shift, hkv;
};

// Sequence b's new tokens: their number, the first row and position; false
// where lengths and offsets do not fit.
struct New {
    int64_t m;
    int o, c;
};
__device__ __forceinline__ bool new_tokens(const Cache& a, int b, New& n) {
    n.c = a.ctx[b];
    n.m = (int64_t)a.ctx_new[b] - n.c;
    n.o = a.offsets[b];
    const int64_t o1 = a.offsets[b + 1];
    return !(n.c < 0 || n.m < 0 || n.o < 0 || o1 < n.o || o1 > a.new_rows || n.m > o1 - n.o || n.m > a.max_new ||
             n.c + n.m > (int64_t)a.max_pages << a.shift);
}

// The fp32 next to d towards zero, its last bit set where that is not d itself:
// on the same side of every border between two codes as d.
__device__ __forceinline__ float to_odd(double d) {
    const float f = (float)d;
    if ((double)f == d) return f;
    uint32_t u = __float_as_uint(f);
    if (fabs((double)f) > fabs(d)) --u;
    return __uint_as_float(u | 1u);
}

// Largest magnitude over the four lanes of a group, NaN if one is.
__device__ __forceinline__ float group_top(const float v[8]) {
    uint32_t t = 0;  // (magnitudes are ordered as their bits, NaN last)
#pragma unroll
    for (int i = 0; i < 8; ++i) t = max(t, __float_as_uint(v[i]) & 0x7fffffffu);
    t = max(t, dpp_u32<0xb1>(0u, t));
    t = max(t, dpp_u32<0x4e>(0u, t));
    return __uint_as_float(t);
}

// Eight values' codes and their group's exponent.
struct Coded {
    uint32_t w;
    int e;
    __device__ __forceinline__ void make(const float v[8]) {
        e = quant::group_exp(group_top(v));
        w = quant::encode8(v, e);
    }
    // the same of values that are off by up to off[]; false: that may matter (of a
    // 0 but for its sign), or one is not finite
    __device__ __forceinline__ bool make(const float v[8], const float off[8]) {
        float hi[8], lo[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            hi[i] = fabsf(v[i]) + off[i];
            lo[i] = fmaxf(fabsf(v[i]) - off[i], 0.f);
        }
        e = quant::group_exp(group_top(hi));
        w = quant::encode8(v, e);
        return quant::group_exp(group_top(lo)) == e && quant::encode8(lo, e) == quant::encode8(hi, e);
    }
};

// Eight values of position r of a block (a head's sixteen positions), and by the
// first lane of a group its exponent.
template <int D, bool V>
__device__ __forceinline__ void store_quant(char* block, int r, int x0, const Coded& c) {
    const int e = c.e;
    const uint32_t w = c.w;
    if constexpr (!V) {
        *reinterpret_cast<uint32_t*>(block + quant::k_code_at<D>(r, x0)) = w;
        if (x0 % 32 == 0) block[quant::k_exp_at<D>(r, x0)] = (char)e;
    } else {
        if constexpr (D == 128) {
            *reinterpret_cast<uint32_t*>(block + quant::v_code_at<D>(r, x0)) = w;
        } else {
            *reinterpret_cast<uint16_t*>(block + quant::v_code_at<D>(r, x0)) = (uint16_t)w;
            *reinterpret_cast<uint16_t*>(block + quant::v_code_at<D>(r, x0 + 4)) = (uint16_t)(w >> 16);
        }
        if (x0 % 32 == 0) block[quant::v_exp_at<D>(r, x0)] = (char)e;
    }
}

// Where position pos of head h lies in its page.
template <int D>
__device__ __forceinline__ int64_t quant_block(const Cache& a, int64_t page, int row, int h) {
    return page * a.page_bytes + ((int64_t)h * ((1 << a.shift) >> 4) + (row >> 4)) * quant::block_bytes(D);
}

// A wave takes some of one token's heads: of its queries, keys and values in
// this order, `per` at a time.
template <typename T, int D, bool Q4, int PAIRS, bool PART>
__global__ __launch_bounds__(kThreads) void append_rope_kernel(Turn turn, Cache a, const T* q, int64_t q_stride,
                                                               T* q_out, int64_t q_out_stride, int32_t hq,
                                                               const T* __restrict__ k_new, int64_t k_stride,
                                                               const T* __restrict__ v_new, int64_t v_stride,
                                                               int32_t segs, int32_t seg_heads) {
    constexpr int kLanes = D / 8, kPer = kWave / kLanes;
    const int mine = lane_id() / kLanes, x0 = lane_id() % kLanes * 8;
    const int hkv = a.hkv;
    const int64_t waves = (int64_t)gridDim.x * kWaves, units = (int64_t)a.batch * a.max_new * segs;
    for (int64_t u = (int64_t)blockIdx.x * kWaves + threadIdx.x / kWave; u < units; u += waves) {
        const int64_t token = u / segs;
        const int seg = (int)(u - token * segs);
        const int b = (int)(token / a.max_new), i = (int)(token - (int64_t)b * a.max_new);
        New n;
        if (!new_tokens(a, b, n)) {
            if (i == 0 && seg == 0 && lane_id() == 0) raise_flag(a.flags, PRESTO_FLAG_BAD_SEQ);
            continue;
        }
        if (i >= n.m) continue;
        const int pos = n.c + i, row = pos & ((1 << a.shift) - 1);
        const int64_t src = n.o + i;
        // this wave's heads of [queries; keys; values]
        const int from = seg * seg_heads, to = from + seg_heads;
        Angles<PAIRS, PART> ang;
        if (from < hq + hkv) ang.make(turn, pos, x0);
        if (from < hq)
            rotate_heads<T, PAIRS, PART>(q + src * q_stride, q_out + src * q_out_stride, D, from, min(to, hq), kPer,
                                         mine, ang);
        if (to <= hq) continue;
        const int page = a.table[(int64_t)b * a.max_pages + (pos >> a.shift)];
        if (page < 0 || page >= a.num_pages) {
            if (lane_id() == 0) raise_flag(a.flags, PRESTO_FLAG_BAD_PAGE);
            continue;
        }
        const int k0 = max(from - hq, 0), k1 = min(to - hq, hkv), v0 = max(from - hq - hkv, 0),
                  v1 = min(to - hq - hkv, hkv);
        if constexpr (!Q4) {
            const int64_t at = page * a.page_bytes + (int64_t)row * hkv * D * sizeof(T);
            if (k0 < k1)
                rotate_heads<T, PAIRS, PART>(k_new + src * k_stride, reinterpret_cast<T*>(a.k + at), D, k0, k1, kPer,
                                             mine, ang);
            for (int h = v0 + mine; h < v1; h += kPer) {
                Eight<T> e;
                e.stream(v_new + src * v_stride + (int64_t)h * D + x0);
                e.store(reinterpret_cast<T*>(a.v + at) + (int64_t)h * D + x0);
            }
        } else {
            // Keys are coded as if rotated in 64 bits: in 32 where no border between
            // two codes is near, else (a few thousandths of the tokens) again.
            const float eps = kTurnError * fabsf(turn.magnitude);
            for (int h = k0 + mine; h < k1; h += kPer) {
                Piece<T, PAIRS> p;
                p.load(k_new + src * k_stride + (int64_t)h * D, ang);
                float f[8], off[8];
                p.turned(ang, f, eps, off);
                Coded code;
                if (__any(!code.make(f, off))) {
                    Angles<PAIRS, PART, double> fine;
                    fine.make(turn, pos, x0);
                    double d[8];
                    p.turned(fine, d);
#pragma unroll
                    for (int j = 0; j < 8; ++j) f[j] = to_odd(d[j]);
                    code.make(f);
                }
                store_quant<D, false>(a.k + quant_block<D>(a, page, row, h), row & 15, x0, code);
            }
            for (int h = v0 + mine; h < v1; h += kPer) {
                Eight<T> e;
                e.stream(v_new + src * v_stride + (int64_t)h * D + x0);
                float f[8];
                e.get(f);
                Coded code;
                code.make(f);
                store_quant<D, true>(a.v + quant_block<D>(a, page, row, h), row & 15, x0, code);
            }
        }
    }
}

// Eight values at x0 of position r of a block.
template <int D, bool V>
__device__ __forceinline__ void load_quant(const char* block, int r, int x0, float v[8]) {
    uint32_t w;
    int e;
    if constexpr (!V) {
        w = *reinterpret_cast<const uint32_t*>(block + quant::k_code_at<D>(r, x0));
        e = (uint8_t)block[quant::k_exp_at<D>(r, x0)];
    } else {
        if constexpr (D == 128)
            w = *reinterpret_cast<const uint32_t*>(block + quant::v_code_at<D>(r, x0));
        else
            w = *reinterpret_cast<const uint16_t*>(block + quant::v_code_at<D>(r, x0)) |
                (uint32_t)*reinterpret_cast<const uint16_t*>(block + quant::v_code_at<D>(r, x0 + 4)) << 16;
        e = (uint8_t)block[quant::v_exp_at<D>(r, x0)];
    }
    const float s = quant::exp_scale(e);
    const uint32_t p[4] = {quant::decode2<0>(w, s), quant::decode2<1>(w, s), quant::decode2<2>(w, s),
                           quant::decode2<3>(w, s)};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        v[2 * j] = e > quant::kMostExp ? NAN : bf16lo(p[j]);
        v[2 * j + 1] = e > quant::kMostExp ? NAN : bf16hi(p[j]);
    }
}

// A wave takes one token.
template <typename T, int D, bool Q4>
__global__ __launch_bounds__(kThreads) void read_kv_kernel(Cache a, T* __restrict__ k_out, int64_t k_stride,
                                                           T* __restrict__ v_out, int64_t v_stride) {
    constexpr int kLanes = D / 8, kPer = kWave / kLanes;
    const int mine = lane_id() / kLanes, x0 = lane_id() % kLanes * 8;
    const int64_t waves = (int64_t)gridDim.x * kWaves, units = (int64_t)a.batch * a.max_new;
    for (int64_t u = (int64_t)blockIdx.x * kWaves + threadIdx.x / kWave; u < units; u += waves) {
        const int b = (int)(u / a.max_new), i = (int)(u - (int64_t)b * a.max_new);
        New n;
        if (!new_tokens(a, b, n)) {
            if (i == 0 && lane_id() == 0) raise_flag(a.flags, PRESTO_FLAG_BAD_SEQ);
            continue;
        }
        if (i >= n.m) continue;
        const int pos = n.c + i, row = pos & ((1 << a.shift) - 1);
        const int page = a.table[(int64_t)b * a.max_pages + (pos >> a.shift)];
        if (page < 0 || page >= a.num_pages) {
            if (lane_id() == 0) raise_flag(a.flags, PRESTO_FLAG_BAD_PAGE);
            continue;
        }
        const int64_t dst = n.o + i;
        for (int h = mine; h < a.hkv; h += kPer) {
            if constexpr (Q4) {
                const int64_t at = quant_block<D>(a, page, row, h);
                float f[8];
                Eight<T> e;
                if (k_out) {
                    load_quant<D, false>(a.k + at, row & 15, x0, f);
                    e.set(f);
                    e.store(k_out + dst * k_stride + (int64_t)h * D + x0);
                }
                if (v_out) {
                    load_quant<D, true>(a.v + at, row & 15, x0, f);
                    e.set(f);
                    e.store(v_out + dst * v_stride + (int64_t)h * D + x0);
                }
            } else {
                const int64_t at = page * a.page_bytes + ((int64_t)row * a.hkv + h) * D * sizeof(T);
                Eight<T> e;
                if (k_out) {
                    e.load(reinterpret_cast<const T*>(a.k + at) + x0);
                    e.store(k_out + dst * k_stride + (int64_t)h * D + x0);
                }
                if (v_out) {
                    e.load(reinterpret_cast<const T*>(a.v + at) + x0);
                    e.store(v_out + dst * v_stride + (int64_t)h * D + x0);
                }
            }
        }
    }
}

}  // namespace rope
}  // namespace presto

namespace presto_host {

using namespace presto;
using namespace presto::rope;

namespace {

constexpr int64_t kMostBlocks = 1 << 20;  // (the rest in turns)

// Heads of a row per wave: few rows are cut so that 1024 waves share the work
// (one on each SIMD; of 256 rows of 40 heads of 128 bf16 values 3.8 us, with 2048
// and 512 of them 4.3 and 4.2, with 4096 4.6), as long as a wave has heads for all
// its lanes.
int heads_per_wave(int64_t rows, int heads, int per) {
    const int pieces = (heads + per - 1) / per;
    const int64_t want = std::max<int64_t>(1, std::min<int64_t>(pieces, rows > 0 ? 1024 / rows : 1));
    return (int)((pieces + want - 1) / want) * per;
}

unsigned grid_of(int64_t units) {
    return (unsigned)std::min<int64_t>((units + kWaves - 1) / kWaves, kMostBlocks);
}

Pairs pairs_of(const presto_rope_desc* r) {
    if (r->rot_dim == 0 || r->interleaved) return kNext;
    return r->rot_dim % 16 == 0 ? kHalf : kHalfOdd;
}

// f(pairs, part) with the two as compile-time constants
template <typename F>
void by_pairs(Pairs p, bool part, F f) {
    auto with = [&](auto pairs) {
        if (part)
            f(pairs, std::true_type{});
        else
            f(pairs, std::false_type{});
    };
    if (p == kNext)
        with(std::integral_constant<int, kNext>{});
    else if (p == kHalf)
        with(std::integral_constant<int, kHalf>{});
    else
        with(std::integral_constant<int, kHalfOdd>{});
}

Cache cache_of(const presto_append_desc* d, void* k, void* v, const int32_t* table, const int32_t* ctx,
               const int32_t* ctx_new, const int32_t* offsets, int32_t* flags) {
    const presto_pages_desc& p = d->pages;
    const int unit = p.dt == PRESTO_DT_BF16 ? 2 : p.dt == PRESTO_DT_F32 ? 4 : 1;
    return {static_cast<char*>(k), static_cast<char*>(v), table, ctx, ctx_new, offsets, flags, p.page_stride * unit,
            d->new_rows, p.batch, d->max_new, p.max_pages, p.num_pages, __builtin_ctz((unsigned)p.page_size), p.hkv};
}

template <typename T>
void run_rope(const presto_rope_desc* r, const uint64_t* steps, const void* x, int64_t x_stride, int64_t rows,
              int32_t heads, int32_t dim, const int32_t* positions, void* out, int64_t out_stride, hipStream_t stream) {
    const Turn turn = {r->rot_dim, r->magnitude, steps};
    const int per = heads_per_wave(rows, heads, kWave / (dim / 8)), segs = (heads + per - 1) / per;
    by_pairs(pairs_of(r), r->rot_dim < dim, [&](auto pairs, auto part) {
        rope_kernel<T, pairs(), part()><<<grid_of(rows * segs), kThreads, 0, stream>>>(
            turn, static_cast<const T*>(x), x_stride, rows, heads, dim, positions, static_cast<T*>(out), out_stride,
            segs, per);
    });
}

template <typename T, int D, bool Q4>
void run_append(const presto_append_desc* d, const presto_rope_desc* r, const uint64_t* steps, const Cache& c,
                const void* q, void* q_out, const void* k_new, const void* v_new, hipStream_t stream) {
    const Turn turn = {r->rot_dim, r->magnitude, steps};
    const int64_t tokens = std::min<int64_t>((int64_t)d->pages.batch * d->max_new, d->new_rows);
    const int hq = q ? d->hq : 0, heads = hq + 2 * d->pages.hkv;
    const int per = heads_per_wave(tokens, heads, kWave / (D / 8)), segs = (heads + per - 1) / per;
    const int64_t units = (int64_t)d->pages.batch * d->max_new * segs;
    by_pairs(pairs_of(r), r->rot_dim < D, [&](auto pairs, auto part) {
        append_rope_kernel<T, D, Q4, pairs(), part()><<<grid_of(units), kThreads, 0, stream>>>(
            turn, c, static_cast<const T*>(q), d->q_stride, static_cast<T*>(q_out), d->q_out_stride, hq,
            static_cast<const T*>(k_new), d->k_stride, static_cast<const T*>(v_new), d->v_stride, segs, per);
    });
}

template <typename T, int D>
void run_read(const presto_append_desc* d, const Cache& c, void* k_out, void* v_out, hipStream_t stream) {
    const unsigned grid = grid_of((int64_t)d->pages.batch * d->max_new);
    if (d->pages.dt == PRESTO_DT_FP4)
        read_kv_kernel<T, D, true><<<grid, kThreads, 0, stream>>>(c, static_cast<T*>(k_out), d->k_stride,
                                                                  static_cast<T*>(v_out), d->v_stride);
    else
        read_kv_kernel<T, D, false><<<grid, kThreads, 0, stream>>>(c, static_cast<T*>(k_out), d->k_stride,
                                                                   static_cast<T*>(v_out), d->v_stride);
}

}  // namespace

presto_status launch_rope(const presto_rope_desc* r, const uint64_t* steps, presto_dtype dt, const void* x,
                          int64_t x_stride, int64_t rows, int32_t heads, int32_t dim, const int32_t* positions,
                          void* out, int64_t out_stride, hipStream_t stream) {
    if (dt == PRESTO_DT_BF16)
        run_rope<uint16_t>(r, steps, x, x_stride, rows, heads, dim, positions, out, out_stride, stream);
    else
        run_rope<float>(r, steps, x, x_stride, rows, heads, dim, positions, out, out_stride, stream);
    return check_launch("rope_kernel");
}

presto_status launch_append_rope(const presto_append_desc* d, const presto_rope_desc* r, const uint64_t* steps,
                                 const void* q, const void* k_new, const void* v_new, const int32_t* offsets,
                                 void* q_out, void* k_pages, void* v_pages, const int32_t* table, const int32_t* ctx,
                                 const int32_t* ctx_new, int32_t* flags, hipStream_t stream) {
    const Cache c = cache_of(d, k_pages, v_pages, table, ctx, ctx_new, offsets, flags);
    auto run = [&](auto type, auto dim) {
        using T = decltype(type);
        if (d->pages.dt == PRESTO_DT_FP4)
            run_append<T, dim(), true>(d, r, steps, c, q, q_out, k_new, v_new, stream);
        else
            run_append<T, dim(), false>(d, r, steps, c, q, q_out, k_new, v_new, stream);
    };
    auto with = [&](auto type) {
        if (d->pages.head_dim == 64)
            run(type, std::integral_constant<int, 64>{});
        else
            run(type, std::integral_constant<int, 128>{});
    };
    if (d->dt == PRESTO_DT_BF16)
        with(uint16_t{});
    else
        with(float{});
    return check_launch("append_rope_kernel");
}

presto_status launch_read_kv(const presto_append_desc* d, const void* k_pages, const void* v_pages,
                             const int32_t* table, const int32_t* ctx, const int32_t* ctx_new, const int32_t* offsets,
                             void* k_out, void* v_out, int32_t* flags, hipStream_t stream) {
    const Cache c = cache_of(d, const_cast<void*>(k_pages), const_cast<void*>(v_pages), table, ctx, ctx_new, offsets,
                             flags);
    if (d->dt == PRESTO_DT_BF16)
        d->pages.head_dim == 64 ? run_read<uint16_t, 64>(d, c, k_out, v_out, stream)
                                : run_read<uint16_t, 128>(d, c, k_out, v_out, stream);
    else
        d->pages.head_dim == 64 ? run_read<float, 64>(d, c, k_out, v_out, stream)
                                : run_read<float, 128>(d, c, k_out, v_out, stream);
    return check_launch("read_kv_kernel");
}

}  // namespace presto_host
