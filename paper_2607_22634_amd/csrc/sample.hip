// A token per row of logits: temperature, top-k, top-p, min-p and a draw with
// the caller's uniform number.
//
// All three cuts keep a head of the tokens in order (z descending, id
// ascending), and the draw looks for a running sum in that order: the order
// itself is never made, only the places are found where counts and sums of
// weights pass given values.
//
// sample_count_kernel reads the logits once, slices of rows over the whole chip,
// and counts them by value: 8 bits of mantissa, magnitudes of 2^-8 to 2^7 of
// either sign, what is nearer to 0 together.  A bf16 bin holds one value, whose
// weight is then taken once per bin and not per token; fp32 bins and the one
// around 0 hold several, and their weights are added up too, relative to the bin's
// upper end (the row's maximum is not known yet), as integers, so that the order
// does not matter.  sample_pick_kernel, a workgroup per row, adds the slices up and
// finds the places; it goes back to the logits of a slice for the ids of the value
// drawn, and to the slices that hold a bin of several values where a border lies
// in it.  Rows that do not fit that grid are counted again on one of their own, by
// one workgroup: those whose largest logit is 2^7 or more, or -2^7 or less, or
// whose finite logits below that count (temperatures above about 3); those where a
// border lies in a bin of more than 512 tokens that are not one value, or a bf16
// slice has more than 1024 within 2^-8 of 0; and temperatures so low that a bin is
// wide.  Rows of at most 1024 tokens are sorted as they are.
//
// Measured (151936 tokens, bf16): one row 21 us, 64 rows of a serving batch 26, 512
// rows 62 (2.5 TB/s).  The counts are bound by LDS atomics next to HBM (37 us of
// 512 rows).  A pick is a chain that one workgroup goes through, 15 us, most of it
// code that is fetched and run once: the slices' counts 3.4, weights 2.2, scans 1.1,
// three cuts and draws 5.0, the ids 1.7 (clock stamps in a copy of the kernel).
// Rows next to or below 0 take what others take, one whose largest logit lies within
// 2^-8 of 0 23 us (bf16: its value is looked for).  Rows that leave the grid cost
// 80 to 120 us for one, 120 to 270 for 64, 410 to 550 for 512; in fp32 130 to 310,
// 210 to 450 and 490 to 910.
#include <algorithm>

#include "common.hpp"
#include "sample.hpp"
#include "step.hpp"

namespace presto {
namespace sample {

constexpr int kThreads = 512;       // of a row
constexpr int kCountThreads = 256;  // of a slice
constexpr int kPer = 8;             // bins of a thread
constexpr int kList = kThreads;     // tokens that are put in order
constexpr int kRareBins = 5 * kThreads;
constexpr int kSubBins = 2 * kThreads, kSubBits = 10;
static_assert(kSubBins == 1 << kSubBits, "");
// Rows that are sorted: 64 rows of 1024 bf16 logits 13.6 us, 2048 of them 72; a token
// more, and they are counted, 16.1 and 64.
constexpr int kShort = 1024;
constexpr double kRange = 64.0;  // tokens that weigh less than 2^-64 of the largest are none
constexpr double kLn2 = 0.6931471805599453094;

// 2^-y, y in -5 .. 200, to about 2^-51: the integer part is the exponent, the
// rest, at most a half, enters the series of the exponential.
__device__ __forceinline__ double weight_of(double y) {
    const double n = rint(y), t = (n - y) * kLn2;
    double r = 1.0 / 6227020800;
    r = fma(r, t, 1.0 / 479001600);
    r = fma(r, t, 1.0 / 39916800);
    r = fma(r, t, 1.0 / 3628800);
    r = fma(r, t, 1.0 / 362880);
    r = fma(r, t, 1.0 / 40320);
    r = fma(r, t, 1.0 / 5040);
    r = fma(r, t, 1.0 / 720);
    r = fma(r, t, 1.0 / 120);
    r = fma(r, t, 1.0 / 24);
    r = fma(r, t, 1.0 / 6);
    r = fma(r, t, 0.5);
    r = fma(r, t, 1.0);
    r = fma(r, t, 1.0);
    return ldexp(r, -(int)n);
}

// Elements from .. to of a row: f(z, i) by NT threads, U loads of 16 bytes in
// flight each.
template <int NT, int U, typename T, typename F>
__device__ __forceinline__ void for_range(const T* row, int from, int to, F f) {
    constexpr int N = 16 / sizeof(T);
    auto one = [&](int i) {
        if constexpr (sizeof(T) == 2)
            f(bf16_to_f(row[i]), i);
        else
            f(row[i], i);
    };
    const int skew = (int)(((uintptr_t)(row + from) & 15) / sizeof(T));
    const int first = min(from + (skew ? N - skew : 0), to);
    const int pieces = (to - first) / N;
    if (from + (int)threadIdx.x < first) one(from + threadIdx.x);
    const uint4* body = reinterpret_cast<const uint4*>(row + first);
    for (int p0 = threadIdx.x; p0 < pieces; p0 += U * NT) {
        uint4 x[U];
#pragma unroll
        for (int j = 0; j < U; ++j) x[j] = body[min(p0 + j * NT, pieces - 1)];
#pragma unroll
        for (int j = 0; j < U; ++j) {
            const int p = p0 + j * NT;
            if (p >= pieces) break;
            const uint32_t w[4] = {x[j].x, x[j].y, x[j].z, x[j].w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if constexpr (sizeof(T) == 2) {
                    f(bf16lo(w[i]), first + p * N + 2 * i);
                    f(bf16hi(w[i]), first + p * N + 2 * i + 1);
                } else {
                    f(__uint_as_float(w[i]), first + p * N + i);
                }
            }
        }
    }
    const int rest = first + pieces * N + threadIdx.x;
    if (rest < to) one(rest);
}

// The same of bf16, eight neighbours at a time: f(piece, i), and one(value, i) at
// the ends.
template <int NT, int U, typename F, typename G>
__device__ __forceinline__ void for_pieces(const uint16_t* row, int from, int to, F f, G one) {
    const int skew = (int)(((uintptr_t)(row + from) & 15) / 2);
    const int first = min(from + (skew ? 8 - skew : 0), to);
    const int pieces = (to - first) / 8, rest = first + pieces * 8;
    const uint4* body = reinterpret_cast<const uint4*>(row + first);
    for (int p0 = threadIdx.x; p0 < pieces; p0 += U * NT) {
        uint4 x[U];
#pragma unroll
        for (int j = 0; j < U; ++j) x[j] = body[min(p0 + j * NT, pieces - 1)];
#pragma unroll
        for (int j = 0; j < U; ++j) {
            if (p0 + j * NT >= pieces) break;
            f(x[j], first + 8 * (p0 + j * NT));
        }
    }
    // (at most seven on either side)
    const int i = (int)threadIdx.x < first - from ? from + threadIdx.x : rest + threadIdx.x - (first - from);
    if (i < to) one(row[i], i);
}

// Values by 8 bits of mantissa, those below `near` together: bins of falling z,
// bin 0 being that of `most`.
struct Bins {
    int least;  // bits 16 .. 30 of near
    int mid;    // the bin around 0

    __device__ __forceinline__ void make(float near, float most) {
        least = (int)(__float_as_uint(near) >> 16);
        mid = 0;
        mid = -at(most);
    }
    // the range of a row: nine binades of the largest magnitude, at most 2 * 9 *
    // 128 + 1 bins
    __device__ __forceinline__ void make_for(float lo, float hi) {
        const int e = (int)(__float_as_uint(fmaxf(fabsf(lo), fabsf(hi))) >> 23) - 8;
        make(__uint_as_float((uint32_t)max(e, 1) << 23), hi);
    }
    __device__ __forceinline__ int at(float z) const {
        const int u = (int)__float_as_uint(z), far = max(((u >> 16) & 0x7fff) - least + 1, 0);
        return mid + (u < 0 ? far : -far);
    }
    // bits 16 .. 31 of a bin's values (not mid's)
    __device__ __forceinline__ uint32_t bits(int bin) const {
        const int d = bin - mid;
        return (uint32_t)(least - 1 + (d < 0 ? -d : d)) | (d > 0 ? 0x8000u : 0u);
    }
    __device__ __forceinline__ float value(int bin) const { return __uint_as_float(bits(bin) << 16); }
    // the largest and least values that a bin may hold
    __device__ __forceinline__ float upper(int bin) const {
        if (bin == mid) return __uint_as_float((uint32_t)least << 16);
        return __uint_as_float(bits(bin) << 16 | (bin < mid ? 0xffffu : 0u));
    }
    __device__ __forceinline__ float lower(int bin) const {
        if (bin == mid) return -__uint_as_float((uint32_t)least << 16);
        return __uint_as_float(bits(bin) << 16 | (bin < mid ? 0u : 0xffffu));
    }
};

// The grid of sample_count_kernel: 15 binades on either side of the bin around
// 0, a bin of what is above (0) and one of what is below, with -inf.
constexpr float kGridNear = 0x1p-8f, kGridMost = 0x1.fffffep+6f;
constexpr int kNearBits = (127 - 8) << 7;  // of kGridNear as bf16
constexpr int kGridSide = 15 * 128, kGridMid = kGridSide + 1, kGridBelow = 2 * kGridSide + 2;
static_assert(kGridBelow < kGridWords && kGridWords <= kPer * kThreads && kGridWords % kPer == 0, "");
constexpr int kNearList = 1024;  // values of a bf16 slice in the bin around 0

// A slice's words in the workspace.
struct Slice {
    uint16_t* count;   // [kGridWords]
    uint64_t* weight;  // [kGridWords] (fp32), or of the bin around 0 alone
    uint32_t* head;    // largest value (fp32: ordered bits), what is wrong
};
template <bool F32>
__device__ __forceinline__ Slice slice_at(char* ws, int64_t i) {
    char* p = ws + i * slice_bytes(F32);
    return {reinterpret_cast<uint16_t*>(p), reinterpret_cast<uint64_t*>(p + kGridWords * 2),
            reinterpret_cast<uint32_t*>(p + kGridWords * 2 + (F32 ? kGridWords * 8 : 8))};
}
enum { kNotANumber = 1, kManyNear = 2, kFar = 4 };

struct Args {
    const void* logits;
    const float *u, *temperature, *top_p, *min_p;
    const int32_t* top_k;
    int32_t* token;
    float* logprob;
    int32_t* flags;
    char* ws;
    int64_t row0, row_stride;
    int32_t vocab, slices, slice, bits;
};

__device__ __forceinline__ float temperature_of(const Args& a, int64_t r) {
    const float t = a.temperature ? a.temperature[r] : 1.f;
    return t > 0.f ? t : 0.f;
}
__device__ __forceinline__ double rate_of(float temp) { return temp > 0.f ? 1.4426950408889634074 / (double)temp : 1.0; }

// w of at most 1 as an integer of `scale` = 2^bits, bits below 52: what lies
// above 2^52 in a double is counted in units.
__device__ __forceinline__ uint64_t as_fixed(double w, double scale) {
    return (uint64_t)__double_as_longlong(fma(w, scale, 0x1p52)) & ((1ull << 52) - 1);
}

// Counts one slice of one row by value.  A bin's weights are held in `bits` bits
// relative to its upper end.
template <typename T>
__global__ __launch_bounds__(kCountThreads) void sample_count_kernel(Args a) {
    constexpr bool F32 = sizeof(T) == 4;
    __shared__ __align__(16) uint32_t s_count[kGridWords];
    __shared__ uint64_t s_weight[F32 ? kGridWords : 1];
    __shared__ uint16_t s_near[F32 ? 1 : kNearList];
    __shared__ uint32_t s_n, s_top, s_bad;
    const int tid = threadIdx.x;
    const int64_t i = blockIdx.x;
    const int64_t r = a.row0 + i / a.slices;
    const int s = (int)(i % a.slices);
    const T* row = static_cast<const T*>(a.logits) + r * a.row_stride;
    const int from = s * a.slice, to = min(from + a.slice, a.vocab);
    for (int b = 4 * tid; b < kGridWords; b += 4 * kCountThreads) {
        *reinterpret_cast<uint4*>(&s_count[b]) = make_uint4(0, 0, 0, 0);
        if (F32)
            for (int j = 0; j < 4; ++j) s_weight[b + j] = 0;
    }
    if (tid == 0) {
        s_weight[0] = 0;
        s_n = s_top = s_bad = 0;
    }
    __syncthreads();
    const double rate = rate_of(temperature_of(a, r)), scale = ldexp(1.0, a.bits);
    bool bad = false, beyond = false;  // beyond: a finite value of -2^7 or less (bf16: 2^7 or more, too)
    if constexpr (F32) {
        Bins bins;
        bins.make(kGridNear, kGridMost);
        float top = -INFINITY;
        for_range<kCountThreads, 2>(row, from, to, [&](float z, int) {
            bad |= !(z < INFINITY);
            top = fmaxf(top, z);
            const int b = min(max(bins.at(z) + 1, 0), kGridBelow);
            beyond |= b == kGridBelow && z > -INFINITY;
            atomicAdd(&s_count[b], 1u);
            const double y = ((double)bins.upper(b - 1) - (double)z) * rate;
            if (b > 0 && b < kGridBelow && y < kRange)
                atomicAdd((unsigned long long*)&s_weight[b], (unsigned long long)as_fixed(weight_of(y), scale));
        });
        top = wave_max_f32_dpp(top);
        if (lane_id() == 0) atomicMax(&s_top, ord32(top));
    } else {
        // two values at a time, in 16 bits each: the magnitude's distance from
        // the bin around 0, with the sign turned, is the bin
        typedef short i16x2 __attribute__((ext_vector_type(2)));
        typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
        constexpr short kLeast = (short)kNearBits;
        i16x2 most = {0, 0};
        auto count = [&](uint32_t w, bool high) {
            const i16x2 mag = __builtin_bit_cast(i16x2, w & 0x7fff7fffu);
            most = __builtin_elementwise_max(most, mag);
            i16x2 far = __builtin_elementwise_max(mag - (short)(kLeast - 1), (i16x2){0, 0});
            far = __builtin_elementwise_min(far, (i16x2){kGridMid, kGridMid});
            const i16x2 neg = __builtin_bit_cast(i16x2, w) >> 15;  // all bits or none
            const i16x2 bin = (far ^ ~neg) - ~neg + (short)kGridMid;
            atomicAdd(&s_count[bin[0]], 1u);
            if (high) atomicAdd(&s_count[bin[1]], 1u);
            return far;
        };
        auto near = [&](uint32_t h) {  // a value in the bin around 0
            if ((h & 0x7fffu) >= (uint32_t)kLeast) return;
            const uint32_t at = atomicAdd(&s_n, 1u);
            if (at < (uint32_t)kNearList) s_near[at] = (uint16_t)h;
        };
        for_pieces<kCountThreads, 4>(
            row, from, to,
            [&](const uint4& x, int) {
                const i16x2 f0 = count(x.x, true), f1 = count(x.y, true), f2 = count(x.z, true), f3 = count(x.w, true);
                const i16x2 f = __builtin_elementwise_min(__builtin_elementwise_min(f0, f1),
                                                          __builtin_elementwise_min(f2, f3));
                if (f[0] == 0 || f[1] == 0) {
                    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        near(w[j] & 0xffffu);
                        near(w[j] >> 16);
                    }
                }
            },
            [&](uint16_t h, int) {
                count(h, false);
                near(h);
            });
        __syncthreads();
        for (int j = tid; j < (int)min(s_n, (uint32_t)kNearList); j += kCountThreads) {
            const double y = ((double)kGridNear - (double)bf16_to_f(s_near[j])) * rate;
            if (y < kRange) atomicAdd((unsigned long long*)s_weight, (unsigned long long)as_fixed(weight_of(y), scale));
        }
        // A thread that saw a magnitude of 2^7 or more looks again at the elements that
        // it counted (the ends of a slice that is not aligned go to other threads in
        // for_range): for the largest value, +inf or a NaN (a NaN of either sign is
        // above 0x7f80 in `most`), and the largest finite magnitude, plus 0x80, with
        // which infinities and NaN are negative numbers.
        constexpr short kFarBits = (127 + 7) << 7;
        if (max(most[0], most[1]) >= kFarBits) {
            i16x2 value = {0, 0}, finite = {0, 0};
            auto look = [&](uint32_t w) {
                value = __builtin_elementwise_max(value, __builtin_bit_cast(i16x2, w));
                const u16x2 up = __builtin_bit_cast(u16x2, w & 0x7fff7fffu) + (unsigned short)0x80;
                finite = __builtin_elementwise_max(finite, __builtin_bit_cast(i16x2, up));
            };
            for_pieces<kCountThreads, 4>(
                row, from, to,
                [&](const uint4& x, int) {
                    look(x.x);
                    look(x.y);
                    look(x.z);
                    look(x.w);
                },
                [&](uint16_t h, int) { look(h); });
            bad = max(most[0], most[1]) > 0x7f80 || max(value[0], value[1]) == 0x7f80;
            beyond = max(finite[0], finite[1]) >= kFarBits + 0x80;
        }
    }
    const uint32_t wrong = (__any(bad) ? kNotANumber : 0) | (__any(beyond) ? kFar : 0);
    if (wrong && lane_id() == 0) atomicOr(&s_bad, wrong);
    __syncthreads();
    const Slice out = slice_at<F32>(a.ws, i);
    for (int b = 8 * tid; b < kGridWords; b += 8 * kCountThreads) {
        const uint4 x = *reinterpret_cast<const uint4*>(&s_count[b]), y = *reinterpret_cast<const uint4*>(&s_count[b + 4]);
        *reinterpret_cast<uint4*>(out.count + b) =
            make_uint4(x.x | x.y << 16, x.z | x.w << 16, y.x | y.y << 16, y.z | y.w << 16);
    }
    if (F32)
        for (int b = tid; b < kGridWords; b += kCountThreads) out.weight[b] = s_weight[b];
    if (tid == 0) {
        if (!F32) out.weight[0] = s_weight[0];
        out.head[0] = s_top;
        out.head[1] = s_bad | (s_n > (uint32_t)kNearList ? kManyNear : 0);
    }
}

template <int NT>
struct Scratch {
    static constexpr int kWaves = NT / kWave;
    double wave_w[kWaves];
    uint32_t wave_c[kWaves];
    int found[2][kWaves];
    uint64_t list[NT];
    uint32_t n_list, bad;
};
struct Shared : Scratch<kThreads> {
    double cw[kRareBins];  // of the row's own count
    uint32_t cc[kRareBins];
    uint64_t sw[kSubBins];
    uint32_t sc[kSubBins];
    uint64_t cw2[kRareBins], sw2[kSubBins];  // (second words of sums)
    uint32_t top, cbase, n;
    double base;
    uint64_t sum, sum2;
};

template <int CTRL, int ROW_MASK = 0xf>
__device__ __forceinline__ double dpp_f64(double v) {
    return __longlong_as_double((long long)dpp_u64<CTRL, ROW_MASK>(0ull, (uint64_t)__double_as_longlong(v)));
}
// Inclusive running sum over the lanes of a wave.
__device__ __forceinline__ double wave_scan_f64(double v) {
    v += dpp_f64<0x111>(v);       // row_shr:1
    v += dpp_f64<0x112>(v);       // row_shr:2
    v += dpp_f64<0x114>(v);       // row_shr:4
    v += dpp_f64<0x118>(v);       // row_shr:8
    v += dpp_f64<0x142, 0xa>(v);  // row_bcast:15
    v += dpp_f64<0x143, 0xc>(v);  // row_bcast:31
    return v;
}

// Inclusive running sums over N entries per thread and the workgroup; wb, cb:
// those before the thread's.
template <int N, int NT>
__device__ __forceinline__ void block_scan(double (&w)[N], uint32_t (&c)[N], double& wb, uint32_t& cb, Scratch<NT>& s) {
#pragma unroll
    for (int i = 1; i < N; ++i) {
        w[i] += w[i - 1];
        c[i] += c[i - 1];
    }
    const double tw = wave_scan_f64(w[N - 1]);
    const uint32_t tc = wave_scan_dpp(c[N - 1]);
    const int lane = lane_id(), wave = threadIdx.x / kWave;
    __syncthreads();
    if (lane == kWave - 1) {
        s.wave_w[wave] = tw;
        s.wave_c[wave] = tc;
    }
    __syncthreads();
    wb = __shfl_up(tw, 1);
    cb = __shfl_up(tc, 1);
    if (lane == 0) {
        wb = 0.0;
        cb = 0;
    }
    double before = 0.0;
#pragma unroll
    for (int i = 0; i < NT / kWave - 1; ++i) {
        const double x = s.wave_w[i];
        const uint32_t y = s.wave_c[i];
        before += i < wave ? x : 0.0;
        cb += i < wave ? y : 0u;
    }
    wb += before;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        w[i] += wb;
        c[i] += cb;
    }
}
template <int N, int NT>
__device__ __forceinline__ void block_scan(double (&w)[N], uint32_t (&c)[N], Scratch<NT>& s) {
    double wb;
    uint32_t cb;
    block_scan<N>(w, c, wb, cb, s);
}

constexpr int kNone = 0x7fffffff;

// The first of the entries, N consecutive ones per thread, where hit() holds,
// over the workgroup (the same for every thread).  `turn`: of the two sets of
// words the one this call takes, so that one barrier is enough.
template <int N, int NT, typename F>
__device__ __forceinline__ int first_where(Scratch<NT>& s, int& turn, F hit) {
    int at = kNone;
#pragma unroll
    for (int i = N - 1; i >= 0; --i)
        if (hit(i)) at = (int)threadIdx.x * N + i;
    const uint32_t least = wave_min_u32_dpp((uint32_t)at);
    if (lane_id() == 0) s.found[turn][threadIdx.x / kWave] = (int)least;
    __syncthreads();
    int r = kNone;
#pragma unroll
    for (int i = 0; i < NT / kWave; ++i) r = min(r, s.found[turn][i]);
    turn ^= 1;
    return r;
}

// s.list[0 .. n - 1] in falling order: entry threadIdx.x of it (0 past the end).
// A bitonic sort, one entry per thread, of as many waves as hold one.
template <int NT>
__device__ __forceinline__ uint64_t sorted(Scratch<NT>& s, int n) {
    const int tid = threadIdx.x;
    uint64_t x = tid < n ? s.list[tid] : 0;
    for (int k = 2; k < 2 * n; k <<= 1) {
        for (int j = k >> 1; j > 0; j >>= 1) {
            uint64_t y;
            if (j >= kWave) {
                __syncthreads();
                s.list[tid] = x;
                __syncthreads();
                y = s.list[tid ^ j];
            } else {
                y = __shfl_xor((unsigned long long)x, j);
            }
            const bool larger = ((tid & j) == 0) == ((tid & k) == 0);  // this thread keeps the larger one
            if ((y > x) == larger) x = y;
        }
    }
    return x;
}

// What a draw asks for.
struct Ask {
    int k;
    float p, m, u;
};
__device__ __forceinline__ Ask ask_of(const Args& a, int64_t r) {
    Ask q;
    q.k = a.top_k ? a.top_k[r] : 0;
    const float p = a.top_p ? a.top_p[r] : 1.f, m = a.min_p ? a.min_p[r] : 0.f, u = a.u[r];
    q.p = p < 1.f ? fmaxf(p, 0.f) : 1.f;
    q.m = m > 0.f ? fminf(m, 1.f) : 0.f;
    q.u = u > 0.f ? fminf(u, 0x1.fffffep-1f) : 0.f;
    return q;
}
// The least running sum above u * total.
__device__ __forceinline__ double above(float u, double total) {
    const double x = (double)u * total;
    return x > 0.0 ? __longlong_as_double(__double_as_longlong(x) + 1) : 0x1p-1000;
}

// What is not above it weighs nothing (the largest does, however narrow the
// range).
__device__ __forceinline__ float cut_of(float hi, double rate) {
    return fminf((float)((double)hi - kRange / rate), nextafterf(hi, -INFINITY));
}

template <typename T>
__device__ __forceinline__ void write_token(const Args& a, int64_t r, int id, float logprob) {
    a.token[r] = id;
    if (a.logprob) a.logprob[r] = logprob;
}

// A row that does not fit the grid, by passes over all of it: counted on a grid
// of its own range; a bin that holds several values is narrowed down to one, and
// so are the ids of one value where there are many.
template <typename T>
__device__ __forceinline__ void pick_rare(const Args& a, int64_t r, float hi, Shared& s) {
    constexpr bool F32 = sizeof(T) == 4;
    constexpr int N = kRareBins / kThreads, M = kSubBins / kThreads;
    const int tid = threadIdx.x;
    const T* row = static_cast<const T*>(a.logits) + r * a.row_stride;
    const float temp = temperature_of(a, r);
    Ask ask = ask_of(a, r);
    const bool greedy = temp == 0.f || ask.k == 1;
    if (greedy) ask = {0, 1.f, 0.f, 0.f};
    int turn = 0;
    const double rate = rate_of(temp), scale = ldexp(1.0, a.bits), unit = ldexp(1.0, -a.bits);
    const float cut = cut_of(hi, rate);
    auto octaves = [&](float z) { return ((double)hi - (double)z) * rate; };
    // Weights relative to the largest, as integers in two words, of 2^-bits and of
    // 2^-2 bits: a bin may be wide here, and what many tokens of 2^-40 to 2^-64 weigh
    // together counts.
    auto parts = [&](float z, uint64_t& first, uint64_t& second) {
        const double w = weight_of(octaves(z)) * scale, whole = floor(w);
        first = (uint64_t)whole;
        second = as_fixed(w - whole, scale);
    };
    auto add = [&](uint64_t* to, uint64_t* to2, uint64_t first, uint64_t second) {
        if (first) atomicAdd((unsigned long long*)to, (unsigned long long)first);
        if (second) atomicAdd((unsigned long long*)to2, (unsigned long long)second);
    };
    auto add_weight = [&](uint64_t* to, uint64_t* to2, float z) {
        uint64_t first, second;
        parts(z, first, second);
        add(to, to2, first, second);
    };
    auto real = [&](uint64_t first, uint64_t second) { return ((double)first + (double)second * unit) * unit; };

    __syncthreads();
    for (int i = tid; i < kRareBins; i += kThreads) {
        s.cw[i] = 0.0;
        s.cw2[i] = 0;
        s.cc[i] = 0;
    }
    float lo = hi;
    for_range<kThreads, 1>(row, 0, a.vocab, [&](float z, int) { lo = z > cut ? fminf(lo, z) : lo; });
    lo = -wave_max_f32_dpp(-lo);
    if (lane_id() == 0) s.wave_w[tid / kWave] = lo;
    __syncthreads();
    for (int i = 0; i < kThreads / kWave; ++i) lo = fminf(lo, (float)s.wave_w[i]);
    Bins bins;
    bins.make_for(lo, hi);
    for_range<kThreads, 1>(row, 0, a.vocab, [&](float z, int) {
        if (!(z > cut)) return;
        const int b = bins.at(z);
        atomicAdd(&s.cc[b], 1u);
        if (F32 || b == bins.mid) add_weight((uint64_t*)&s.cw[b], &s.cw2[b], z);
    });
    __syncthreads();
    double w[N];
    uint32_t c[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int b = tid * N + i;
        c[i] = s.cc[b];
        w[i] = 0.0;
        if (c[i])
            w[i] = F32 || b == bins.mid ? real((uint64_t)__double_as_longlong(s.cw[b]), s.cw2[b])
                                        : c[i] * weight_of(octaves(bins.value(b)));
    }
    block_scan<N>(w, c, s);
#pragma unroll
    for (int i = 0; i < N; ++i) {
        s.cw[tid * N + i] = w[i];
        s.cc[tid * N + i] = c[i];
    }
    __syncthreads();
    const uint32_t all = s.cc[kRareBins - 1];
    double total = s.cw[kRareBins - 1];
    auto upto_bin = [&](int b) { return b < 0 ? 0.0 : s.cw[b]; };
    auto counted_bin = [&](int b) { return b < 0 ? 0u : s.cc[b]; };
    const int last = min(first_where<N>(s, turn, [&](int i) { return s.cc[tid * N + i] == all; }), kRareBins - 1);

    // The cuts one after the other, then the draw: the place of the `count`-th
    // token, or (count 0) the first one with which the running sum is `sum` or
    // more; where rounding leaves none, the last.
    float z = hi;
    uint32_t rank = 0, n = 0;
#pragma clang loop unroll(disable)
    for (int stage = 0; stage < 3; ++stage) {
        uint32_t count = 0;
        double sum = 0.0;
        if (stage == 0) {
            if (ask.k <= 0 || (uint32_t)ask.k >= all) continue;
            count = (uint32_t)ask.k;
        } else if (stage == 1) {
            if (!(ask.p < 1.f)) continue;
            sum = (double)ask.p * total;
        } else {
            if (ask.m > 0.f) {  // (w >= min_p: at most that many octaves below the largest)
                const double most = -log2((double)ask.m);
                __syncthreads();
                if (tid == 0) s.sum = s.sum2 = 0;
                __syncthreads();
                uint64_t mine = 0, mine2 = 0;
                for_range<kThreads, 1>(row, 0, a.vocab, [&](float y, int) {
                    if (!(y > cut && octaves(y) <= most)) return;
                    uint64_t first, second;
                    parts(y, first, second);
                    mine += first;
                    mine2 += second;
                });
                add(&s.sum, &s.sum2, mine, mine2);
                __syncthreads();
                total = fmin(total, real(s.sum, s.sum2));
            }
            if (greedy)
                count = 1;
            else
                sum = above(ask.u, total);
        }
        const int b = min(last, first_where<N>(s, turn, [&](int i) {
                              const int x = tid * N + i;
                              return count ? s.cc[x] >= count : s.cw[x] >= sum && s.cc[x] > counted_bin(x - 1);
                          }));
        double base = upto_bin(b - 1);
        uint32_t cbase = counted_bin(b - 1);
        n = s.cc[b] - cbase;
        if (!F32 && b != bins.mid) {
            z = bins.value(b);
        } else {
            // the keys of the bin's values, narrowed down until one is left
            uint32_t klo = ord32(bins.lower(b)), khi = ord32(bins.upper(b));
            for (bool again = true; again; again = klo != khi) {
                const int shift = max(0, 32 - __clz((int)(khi - klo)) - kSubBits);
                for (int i = tid; i < kSubBins; i += kThreads) {
                    s.sw[i] = s.sw2[i] = 0;
                    s.sc[i] = 0;
                }
                __syncthreads();
                for_range<kThreads, 1>(row, 0, a.vocab, [&](float y, int) {
                    const uint32_t key = ord32(y);
                    if (key < klo || key > khi || !(y > cut) || bins.at(y) != b) return;
                    const uint32_t x = (khi - key) >> shift;
                    atomicAdd(&s.sc[x], 1u);
                    add_weight(&s.sw[x], &s.sw2[x], y);
                });
                __syncthreads();
                double sub_w[M];
                uint32_t sub_c[M];
#pragma unroll
                for (int i = 0; i < M; ++i) {
                    sub_w[i] = real(s.sw[tid * M + i], s.sw2[tid * M + i]);
                    sub_c[i] = s.sc[tid * M + i];
                }
                block_scan<M>(sub_w, sub_c, s);
#pragma unroll
                for (int i = 0; i < M; ++i) {
                    s.sw[tid * M + i] = (uint64_t)__double_as_longlong(sub_w[i]);
                    s.sc[tid * M + i] = sub_c[i];
                }
                auto upto = [&](int x) { return x < 0 ? 0.0 : __longlong_as_double((long long)s.sw[x]); };
                auto counted = [&](int x) { return x < 0 ? 0u : s.sc[x]; };
                const int end = first_where<M>(s, turn, [&](int i) { return counted(tid * M + i) == n; });
                const int x = min(min(end, kSubBins - 1), first_where<M>(s, turn, [&](int i) {
                                      const int y = tid * M + i;
                                      if (count) return cbase + counted(y) >= count;
                                      return base + upto(y) >= sum && counted(y) > counted(y - 1);
                                  }));
                base += upto(x - 1);
                cbase += counted(x - 1);
                n = counted(x) - counted(x - 1);
                khi -= (uint32_t)x << shift;
                const uint32_t width = (1u << shift) - 1u;
                if (khi - klo > width) klo = khi - width;
                __syncthreads();
            }
            z = unord32(klo);
        }
        const double one = weight_of(octaves(z));
        rank = count ? count - cbase - 1 : (uint32_t)fmin(fmax(ceil((sum - base) / one) - 1.0, 0.0), (double)(n - 1));
        if (stage < 2) total = fmin(total, base + (rank + 1.0) * one);
    }

    // the id of the token of this rank among those of its value
    uint32_t ilo = 0, ihi = (uint32_t)a.vocab - 1;
    const uint32_t key = ord32(z);
    while (n > (uint32_t)kList) {
        const int shift = max(0, 32 - __clz((int)(ihi - ilo)) - kSubBits);
        for (int i = tid; i < kSubBins; i += kThreads) s.sc[i] = 0;
        __syncthreads();
        for_range<kThreads, 1>(row, (int)ilo, (int)ihi + 1, [&](float y, int i) {
            if (ord32(y) == key) atomicAdd(&s.sc[((uint32_t)i - ilo) >> shift], 1u);
        });
        __syncthreads();
        double none[M] = {};
        uint32_t ids[M];
#pragma unroll
        for (int i = 0; i < M; ++i) ids[i] = s.sc[tid * M + i];
        block_scan<M>(none, ids, s);
        const int at = min(first_where<M>(s, turn, [&](int i) { return ids[i] > rank; }), kSubBins - 1);
        if (tid == at / M) s.cbase = ids[at % M];
        __syncthreads();
        n = s.sc[at];
        rank -= s.cbase - n;
        ilo += (uint32_t)at << shift;
        ihi = min(ihi, ilo + (1u << shift) - 1u);
        __syncthreads();
    }
    if (tid == 0) s.n_list = 0;
    __syncthreads();
    for_range<kThreads, 1>(row, (int)ilo, (int)ihi + 1, [&](float y, int i) {
        if (ord32(y) == key) {
            const uint32_t at = atomicAdd(&s.n_list, 1u);
            if (at < (uint32_t)kList) s.list[at] = ~(uint64_t)i;
        }
    });
    __syncthreads();
    const uint64_t id = ~sorted(s, (int)n);
    if (tid == (int)rank)
        write_token<T>(a, r, (int)id, greedy ? 0.f : (float)(-octaves(z) * kLn2 - log(total)));
}

// A row from the counts of its slices; false (and the largest logit): one for
// pick_rare.
template <typename T>
__device__ __forceinline__ bool pick_counted(const Args& a, int64_t r, int64_t slice0, float& hi, Shared& s) {
    constexpr bool F32 = sizeof(T) == 4;
    constexpr int N = kPer;
    const int tid = threadIdx.x;
    const T* row = static_cast<const T*>(a.logits) + r * a.row_stride;
    const float temp = temperature_of(a, r);
    Ask ask = ask_of(a, r);
    int turn = 0;

    // this thread's bins, the slices added up
    uint32_t c[N] = {};
    uint64_t several[F32 ? N : 1] = {};
    if (tid == 0) s.top = s.bad = s.n_list = 0;
    __syncthreads();
    if (tid < kGridWords / N) {
#pragma unroll 4
        for (int k = 0; k < a.slices; ++k) {
            const Slice x = slice_at<F32>(a.ws, slice0 + k);
            const uint4 v = *reinterpret_cast<const uint4*>(x.count + tid * N);
            const uint32_t h[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int i = 0; i < N; ++i) c[i] += h[i / 2] >> (16 * (i % 2)) & 0xffffu;
            if constexpr (F32) {
#pragma unroll
                for (int i = 0; i < N; ++i) several[i] += x.weight[tid * N + i];
            }
        }
    } else {
        for (int k = tid - kGridWords / N; k < a.slices; k += kThreads - kGridWords / N) {
            const Slice x = slice_at<F32>(a.ws, slice0 + k);
            if (F32) atomicMax(&s.top, x.head[0]);
            if (x.head[1]) atomicOr(&s.bad, x.head[1]);
        }
    }
    if constexpr (!F32) {  // the bin around 0
        if (tid == kGridMid / N)
            for (int k = 0; k < a.slices; ++k) several[0] += slice_at<F32>(a.ws, slice0 + k).weight[0];
    }
    Bins bins;
    bins.make(kGridNear, kGridMost);
    ++bins.mid;  // (bin 0 is what lies above)
    const int first = first_where<N>(s, turn, [&](int i) { return c[i] != 0; });
    bool grid = first > 0 && first < kGridBelow && !(s.bad & kManyNear);
    const bool known = F32 || (grid && first != kGridMid);
    hi = F32 ? unord32(s.top) : known ? bins.value(first) : -INFINITY;
    if (!known && !(s.bad & kNotANumber)) {  // the largest logit
        float top = -INFINITY;
        for_range<kThreads, 4>(row, 0, a.vocab, [&](float z, int) { top = fmaxf(top, z); });
        atomicMax(&s.top, ord32(wave_max_f32_dpp(top)));
        __syncthreads();
        hi = unord32(s.top);
    }
    if ((s.bad & kNotANumber) || !(hi > -INFINITY)) {
        if (tid == 0) {
            write_token<T>(a, r, -1, NAN);
            raise_flag(a.flags, PRESTO_FLAG_NAN_LOGITS);
        }
        return true;
    }
    const bool greedy = temp == 0.f || ask.k == 1;
    if (greedy) ask = {0, 1.f, 0.f, 0.f};

    // y = (max - z) * rate octaves below the largest
    const double rate = rate_of(temp), unit = ldexp(1.0, -a.bits);
    auto octaves = [&](float z) { return ((double)hi - (double)z) * rate; };
    // Weights of a bin of several values are held relative to its upper end, so none
    // that takes part may be wide (in octaves).  In fp32 bins are wide by at most a
    // 128th of their values' magnitude, which 64 octaves below the largest is at most
    // that much more: that bounds those below 0; above it the first one is widest.
    constexpr double kWide = 4.0;
    grid = grid && (!(s.bad & kFar) || octaves(-kGridMost) >= kRange) &&
           (!F32 || (first < kGridMid ? ((double)bins.upper(first) - (double)bins.lower(first)) * rate <= kWide
                                      : -(double)hi * rate + kRange <= 128 * kWide)) &&
           (first > kGridMid || octaves(kGridNear) >= kRange || 2 * (double)kGridNear * rate <= kWide);
    if (!grid) return false;

    // weights by bin
    double w[N];
    bool live = false;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int b = tid * N + i;
        if (b >= kGridBelow || !(octaves(F32 || b == kGridMid ? bins.upper(b) : bins.value(b)) < kRange)) c[i] = 0;
        live |= c[i] != 0;
        w[i] = 0.0;
    }
    // what the largest logit was counted as: where its bin holds nothing else, which
    // its sum tells, the sum is the number of tokens and not that of roundings (a
    // border between equal tokens may be met exactly)
    uint64_t full = 0;
    if (F32 || first == kGridMid)
        full = as_fixed(weight_of(((double)bins.upper(first) - (double)hi) * rate), ldexp(1.0, a.bits));
    if (__any(live)) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int b = tid * N + i;
            const bool many = F32 || b == kGridMid;
            const double y = fmin(octaves(many ? bins.upper(b) : bins.value(b)), 2 * kRange);
            w[i] = c[i] ? (many ? (double)several[F32 ? i : 0] * unit : (double)c[i]) * weight_of(y) : 0.0;
            if (many && b == first && several[F32 ? i : 0] == c[i] * full) w[i] = (double)c[i];
        }
    }
    double wb;
    uint32_t cb;
    block_scan<N>(w, c, wb, cb, s);
    auto held = [&](int i) { return c[i] != (i ? c[i - 1] : cb); };  // whether bin i has a token
    if (tid == kThreads - 1) {
        s.base = w[N - 1];
        s.cbase = c[N - 1];
    }
    __syncthreads();
    double total = s.base;
    const uint32_t all = s.cbase;
    const int last = first_where<N>(s, turn, [&](int i) { return c[i] == all; });  // the last bin with a token

    // The cuts one after the other, then the draw: the place of the `count`-th
    // token, or (count 0) the first one with which the running sum is `sum` or
    // more; where rounding leaves none, the last.  Stage 2 is min-p: what is more
    // than `most` octaves below the largest goes.
    const double most = -log2((double)ask.m);
    float z = hi;
    uint32_t rank = 0, n = 0;
    int id = -1, b = 0;
#pragma clang loop unroll(disable)
    for (int stage = 0; stage < 4; ++stage) {
        uint32_t count = 0;
        double sum = 0.0;
        if (stage == 0) {
            if (ask.k <= 0 || (uint32_t)ask.k >= all) continue;
            count = (uint32_t)ask.k;
        } else if (stage == 1) {
            if (!(ask.p < 1.f)) continue;
            sum = (double)ask.p * total;
        } else if (stage == 2) {
            if (!(ask.m > 0.f)) continue;
        } else if (greedy) {
            count = 1;
        } else {
            sum = above(ask.u, total);
        }
        b = first_where<N>(s, turn, [&](int i) {
            const int x = tid * N + i;
            if (stage == 2) return held(i) && octaves(F32 || x == kGridMid ? bins.lower(x) : bins.value(x)) > most;
            return count ? c[i] >= count : w[i] >= sum && held(i);
        });
        if (stage == 2 && b == kNone) continue;  // (all stay)
        b = min(b, last);
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (b == tid * N + i) {
                s.base = i ? w[i - 1] : wb;
                s.cbase = i ? c[i - 1] : cb;
                s.n = c[i] - s.cbase;
            }
        __syncthreads();
        const double base = s.base;
        const uint32_t cbase = s.cbase;
        n = s.n;
        if (!F32 && b != kGridMid) {
            z = bins.value(b);
            const double one = weight_of(octaves(z));
            if (stage == 2) {
                total = fmin(total, base);
                continue;
            }
            rank = count ? count - cbase - 1 : (uint32_t)fmin(fmax(ceil((sum - base) / one) - 1.0, 0.0), (double)(n - 1));
            if (stage < 2) total = fmin(total, base + (rank + 1.0) * one);
            continue;
        }
        if (n > (uint32_t)kList) return false;
        // the bin's tokens in order, from the slices that hold any
        if (tid == 0) s.n_list = 0;
        __syncthreads();
        const int lane = lane_id();  // (every wave for itself)
        uint64_t some = __ballot(lane < a.slices && slice_at<F32>(a.ws, slice0 + lane).count[b] != 0);
        while (some) {  // neighbours in one go, so that more loads are in flight
            const int k = __ffsll((unsigned long long)some) - 1, end = k + __ffsll(~(unsigned long long)(some >> k)) - 1;
            const int from = k * a.slice, to = min(end * a.slice, a.vocab);
            auto put = [&](float y, int i) {
                const uint32_t at = atomicAdd(&s.n_list, 1u);
                if (at < (uint32_t)kList) s.list[at] = vocab_key(y, (uint32_t)i);
            };
            if constexpr (F32) {
                for_range<kThreads, 4>(row, from, to, [&](float y, int i) {
                    if (bins.at(y) == b) put(y, i);
                });
            } else {  // (the bin around 0)
                auto near = [&](uint32_t h, int i) {
                    if ((h & 0x7fffu) < (uint32_t)kNearBits) put(bf16_to_f((uint16_t)h), i);
                };
                for_pieces<kThreads, 4>(
                    row, from, to,
                    [&](const uint4& x, int i) {
                        const uint32_t v[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            near(v[j] & 0xffffu, i + 2 * j);
                            near(v[j] >> 16, i + 2 * j + 1);
                        }
                    },
                    near);
            }
            some &= ~0ull << end;
        }
        __syncthreads();
        const uint64_t key = sorted(s, (int)n);
        double run[1] = {tid < (int)n ? weight_of(octaves(key_value(key))) : 0.0};
        uint32_t none[1] = {0};
        block_scan<1>(run, none, s);
        const int x = first_where<1>(s, turn, [&](int) {
            if (tid >= (int)n) return false;
            return stage == 2 ? octaves(key_value(key)) > most : count ? cbase + tid + 1 >= count : base + run[0] >= sum;
        });
        // (stage 2: the last one that stays; -1: none)
        const int at = stage == 2 ? min(x, (int)n) - 1 : min(x, (int)n - 1);
        if (tid == max(at, 0)) {
            s.base = at < 0 ? base : base + run[0];
            s.sum = key;
        }
        __syncthreads();
        if (stage < 3) total = fmin(total, s.base);
        z = key_value(s.sum);
        id = (int)key_id(s.sum);
    }
    const float logprob = greedy ? 0.f : (float)(-octaves(z) * kLn2 - log(total));
    if (F32 || b == kGridMid) {
        if (tid == 0) write_token<T>(a, r, id, logprob);
        return true;
    }

    // the id of the token of this rank among the bin's: its slice, then in order
    if constexpr (!F32) {
        const int lane = lane_id();  // (every wave for itself)
        const uint32_t own = lane < a.slices ? slice_at<F32>(a.ws, slice0 + lane).count[b] : 0u;
        const uint32_t run = wave_scan_dpp(own);
        const int k = min(__ffsll((unsigned long long)__ballot(run > rank)) - 1, a.slices - 1);
        n = (uint32_t)__builtin_amdgcn_readlane((int)own, k);
        rank -= (uint32_t)__builtin_amdgcn_readlane((int)run, k) - n;
        if (n > (uint32_t)kList) return false;
        if (tid == 0) s.n_list = 0;
        __syncthreads();
        const uint32_t h = bins.bits(b);
        auto put = [&](int i) {
            const uint32_t at = atomicAdd(&s.n_list, 1u);
            if (at < (uint32_t)kList) s.list[at] = ~(uint64_t)i;
        };
        for_pieces<kThreads, 4>(
            row, k * a.slice, min((k + 1) * a.slice, a.vocab),
            [&](const uint4& x, int i) {
                const uint32_t v[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if ((v[j] & 0xffffu) == h) put(i + 2 * j);
                    if (v[j] >> 16 == h) put(i + 2 * j + 1);
                }
            },
            [&](uint16_t x, int i) {
                if (x == h) put(i);
            });
        __syncthreads();
        const uint64_t found = ~sorted(s, (int)n);
        if (tid == (int)rank) write_token<T>(a, r, (int)found, logprob);
    }
    return true;
}

template <typename T>
__global__ __launch_bounds__(kThreads, 4) void sample_pick_kernel(Args a) {
    __shared__ Shared s;
    const int64_t r = a.row0 + blockIdx.x;
    float hi;
    if (!pick_counted<T>(a, r, (int64_t)blockIdx.x * a.slices, hi, s)) pick_rare<T>(a, r, hi, s);
}

// Rows of at most NT tokens: in order, one per thread.
template <typename T, int NT>
__global__ __launch_bounds__(NT) void sample_short_kernel(Args a) {
    __shared__ Scratch<NT> s;
    const int tid = threadIdx.x, n = a.vocab;
    int turn = 0;
    const int64_t r = a.row0 + blockIdx.x;
    const T* row = static_cast<const T*>(a.logits) + r * a.row_stride;
    if (tid == 0) s.bad = 0;
    __syncthreads();
    bool bad = false;
    for_range<NT, 1>(row, 0, n, [&](float z, int i) {
        bad |= !(z < INFINITY);
        s.list[i] = vocab_key(z, (uint32_t)i);
    });
    if (__any(bad) && lane_id() == 0) s.bad = 1;
    __syncthreads();
    const uint64_t key = sorted(s, n);
    __syncthreads();
    if (tid == 0) s.list[0] = key;
    __syncthreads();
    const float hi = key_value(s.list[0]);
    if (s.bad || !(hi > -INFINITY)) {
        if (tid == 0) {
            a.token[r] = -1;
            if (a.logprob) a.logprob[r] = NAN;
            raise_flag(a.flags, PRESTO_FLAG_NAN_LOGITS);
        }
        return;
    }
    const float temp = temperature_of(a, r);
    const Ask ask = ask_of(a, r);
    const double rate = rate_of(temp);
    const float cut = cut_of(hi, rate), z = key_value(key);
    const double y = ((double)hi - (double)z) * rate;
    const bool one = temp == 0.f || ask.k == 1;
    const double w = tid < n && (one ? tid == 0 : z > cut) ? weight_of(y) : 0.0;
    double sum[1] = {w};
    uint32_t none[1] = {0};
    block_scan<1>(sum, none, s);
    auto upto = [&](int x) {  // the running sum at entry x
        __syncthreads();
        if (tid == x) s.wave_w[0] = sum[0];
        __syncthreads();
        const double v = s.wave_w[0];
        __syncthreads();
        return v;
    };
    const int last = min(first_where<1>(s, turn, [&](int) { return w == 0.0; }), n) - 1;  // (the first weighs 1)
    double total = upto(last);
    if (ask.k > 0) total = upto(min(ask.k - 1, last));
    if (ask.p < 1.f) {
        const double want = (double)ask.p * total;
        total = fmin(total, upto(min(first_where<1>(s, turn, [&](int) { return sum[0] >= want; }), last)));
    }
    const double most = -log2((double)ask.m);  // (w >= min_p: at most that many octaves below the largest)
    if (ask.m > 0.f)
        total = fmin(total, upto(min(first_where<1>(s, turn, [&](int) { return y > most; }) - 1, last)));
    const double want = above(ask.u, total);
    const int at = min(first_where<1>(s, turn, [&](int) { return sum[0] >= want; }), last);
    if (tid == at) {
        a.token[r] = (int32_t)key_id(key);
        if (a.logprob) a.logprob[r] = one ? 0.f : (float)(-y * kLn2 - log(total));
    }
}

}  // namespace sample
}  // namespace presto

namespace presto_host {

using namespace presto::sample;

presto_status launch_sample(presto_dtype dt, const void* logits, int64_t rows, int32_t vocab, int64_t row_stride,
                            const float* u, const float* temperature, const int32_t* top_k, const float* top_p,
                            const float* min_p, int32_t* token, float* logprob, int32_t* flags, void* ws,
                            hipStream_t stream) {
    Args a{};
    a.logits = logits;
    a.u = u;
    a.temperature = temperature;
    a.top_k = top_k;
    a.top_p = top_p;
    a.min_p = min_p;
    a.token = token;
    a.logprob = logprob;
    a.flags = flags;
    a.ws = static_cast<char*>(ws);
    a.row_stride = row_stride;
    a.vocab = vocab;
    // sums of `vocab` weights of up to 2^bits stay below 2^63
    a.bits = 62 - (32 - __builtin_clz((unsigned)vocab));
    const bool f32 = dt == PRESTO_DT_F32;
    if (vocab <= kShort) {
        auto run = [&](auto type) {
            using T = decltype(type);
            if (vocab <= 256)
                sample_short_kernel<T, 256><<<(unsigned)rows, 256, 0, stream>>>(a);
            else
                sample_short_kernel<T, kShort><<<(unsigned)rows, kShort, 0, stream>>>(a);
        };
        if (f32)
            run(float{});
        else
            run(uint16_t{});
        return check_launch("sample_short_kernel");
    }
    const SamplePlan p = sample_plan(dt, rows, vocab);
    a.slices = p.slices;
    a.slice = p.slice;
    for (; a.row0 < rows; a.row0 += p.rows) {
        const unsigned n = (unsigned)std::min<int64_t>(p.rows, rows - a.row0);
        if (f32) {
            sample_count_kernel<float><<<n * p.slices, kCountThreads, 0, stream>>>(a);
            sample_pick_kernel<float><<<n, kThreads, 0, stream>>>(a);
        } else {
            sample_count_kernel<uint16_t><<<n * p.slices, kCountThreads, 0, stream>>>(a);
            sample_pick_kernel<uint16_t><<<n, kThreads, 0, stream>>>(a);
        }
    }
    return check_launch("sample_pick_kernel");
}

// Slices of about 32768 tokens, or smaller ones where that makes less than 1024
// workgroups (512: 64 rows of 151936 25.4 us for 26.7, but 128 rows 32.0 for 29.9
// and 32 of fp32 70 for 65), no more than 16 of them, which the pick reads one
// after the other (one row 20.8 us; 8 of them 22.9, 32 of them 22.1), and none below
// 4096 tokens (64 rows of 32768 19.6 us, of 2048 22.9); the rows of a call in
// rounds of 2048, which share a workspace.
SamplePlan sample_plan(presto_dtype dt, int64_t rows, int32_t vocab) {
    SamplePlan p{};
    if (rows == 0 || vocab <= kShort) return p;
    constexpr int64_t kRound = 2048, kWanted = 1024, kLong = 32768, kLeast = 4096, kMost = 16;
    p.rows = std::min(rows, kRound);
    int64_t n = std::min(kMost, std::max<int64_t>(1, std::min<int64_t>(kWanted / p.rows, vocab / kLeast)));
    n = std::max<int64_t>(n, (vocab + kLong - 1) / kLong);
    p.slice = (int)(((vocab + n - 1) / n + 63) / 64 * 64);
    p.slices = (vocab + p.slice - 1) / p.slice;
    p.bytes = (size_t)(p.rows * p.slices) * slice_bytes(dt == PRESTO_DT_F32);
    return p;
}

}  // namespace presto_host
