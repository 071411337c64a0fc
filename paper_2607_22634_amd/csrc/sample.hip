// A token per row of logits: temperature, top-k, top-p, min-p and a draw with
// the caller's uniform number.
//
// All three cuts keep a head of the tokens in order (z descending, id
// ascending), and the draw looks for a running sum in that order: no sort is
// needed, only the places where counts and sums of weights pass given values.
// A workgroup takes a row: one pass for its range, one that counts the tokens
// by value in LDS, and one for the ids of the value that is drawn.  bf16 logits
// have few distinct values: almost every bin of the count holds one, whose
// weight is taken once per bin; where a bin holds several (fp32, and the values
// close to 0 of a wide range) their weights are added up as integers, so that the
// order does not matter, and the bin is looked into again when a border lies in
// it.
#include <algorithm>

#include "common.hpp"
#include "step.hpp"

namespace presto {
namespace sample {

constexpr int kThreads = 1024;
constexpr int kWaves = kThreads / kWave;
constexpr int kBins = 3 * kThreads;
constexpr int kSubBins = 2 * kThreads;
constexpr int kList = kThreads;
constexpr double kRange = 64.0;  // tokens that weigh less than 2^-64 of the largest are none

// 2^-y, y in 0 .. 65, to about 2^-51: the integer part is the exponent, the
// rest, at most a half, enters the series of the exponential.
__device__ __forceinline__ double weight_of(double y) {
    const double n = rint(y), t = (n - y) * 0.6931471805599453094;
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

// The row: z(i) for every i, to f(z, i).
template <typename T, typename F>
__device__ __forceinline__ void for_row(const T* row, int vocab, F f) {
    constexpr int N = 16 / sizeof(T);
    auto one = [&](int i) {
        if constexpr (sizeof(T) == 2)
            f(bf16_to_f(row[i]), i);
        else
            f(row[i], i);
    };
    const int skew = (int)(((uintptr_t)row & 15) / sizeof(T));
    const int head = min(skew ? N - skew : 0, vocab);
    const int pieces = (vocab - head) / N;
    if ((int)threadIdx.x < head) one(threadIdx.x);
    const uint4* body = reinterpret_cast<const uint4*>(row + head);
    constexpr int U = 4;
    for (int p0 = threadIdx.x; p0 < pieces; p0 += U * kThreads) {
        uint4 x[U];
#pragma unroll
        for (int j = 0; j < U; ++j) x[j] = body[min(p0 + j * kThreads, pieces - 1)];
#pragma unroll
        for (int j = 0; j < U; ++j) {
            const int p = p0 + j * kThreads;
            if (p >= pieces) break;
            const uint32_t w[4] = {x[j].x, x[j].y, x[j].z, x[j].w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if constexpr (sizeof(T) == 2) {
                    f(bf16lo(w[i]), head + p * N + 2 * i);
                    f(bf16hi(w[i]), head + p * N + 2 * i + 1);
                } else {
                    f(__uint_as_float(w[i]), head + p * N + i);
                }
            }
        }
    }
    for (int i = head + pieces * N + threadIdx.x; i < vocab; i += kThreads) one(i);
}

// Values by 8 bits of mantissa, those near 0 together: a falling function of z.
struct Bins {
    uint32_t thr;   // key (16 bits) of the least magnitude that has bins of its own
    uint32_t nthr;  // of its negative
    int top;        // of the row's maximum
    float near;     // that magnitude

    static __device__ __forceinline__ uint32_t key16(float z) { return ord32(z) >> 16; }
    __device__ __forceinline__ int raw(float z) const {
        const uint32_t k = key16(z);
        if (z >= near) return (int)(0xff80u - k);
        const int mid = (int)(0xff80u - thr) + 1;
        if (z > -near) return mid;
        return mid + 1 + (int)(nthr - k);
    }
    __device__ __forceinline__ void make(float lo, float hi) {
        // nine binades of the largest magnitude: at most 2 * 9 * 128 + 1 bins
        // (an fp32 value of -near's binade shares its key with no other bin)
        const float m = fmaxf(fabsf(lo), fabsf(hi));
        const int e = (int)(__float_as_uint(m) >> 23) - 8;
        near = __uint_as_float((uint32_t)max(e, 1) << 23);
        thr = key16(near);
        nthr = key16(-near);
        top = 0;
        top = raw(hi);
    }
    __device__ __forceinline__ int at(float z) const { return raw(z) - top; }
    __device__ __forceinline__ bool several(int bin) const { return bin + top == (int)(0xff80u - thr) + 1; }
    // the keys (32 bits) between which a bin's values lie
    __device__ __forceinline__ void keys(int bin, uint32_t& klo, uint32_t& khi) const {
        const int r = bin + top, mid = (int)(0xff80u - thr) + 1;
        const uint32_t k0 = r < mid ? 0xff80u - r : nthr - (uint32_t)(r - mid - 1);
        klo = (r == mid ? nthr : k0) << 16;
        khi = (r == mid ? thr : k0) << 16 | 0xffffu;
    }
    // the value of a bin that holds one (bf16)
    __device__ __forceinline__ float value(int bin) const {
        const int r = bin + top, mid = (int)(0xff80u - thr) + 1;
        const uint32_t k = r < mid ? 0xff80u - r : nthr - (uint32_t)(r - mid - 1);
        return unord32(k < 0x8000u ? k << 16 | 0xffffu : k << 16);
    }
};

struct Shared {
    double cw[kBins];     // running sums over the bins, and of counts
    uint32_t cc[kBins];
    uint64_t sw[kSubBins];
    uint32_t sc[kSubBins];
    uint64_t list[kList];
    double wave_w[kWaves];
    uint32_t wave_c[kWaves];
    uint32_t n_list;
    int found;
    uint64_t key;
    int bad;
};

// Inclusive running sums over N bins per thread and the workgroup.
template <int N>
__device__ __forceinline__ void block_scan(double (&w)[N], uint32_t (&c)[N], Shared& s) {
#pragma unroll
    for (int i = 1; i < N; ++i) {
        w[i] += w[i - 1];
        c[i] += c[i - 1];
    }
    double tw = w[N - 1];
    uint32_t tc = c[N - 1];
    const int lane = lane_id(), wave = threadIdx.x / kWave;
    for (int o = 1; o < kWave; o <<= 1) {
        const double a = __shfl_up(tw, o);
        const uint32_t b = __shfl_up(tc, o);
        if (lane >= o) {
            tw += a;
            tc += b;
        }
    }
    __syncthreads();
    if (lane == kWave - 1) {
        s.wave_w[wave] = tw;
        s.wave_c[wave] = tc;
    }
    __syncthreads();
    double bw = 0;
    uint32_t bc = 0;
    for (int i = 0; i < wave; ++i) {
        bw += s.wave_w[i];
        bc += s.wave_c[i];
    }
    const double pw = __shfl_up(tw, 1);
    const uint32_t pc = __shfl_up(tc, 1);
    if (lane > 0) {
        bw += pw;
        bc += pc;
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
        w[i] += bw;
        c[i] += bc;
    }
}

// The first of this thread's N consecutive entries where hit() holds, over the
// workgroup: its index (the same for every thread).
template <int N, typename F>
__device__ __forceinline__ int first_where(Shared& s, F hit) {
    __syncthreads();
    if (threadIdx.x == 0) s.found = 0x7fffffff;
    __syncthreads();
#pragma unroll
    for (int i = N - 1; i >= 0; --i)
        if (hit(i)) atomicMin(&s.found, (int)threadIdx.x * N + i);
    __syncthreads();
    return s.found;
}

// Where a search stands in the order: what the tokens before weigh and count.
struct Place {
    double sum;  // up to and with the place
    float z;     // its value
    uint32_t rank;  // among the tokens of that value, from 0
    uint32_t ties;  // how many there are
};

template <typename T>
__global__ __launch_bounds__(kThreads) void sample_kernel(const T* __restrict__ logits, int64_t rows, int32_t vocab,
                                                          int64_t row_stride, const float* __restrict__ u,
                                                          const float* __restrict__ temperature,
                                                          const int32_t* __restrict__ top_k,
                                                          const float* __restrict__ top_p,
                                                          const float* __restrict__ min_p, int32_t* __restrict__ token,
                                                          float* __restrict__ logprob, int32_t* __restrict__ flags,
                                                          int32_t bits) {
    constexpr bool F32 = sizeof(T) == 4;
    __shared__ Shared s;
    const int tid = threadIdx.x;
    const int64_t r = blockIdx.x;
    const T* row = logits + r * row_stride;

    // the range, the first of the largest, and whether all of it can be used
    uint64_t best = 0;
    float lo = INFINITY;
    bool bad = false;
    for_row<T>(row, vocab, [&](float z, int i) {
        bad |= !(z < INFINITY);
        best = max(best, vocab_key(z, (uint32_t)i));
        if (z > -INFINITY) lo = fminf(lo, z);
    });
    if (tid == 0) {
        s.key = 0;
        s.bad = 0;
    }
    __syncthreads();
    best = wave_max_u64_dpp(best);
    lo = -wave_max_f32_dpp(-lo);
    if (__any(bad) && lane_id() == 0) s.bad = 1;
    if (lane_id() == 0) {
        s.wave_w[tid / kWave] = lo;
        atomicMax((unsigned long long*)&s.key, (unsigned long long)best);
    }
    __syncthreads();
    best = s.key;
    for (int i = 0; i < kWaves; ++i) lo = fminf(lo, (float)s.wave_w[i]);
    const float hi = key_value(best);
    if (s.bad || !(hi > -INFINITY)) {
        if (tid == 0) {
            token[r] = -1;
            if (logprob) logprob[r] = NAN;
            raise_flag(flags, PRESTO_FLAG_NAN_LOGITS);
        }
        return;
    }
    float temp = temperature ? temperature[r] : 1.f;
    const int k = top_k ? top_k[r] : 0;
    if (!(temp > 0.f) || k == 1) {
        if (tid == 0) {
            token[r] = (int32_t)key_id(best);
            if (logprob) logprob[r] = 0.f;
        }
        return;
    }

    // y = (max - z) * rate octaves below the largest
    const double rate = 1.4426950408889634074 / (double)temp;
    auto octaves = [&](float z) { return ((double)hi - (double)z) * rate; };
    // what is not above it weighs nothing (the largest does, however narrow the range)
    const float cut = fminf((float)((double)hi - kRange / rate), nextafterf(hi, -INFINITY));
    auto fixed = [&](float z) { return (uint64_t)rint(ldexp(weight_of(octaves(z)), bits)); };
    auto real = [&](uint64_t w) { return ldexp((double)w, -bits); };
    Bins bins;
    bins.make(fmaxf(lo, cut), hi);

    for (int i = tid; i < kBins; i += kThreads) {
        s.cw[i] = 0.0;
        s.cc[i] = 0;
    }
    __syncthreads();
    for_row<T>(row, vocab, [&](float z, int) {
        if (!(z > cut)) return;
        const int b = bins.at(z);
        atomicAdd(&s.cc[b], 1u);
        if (F32 || bins.several(b)) atomicAdd((unsigned long long*)&s.cw[b], (unsigned long long)fixed(z));
    });
    __syncthreads();
    {
        constexpr int N = kBins / kThreads;
        double w[N];
        uint32_t c[N];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int b = tid * N + i;
            c[i] = s.cc[b];
            w[i] = 0.0;
            if (c[i]) {
                if (F32 || bins.several(b))
                    w[i] = real((uint64_t)__double_as_longlong(s.cw[b]));
                else
                    w[i] = c[i] * weight_of(octaves(bins.value(b)));
            }
        }
        block_scan<N>(w, c, s);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            s.cw[tid * N + i] = w[i];
            s.cc[tid * N + i] = c[i];
        }
        __syncthreads();
    }

    const uint32_t all = s.cc[kBins - 1];

    // The place of the `count`-th token, or (count 0) the first one with which
    // the running sum is `sum` or more; where rounding leaves none, the last.
    auto locate = [&](uint32_t count, double sum) -> Place {
        constexpr int N = kBins / kThreads;
        const int last = first_where<N>(s, [&](int i) { return s.cc[tid * N + i] == all; });
        const int b = min(min(last, kBins - 1), first_where<N>(s, [&](int i) {
                              const int x = tid * N + i;
                              if (count) return s.cc[x] >= count;
                              return s.cw[x] >= sum && s.cc[x] > (x ? s.cc[x - 1] : 0u);
                          }));
        double base = b ? s.cw[b - 1] : 0.0;
        uint32_t cbase = b ? s.cc[b - 1] : 0u, n = s.cc[b] - cbase;
        Place p;
        if (!(F32 || bins.several(b))) {
            p.z = bins.value(b);
        } else {
            // the keys of the bin's values, narrowed down until one is left
            uint32_t klo, khi;
            bins.keys(b, klo, khi);
            for (bool first = true; first || klo != khi; first = false) {
                const int shift = max(0, 32 - __clz((int)(khi - klo)) - 11);
                for (int i = tid; i < kSubBins; i += kThreads) {
                    s.sw[i] = 0;
                    s.sc[i] = 0;
                }
                __syncthreads();
                for_row<T>(row, vocab, [&](float z, int) {
                    const uint32_t key = ord32(z);
                    if (!(z > cut) || key < klo || key > khi || bins.at(z) != b) return;
                    const uint32_t x = (khi - key) >> shift;
                    atomicAdd(&s.sc[x], 1u);
                    atomicAdd((unsigned long long*)&s.sw[x], (unsigned long long)fixed(z));
                });
                __syncthreads();
                constexpr int M = kSubBins / kThreads;
                double w[M];
                uint32_t c[M];
#pragma unroll
                for (int i = 0; i < M; ++i) {
                    w[i] = real(s.sw[tid * M + i]);
                    c[i] = s.sc[tid * M + i];
                }
                block_scan<M>(w, c, s);
#pragma unroll
                for (int i = 0; i < M; ++i) {
                    s.sw[tid * M + i] = (uint64_t)__double_as_longlong(w[i]);
                    s.sc[tid * M + i] = c[i];
                }
                auto upto = [&](int x) { return x < 0 ? 0.0 : __longlong_as_double((long long)s.sw[x]); };
                auto counted = [&](int x) { return x < 0 ? 0u : s.sc[x]; };
                const int end = first_where<M>(s, [&](int i) { return counted(tid * M + i) == n; });
                const int x = min(min(end, kSubBins - 1), first_where<M>(s, [&](int i) {
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
            p.z = unord32(klo);
        }
        const double w = weight_of(octaves(p.z));
        p.ties = n;
        if (count)
            p.rank = count - cbase - 1;
        else
            p.rank = (uint32_t)fmin(fmax(ceil((sum - base) / w) - 1.0, 0.0), (double)(n - 1));
        p.sum = base + (p.rank + 1.0) * w;
        return p;
    };

    double total = s.cw[kBins - 1];
    if (k > 0 && (uint32_t)k < all) total = locate((uint32_t)k, 0.0).sum;
    const float tp = top_p ? top_p[r] : 1.f;
    if (tp < 1.f) {
        const Place p = locate(0, fmax((double)tp, 0.0) * total);
        total = fmin(total, p.sum);
    }
    float mp = min_p ? min_p[r] : 0.f;
    if (mp > 0.f) {
        mp = fminf(mp, 1.f);
        // the tokens of at least mp of the largest's weight
        if (tid == 0) s.key = 0;
        __syncthreads();
        uint64_t sum = 0;
        for_row<T>(row, vocab, [&](float z, int) {
            if (!(z > cut)) return;
            const double w = weight_of(octaves(z));
            if (w >= (double)mp) sum += (uint64_t)rint(ldexp(w, bits));
        });
        for (int o = 32; o; o >>= 1) sum += __shfl_xor((unsigned long long)sum, o);
        if (lane_id() == 0) atomicAdd((unsigned long long*)&s.key, (unsigned long long)sum);
        __syncthreads();
        total = fmin(total, real(s.key));
        __syncthreads();
    }

    float x = u[r];
    x = x > 0.f ? fminf(x, 0x1.fffffep-1f) : 0.f;
    // the first running sum above x * total: the next double or more
    const double target = (double)x * total;
    const Place p = locate(0, target > 0.0 ? __longlong_as_double(__double_as_longlong(target) + 1) : 0x1p-1000);

    // the id of the token of this rank among those of its value
    uint32_t rank = p.rank, ilo = 0, ihi = (uint32_t)vocab - 1, n = p.ties;
    const uint32_t key = ord32(p.z);
    while (n > (uint32_t)kList) {
        const int shift = max(0, 32 - __clz((int)(ihi - ilo)) - 11);
        for (int i = tid; i < kSubBins; i += kThreads) s.sc[i] = 0;
        __syncthreads();
        for_row<T>(row, vocab, [&](float z, int i) {
            if (ord32(z) == key && (uint32_t)i >= ilo && (uint32_t)i <= ihi)
                atomicAdd(&s.sc[((uint32_t)i - ilo) >> shift], 1u);
        });
        __syncthreads();
        constexpr int M = kSubBins / kThreads;
        double w[M] = {};
        uint32_t c[M];
#pragma unroll
        for (int i = 0; i < M; ++i) c[i] = s.sc[tid * M + i];
        block_scan<M>(w, c, s);
        const int at = min(first_where<M>(s, [&](int i) { return c[i] > rank; }), kSubBins - 1);
        if (tid == at / M) s.wave_c[0] = c[at % M];
        __syncthreads();
        n = s.sc[at];
        rank -= s.wave_c[0] - n;
        ilo += (uint32_t)at << shift;
        ihi = min(ihi, ilo + (1u << shift) - 1u);
        __syncthreads();
    }
    if (tid == 0) s.n_list = 0;
    __syncthreads();
    for_row<T>(row, vocab, [&](float z, int i) {
        if (ord32(z) == key && (uint32_t)i >= ilo && (uint32_t)i <= ihi) {
            const uint32_t at = atomicAdd(&s.n_list, 1u);
            if (at < (uint32_t)kList) s.list[at] = (uint64_t)i;
        }
    });
    __syncthreads();
    // (each of the few counts those before it)
    if (tid < (int)n) {
        const uint64_t id = s.list[tid];
        uint32_t before = 0;
        for (uint32_t i = 0; i < n; ++i) before += s.list[i] < id;
        if (before == rank) {
            token[r] = (int32_t)id;
            if (logprob) logprob[r] = (float)(-octaves(p.z) * 0.6931471805599453094 - log(total));
        }
    }
}

}  // namespace sample
}  // namespace presto

namespace presto_host {

presto_status launch_sample(presto_dtype dt, const void* logits, int64_t rows, int32_t vocab, int64_t row_stride,
                            const float* u, const float* temperature, const int32_t* top_k, const float* top_p,
                            const float* min_p, int32_t* token, float* logprob, int32_t* flags, hipStream_t stream) {
    // sums of `vocab` weights of 2^bits at most stay below 2^63
    const int bits = 62 - (32 - __builtin_clz((unsigned)vocab));
    using namespace presto::sample;
    if (dt == PRESTO_DT_BF16)
        sample_kernel<uint16_t><<<(unsigned)rows, kThreads, 0, stream>>>(
            static_cast<const uint16_t*>(logits), rows, vocab, row_stride, u, temperature, top_k, top_p, min_p, token,
            logprob, flags, bits);
    else
        sample_kernel<float><<<(unsigned)rows, kThreads, 0, stream>>>(static_cast<const float*>(logits), rows, vocab,
                                                                      row_stride, u, temperature, top_k, top_p, min_p,
                                                                      token, logprob, flags, bits);
    return check_launch("sample_kernel");
}

}  // namespace presto_host
