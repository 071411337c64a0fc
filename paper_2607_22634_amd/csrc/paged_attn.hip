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
// rows of a workgroup see are one list: the sinks, then the keys from the
// window's start to the last row's position; what lies between is never
// touched, so its pages may have been given back.
#include <math.h>

#include <type_traits>

#include "common.hpp"
#include "paged.hpp"

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
    // partials: the output normalised by the part's own sum [part, rho, D] fp32
    // and (reference in log2 units, sum) [part, rho]; part = (b, g, split), or
    // (g, piece)
    float* part_o;
    float2* part_ml;
    int32_t* flags;
    int64_t q_stride, page_stride;  // elements
    int64_t total_q;
    int32_t batch, hq, hkv, G, max_q, max_ctx, num_pages, max_pages, page_shift;
    int32_t window, sinks;
    int32_t row_blocks, block_rows, splits, split_tiles;
    int32_t order;  // of the row blocks: kByLength, kBySequence, kByGrid
    // pieces > 0: every sequence is cut into pieces of one length, such that the
    // batch has `pieces` of them and one more per sequence at most (n_slots)
    int32_t pieces, n_slots;
    int2* slots;  // [batch] a sequence's first and last piece, counted over the batch
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

// Row block number idx of the batch, counting those that hold rows: its sequence
// and its place from the sequence's end (the last block has the longest key
// range).  kByLength: the last blocks of all sequences, then those before them,
// and so on (batches of up to a wave's lanes); kBySequence: one sequence after
// the other; kByGrid: idx counts `row_blocks` for every sequence, whether it has
// them or not (batches too large to look through).  Counted by grid, blocks
// without rows would lie in between at a fixed stride, and those with rows all
// fall on the same shader engines: four ragged windowed prompts of up to 4026
// tokens (bf16, 32/8 heads of 128) 264 us, 239 counted.
// false: there is no such block.
enum { kByLength, kBySequence, kByGrid };
__device__ __forceinline__ bool find_block(const Args& a, int idx, bool first, int& b, int& rev, Seq& sq) {
    const int lane = lane_id();
    // (a lane's sequence in sq; that of the lane which is asked for at the end)
    auto blocks_of = [&](int bb, bool& bad) {
        if (bb >= a.batch) return 0;
        sq = seq_of(a, bb);
        bad |= sq.bad;
        return (sq.n * a.G + a.block_rows - 1) / a.block_rows;
    };
    auto of_lane = [&](int l) {
        sq.r0 = __builtin_amdgcn_readlane((int)sq.r0, l);
        sq.n = __builtin_amdgcn_readlane(sq.n, l);
        sq.pos0 = __builtin_amdgcn_readlane(sq.pos0, l);
    };
    bool bad = false, found = false;
    b = rev = 0;
    if (a.order == kByLength && a.batch == 1) {
        rev = idx;
        found = idx < blocks_of(0, bad);
    } else if (a.order == kByLength) {
        const int n = blocks_of(lane, bad);
        auto upto = [&](int r) {  // blocks with rev < r
            return __builtin_amdgcn_readlane((int)wave_scan_dpp(min(n, r)), kWave - 1);
        };
        int lo = 0, hi = a.row_blocks;  // upto(lo) <= idx < upto(hi), if any
        found = idx < upto(hi);
        while (found && hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (upto(mid) <= idx)
                lo = mid;
            else
                hi = mid;
        }
        const int j = idx - upto(lo);
        const int incl = (int)wave_scan_dpp(n > lo ? 1 : 0);
        const uint64_t hit = __ballot(incl > j);
        b = uniform(hit ? __ffsll((unsigned long long)hit) - 1 : 0);
        of_lane(b);
        rev = lo;
    } else if (a.order == kBySequence) {
        int base = 0;
        Seq got{};
        for (int b0 = 0; b0 < a.batch && (!found || first); b0 += kWave) {
            const int n = blocks_of(b0 + lane, bad), incl = (int)wave_scan_dpp(n);
            const uint64_t hit = __ballot(base + incl > idx);
            if (hit && !found) {
                const int at = uniform(__ffsll((unsigned long long)hit) - 1);
                of_lane(at);
                got = sq;
                b = b0 + at;
                rev = idx - base - __builtin_amdgcn_readlane(incl - n, at);
                found = true;
            }
            base += __builtin_amdgcn_readlane(incl, kWave - 1);
        }
        sq = got;
    } else {
        b = idx % a.batch;
        rev = idx / a.batch;
        found = rev < blocks_of(b, bad);
        first = rev == 0;
    }
    if (first && __ballot(bad) && lane == 0) raise_flag(a.flags, PRESTO_FLAG_BAD_SEQ);
    b = uniform(b);
    rev = uniform(rev);
    sq.r0 = uniform((int)sq.r0);
    sq.n = uniform(sq.n);
    sq.pos0 = uniform(sq.pos0);
    return found;
}

// Keys that rows at positions p_lo .. p_hi see, [0, sinks) and [lo, hi), as a
// list of n entries: entry v is key v below `head`, and key v + gap from there
// on.  Head and gap are multiples of 16, so that sixteen entries from a
// multiple of 16 lie in one page.
struct Span {
    int lo, hi, head, gap, n;
};
__device__ __forceinline__ Span span_of(const Args& a, int p_lo, int p_hi) {
    Span s;
    s.hi = max(p_hi + 1, 0);
    s.lo = a.window > 0 ? max(max(p_lo, 0) - a.window + 1, 0) : 0;
    const int start = s.lo & ~15, head = (a.sinks + 15) & ~15;
    s.head = head < start ? head : 0;
    s.gap = head < start ? start - head : 0;
    s.n = s.hi - s.gap;
    return s;
}
__device__ __forceinline__ int key_of(const Span& s, int v) { return v < s.head ? v : v + s.gap; }

__device__ __forceinline__ bool sees(const Args& a, int pos, int key) {
    return key <= pos && (a.window == 0 || key > pos - a.window || key < a.sinks);
}

// The kernel's arguments, read again: what a path taken rarely needs would
// otherwise stay in scalar registers over the key loop (prompts 7% slower).
__device__ __forceinline__ const Args& args_again() {
    auto p = (const __attribute__((address_space(4))) Args*)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(p));
    return *(const Args*)p;
}

// What the matrix instructions cannot do: a row that does not see a key whose V
// is not finite still meets it, as 0 * inf.  Only keys that some rows of a
// block see and others do not can do that: the positions of the block's own
// tokens, and as many at the window's start.  Does one of them hold a V that is
// not finite?  (This thread's part of the answer.)
template <bool BF16, int D>
__device__ bool edge_not_finite(const Args& a, int b, int g, int p_lo, int p_hi) {
    constexpr int E = BF16 ? 2 : 4, CPR = D * E / 16;
    const int after = max(p_lo + 1, 0), n_after = max(p_hi + 1 - after, 0);
    const int at_start = max(max(p_lo - a.window + 1, a.sinks), 0);
    const int n_start = a.window > 0 ? max(p_hi - a.window + 1 - at_start, 0) : 0;
    bool found = false;
    for (int i = threadIdx.x; i < (n_after + n_start) * CPR; i += blockDim.x) {
        const int k = i / CPR, key = k < n_after ? after + k : at_start + k - n_after;
        const int page = a.table[(int64_t)b * a.max_pages + (key >> a.page_shift)];
        if (page < 0 || page >= a.num_pages) continue;
        const int64_t row = page * a.page_stride + ((int64_t)(key & ((1 << a.page_shift) - 1)) * a.hkv + g) * D;
        const uint4 u = *reinterpret_cast<const uint4*>(a.vp + row * E + i % CPR * 16);
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
        for (int j = 0; j < 4; ++j) {
            // (an exponent of ones: in fp32, and in the upper and lower bf16)
            found |= (w[j] & 0x7f800000u) == 0x7f800000u || (BF16 && (w[j] & 0x7f80u) == 0x7f80u);
        }
    }
    return found;
}

// One row on its own, by all NT threads: entries v0 .. v1 - 1 of the list, with
// the keys that the row does not see left out of the sums.  A thread scores a
// key of NT, then sums 16 bytes of V over every (NT / CPR)-th of them.  O,
// normalised, in scratch[0 .. D - 1]; (reference, sum) returned.  About 0.2 ms
// per row and 10,000 keys: for caches that hold infinities, not a path to take
// often.
template <int D, int E, int NT>
constexpr int kAloneFloats = D + NT + 2 * NT + 2 * (NT / kWave) + NT / (D * E / 16) * D;

template <bool BF16, int D, int NT>
__device__ float2 row_alone(const Args& a, const Span& sp, int b, int g, int64_t qrow, int head, int pos, int v0,
                            int v1, float* scratch) {
    constexpr int E = BF16 ? 2 : 4, CPR = D * E / 16, EPC = 16 / E;  // values per 16 bytes
    constexpr int LANES = NT / CPR, NW = NT / kWave;
    float* const s_q = scratch;
    int64_t* const s_at = reinterpret_cast<int64_t*>(s_q + D);  // -1: not seen
    float* const s_p = reinterpret_cast<float*>(s_at + NT);
    float* const s_w = s_p + NT;
    float* const s_part = s_w + 2 * NW;  // [LANES][D]
    const int tid = threadIdx.x, wave = tid / kWave, lane = lane_id();
    const int keys = min(v1, sp.n) - v0;
    auto values = [](const char* p, float (&x)[EPC]) {
        const uint4 u = *reinterpret_cast<const uint4*>(p);
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
        for (int j = 0; j < 4; ++j) {
            if constexpr (BF16) {
                x[2 * j] = bf16lo(w[j]);
                x[2 * j + 1] = bf16hi(w[j]);
            } else {
                x[j] = __uint_as_float(w[j]);
            }
        }
    };
    __syncthreads();
    if (tid < CPR) {
        float x[EPC];
        values(a.q + (qrow * a.q_stride + (int64_t)head * D) * E + tid * 16, x);
        for (int j = 0; j < EPC; ++j) s_q[tid * EPC + j] = x[j];
    }
    const int chunk = tid % CPR, part = tid / CPR;
    float acc[EPC], m = -INFINITY, l = 0.f;
    for (int j = 0; j < EPC; ++j) acc[j] = 0.f;
    for (int i0 = 0; i0 < keys; i0 += NT) {
        __syncthreads();
        float s = -INFINITY;
        int64_t at = -1;
        if (i0 + tid < keys) {
            const int key = key_of(sp, v0 + i0 + tid);
            if (sees(a, pos, key)) {
                const int page = a.table[(int64_t)b * a.max_pages + (key >> a.page_shift)];
                if (page >= 0 && page < a.num_pages) {
                    at = (page * a.page_stride + ((int64_t)(key & ((1 << a.page_shift) - 1)) * a.hkv + g) * D) * E;
                    s = 0.f;
                    for (int c = 0; c < CPR; ++c) {
                        float x[EPC];
                        values(a.kp + at + c * 16, x);
                        for (int j = 0; j < EPC; ++j) s = fmaf(s_q[c * EPC + j], x[j], s);
                    }
                    s *= a.scale_log2;
                }
            }
        }
        const float mw = wave_max_f32_dpp(s);
        if (lane == 0) s_w[wave] = mw;
        __syncthreads();
        float mn = m;
        for (int w = 0; w < NW; ++w) mn = fmaxf(mn, s_w[w]);
        const float f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - mn);
        m = mn;
        const float p = at < 0 ? 0.f : __builtin_amdgcn_exp2f(s - (m == -INFINITY ? 0.f : m));
        s_p[tid] = p;
        s_at[tid] = at;
        l = l * f + p;
        if (i0 > 0)
            for (int j = 0; j < EPC; ++j) acc[j] *= f;
        __syncthreads();
        for (int i = part; i < min(NT, keys - i0); i += LANES) {
            if (s_at[i] < 0) continue;
            float x[EPC];
            values(a.vp + s_at[i] + chunk * 16, x);
            for (int j = 0; j < EPC; ++j) acc[j] = fmaf(s_p[i], x[j], acc[j]);
        }
    }
    const float lw = wave_sum_f32_dpp(l);
    if (lane == 0) s_w[NW + wave] = lw;
    for (int j = 0; j < EPC; ++j) s_part[part * D + chunk * EPC + j] = acc[j];
    __syncthreads();
    l = 0.f;
    for (int w = 0; w < NW; ++w) l += s_w[NW + w];
    const float inv = l == 0.f ? 0.f : 1.f / l;
    for (int d = tid; d < D; d += NT) {
        float o = 0.f;
        for (int i = 0; i < LANES; ++i) o += s_part[i * D + d];
        s_q[d] = o * inv;
    }
    __syncthreads();
    return make_float2(m, l);
}

// The keys from memory into the registers of the matrix instructions: nothing
// is shared between waves, so there is no barrier in the key loop.  A
// workgroup's four waves take every fourth tile of its keys (32 in bf16, 16 in
// fp32) and its 16 NB rows, and their states (reference, sum, O) are joined
// through LDS at the end.
//
// Scores are computed transposed, S^T = K Q^T with 16x16 instructions: lane
// (t16, tq) takes key t16 of sixteen and 16 bytes of its row per step, and
// holds row t16's scores of keys 4 tq .. 4 tq + 3.  O^T = V^T P^T contracts
// over keys in the order the scores are in: lane (t16, tq) reads the rows of
// just those keys, D / 16 neighbouring dims of each (so sixteen lanes read a
// whole row), and the dims of an instruction are t16 * (D / 16) + t.  In fp32
// that is the operand; in bf16 it takes one v_perm per pair of keys and dim.
// K is read whole rows at a time too and turned through LDS, by each wave for
// itself (chunks permuted: no bank conflicts): read as the instruction wants
// it, 64 bytes of sixteen rows at a time, a long cache came at 5.65 TB/s, and
// at 6.3 this way (6.7 with the steps after it).
//
// The reference m of a row moves only when a score exceeds it by 8 (in log2
// units), so that the common tile needs no reduction across lanes.
//
// kOnce: a sequence's keys are read by one workgroup per KV head, past the
// caches (bf16, 32/8 heads of 128, 16 x 32768 keys: 318 us past them, 362
// through them).  Pages that several sequences share are then fetched once for
// each: 16 samples of one prompt of 32000 keys take 168 us, 107 through the
// caches, 64 of 1792 keys 46 and 40 (what is shared is known to the table only).
constexpr int kWaves = 4;
enum { kCached, kOnce };

template <int MODE>
__device__ __forceinline__ uint4 load16(const char* p) {
    if constexpr (MODE != kCached) return load_stream16(p);
    return *reinterpret_cast<const uint4*>(p);
}

// Tiles of a sequence, at least one (so that some workgroup clears the rows of
// an empty one).
template <int T>
__device__ __forceinline__ int tiles_of(const Args& a, int b) {
    if (b >= a.batch) return 0;
    const Seq sq = seq_of(a, b);
    return max((span_of(a, sq.pos0, sq.pos0 + max(sq.n, 1) - 1).n + T - 1) / T, 1);
}

template <bool BF16, int D, int NB, int MODE>
__global__ __launch_bounds__(kWaves * kWave, NB == 1 ? 3 : 2) void paged_attn_rows_kernel(Args a) {
    constexpr int E = BF16 ? 2 : 4;
    constexpr int KB = BF16 ? 2 : 1;  // 16-key groups per tile
    constexpr int T = 16 * KB;
    constexpr int KC = D * E / 64;        // 16-byte chunks of a K row per lane and operand
    constexpr int CPR = D * E / 16;       // 16-byte chunks of a row
    constexpr int KL = T * CPR / 64;      // loads of a K tile per lane
    constexpr int VD = D / 16;            // dims of a V row per lane
    constexpr int VW = VD * E / 4;        // the same in words
    constexpr int R = 16 * NB;            // rows of the workgroup
    constexpr int SD = D + 4;             // row stride of the states in LDS
    constexpr int NT = kWaves * kWave;
    __shared__ __align__(16) float s_o[kWaves * R * SD];  // a wave's part: its K tile first
    static_assert(R * SD * 4 >= T * D * E, "a K tile fits");
    __shared__ float s_ml[2 * kWaves * R];
    __shared__ int s_bad[R];

    const int tid = threadIdx.x;
    const int wave = uniform(tid / kWave);

    // ---- which keys and rows: tiles t_begin .. t_end - 1 of row block rb, to part
    // `part`, or with part < 0 (the rows' only one) to the output.
    // Neighbouring blocks differ in the split or piece, so that an XCD (every
    // eighth block) meets all KV heads: rows of one head alone fall on few of
    // its L2's channels (a long cache at 5.65 against 6.2 TB/s).
    int id = blockIdx.x;
    int g, b, rev = 0, t_begin, t_end, part = -1;
    Seq sq{};
    if (MODE == kOnce && a.pieces > 0) {
        const int lane = lane_id(), idx = id % a.n_slots;
        g = id / a.n_slots;
        int total = 0;
        for (int b0 = 0; b0 < a.batch; b0 += kWave)
            total += __builtin_amdgcn_readlane((int)wave_scan_dpp(tiles_of<T>(a, b0 + lane)), kWave - 1);
        // whole rounds of the waves; at least one
        const int len = ((total + a.pieces - 1) / a.pieces + kWaves - 1) / kWaves * kWaves;
        int base = 0, count = 0;
        b = -1;
        for (int b0 = 0; b0 < a.batch && b < 0; b0 += kWave) {
            const int n = (tiles_of<T>(a, b0 + lane) + len - 1) / len, incl = (int)wave_scan_dpp(n);
            const uint64_t hit = __ballot(base + incl > idx);
            if (hit) {
                const int at = __ffsll((unsigned long long)hit) - 1;
                b = b0 + at;
                count = __builtin_amdgcn_readlane(n, at);
                base += __builtin_amdgcn_readlane(incl, at) - count;
            } else {
                base += __builtin_amdgcn_readlane(incl, kWave - 1);
            }
        }
        if (b < 0) return;
        t_begin = (idx - base) * len;
        t_end = t_begin + len;
        if (count > 1) part = g * a.n_slots + idx;
        if (idx == base && g == 0 && tid == 0) a.slots[b] = make_int2(idx, idx + count - 1);
    } else {
        const int split = id % a.splits;
        id /= a.splits;
        g = id % a.hkv;
        id /= a.hkv;
        b = id;
        if (MODE == kCached && !find_block(a, id, id == 0 && g == 0 && split == 0, b, rev, sq)) return;
        t_begin = split * a.split_tiles;
        t_end = t_begin + a.split_tiles;
        if (a.splits > 1) part = (b * a.hkv + g) * a.splits + split;
    }
    // (the same for the whole workgroup: scalars from here on)
    b = uniform(b), g = uniform(g), rev = uniform(rev);
    t_begin = uniform(t_begin), t_end = uniform(t_end), part = uniform(part);
    if (MODE == kOnce) sq = seq_of(a, b);
    if (MODE == kOnce && sq.bad && g == 0 && t_begin == 0 && tid == 0) raise_flag(a.flags, PRESTO_FLAG_BAD_SEQ);
    if (sq.n == 0) return;
    const int rb = MODE == kOnce ? 0 : (sq.n * a.G + R - 1) / R - 1 - rev;
    const int lane = lane_id();
    const int rows = sq.n * a.G;
    const int row0 = rb * R;
    const int p_lo = sq.pos0 + row0 / a.G, p_hi = sq.pos0 + (min(row0 + R, rows) - 1) / a.G;
    const Span sp = span_of(a, p_lo, p_hi);
    t_end = min(t_end, (sp.n + T - 1) / T);
    if (t_begin > 0 && t_begin >= t_end) return;  // the merge knows

    const int t16 = lane & 15, tq = lane >> 4;
    const uint32_t RS = (uint32_t)(a.hkv * D * E);  // bytes from a cache row to the next

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
        int key0[KB];
        int page[KB];  // -1: nothing to read
    };
    bool bad_page = false;
    const int32_t* trow = a.table + (int64_t)b * a.max_pages;
    auto locate = [&](int t) {
        Tile x;
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) {
            // (sixteen keys that no row sees may be without a page)
            const int k0 = uniform(key_of(sp, t * T + 16 * kb));
            const bool wanted = k0 < sp.hi && (k0 + 16 > sp.lo || k0 < a.sinks);
            x.key0[kb] = k0;
            x.page[kb] = wanted ? trow[k0 >> a.page_shift] : -1;
            if (wanted && (uint32_t)x.page[kb] >= (uint32_t)a.num_pages) {
                bad_page = true;
                x.page[kb] = -1;
            }
        }
        return x;
    };
    auto group = [&](const char* pool, const Tile& x, int kb) {
        const int r = x.key0[kb] & ((1 << a.page_shift) - 1);
        const int64_t at = x.page[kb] < 0 ? 0 : x.page[kb] * a.page_stride + (int64_t)r * a.hkv * D;
        return pool + (at + g * D) * E;  // (page 0 stands for one that is not there)
    };
    // K: load j covers rows j * 64 / CPR .. of the tile; row r's chunk c lies
    // at c ^ swz(r) in LDS, and operand (key t16, chunk 4 i + tq) is read back
    auto swz = [](int r) { return CPR == 8 ? (r >> 1) & 7 : r & 15; };
    char* const s_k = reinterpret_cast<char*>(s_o + wave * R * SD);
    uint4 kf[KL];
    uint32_t vf[4 * KB][VW];
    const uint32_t k_off = lane / CPR * RS + lane % CPR * 16;
    const uint32_t v_off = 4 * tq * RS + t16 * VW * 4;
    // (the steps from load to load go to the scalar base: in the offset they
    // would cost a register each)
    auto load_k = [&](const Tile& x) {
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) {
            const char* p = group(a.kp, x, kb);
#pragma unroll
            for (int j = 0; j < KL / KB; ++j) kf[kb * (KL / KB) + j] = load16<MODE>(p + (int64_t)(j * (64 / CPR)) * RS + k_off);
        }
    };
    auto store_k = [&]() {
#pragma unroll
        for (int j = 0; j < KL; ++j) {
            const int r = j * (64 / CPR) + lane / CPR;
            *reinterpret_cast<uint4*>(s_k + r * (D * E) + ((lane % CPR) ^ swz(r)) * 16) = kf[j];
        }
    };
    auto k_at = [&](int kb, int i) {
        const int r = 16 * kb + t16;
        return *reinterpret_cast<const uint4*>(s_k + r * (D * E) + ((4 * i + tq) ^ swz(r)) * 16);
    };
    auto load_v = [&](const Tile& x) {
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) {
            const char* p = group(a.vp, x, kb);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const char* pr = p + (int64_t)r * RS + v_off;
                if constexpr (VW == 2) {
                    const uint2 u = *reinterpret_cast<const uint2*>(pr);
                    vf[4 * kb + r][0] = u.x;
                    vf[4 * kb + r][1] = u.y;
                } else {
#pragma unroll
                    for (int w = 0; w < VW; w += 4) {
                        const uint4 u = load16<MODE>(pr + w * 4);
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
        // ---- scores (a wave's LDS accesses stay in order)
        store_k();
        if (more) load_k(nxt);
        __builtin_amdgcn_wave_barrier();
        floatx4 S[NB][KB];
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int kb = 0; kb < KB; ++kb) S[nb][kb] = (floatx4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
            for (int i = 0; i < KC; ++i) {
                const uint4 ku = k_at(kb, i);
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) {
                    if constexpr (BF16) {
                        S[nb][kb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                            __builtin_bit_cast(bf16x8, ku), __builtin_bit_cast(bf16x8, qf[nb][i]), S[nb][kb], 0, 0, 0);
                    } else {
                        const floatx4 kv = __builtin_bit_cast(floatx4, ku);
                        const floatx4 qv = __builtin_bit_cast(floatx4, qf[nb][i]);
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            S[nb][kb] = __builtin_amdgcn_mfma_f32_16x16x4f32(kv[e], qv[e], S[nb][kb], 0, 0, 0);
                    }
                }
            }
        __builtin_amdgcn_wave_barrier();

        // ---- masks, on the tiles that need them
        bool edge = false;
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) {
            const int k0 = cur.key0[kb];
            edge |= cur.page[kb] < 0 || k0 + 16 > p_lo + 1 ||
                    (a.window > 0 && k0 <= p_hi - a.window && k0 + 16 > a.sinks);
        }
        if (edge) {
#pragma unroll
            for (int kb = 0; kb < KB; ++kb)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int key = cur.key0[kb] + 4 * tq + r;
                    const bool here = cur.page[kb] >= 0;
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb)
                        S[nb][kb][r] = here && sees(a, pos[nb], key) ? S[nb][kb][r] : -INFINITY;
                    // rows that nobody sees may hold anything
                    const bool any = here && key < sp.hi && (key >= sp.lo || key < a.sinks);
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
            // A probability enters as two bf16, the second what the rounding of
            // the first left (16 bits between them; their sum is taken before).
            // The second products hide behind the keys' arrival: 16 x 32768
            // keys 319 us with one and with two, the listed decodes within
            // 0.7%, short prompts 1 to 3% slower; the error of an output is that
            // of its own rounding, 1.66e-3 in norm, where one makes it 2.1e-3.
            bf16x8 ph[NB], pl[NB];
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
                uint32_t hi[4], lo[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float p0 = S[nb][i / 2][2 * (i % 2)], p1 = S[nb][i / 2][2 * (i % 2) + 1];
                    hi[i] = pack2(p0, p1);
                    lo[i] = pack2(p0 - bf16lo(hi[i]), p1 - bf16hi(hi[i]));
                    l[nb] += p0 + p1;
                }
                ph[nb] = __builtin_bit_cast(bf16x8, make_uint4(hi[0], hi[1], hi[2], hi[3]));
                pl[nb] = __builtin_bit_cast(bf16x8, make_uint4(lo[0], lo[1], lo[2], lo[3]));
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
                for (int nb = 0; nb < NB; ++nb) {
                    o[nb][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va, pl[nb], o[nb][i], 0, 0, 0);
                    o[nb][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va, ph[nb], o[nb][i], 0, 0, 0);
                }
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

    const int64_t prow = (int64_t)part * a.G * a.max_q;
    auto put = [&](int rho, int d, floatx4 v) {
        if (part >= 0) {
            *reinterpret_cast<floatx4*>(a.part_o + (prow + rho) * D + d) = v;
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
        if (part >= 0) a.part_ml[prow + rho] = make_float2(M, L);
    };
    bool bad = false;
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
        if (!fine) {
            s_bad[r] = 1;
            bad = true;
        }
        put(rho, d, acc);
        if (d == 0) put_ml(rho, M, L);
    }
    // ---- rows of several positions whose sums are not all finite: a key that
    // only others see may be the cause
    static_assert(kAloneFloats<D, E, NT> <= kWaves * R * SD, "the states' room is enough");
    if (p_lo == p_hi || !__syncthreads_or(bad)) return;
    const Args& a2 = args_again();
    if (!__syncthreads_or(edge_not_finite<BF16, D>(a2, b, g, p_lo, p_hi))) return;
    for (int r = 0; r < R; ++r) {
        if (!s_bad[r]) continue;
        const int rho = row0 + r, tok = rho / a2.G;
        const float2 ml = row_alone<BF16, D, NT>(a2, sp, b, g, sq.r0 + tok, g * a2.G + rho - tok * a2.G, sq.pos0 + tok,
                                                 t_begin * T, t_end * T, s_o);
        for (int d = tid * 4; d < D; d += NT * 4) put(rho, d, *reinterpret_cast<const floatx4*>(&s_o[d]));
        if (tid == 0) put_ml(rho, ml.x, ml.y);
    }
}

// Many query rows per KV head (bf16): tiles of 64 keys go from memory straight
// into LDS (a ring of four: one consumed, one resident, two in flight), where
// eight waves of 32 rows each read them, so that a key is fetched once for 256
// rows.  32x32x16 instructions, S^T = K Q^T and O^T = V^T P^T as above; a lane
// holds one row and 16 of a block's 32 keys, and the probabilities are the
// second product's operand as they are.  K rows lie in LDS with their 16-byte
// chunks permuted by chunk ^ (row mod 16), V rows by chunk ^ 4 (row mod 4), so
// that neither the b128 reads of K nor the transposed reads of V meet bank
// conflicts.
//
// Three blocks of 32 keys are in work per wave: a step issues the P V products
// of block i, the exponentials of block i + 1 and the scores of block i + 2
// between one another.  Scores start from -m, so that a probability is
// exp2(c S); the reference m moves only where a block's sum exceeds 2^8 or a
// row has no mass yet, or next to none (kLeastMass: keys that a row does not see
// may come first, and all of its scores may lie far below 0).
//
// The page numbers of the workgroup's keys are looked up once and kept in LDS:
// eight rows of a tile, one wave's share of its loads, lie in one page.
typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef short shortx4 __attribute__((ext_vector_type(4)));

constexpr int kKeyTile = 64;
constexpr int kRing = 4;
constexpr int kTileWaves = 8;
constexpr int kTileRows = kTileWaves * 32;
constexpr int kTilePages = 4096;  // page numbers in LDS

// 16 bytes per lane from memory to LDS: lane l's land at lds + 16 l.  In inline
// assembly, because the compiler would put a wait for all loads before every
// later LDS read; the kernel waits for each tile itself.
__device__ __forceinline__ void lds_load16(const void* lane_ptr, uint32_t lds) {
    const uint32_t m0v = (uint32_t)__builtin_amdgcn_readfirstlane(lds);
    asm volatile("global_load_lds_dwordx4 %0, off" ::"v"(lane_ptr), "{m0}"(m0v) : "memory");
}
// the same with a wave-uniform base and a 32-bit offset per lane
__device__ __forceinline__ void lds_load16(const void* base, uint32_t off, uint32_t lds) {
    const uint64_t b = (uint64_t)(uintptr_t)base;
    const uint32_t lo = (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)b);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)(b >> 32));
    const uint64_t sb = ((uint64_t)hi << 32) | (uint64_t)lo;
    const uint32_t m0v = (uint32_t)__builtin_amdgcn_readfirstlane(lds);
    asm volatile("global_load_lds_dwordx4 %0, %1" ::"v"(off), "s"(sb), "{m0}"(m0v) : "memory");
}

// A barrier for what is in LDS: loads and stores of global memory stay on their
// way across it.
__device__ __forceinline__ void lds_barrier() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

template <int D>
__global__ __launch_bounds__(kTileWaves * kWave) void paged_attn_tiles_kernel(Args a) {
    constexpr int T = kKeyTile;
    constexpr int KS = D / 16;                // contraction steps of a score block
    constexpr int DB = D / 32;                // 32-dim blocks of the output
    constexpr int CH = D / 8;                 // 16-byte chunks per row
    constexpr int NT = kTileWaves * kWave;
    constexpr int RPL = 64 / CH;              // key rows per load instruction
    constexpr int LPT = T / RPL / kTileWaves; // loads per thread and tile, K and V each
    constexpr int kTile = T * D * 2;          // bytes of a K or V tile
    constexpr int kV = kRing * kTile;         // K tiles first, then V tiles
    static_assert(LPT * RPL == 8, "a wave loads eight rows of a tile");
    __shared__ __align__(16) char s_kv[2 * kRing * kTile];
    __shared__ int32_t s_page[kTilePages];
    __shared__ int s_bad[kTileRows], s_any;

    // Neighbouring blocks differ in the KV head, so that the row blocks of one
    // head, which read the same keys, meet in the L2 of one XCD (every eighth
    // block).
    int id = blockIdx.x;
    const int g = id % a.hkv;
    id /= a.hkv;
    const int split = id % a.splits;
    id /= a.splits;
    int b, rev;
    Seq sq{};
    if (!find_block(a, id, id == 0 && g == 0 && split == 0, b, rev, sq)) return;
    const int rows = sq.n * a.G;
    const int rb = (rows + a.block_rows - 1) / a.block_rows - 1 - rev;
    const int tid = threadIdx.x, lane = lane_id();
    const int wave = uniform(tid / kWave);
    const int row0 = rb * a.block_rows;  // (a multiple of 32, at most kTileRows)
    const int row_end = min(row0 + a.block_rows, rows);
    const Span sp = span_of(a, sq.pos0 + row0 / a.G, sq.pos0 + (row_end - 1) / a.G);
    const int t_begin = split * a.split_tiles, t_end = min(t_begin + a.split_tiles, (sp.n + T - 1) / T);
    if (split > 0 && t_begin >= t_end) return;  // the merge knows
    const int64_t prow = (((int64_t)b * a.hkv + g) * a.splits + split) * a.G * a.max_q;

    const int l32 = lane & 31, h = lane >> 5;
    const int wrow0 = row0 + wave * 32;  // this wave's first row
    const int rho = wrow0 + l32;
    const int rq = min(rho, row_end - 1);
    const int tok = rq / a.G, qh = rq - tok * a.G;
    const int pos = sq.pos0 + tok;
    const int p_lo = uniform(sq.pos0 + min(wrow0, row_end - 1) / a.G);
    const int p_hi = uniform(sq.pos0 + min(wrow0 + 31, row_end - 1) / a.G);
    const float c = a.scale_log2;
    // ---- page numbers: those of the entries before the gap, then of the others
    const int va = t_begin * T, va_end = min(sp.head, t_end * T);
    const int pa = va >> a.page_shift;
    const int na = va < va_end ? ((va_end - 1) >> a.page_shift) - pa + 1 : 0;
    const int kb = max(va, sp.head) + sp.gap, kb_end = min(sp.hi, t_end * T + sp.gap);
    const int pb = kb >> a.page_shift;
    const int nb = kb < kb_end ? ((kb_end - 1) >> a.page_shift) - pb + 1 : 0;
    // (the first number of each thread is asked for before the queries, so that
    // waiting for it leaves them on their way)
    const int32_t* trow = a.table + (int64_t)b * a.max_pages;
    const int pages = min(na + nb, kTilePages);
    auto column = [&](int i) { return i < na ? pa + i : pb + i - na; };
    const int first_page = tid < pages ? trow[column(tid)] : 0;
    // queries, second operand of S^T: row l32, dims ks * 16 + h * 8 ..
    bf16x8 qf[KS];
    {
        const char* qp = a.q + ((sq.r0 + tok) * a.q_stride + (int64_t)(g * a.G + qh) * D + h * 8) * 2;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
            qf[ks] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const uint4*>(qp + ks * 32));
    }
    bool bad_page = na + nb > kTilePages;  // (the host's choice of splits rules it out)
    for (int i = tid; i < pages; i += NT) {
        const int x = column(i);
        const int k0 = max(x << a.page_shift, i < na ? va : kb), k1 = min((x + 1) << a.page_shift, kb_end);
        const bool wanted = k0 < a.sinks || (i >= na && k1 > sp.lo);
        const int page = !wanted ? 0 : i == tid ? first_page : trow[x];
        const bool ok = (uint32_t)page < (uint32_t)a.num_pages;
        bad_page |= !ok;
        s_page[i] = ok ? page : 0;
    }
    if (tid < kTileRows) s_bad[tid] = 0;
    if (tid == 0) s_any = 0;
    lds_barrier();
    if (bad_page) s_any = 1;
    lds_barrier();
    const bool skip = s_any != 0;
    if (skip) {
        // a page that is not there: its keys are left out, row by row
        if (tid == 0) raise_flag(a.flags, PRESTO_FLAG_BAD_PAGE);
        if (tid < row_end - row0) s_bad[tid] = 1;
    }

    floatx16 o[DB];
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[db][i] = 0.f;
    float m = 0.f, l_run = 0.f;  // reference (score units) and sum of the row

    if (!skip && t_begin < t_end) {
        // ---- loads: instruction j of this wave covers rows 8 wave + RPL j ..
        // of a tile; lane l writes chunk l % CH of row l / CH and fetches the
        // chunk that the row's permutation puts there
        uint32_t goff_k[LPT], goff_v[LPT];
        int lrow[LPT], lck[LPT], lcv[LPT];
#pragma unroll
        for (int j = 0; j < LPT; ++j) {
            const int r = 8 * wave + RPL * j + lane / CH, pc = lane % CH;
            lrow[j] = r;
            lck[j] = pc ^ (r & (CH - 1) & 15);
            lcv[j] = pc ^ ((4 * (r & 3)) & (CH - 1));
            goff_k[j] = (uint32_t)(((r - 8 * wave) * a.hkv * D + lck[j] * 8) * 2);
            goff_v[j] = (uint32_t)(((r - 8 * wave) * a.hkv * D + lcv[j] * 8) * 2);
        }
        const uint32_t lds_kv = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)s_kv;
        const int pmask = (1 << a.page_shift) - 1;
        auto page_of = [&](bool head, int key) __attribute__((always_inline)) {
            return s_page[(key >> a.page_shift) - (head ? pa : pb - na)];
        };
        auto load_tile = [&](int t, int buf) __attribute__((always_inline)) {
            const uint32_t kdst = lds_kv + buf * kTile + wave * LPT * 1024;
            const uint32_t vdst = kdst + kV;
            const int v0 = t * T, key0 = v0 + sp.gap;
            if (t < t_end && v0 >= sp.head && key0 + T <= sp.hi && (key0 >= sp.lo || key0 + T <= a.sinks)) {
                const int kw = key0 + 8 * wave;
                const int64_t at = uniform(page_of(false, kw)) * a.page_stride + ((int64_t)(kw & pmask) * a.hkv + g) * D;
#pragma unroll
                for (int j = 0; j < LPT; ++j) {
                    lds_load16(a.kp + at * 2, goff_k[j], kdst + j * 1024);
                    lds_load16(a.vp + at * 2, goff_v[j], vdst + j * 1024);
                }
            } else {
                // entries that no query of the workgroup sees repeat one of
                // their tile that some query does (nothing else is read: there
                // may be no page, and V must be a number where P is 0); past
                // the last tile, its last entry
                const int vt = min(t, t_end - 1) * T;
#pragma unroll
                for (int j = 0; j < LPT; ++j) {
                    const int v = t < t_end ? v0 + lrow[j] : vt + T - 1;
                    const bool head = v < sp.head;
                    int key = head ? min(v, a.sinks - 1) : min(v + sp.gap, sp.hi - 1);
                    if (!head && key < sp.lo && key >= a.sinks) key = sp.gap == 0 && vt < a.sinks ? a.sinks - 1 : sp.lo;
                    const int64_t at = page_of(head, key) * a.page_stride + ((int64_t)(key & pmask) * a.hkv + g) * D;
                    lds_load16(a.kp + (at + lck[j] * 8) * 2, kdst + j * 1024);
                    lds_load16(a.vp + (at + lcv[j] * 8) * 2, vdst + j * 1024);
                }
            }
        };
        // vmcnt(n) with the other counters left alone
#define PRESTO_WAIT_VM(n) __builtin_amdgcn_s_waitcnt(((n) & 15) | (((n) >> 4) << 14) | 0x0f70)

        // the blocks of the workgroup, and of this wave up to its last row's
        // position
        const int ntiles = t_end - t_begin;
        const int nblocks = (min(min(p_hi + 1 - sp.gap, sp.n), t_end * T) - t_begin * T + 31) / 32;
        const bool active = wrow0 < row_end && nblocks > 0;

        // per-lane LDS addresses of the fragment reads (ring slot 0, block 0)
        const int vr = 4 * h + ((lane & 15) >> 2);
        const int vc = ((lane >> 4) & 1) * 2 + ((lane & 3) >> 1);
        uint32_t kaddr[KS], vaddr[DB];
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
            kaddr[ks] = (l32 * (D * 2) + ((h ^ (l32 & 15)) & (CH - 1)) * 16) ^ (ks << 5);
#pragma unroll
        for (int db = 0; db < DB; ++db)
            vaddr[db] = kV + ((vr * (D * 2) + ((4 * (vr & 3) + vc) & (CH - 1)) * 16 + (lane & 1) * 8) ^ (db << 6));

        const bf16x2 ones = {(__bf16)1.0f, (__bf16)1.0f};
        floatx16 negm;
#pragma unroll
        for (int e = 0; e < 16; ++e) negm[e] = 0.f;
        typedef __attribute__((address_space(3))) shortx4* lds_s4;

        auto half_swap = [&](float v) __attribute__((always_inline)) {
            const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
            return __uint_as_float(h == 0 ? sw[1] : sw[0]);
        };
        auto row_max = [&](const floatx16& S) __attribute__((always_inline)) {
            float mx = S[0];
#pragma unroll
            for (int e = 1; e < 16; ++e) mx = fmaxf(mx, S[e]);
            return fmaxf(mx, half_swap(mx));
        };
        auto row_sum = [&](float v) __attribute__((always_inline)) { return v + half_swap(v); };
        auto masked = [&](int i) __attribute__((always_inline)) {
            const int v0 = t_begin * T + 32 * i, k0 = v0 + sp.gap;
            return k0 + 32 > p_lo + 1 || v0 < sp.head || (a.window > 0 && k0 <= p_hi - a.window && k0 + 32 > a.sinks);
        };
        // the block's 32 entries as bits, then a test and a select per element
        auto apply_mask = [&](floatx16& S, int i) __attribute__((always_inline)) {
            const int v0 = t_begin * T + 32 * i;
            auto below = [](int n) { return n >= 32 ? ~0u : (n <= 0 ? 0u : (1u << n) - 1u); };
            uint32_t vis = below(pos + 1 - sp.gap - v0);
            if (a.window > 0) {
                vis &= ~below(max(pos - a.window + 1 - sp.gap, sp.head) - v0);
                vis |= below(min(a.sinks, pos + 1) - v0);
            }
            vis >>= 4 * h;
#pragma unroll
            for (int e = 0; e < 16; ++e) S[e] = (vis >> (8 * (e >> 2) + (e & 3))) & 1u ? S[e] : -INFINITY;
        };
        auto qk = [&](auto bufc, int blk, floatx16& Sx) __attribute__((always_inline)) {
            constexpr int buf = decltype(bufc)::value;
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                const uint4 u = *reinterpret_cast<const uint4*>(s_kv + kaddr[ks] + buf * kTile + blk * 32 * D * 2);
                Sx = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, u), qf[ks],
                                                             ks == 0 ? negm : Sx, 0, 0, 0);
            }
        };
        // two probabilities, rounded to the product's bf16; the sum takes the
        // rounded values (one bf16: the matrix cores bound this kernel, and a
        // second one, as the kernel of rows takes, would be half as many
        // instructions again; 2.3e-3 in norm for the output rounding's 1.66e-3)
        auto pair = [&](const floatx16& S, int e, float& ls) __attribute__((always_inline)) {
            const uint32_t w = pack2(__builtin_amdgcn_exp2f(S[e] * c), __builtin_amdgcn_exp2f(S[e + 1] * c));
            ls = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, w), ones, ls, false);
            return w;
        };
        // moves m to the block's maximum in the rows that need it and takes the
        // block's probabilities again (Sy: a block scored against the old m)
        auto exact = [&](floatx16& Sx, uint32_t(&Px)[8], float& ls, bool need, floatx16& Sy) __attribute__((always_inline)) {
            const float mx = row_max(Sx);
            const float delta = need && mx != -INFINITY ? mx : 0.f;
            const float alpha = l_run > 0.f ? __builtin_amdgcn_exp2f(-delta * c) : 0.f;
            m += delta;
            l_run *= alpha;
#pragma unroll
            for (int db = 0; db < DB; ++db) o[db] *= alpha;
            ls = 0.f;
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                Sx[e] -= delta;
                Sy[e] -= delta;
                negm[e] = -m;
            }
#pragma unroll
            for (int e = 0; e < 16; e += 2) Px[e >> 1] = pair(Sx, e, ls);
            ls = row_sum(ls);
        };

        constexpr int EPK = 16 / KS;  // exponentials per score instruction
        static_assert(EPK * KS == 16 && EPK % 2 == 0 && KS == 2 * DB, "head_dim 64 or 128");
        floatx16 Sa = negm, Sb = negm;  // scores of blocks i + 1 and i + 2
        uint32_t Pp[8];                 // probabilities of block i
        auto step = [&](auto bvc, auto bkc, int i, int q) __attribute__((always_inline)) {
            constexpr int bv = decltype(bvc)::value, bk = decltype(bkc)::value;
            const bool more = i + 1 < nblocks;
            if (more && masked(i + 1)) apply_mask(Sa, i + 1);
            uint32_t Pn[8];
            float ls = 0.f;
#pragma unroll
            for (int st = 0; st < 2; ++st) {
                const bf16x8 pv =
                    __builtin_bit_cast(bf16x8, make_uint4(Pp[4 * st], Pp[4 * st + 1], Pp[4 * st + 2], Pp[4 * st + 3]));
#pragma unroll
                for (int db = 0; db < DB; ++db) {
                    const uint32_t v0 = vaddr[db] + bv * kTile + q * 32 * D * 2 + st * 16 * D * 2;
                    const shortx4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4)(s_kv + v0));
                    const shortx4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4)(s_kv + v0 + 8 * D * 2));
                    const uint2 ul = __builtin_bit_cast(uint2, lo), uh = __builtin_bit_cast(uint2, hi);
                    o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                        __builtin_bit_cast(bf16x8, make_uint4(ul.x, ul.y, uh.x, uh.y)), pv, o[db], 0, 0, 0);
                    const int ks = st * DB + db;
                    const uint4 u = *reinterpret_cast<const uint4*>(s_kv + kaddr[ks] + bk * kTile + q * 32 * D * 2);
                    Sb = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, u), qf[ks],
                                                                 ks == 0 ? negm : Sb, 0, 0, 0);
#pragma unroll
                    for (int e = ks * EPK; e < ks * EPK + EPK; e += 2) Pn[e >> 1] = pair(Sa, e, ls);
                }
            }
            if (more) {
                ls = row_sum(ls);
                const bool need = !(ls <= 256.f) || l_run + ls < kLeastMass;
                if (__ballot(need)) exact(Sa, Pn, ls, need, Sb);
                l_run += ls;
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) Pp[j] = Pn[j];
            Sa = Sb;
        };
        // one tile: its two blocks, the load of tile t + 3 into the slot that
        // every wave left before the last barrier, the wait for tile t + 2
        // (where no more tiles follow, for all that is on its way: loads of
        // the last entry in their place cost short lists up to 5%)
        auto tile = [&](auto uc, int t) __attribute__((always_inline)) {
            constexpr int u = decltype(uc)::value;
            using BV = std::integral_constant<int, u>;
            using BK = std::integral_constant<int, (u + 1) % kRing>;
            if (t + 3 < ntiles)
                load_tile(t_begin + t + 3, (u + 3) % kRing);
            else
                PRESTO_WAIT_VM(0);
            if (active) {
                if (2 * t < nblocks) step(BV{}, BK{}, 2 * t, 0);
                if (2 * t + 1 < nblocks) step(BV{}, BK{}, 2 * t + 1, 1);
            }
            PRESTO_WAIT_VM(2 * LPT);
            __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0): this wave's LDS reads are done
            __builtin_amdgcn_s_barrier();
        };
        load_tile(t_begin, 0);
        load_tile(t_begin + 1, 1);
        load_tile(t_begin + 2, 2);
        PRESTO_WAIT_VM(2 * LPT);  // (the queries too: they were asked for first)
        lds_barrier();
        if (active) {
            using B0 = std::integral_constant<int, 0>;
            floatx16 S0 = negm;
            qk(B0{}, 0, S0);
            if (masked(0)) apply_mask(S0, 0);
            float ls;
            exact(S0, Pp, ls, true, Sb);
            l_run = ls;
            qk(B0{}, 1, Sa);
        }
        for (int t = 0; t < ntiles; t += kRing) {
            tile(std::integral_constant<int, 0>{}, t);
            if (t + 1 < ntiles) tile(std::integral_constant<int, 1>{}, t + 1);
            if (t + 2 < ntiles) tile(std::integral_constant<int, 2>{}, t + 2);
            if (t + 3 < ntiles) tile(std::integral_constant<int, 3>{}, t + 3);
        }
        PRESTO_WAIT_VM(0);  // no load into LDS outlives its buffer
#undef PRESTO_WAIT_VM
    }

    // ---- lane: row rho, dims db * 32 + 8 q4 + 4 h + 0 .. 3
    const float inv = l_run == 0.f ? 0.f : 1.f / l_run;
    bool fine = true;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            o[db][e] *= inv;
            fine &= fabsf(o[db][e]) < INFINITY;
        }
    if (!fine && rho < row_end) {
        s_bad[rho - row0] = 1;
        s_any = 1;
    }
    lds_barrier();  // (the ring is free, too)
    const bool any = s_any != 0;
    auto out_row = [&](int r) {
        const int tk = r / a.G;
        return reinterpret_cast<uint16_t*>(a.out) + ((sq.r0 + tk) * a.hq + g * a.G + r - tk * a.G) * D;
    };
    auto part_row = [&](int r) { return a.part_o + (prow + r) * D; };
    if (a.splits == 1) {
        // through this wave's part of the ring: whole rows, 16 bytes per lane
        char* const w = s_kv + wave * (32 * D * 2);
        static_assert(kTileWaves * 32 * D * 2 <= 2 * kRing * kTile, "the rows fit");
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int q4 = 0; q4 < 4; ++q4)
                *reinterpret_cast<uint2*>(w + l32 * (D * 2) + (((4 * db + q4) ^ (l32 & (CH - 1))) * 16 + 8 * h)) =
                    make_uint2(pack2(o[db][4 * q4], o[db][4 * q4 + 1]), pack2(o[db][4 * q4 + 2], o[db][4 * q4 + 3]));
        __builtin_amdgcn_wave_barrier();  // (a wave's LDS accesses stay in order)
#pragma unroll
        for (int j = 0; j < 32 / RPL; ++j) {
            const int r = j * RPL + lane / CH, ck = lane % CH;
            const uint4 u = *reinterpret_cast<const uint4*>(w + r * (D * 2) + ((ck ^ (r & (CH - 1))) * 16));
            if (wrow0 + r < row_end) *reinterpret_cast<uint4*>(out_row(wrow0 + r) + ck * 8) = u;
        }
    } else if (rho < row_end) {
        float* op = part_row(rho);
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int q4 = 0; q4 < 4; ++q4)
                *reinterpret_cast<floatx4*>(op + db * 32 + 8 * q4 + 4 * h) =
                    (floatx4){o[db][4 * q4], o[db][4 * q4 + 1], o[db][4 * q4 + 2], o[db][4 * q4 + 3]};
        if (h == 0) a.part_ml[prow + rho] = make_float2(l_run == 0.f ? -INFINITY : m * c, l_run);
    }
    // ---- rows whose sums are not all finite: a key that only others see may
    // be the cause; or all rows, where a page is not there
    if (!any) return;
    const Args& a2 = args_again();
    if (!skip && !__syncthreads_or(edge_not_finite<true, D>(a2, b, g, sq.pos0 + row0 / a2.G,
                                                            sq.pos0 + (row_end - 1) / a2.G)))
        return;
    float* const f = reinterpret_cast<float*>(s_kv);
    static_assert(kAloneFloats<D, 2, NT> * 4 <= 2 * kRing * kTile, "the ring's room is enough");
    for (int r = 0; r < row_end - row0; ++r) {
        if (!s_bad[r]) continue;
        const int rr = row0 + r, tk = rr / a2.G;
        const float2 ml = row_alone<true, D, NT>(a2, sp, b, g, sq.r0 + tk, g * a2.G + rr - tk * a2.G, sq.pos0 + tk,
                                                 t_begin * T, t_end * T, f);
        for (int d = tid; d < D / 2; d += NT) {
            if (a.splits == 1)
                *reinterpret_cast<uint32_t*>(out_row(rr) + 2 * d) = pack2(f[2 * d], f[2 * d + 1]);
            else
                *reinterpret_cast<float2*>(part_row(rr) + 2 * d) = make_float2(f[2 * d], f[2 * d + 1]);
        }
        if (tid == 0 && a.splits > 1) a.part_ml[prow + rr] = ml;
    }
}

// Joins the splits of a row.  D / 4 lanes read a split's row; `parts` groups of
// them share a row's splits and join theirs through LDS, so that all of a row's
// partials are asked for at once (32 rows of 32 splits: 13.9 us with one group,
// a memory round trip per eight splits).  Splits past a sequence's keys have
// written nothing.
constexpr int kMergeThreads = 256;

template <bool BF16, int D, int T>
__global__ __launch_bounds__(kMergeThreads) void paged_attn_merge_kernel(Args a, int parts) {
    constexpr int E = BF16 ? 2 : 4;
    constexpr int LR = D / 4;  // lanes per row and part: 16 or 32
    constexpr int GROUPS = kMergeThreads / LR;
    __shared__ __align__(16) float s_acc[GROUPS][D];
    __shared__ float s_ml[2][GROUPS];
    const int per_seq = a.max_q * a.hq;
    const int grp = threadIdx.x / LR, ln = threadIdx.x % LR, part = grp % parts;
    const int64_t idx = (int64_t)blockIdx.x * (GROUPS / parts) + grp / parts;
    const int b = (int)(idx / per_seq), rest = (int)(idx % per_seq);
    const bool in = b < a.batch;
    const Seq sq = in ? seq_of(a, b) : Seq{0, 0, 0, false};
    const int tok = rest / a.hq, head = rest - tok * a.hq;
    const bool live_row = tok < sq.n;
    int live = 1;
    float M = -INFINITY, L = 0.f;
    floatx4 acc = {0.f, 0.f, 0.f, 0.f};
    if (live_row) {
        const int g = head / a.G, rho = tok * a.G + head - g * a.G;
        const int64_t all = (int64_t)a.G * a.max_q;
        int64_t first;
        if (a.pieces > 0) {
            const int2 s = a.slots[b];
            first = (int64_t)g * a.n_slots + s.x;
            live = s.y - s.x + 1;
        } else {
            const int row0 = rho / a.block_rows * a.block_rows;
            const Span sp = span_of(a, sq.pos0 + row0 / a.G, sq.pos0 + (min(row0 + a.block_rows, sq.n * a.G) - 1) / a.G);
            first = ((int64_t)b * a.hkv + g) * a.splits;
            live = max(min(((sp.n + T - 1) / T + a.split_tiles - 1) / a.split_tiles, a.splits), 1);
        }
        const int64_t prow = first * all + rho;
        const float2* ml = a.part_ml + prow;
        const float* po = a.part_o + prow * D + ln * 4;
        for (int s0 = part; s0 < (a.pieces > 0 && live == 1 ? 0 : live); s0 += 4 * parts) {
            floatx4 v[4];
            float2 x[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int s = min(s0 + j * parts, live - 1);
                v[j] = *reinterpret_cast<const floatx4*>(po + (int64_t)s * all * D);
                x[j] = ml[s * all];
            }
            // (a split in which the row sees nothing has reference -inf and sum 0)
            float mn = M;
#pragma unroll
            for (int j = 0; j < 4; ++j) mn = fmaxf(mn, x[j].x);
            const float f = M == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(M - mn);
            M = mn;
            if (L != 0.f) {
                L *= f;
                acc *= f;
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (s0 + j * parts >= live || x[j].y == 0.f) continue;
                const float w = x[j].y * __builtin_amdgcn_exp2f(x[j].x - M);
                L += w;
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[e] = fmaf(w, v[j][e], acc[e]);
            }
        }
    }
    if (parts > 1) {
        *reinterpret_cast<floatx4*>(&s_acc[grp][ln * 4]) = acc;
        if (ln == 0) {
            s_ml[0][grp] = M;
            s_ml[1][grp] = L;
        }
        __syncthreads();
        if (part != 0) return;
        const float own = M;
        for (int i = 1; i < parts; ++i) M = fmaxf(M, s_ml[0][grp + i]);
        const float f = L == 0.f ? 0.f : __builtin_amdgcn_exp2f(own - M);
        if (L != 0.f) {
            L *= f;
            acc *= f;
        }
        for (int i = 1; i < parts; ++i) {
            const float l = s_ml[1][grp + i];
            if (l == 0.f) continue;
            const float w = __builtin_amdgcn_exp2f(s_ml[0][grp + i] - M);
            L = fmaf(w, l, L);
            const floatx4 v = *reinterpret_cast<const floatx4*>(&s_acc[grp + i][ln * 4]);
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[e] = fmaf(w, v[e], acc[e]);
        }
    }
    if (!live_row || (a.pieces > 0 && live == 1)) return;  // (a sequence in one piece is written already)
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

int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Entries of the longest key list of a block of `rows` rows: all of the
// context, or the sinks and the window of its first to its last row.
int64_t longest_list(const presto_paged_attn_desc* d, int64_t rows) {
    const int64_t all = d->max_ctx > 0 ? d->max_ctx : 1;
    if (d->window == 0) return all;
    const int G = d->hq / d->pages.hkv;
    const int64_t span = (int64_t)d->window + (rows - 1) / G + 1 + 15 + (d->sinks + 15) / 16 * 16;
    return span < all ? span : all;
}

// Row blocks of a grid, and how they are counted (find_block).
int64_t counted_blocks(const presto_paged_attn_desc* d, PagedPlan& p) {
    const int64_t batch = d->pages.batch, all = batch * p.row_blocks;
    p.order = batch <= kWave ? kByLength : batch <= 2048 ? kBySequence : kByGrid;
    // (sequences end in a part of a block each)
    const int64_t most = d->total_q * (d->hq / d->pages.hkv) / p.block_rows + batch;
    return p.order != kByGrid && most < all ? most : all;
}

// The kernel of tiles: rows per workgroup and splits, by modelled time in us.
// A workgroup takes about 8 beside its tiles (page numbers, queries, first
// tiles, output), a tile of 64 keys 1.75 with two waves of rows per SIMD and
// 1.25 with one (up to 128 rows), at head_dim 64 three quarters of that (off by
// 9% r.m.s. over 149 shapes), a merge 5 and its partials' traffic.  One
// workgroup per CU: whole rounds where all are alike, else the longest or the
// sum.  Measured, bf16, 32/8 heads of 128, forced to blocks of 64, 128 and 256
// rows: 1000 new tokens alone 34, 27 and 41 us; 64 on 65536 cached 182, 111 and
// 98; 16 x 300 on 1700 365, 193 and 152.
// (Every sequence is counted with max_q tokens: a chunk that shares its call
// with decode rows is cut too little, 512 tokens on 30720 keys 244 us alone, 408
// beside one row and 777 beside seven, which alone take 26.)
double plan_tiles(const presto_paged_attn_desc* d, int64_t rows, PagedPlan& p) {
    const int64_t heads = (int64_t)d->pages.batch * d->pages.hkv;
    const int64_t most = (int64_t)(kTilePages - 8) * d->pages.page_size / kKeyTile;  // page numbers in LDS
    const bool narrow = d->pages.head_dim == 64;
    const double start = narrow ? 6.2 : 8.0;
    double best = 1e300;
    for (int r = kTileRows; r >= 64; r /= 2) {
        const int64_t blocks = heads * cdiv(rows, r), list = longest_list(d, r), tiles = cdiv(list, kKeyTile);
        // the earlier row blocks of a sequence see fewer keys
        const int64_t mean = list - (list == d->max_ctx ? (d->max_q < list ? d->max_q : list) / 2 : 0);
        const int64_t least = cdiv(tiles, most);
        for (int64_t want = least; want <= tiles && (want == least || blocks * want <= 4096); want += 1 + want / 8) {
            const int64_t per = cdiv(tiles, want), s = cdiv(tiles, per);
            const double step = (r > 128 ? 1.75 : 1.25) * (narrow ? 0.75 : 1.0);
            const double longest = start + (double)per * step;
            double cost = (double)cdiv(blocks * s, 256) * longest;
            if (10 * mean < 9 * list) {
                const double sum = (double)(blocks * s) * (start + (double)per * step * (double)mean / (double)list) / 256;
                cost = longest > 1.1 * sum ? longest : 1.1 * sum;
            }
            if (s > 1) cost += 5.0 + 2.0 * (double)(heads * s * rows) * d->pages.head_dim * 4 / 8e6;
            if (cost < best) {
                best = cost;
                p.block_rows = r;
                p.splits = (int)s;
                p.split_tiles = (int)per;
            }
        }
    }
    p.row_blocks = (int)cdiv(rows, p.block_rows);
    p.blocks = heads / d->pages.batch * counted_blocks(d, p) * p.splits;
    // K and V of a head past the 4 MB of an XCD's L2: its row blocks side by
    // side (bf16, 32/8 heads of 128, 4 sequences of 2048 new tokens: on 30720
    // cached 3979 -> 3836 us; on 4096 it would be 616 -> 623)
    if (p.order == kByLength && longest_list(d, p.block_rows) * d->pages.head_dim * 4 > (4 << 20))
        p.order = kBySequence;
    return best;
}

// The kernel of rows on more than sixteen: 16 or 32 rows per workgroup and
// splits, by modelled time in us.  A round (a tile for each of the four waves)
// takes a workgroup a + b nb, more where others share its CU, and the chip gets
// through 256 of them in c + d nb: with 32 rows a key is fetched for twice as
// many rows, with 16 there are twice as many workgroups of half the work (in
// bf16 they win by more than the model has it: `wide`).  Fitted by least squares
// to the times of 2200 plans of 320 shapes (heads, dims, types, lengths and
// windows drawn over their ranges, a sequence's new tokens and context evenly
// between two bounds): off by 14% and 12% r.m.s.  Measured, 16 and 32 rows: fp32,
// 4/2 heads of 64, 3 sequences of up to 77 tokens 8.5 and 9.8 us; fp32, 32/8 of
// 128, 2048 tokens alone 363 and 326; bf16, 32/8 of 128, 4 x 8 tokens on 8000
// keys 36 both.  Against the kernel of tiles the shorter modelled time decides,
// rows and tiles: 4 x 54 tokens on 182, 8/4 heads of 64, 8.3 and 9.3 us; 28 x 41
// alone, 56/8 of 128, 37 and 20.  On shapes drawn like the fitted ones that was
// within 1 or 2% of the better kernel on average; single shapes miss by more
// (512 tokens on 512 cached, 32/8 heads of 128: 31 us in tiles, 24 in rows).
struct RowsCost {
    double start, a, b, shared, round, c, d, merge, partials, keys, ends, wide;
};
constexpr RowsCost kRowsF32{5.4, 0.2, 1.4, 0.5, 0.45, 0.2, 1.5, 3.4, 0.7, 0.06, 0.0, 1.0};
constexpr RowsCost kRowsBf16{4.7, 0.6, 0.9, 0.15, 1.2, 0.05, 0.95, 3.2, 0.8, 0.09, 1.0, 1.15};

double plan_many_rows(const presto_paged_attn_desc* d, int64_t rows, PagedPlan& p) {
    const bool bf16 = d->pages.dt == PRESTO_DT_BF16;
    const RowsCost& k = bf16 ? kRowsBf16 : kRowsF32;
    const int T = bf16 ? 32 : 16;
    const double dims = d->pages.head_dim / 128.0, batch = d->pages.batch;
    const double ctx = d->total_ctx > 0 ? d->total_ctx / batch : d->max_ctx;
    double best = 1e300, us = best;
    for (int nb = 2; nb >= 1; --nb) {
        PagedPlan x = p;
        x.nb = nb;
        x.block_rows = 16 * nb;
        x.row_blocks = (int)cdiv(rows, x.block_rows);
        const int64_t blocks = d->pages.hkv * counted_blocks(d, x);
        const int64_t list = longest_list(d, x.block_rows), tiles = cdiv(list, T);
        // the keys of a mean block: the earlier ones of a sequence see fewer
        double mean = ctx < list ? ctx : list;
        if (list == d->max_ctx) mean -= d->total_q / batch / 2;
        mean = mean < 1 ? 1 / (double)list : mean / list;
        const double kv_mb = batch * d->pages.hkv * list * d->pages.head_dim * (bf16 ? 4e-6 : 8e-6);
        for (int64_t want = 1; want <= tiles && (want == 1 || blocks * want <= 4096); want += 1 + want / 8) {
            const int64_t per = cdiv(tiles, want), s = cdiv(tiles, per);
            const double rounds = (double)cdiv(per, kWaves), load = (double)(blocks * s) / 256;
            const double alone = k.start + rounds * (k.a + k.b * nb * dims) * (1 + k.shared * (load < 1 ? load : 1));
            const double some = rounds * mean + k.ends < rounds ? rounds * mean + k.ends : rounds;
            const double chip = k.start / 2 + load * (k.round + some * (k.c + k.d * nb) * dims);
            const double fetch = k.start + kv_mb * x.row_blocks * k.keys;
            double cost = alone > chip ? alone : chip;
            if (cost < fetch) cost = fetch;
            if (s > 1) cost += k.merge + k.partials * 4e-6 * (double)(d->total_q * s) * d->hq * d->pages.head_dim;
            const double weighed = nb == 2 ? cost * k.wide : cost;
            if (weighed < best) {
                best = weighed;
                us = cost;
                p = x;
                p.splits = (int)s;
                p.split_tiles = (int)per;
                p.blocks = blocks * s;
            }
        }
    }
    return us;
}

// The kernel of rows.
void plan_rows(const presto_paged_attn_desc* d, int64_t rows, PagedPlan& p) {
    const bool bf16 = d->pages.dt == PRESTO_DT_BF16;
    const int T = bf16 ? 32 : 16;
    p.nb = rows > 16 ? 2 : 1;
    p.block_rows = 16 * p.nb;
    p.row_blocks = 1;
    const int64_t longest = longest_list(d, p.block_rows), tiles = cdiv(longest, T);
    const int64_t all = (int64_t)d->pages.batch * d->pages.hkv;
    int64_t mean = longest;
    if (d->total_ctx > 0 && d->total_ctx / d->pages.batch < mean) mean = d->total_ctx / d->pages.batch + 1;
    const bool even = d->total_ctx > 0 && 10 * mean >= 9 * longest;
    if (rows > 32 || (rows > 16 && (even || d->pages.batch == 1 || tiles <= 3 * kWaves))) {
        plan_many_rows(d, rows, p);
        return;
    }
    // Workgroups that the chip holds at once: three per CU by registers at
    // head_dim 128, two where they have 32 rows
    const int wgs = 256 * (d->pages.head_dim == 64 ? (p.nb == 1 ? 4 : 3) : (p.nb == 1 ? 3 : 2));
    // Few rows are a stream of the cache: what counts is that all CUs end
    // together, and few launches.
    // (bf16, 32/8 heads of 128:)
    // * Sequences of up to three tiles per wave are not cut (no merge: 384 keys
    //   8.8 against 11.5 us).
    // * Sequences of about one length (known from total_ctx) are cut into as
    //   many splits as fill one round: 32 x 2048 keys in 3 splits 48 us, in 6
    //   52; 80 x 2048 uncut 114, in 2 splits 143.
    // * Others in pieces of one length: about one round of them, three where
    //   there are many sequences, each with an end that is not full (us: 16 of
    //   1024 .. 8192 keys 61 in one round, 62 in three; 40 of 1000 .. 9000 155
    //   and 138; 24 of 200 .. 12000 in splits of the longest 157, in pieces 102).
    p.splits = all < wgs ? (int)(wgs / all) : 1;
    p.split_tiles = (int)(cdiv(cdiv(tiles, p.splits), kWaves) * kWaves);
    if (tiles <= 3 * kWaves || p.split_tiles > tiles) p.split_tiles = (int)tiles;
    p.splits = (int)cdiv(tiles, p.split_tiles);
    p.blocks = all * p.splits;
    // (every workgroup looks through the batch for its piece)
    const bool can = d->pages.batch <= 2048 && d->pages.batch * tiles < ((int64_t)1 << 30);
    if (tiles > 3 * kWaves && !even && can) {
        int round = wgs / d->pages.hkv > 0 ? wgs / d->pages.hkv : 1;
        if (4 * d->pages.batch > round) round *= 3;
        // every sequence may end in a piece that is not full
        p.pieces = round > 2 * d->pages.batch ? round - d->pages.batch : (round + 1) / 2;
        p.n_slots = p.pieces + d->pages.batch;
        p.blocks = (int64_t)p.n_slots * d->pages.hkv;
        p.splits = 1;
    }
}

}  // namespace

PagedPlan paged_plan(const presto_paged_attn_desc* d) {
    PagedPlan p{};
    // output rows are numbered in 32 bits, and a grid holds fewer than 2^32 threads
    if ((double)d->pages.batch * d->max_q * d->hq >= 2147483648.0) return p;
    const int64_t out_rows = (int64_t)d->pages.batch * d->max_q * d->hq;
    const int64_t rows = (int64_t)(d->hq / d->pages.hkv) * d->max_q;
    p.tiles = d->pages.dt == PRESTO_DT_BF16 && d->max_q > 1 && rows > 32;
    if (p.tiles) {
        const double tiles_us = plan_tiles(d, rows, p);
        PagedPlan x{};
        if (plan_many_rows(d, rows, x) < tiles_us) p = x;  // (x.tiles: false)
    } else {
        plan_rows(d, rows, p);
    }
    const bool cut = p.splits > 1 || p.pieces > 0;
    if (cut) {
        // four splits or fewer per part
        const int groups = kMergeThreads / (d->pages.head_dim / 4);
        const int each = p.pieces ? p.pieces / d->pages.batch + 2 : p.splits;
        p.merge_parts = 1;
        while (p.merge_parts < groups && p.merge_parts * 4 < each) p.merge_parts *= 2;
        p.merge_blocks = cdiv(out_rows, groups / p.merge_parts);
    }
    p.fits = p.blocks < ((int64_t)1 << 23) && p.merge_blocks < ((int64_t)1 << 24);
    if (cut && p.fits) {
        const int64_t parts = d->pages.hkv * (p.pieces ? (int64_t)p.n_slots : (int64_t)d->pages.batch * p.splits);
        p.o_bytes = (size_t)(parts * rows) * d->pages.head_dim * sizeof(float);
        p.ml_bytes = (size_t)(parts * rows) * sizeof(float2);
        p.bytes = p.o_bytes + p.ml_bytes + (p.pieces ? (size_t)d->pages.batch * sizeof(int2) : 0);
    }
    return p;
}

namespace {

template <bool BF16, int D, int NB>
void launch_rows(const PagedPlan& p, const Args& a, hipStream_t stream) {
    const unsigned grid = (unsigned)p.blocks;
    if (p.row_blocks == 1)
        paged_attn_rows_kernel<BF16, D, NB, kOnce><<<grid, kWaves * kWave, 0, stream>>>(a);
    else
        paged_attn_rows_kernel<BF16, D, NB, kCached><<<grid, kWaves * kWave, 0, stream>>>(a);
}

template <bool BF16, int D>
void launch_attn(const PagedPlan& p, const Args& a, hipStream_t stream) {
    if (p.tiles) {
        if constexpr (BF16)
            paged_attn_tiles_kernel<D><<<(unsigned)p.blocks, kTileWaves * kWave, 0, stream>>>(a);
    } else if (p.nb == 1) {
        launch_rows<BF16, D, 1>(p, a, stream);
    } else {
        launch_rows<BF16, D, 2>(p, a, stream);
    }
    if (p.splits > 1 || p.pieces > 0) {
        constexpr int T = BF16 ? 32 : 16;
        const unsigned grid = (unsigned)p.merge_blocks;
        const int parts = p.merge_parts;
        if (p.tiles)
            paged_attn_merge_kernel<BF16, D, kKeyTile>
                <<<grid, kMergeThreads, 0, stream>>>(a, parts);
        else
            paged_attn_merge_kernel<BF16, D, T><<<grid, kMergeThreads, 0, stream>>>(a, parts);
    }
}

}  // namespace

presto_status launch_paged_attn(const presto_paged_attn_desc* d, const PagedPlan& p, const void* q, const int32_t* q_off,
                                const void* kp, const void* vp, const int32_t* table, const int32_t* ctx, void* out,
                                int32_t* flags, void* ws, hipStream_t stream) {
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
    a.block_rows = p.block_rows;
    a.order = p.order;
    a.splits = p.splits;
    a.split_tiles = p.split_tiles;
    a.pieces = p.pieces;
    a.n_slots = p.n_slots;
    a.slots = reinterpret_cast<int2*>(static_cast<char*>(ws) + p.o_bytes + p.ml_bytes);
    a.scale_log2 = d->scale * kLog2e;
    const bool bf16 = d->pages.dt == PRESTO_DT_BF16;
    if (d->pages.head_dim == 128)
        bf16 ? launch_attn<true, 128>(p, a, stream) : launch_attn<false, 128>(p, a, stream);
    else
        bf16 ? launch_attn<true, 64>(p, a, stream) : launch_attn<false, 64>(p, a, stream);
    return check_launch("paged_attn kernel");
}

}  // namespace presto_host
