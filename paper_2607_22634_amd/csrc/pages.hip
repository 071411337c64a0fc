// Bookkeeping of a paged KV cache: giving pages to sequences, sharing them
// between sequences, giving them back, and moving the live ones together.
//
// refs[p] is the number of page-table entries that hold page p (0: free); it
// is all the state there is.  Pages are handed out lowest first, so that the
// result does not depend on the order in which anything runs.  The planning
// kernels are one workgroup each: a pool has 10^2 .. 10^5 pages, whose counts
// one workgroup reads in a few memory round trips, and every step needs the
// totals of the one before.  What is bound by memory bandwidth, moving the
// pages of all layers and writing new rows, runs on the whole chip.
#include <algorithm>

#include "common.hpp"

namespace presto {
namespace pages {

constexpr int kPlanThreads = 1024;
constexpr int kSeqLanes = 16;  // lanes that look at one sequence's columns

// Exclusive prefix sum over the workgroup; `total` for every thread.
__device__ __forceinline__ int block_scan(int v, int* s_wave, int& total) {
    const int incl = (int)wave_scan_dpp((uint32_t)v);
    const int wave = threadIdx.x / kWave, lane = lane_id();
    __syncthreads();  // s_wave may still be read
    if (lane == kWave - 1) s_wave[wave] = incl;
    __syncthreads();
    constexpr int NW = kPlanThreads / kWave;
    const int mine = lane < NW ? s_wave[lane] : 0;
    const int pre = (int)wave_scan_dpp((uint32_t)mine);
    total = __builtin_amdgcn_readlane(pre, NW - 1);
    const int before = wave == 0 ? 0 : __builtin_amdgcn_readlane(pre, __builtin_amdgcn_readfirstlane(wave) - 1);
    return before + incl - v;
}

// Keeps a load where it is written: without a use before the branch that needs
// it, the compiler moves it there, and the loads of a thread then wait for one
// another.
__device__ __forceinline__ void arrived(const uint4& u) { asm volatile("" ::"v"(u.x), "v"(u.y), "v"(u.z), "v"(u.w)); }

struct Four {
    int32_t v[4];
};
// refs[p .. p + 3], `past` beyond the pool
__device__ __forceinline__ Four refs_at(const int32_t* refs, int64_t p, int n, int32_t past) {
    Four f;
    if (p + 4 <= n) {
        __builtin_memcpy(&f, refs + p, sizeof(f));
    } else {
        for (int i = 0; i < 4; ++i) f.v[i] = p + i < n ? refs[p + i] : past;
    }
    return f;
}

// The first `want` free pages in order, into list; returns how many there are
// (at most `want`).  `head`: this thread's counts of the first 4096 pages, asked
// for before the work that says how many pages are wanted.
__device__ __forceinline__ Four pool_head(const int32_t* refs, int n) { return refs_at(refs, 4 * threadIdx.x, n, 1); }
__device__ __forceinline__ int free_pages(const int32_t* refs, const Four& head, int n, int want, int32_t* list,
                                          int* s_wave) {
    int found = 0;
    for (int64_t p0 = 0; p0 < n && found < want; p0 += 4 * kPlanThreads) {
        const int64_t p = p0 + 4 * threadIdx.x;
        const Four f = p0 == 0 ? head : refs_at(refs, p, n, 1);
        int mine = 0, total;
        for (int i = 0; i < 4; ++i) mine += f.v[i] <= 0;
        int at = found + block_scan(mine, s_wave, total);
        for (int i = 0; i < 4; ++i)
            if (f.v[i] <= 0) {
                if (at < want) list[at] = (int32_t)(p + i);
                ++at;
            }
        found += total;
    }
    __syncthreads();
    return min(found, want);
}

// Sum over the kSeqLanes lanes of a sequence.
__device__ __forceinline__ int seq_sum(int v) {
#pragma unroll
    for (int o = kSeqLanes / 2; o > 0; o >>= 1) v += __shfl_xor(v, o, kSeqLanes);
    return v;
}
// This lane's rank among the lanes of its sequence where `set` holds, and
// their number.
__device__ __forceinline__ int seq_rank(bool set, int& count) {
    const int base = lane_id() & ~(kSeqLanes - 1);
    const uint32_t bits = (uint32_t)(__ballot(set) >> base) & ((1u << kSeqLanes) - 1u);
    count = __popc(bits);
    return __popc(bits & ((1u << (lane_id() - base)) - 1u));
}

// Columns ceil(ctx / page) .. ceil(new / page) - 1 of a sequence that hold no
// page get one.  Sequences are served in order; one that does not fit, and
// those after it that need pages, keep their length.
__global__ __launch_bounds__(kPlanThreads) void pages_reserve_kernel(
    int32_t* __restrict__ refs, int32_t* __restrict__ table, const int32_t* ctx, const int32_t* __restrict__ add,
    int32_t extra, int32_t* ctx_out, int32_t batch, int32_t max_pages, int32_t num_pages, int32_t shift,
    int32_t* __restrict__ list, int32_t* __restrict__ need, int32_t* __restrict__ flags) {
    __shared__ int s_wave[kPlanThreads / kWave];
    const int tid = threadIdx.x, sl = tid % kSeqLanes;
    const Four head = pool_head(refs, num_pages);
    constexpr int PER = kPlanThreads / kSeqLanes;
    const int page = 1 << shift;
    // length after the call, -1: not a length
    auto grown = [&](int b, int c) {
        const int64_t a = add ? add[b] : 0, n = (int64_t)c + a + extra;
        return c < 0 || a < 0 || a + extra < 0 || n > (int64_t)max_pages * page ? -1 : (int)n;
    };
    auto cols = [&](int n) { return (int)(((int64_t)n + page - 1) >> shift); };
    bool odd = false;
    for (int b = tid / kSeqLanes; b < batch; b += PER) {
        const int c = ctx[b], n = grown(b, c);
        int miss = 0;
        if (n >= 0)
            for (int x = cols(c) + sl; x < cols(n); x += kSeqLanes) miss += table[(int64_t)b * max_pages + x] < 0;
        miss = seq_sum(miss);
        if (sl == 0) need[b] = miss;
        odd |= n < 0;
    }
    if (odd) raise_flag(flags, PRESTO_FLAG_BAD_SEQ);
    __syncthreads();
    // exclusive prefix of the needs, in place (at most 2^20 columns: the sums
    // of 1024 sequences fit; past 2^31 pages no pool is large enough)
    int64_t total = 0;
    for (int b0 = 0; b0 < batch; b0 += kPlanThreads) {
        const int v = b0 + tid < batch ? need[b0 + tid] : 0;
        int sum;
        const int64_t pre = total + block_scan(v, s_wave, sum);
        if (b0 + tid < batch) need[b0 + tid] = (int)min(pre, (int64_t)0x7fffffff);
        total += sum;
    }
    const int want = (int)min(total, (int64_t)num_pages);
    const int found = free_pages(refs, head, num_pages, want, list, s_wave);
    bool out_of_pages = false;
    for (int b = tid / kSeqLanes; b < batch; b += PER) {
        const int c = ctx[b], n = grown(b, c), pre = need[b];
        int64_t end = pre;  // where this sequence's pages end in the list
        int at = pre;
        if (n >= 0) {
            const int x0 = cols(c), x1 = cols(n);
            int miss = 0;
            for (int x = x0 + sl; x < x1; x += kSeqLanes) miss += table[(int64_t)b * max_pages + x] < 0;
            end += seq_sum(miss);
            if (end == pre || end <= found)
                for (int xb = x0; xb < x1; xb += kSeqLanes) {
                    const int x = xb + sl;
                    const bool none = x < x1 && table[(int64_t)b * max_pages + x] < 0;
                    int count;
                    const int r = seq_rank(none, count);
                    if (none) {
                        const int p = list[at + r];
                        table[(int64_t)b * max_pages + x] = p;
                        refs[p] = 1;
                    }
                    at += count;
                }
        }
        const bool ok = n >= 0 && (end == pre || end <= found);
        out_of_pages |= n >= 0 && !ok;
        if (sl == 0) ctx_out[b] = ok ? n : c;
    }
    if (out_of_pages) raise_flag(flags, PRESTO_FLAG_NO_PAGES);
}

// Moves for pages_move_kernel: (source page, destination page, rows).
struct Move {
    int32_t src, dst, rows, pad;
};

// A child takes its parent's length, shares its full pages and gets a page of
// its own for the rows of the last one.  Wave per fork.
__global__ __launch_bounds__(kPlanThreads) void pages_fork_kernel(
    int32_t* __restrict__ refs, int32_t* __restrict__ table, int32_t* __restrict__ ctx,
    const int32_t* __restrict__ parent, const int32_t* __restrict__ child, int32_t n, int32_t batch,
    int32_t max_pages, int32_t num_pages, int32_t shift, int32_t* list, int32_t* need,
    int32_t* lens, int32_t* first, Move* __restrict__ moves, int32_t* __restrict__ n_moves,
    int32_t* __restrict__ flags) {
    __shared__ int s_wave[kPlanThreads / kWave];
    __shared__ int32_t s_need[kPlanThreads], s_len[kPlanThreads], s_list[kPlanThreads];
    const int tid = threadIdx.x, wave = tid / kWave, lane = lane_id();
    const Four head = pool_head(refs, num_pages);
    const bool few = n <= kPlanThreads;
    if (few) {  // few forks keep their words in LDS
        list = s_list;
        need = s_need;
        lens = s_len;
    } else {  // the first fork that names a child
        for (int i = tid; i < batch; i += kPlanThreads) first[i] = n;
        __syncthreads();
        for (int i = tid; i < n; i += kPlanThreads) {
            const int c = child[i];
            if (c >= 0 && c < batch) atomicMin(&first[c], i);
        }
        __syncthreads();
    }
    constexpr int NW = kPlanThreads / kWave;
    const int page = 1 << shift;
    bool bad = false, short_of = false;
    // everything is read before anything is written
    for (int i = wave; i < n; i += NW) {
        const int p = parent[i], c = child[i];
        bool ok = p >= 0 && p < batch && c >= 0 && c < batch && p != c;
        const int len = ok ? ctx[p] : 0, own = ok ? ctx[c] : 0;
        ok = ok && len >= 0 && len <= (int64_t)max_pages * page && own == 0;
        if (ok) {
            const int used = (int)(((int64_t)len + page - 1) >> shift);
            bool here = true;
            for (int x = lane; x < max_pages; x += kWave) {
                const int e = table[(int64_t)p * max_pages + x];
                here &= table[(int64_t)c * max_pages + x] < 0;
                if (x < used) {
                    // (-1: a page given back; the last one is needed)
                    const bool held = e >= 0 && e < num_pages && refs[e] > 0;
                    here &= held || (e < 0 && !(x == used - 1 && (len & (page - 1))));
                }
            }
            if (few)
                for (int j = lane; j < i; j += kWave) here &= child[j] != c;
            else
                here &= __hip_atomic_load(&first[c], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == i;
            ok = __ballot(!here) == 0;
        }
        if (lane == 0) {
            need[i] = ok && (len & (page - 1)) ? 1 : 0;
            lens[i] = ok ? len : -1;
        }
        bad |= !ok;
    }
    if (bad) raise_flag(flags, PRESTO_FLAG_BAD_SEQ);
    __syncthreads();
    int total = 0;
    for (int i0 = 0; i0 < n; i0 += kPlanThreads) {
        const int v = i0 + tid < n ? need[i0 + tid] : 0;
        int sum;
        const int pre = total + block_scan(v, s_wave, sum);
        if (i0 + tid < n) need[i0 + tid] = pre;
        total += sum;
    }
    const int found = free_pages(refs, head, num_pages, min(total, num_pages), list, s_wave);
    if (tid == 0) *n_moves = found;  // (the forks that get a page are the first ones that need one)
    for (int i = wave; i < n; i += NW) {
        const int len = lens[i];
        if (len < 0) continue;
        const int part = len & (page - 1), full = len >> shift, at = need[i];
        if (part && at >= found) {
            short_of = true;
            continue;
        }
        const int32_t* from = table + (int64_t)parent[i] * max_pages;
        int32_t* to = table + (int64_t)child[i] * max_pages;
        for (int x = lane; x < full; x += kWave) {
            const int e = from[x];
            to[x] = e;
            if (e >= 0) atomicAdd(&refs[e], 1);
        }
        if (lane == 0) {
            if (part) {
                const int p = list[at];
                to[full] = p;
                refs[p] = 1;
                moves[at] = {from[full], p, part, 0};
            }
            ctx[child[i]] = len;
        }
    }
    if (short_of) raise_flag(flags, PRESTO_FLAG_NO_PAGES);
}

// Takes one reference of the entry away; true if something was wrong with it.
__device__ __forceinline__ bool drop(int32_t* refs, int32_t* entry, int32_t num_pages) {
    if (*entry < 0) return false;
    const int e = atomicExch(entry, -1);  // (a sequence named twice is dropped once)
    if (e < 0) return false;
    if (e >= num_pages) return true;
    if (atomicSub(&refs[e], 1) > 0) return false;
    atomicAdd(&refs[e], 1);
    return true;
}

// One workgroup per sequence to drop.
__global__ __launch_bounds__(256) void pages_free_kernel(int32_t* refs, int32_t* table, int32_t* ctx,
                                                         const int32_t* __restrict__ rows, int32_t batch,
                                                         int32_t max_pages, int32_t num_pages, int32_t* flags) {
    const int b = rows[blockIdx.x];
    if (b < 0 || b >= batch) {
        if (threadIdx.x == 0) raise_flag(flags, PRESTO_FLAG_BAD_SEQ);
        return;
    }
    bool bad = false;
    for (int x = threadIdx.x; x < max_pages; x += 256)
        bad |= drop(refs, table + (int64_t)b * max_pages + x, num_pages);
    if (threadIdx.x == 0) ctx[b] = 0;
    if (bad) raise_flag(flags, PRESTO_FLAG_BAD_PAGE);
}

// Pages that hold only positions which no query at position ctx - 1 or later
// sees: those from the sinks' end to the window's start.
__global__ __launch_bounds__(256) void pages_trim_kernel(int32_t* refs, int32_t* table,
                                                         const int32_t* __restrict__ ctx, int32_t max_pages,
                                                         int32_t num_pages, int32_t shift, int32_t window,
                                                         int32_t sinks, int32_t* flags) {
    const int b = blockIdx.x;
    const int64_t len = ctx[b];
    if (len < 0 || len > (int64_t)max_pages << shift) {  // not a length: nothing is given back on its word
        if (threadIdx.x == 0) raise_flag(flags, PRESTO_FLAG_BAD_SEQ);
        return;
    }
    const int64_t x0 = ((int64_t)sinks + (1 << shift) - 1) >> shift;
    const int64_t x1 = len > window ? (len - window) >> shift : 0;
    bool bad = false;
    for (int64_t x = x0 + threadIdx.x; x < x1; x += 256) bad |= drop(refs, table + b * (int64_t)max_pages + x, num_pages);
    if (bad) raise_flag(flags, PRESTO_FLAG_BAD_PAGE);
}

// With L live pages, the i-th free page below L takes the i-th live page from
// L on.  map[p]: where live page p is afterwards, -1 for a free one.
__global__ __launch_bounds__(kPlanThreads) void pages_compact_kernel(const int32_t* refs, int32_t* refs_out,
                                                                     int32_t num_pages, int32_t page,
                                                                     int32_t* __restrict__ map,
                                                                     int32_t* __restrict__ list,
                                                                     Move* __restrict__ moves,
                                                                     int32_t* __restrict__ n_moves,
                                                                     int32_t* __restrict__ n_live) {
    __shared__ int s_wave[kPlanThreads / kWave];
    const int tid = threadIdx.x;
    int mine = 0, live;
    for (int64_t p = 4 * tid; p < num_pages; p += 4 * kPlanThreads) {
        const Four f = refs_at(refs, p, num_pages, 0);
        for (int i = 0; i < 4; ++i) mine += f.v[i] > 0;
    }
    block_scan(mine, s_wave, live);
    if (tid == 0) *n_live = live;
    // below L: live pages stay, free ones are listed (refs_out may be refs:
    // every thread has read its four counts before it writes them)
    int holes = 0;
    for (int64_t p0 = 0; p0 < live; p0 += 4 * kPlanThreads) {
        const int64_t p = p0 + 4 * tid;
        const Four f = refs_at(refs, p, live, 1);
        int free = 0, total;
        for (int i = 0; i < 4; ++i) free += f.v[i] <= 0;
        int at = holes + block_scan(free, s_wave, total);
        for (int i = 0; i < 4; ++i) {
            if (p + i >= live) break;
            if (f.v[i] <= 0) {
                list[at++] = (int32_t)(p + i);
                map[p + i] = -1;
            } else {
                map[p + i] = (int32_t)(p + i);
                refs_out[p + i] = f.v[i];
            }
        }
        holes += total;
    }
    __syncthreads();
    if (tid == 0) *n_moves = holes;  // as many live pages lie from L on
    int done = 0;
    for (int64_t p0 = live; p0 < num_pages; p0 += 4 * kPlanThreads) {
        const int64_t p = p0 + 4 * tid;
        const Four f = refs_at(refs, p, num_pages, 0);
        int cnt = 0, total;
        for (int i = 0; i < 4; ++i) cnt += f.v[i] > 0;
        int at = done + block_scan(cnt, s_wave, total);
        for (int i = 0; i < 4; ++i) {
            if (p + i >= num_pages) break;
            int to = -1;
            if (f.v[i] > 0) {
                to = list[at];
                moves[at++] = {(int32_t)(p + i), to, page, 0};
                refs_out[to] = f.v[i];
            }
            map[p + i] = to;
            refs_out[p + i] = 0;
        }
        done += total;
    }
}

// table_out[i] = map[table[i]]; an entry without a page stays without one.
__global__ __launch_bounds__(256) void pages_remap_kernel(const int32_t* table, int32_t* table_out, int64_t n,
                                                          int32_t num_pages, const int32_t* __restrict__ map,
                                                          int32_t* __restrict__ map_out, int32_t* flags) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    bool bad = false;
    if (i < n) {
        const int e = table[i];
        int to = -1;
        if (e >= 0) {
            to = e < num_pages ? map[e] : -1;
            bad = to < 0;
        }
        table_out[i] = to;
    }
    if (map_out && i < num_pages) map_out[i] = map[i];
    if (bad) raise_flag(flags, PRESTO_FLAG_BAD_PAGE);
}

// Copies the first `rows` rows of page src to page dst, in every layer, of K
// and of V.  A unit is a stretch of kMoveBytes of one page; the pages of a
// call's moves are all different, so units run in any order.  Neighbouring
// units belong to different pools (layers, K and V): every eighth block runs on
// one XCD, which so touches few pools' address translations.  STREAM: past the
// caches, for a compaction's pages, which nobody reads next (1.5 GB moved: 326
// us through them, 310 past them: 5.05 TB/s read and written).
constexpr int kMoveThreads = 256;
constexpr int kMoveLoads = 4;
constexpr int kMoveBytes = kMoveThreads * kMoveLoads * 16;

template <bool STREAM>
__global__ __launch_bounds__(kMoveThreads) void pages_move_kernel(char* __restrict__ k, char* __restrict__ v,
                                                                  const Move* __restrict__ moves,
                                                                  const int32_t* __restrict__ n_moves,
                                                                  int32_t layers, int32_t stretches,
                                                                  int64_t row_bytes, int64_t page_bytes,
                                                                  int64_t layer_bytes) {
    const int64_t units = (int64_t)*n_moves * layers * 2 * stretches;
    for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
        const int pool_id = (int)(u % (2 * layers)), layer = pool_id >> 1;
        char* pool = pool_id & 1 ? v : k;
        const int64_t r = u / (2 * layers);
        const int s = (int)(r % stretches);
        const Move mv = moves[r / stretches];
        const int64_t bytes = mv.rows * row_bytes;
        const int64_t at = (int64_t)s * kMoveBytes + threadIdx.x * 16;
        const char* from = pool + layer * layer_bytes + mv.src * page_bytes;
        char* to = pool + layer * layer_bytes + mv.dst * page_bytes;
        if (at >= bytes) continue;
        uint4 x[kMoveLoads];  // (past the end the last piece is read again)
#pragma unroll
        for (int j = 0; j < kMoveLoads; ++j) {
            const char* p = from + min(at + j * (kMoveThreads * 16), bytes - 16);
            if constexpr (STREAM)
                x[j] = load_stream16(p);
            else
                x[j] = *reinterpret_cast<const uint4*>(p);
        }
#pragma unroll
        for (int j = 0; j < kMoveLoads; ++j) arrived(x[j]);
#pragma unroll
        for (int j = 0; j < kMoveLoads; ++j) {
            const int64_t o = at + j * (kMoveThreads * 16);
            if (o >= bytes) break;
            if constexpr (STREAM)
                __builtin_nontemporal_store((u32x4){x[j].x, x[j].y, x[j].z, x[j].w}, reinterpret_cast<u32x4*>(to + o));
            else
                *reinterpret_cast<uint4*>(to + o) = x[j];
        }
    }
}

// New rows of sequence b go to positions ctx[b] .. ctx_new[b] - 1, a few rows
// of one sequence per workgroup, read past the caches (17,600 rows of 2 KB, K
// and V: 26 us, 31 with the reservation before it; 144 MB at the 5.05 TB/s of a
// compaction take 28.5.  Sixteen rows per workgroup took 10 us more than four).
constexpr int kAppendThreads = 256;
constexpr int kAppendRows = 4;

__global__ __launch_bounds__(kAppendThreads) void append_kv_kernel(
    const char* __restrict__ k_new, const char* __restrict__ v_new, int64_t new_bytes, int64_t new_rows,
    const int32_t* __restrict__ offsets, const int32_t* __restrict__ ctx, const int32_t* __restrict__ ctx_new,
    const int32_t* __restrict__ table, char* __restrict__ k, char* __restrict__ v, int32_t batch, int32_t blocks,
    int32_t max_new, int32_t max_pages, int32_t num_pages, int32_t shift, int32_t row16, int64_t page_bytes,
    int32_t* __restrict__ flags) {
    const int b = blockIdx.x / blocks, i0 = (blockIdx.x % blocks) * kAppendRows;
    const int c = ctx[b];
    const int64_t m = (int64_t)ctx_new[b] - c;
    const int o0 = offsets[b], o1 = offsets[b + 1];
    const int page = 1 << shift;
    const bool bad = c < 0 || m < 0 || o0 < 0 || o1 < o0 || o1 > new_rows || m > o1 - o0 || m > max_new ||
                     (int64_t)c + m > (int64_t)max_pages * page;
    if (bad) {
        if (threadIdx.x == 0 && i0 == 0) raise_flag(flags, PRESTO_FLAG_BAD_SEQ);
        return;
    }
    if (i0 >= m) return;
    const int rows = (int)min((int64_t)kAppendRows, m - i0);
    bool lost = false;
    // four pieces of K and V in flight per thread; past the end the last piece
    // is read again
    constexpr int U = 4;
    const int pieces = rows * row16;
    for (int p0 = threadIdx.x; p0 < pieces; p0 += U * kAppendThreads) {
        int e[U], at[U];
        uint4 kv[U], vv[U];
#pragma unroll
        for (int j = 0; j < U; ++j) {
            const int i = min(p0 + j * kAppendThreads, pieces - 1);
            const int r = i / row16, x = i - r * row16, pos = c + i0 + r;
            e[j] = table[(int64_t)b * max_pages + (pos >> shift)];
            at[j] = (pos & (page - 1)) * row16 + x;
            const int64_t src = (o0 + i0 + r) * new_bytes + x * 16;
            kv[j] = load_stream16(k_new + src);
            vv[j] = load_stream16(v_new + src);
        }
#pragma unroll
        for (int j = 0; j < U; ++j) {
            arrived(kv[j]);
            arrived(vv[j]);
        }
#pragma unroll
        for (int j = 0; j < U; ++j) {
            if (p0 + j * kAppendThreads >= pieces) continue;
            if (e[j] < 0 || e[j] >= num_pages) {
                lost = true;
                continue;
            }
            const int64_t dst = e[j] * page_bytes + (int64_t)at[j] * 16;
            *reinterpret_cast<uint4*>(k + dst) = kv[j];
            *reinterpret_cast<uint4*>(v + dst) = vv[j];
        }
    }
    if (lost) raise_flag(flags, PRESTO_FLAG_BAD_PAGE);
}

}  // namespace pages
}  // namespace presto

namespace presto_host {

using namespace presto;
using namespace presto::pages;

namespace {

int64_t up16(int64_t b) { return (b + 15) / 16 * 16; }

// Workspace: the moves (at most one per page of the pool), the list of free
// pages, the map and three words per sequence or fork.
struct PagesWs {
    Move* moves;
    int32_t *list, *map, *need, *lens, *first, *n_moves;
    size_t bytes;
};
PagesWs pages_ws(void* ws, int64_t num_pages, int64_t n) {
    PagesWs w{};
    const uintptr_t at = reinterpret_cast<uintptr_t>(ws);  // (null where only the size is asked for)
    auto take = [&](int64_t bytes) {
        const uintptr_t p = at + w.bytes;
        w.bytes += (size_t)up16(bytes);
        return p;
    };
    w.moves = reinterpret_cast<Move*>(take(num_pages * (int64_t)sizeof(Move)));
    w.list = reinterpret_cast<int32_t*>(take(num_pages * 4));
    w.map = reinterpret_cast<int32_t*>(take(num_pages * 4));
    w.need = reinterpret_cast<int32_t*>(take(n * 4));
    w.lens = reinterpret_cast<int32_t*>(take(n * 4));
    w.first = reinterpret_cast<int32_t*>(take(n * 4));
    w.n_moves = reinterpret_cast<int32_t*>(take(4));
    return w;
}

int esize(const presto_pages_desc* d) { return d->dt == PRESTO_DT_BF16 ? 2 : 4; }

template <bool STREAM>
void launch_move(const presto_pages_desc* d, void* k, void* v, const PagesWs& w, int64_t max_moves,
                 hipStream_t stream) {
    const int64_t row = (int64_t)d->hkv * d->head_dim * esize(d);
    const int stretches = (int)((row * d->page_size + kMoveBytes - 1) / kMoveBytes);
    // (the number of moves is known to the device only)
    const int64_t units = max_moves * d->layers * 2 * stretches;
    if (units == 0) return;  // (a pool of one page has none to fill)
    const unsigned grid = (unsigned)std::min<int64_t>(units, 256 * 64);
    pages_move_kernel<STREAM><<<grid, kMoveThreads, 0, stream>>>(static_cast<char*>(k), static_cast<char*>(v), w.moves,
                                                         w.n_moves, d->layers, stretches, row,
                                                         d->page_stride * esize(d), d->layer_stride * esize(d));
}

}  // namespace

size_t pages_workspace_bytes(const presto_pages_desc* d, int64_t n) {
    return pages_ws(nullptr, d->num_pages, n).bytes;
}

presto_status launch_pages_reserve(const presto_pages_desc* d, int32_t* refs, int32_t* table, const int32_t* ctx,
                                   const int32_t* add, int32_t extra, int32_t* ctx_out, int32_t* flags, void* ws,
                                   hipStream_t stream) {
    const PagesWs w = pages_ws(ws, d->num_pages, d->batch);
    pages_reserve_kernel<<<1, kPlanThreads, 0, stream>>>(refs, table, ctx, add, extra, ctx_out, d->batch,
                                                         d->max_pages, d->num_pages,
                                                         __builtin_ctz((unsigned)d->page_size), w.list, w.need,
                                                         flags);
    return check_launch("pages_reserve_kernel");
}

presto_status launch_pages_fork(const presto_pages_desc* d, int32_t* refs, int32_t* table, int32_t* ctx,
                                const int32_t* parent, const int32_t* child, int32_t n, void* k, void* v,
                                int32_t* flags, void* ws, hipStream_t stream) {
    const PagesWs w = pages_ws(ws, d->num_pages, d->batch);
    pages_fork_kernel<<<1, kPlanThreads, 0, stream>>>(refs, table, ctx, parent, child, n, d->batch, d->max_pages,
                                                      d->num_pages, __builtin_ctz((unsigned)d->page_size), w.list,
                                                      w.need, w.lens, w.first, w.moves, w.n_moves, flags);
    launch_move<false>(d, k, v, w, n, stream);
    return check_launch("pages_fork_kernel");
}

presto_status launch_pages_free(const presto_pages_desc* d, int32_t* refs, int32_t* table, int32_t* ctx,
                                const int32_t* rows, int32_t n, int32_t* flags, hipStream_t stream) {
    pages_free_kernel<<<(unsigned)n, 256, 0, stream>>>(refs, table, ctx, rows, d->batch, d->max_pages, d->num_pages,
                                                       flags);
    return check_launch("pages_free_kernel");
}

presto_status launch_pages_trim(const presto_pages_desc* d, int32_t* refs, int32_t* table, const int32_t* ctx,
                                int32_t window, int32_t sinks, int32_t* flags, hipStream_t stream) {
    pages_trim_kernel<<<(unsigned)d->batch, 256, 0, stream>>>(refs, table, ctx, d->max_pages, d->num_pages,
                                                              __builtin_ctz((unsigned)d->page_size), window, sinks,
                                                              flags);
    return check_launch("pages_trim_kernel");
}

presto_status launch_pages_compact(const presto_pages_desc* d, const int32_t* refs, int32_t* refs_out,
                                   const int32_t* table, int32_t* table_out, int32_t* n_live, int32_t* map_out,
                                   void* k, void* v, int32_t* flags, void* ws, hipStream_t stream) {
    const PagesWs w = pages_ws(ws, d->num_pages, d->batch);
    pages_compact_kernel<<<1, kPlanThreads, 0, stream>>>(refs, refs_out, d->num_pages, d->page_size, w.map, w.list,
                                                         w.moves, w.n_moves, n_live);
    const int64_t entries = (int64_t)d->batch * d->max_pages;
    const int64_t items = std::max<int64_t>(entries, map_out ? d->num_pages : 0);
    if (items > 0)
        pages_remap_kernel<<<(unsigned)((items + 255) / 256), 256, 0, stream>>>(table, table_out, entries,
                                                                                d->num_pages, w.map, map_out, flags);
    launch_move<true>(d, k, v, w, d->num_pages / 2, stream);
    return check_launch("pages_compact_kernel");
}

presto_status launch_append_kv(const presto_pages_desc* d, const void* k_new, const void* v_new, int64_t new_stride,
                               int64_t new_rows, const int32_t* offsets, int32_t max_new, void* k, void* v,
                               const int32_t* table, const int32_t* ctx, const int32_t* ctx_new, int32_t* flags,
                               hipStream_t stream) {
    const int e = esize(d);
    const int blocks = (max_new + kAppendRows - 1) / kAppendRows;
    append_kv_kernel<<<(unsigned)((int64_t)blocks * d->batch), kAppendThreads, 0, stream>>>(
        static_cast<const char*>(k_new), static_cast<const char*>(v_new), new_stride * e, new_rows, offsets, ctx,
        ctx_new, table, static_cast<char*>(k), static_cast<char*>(v), d->batch, blocks, max_new, d->max_pages,
        d->num_pages, __builtin_ctz((unsigned)d->page_size), (int)((int64_t)d->hkv * d->head_dim * e / 16),
        d->page_stride * e, flags);
    return check_launch("append_kv_kernel");
}

}  // namespace presto_host
