// metok_paged_append and metok_paged_evict: rows into a paged K/V cache, and out of it by accumulated attention weight.
#include "launchers.h"
#include "paged.cuh"

namespace metok {

namespace {

// ---- append -------------------------------------------------------------------------
// A warp copies kAppendChunks 16-byte chunks per lane of one new row (all heads, K then V): a row of 4 heads of 128 bf16 is
// one warp's work, one of 40 fp32 heads that of twenty, so that a step of few rows still fills the SMs.  Reads and writes are
// contiguous pieces of dh elements; what bounds a long call is HBM (53 650 rows of 4 heads of 128: 42 us, 5.2 TB/s), a step's call its launch
// and three round trips (the offsets and lengths, the page, the copy): 6 us.
constexpr int kAppendWarps = 8, kAppendChunks = 4;

struct AppendArgs {
    PagedDims d;
    const uint4 *k_new, *v_new;
    uint4 *k_pool, *v_pool;
    long long k_head, k_row, v_head, v_row;            // in 16-byte chunks
    int n_new, parts;
    const int32_t *block_table, *kv_len, *offsets, *pos_new;
    int32_t* positions;
    float* mass;
    const float* mass_new;
    int32_t *new_len, *status;
};

// Where the new rows of sequences lie, as given by ascending offsets; with offsets that descend anywhere nothing is appended, as a search
// among them would find some sequences' rows and not others'.
struct NewRows {
    int b, lo, hi, len;                                // a sequence, its new rows, and the rows that it holds
};
// The sequence of new row i, one of more than 32: the number of offsets[1 .. n) that are <= i.  Whole warp, 32-ary search.
__device__ __forceinline__ int sequence_of(const int32_t* __restrict__ offsets, int n, int i, int lane) {
    int lo = 0, left = n - 1;                          // it lies in [lo, lo + left]
    while (left > 0) {
        const int step = (left + 31) >> 5, at = lane * step + step - 1;
        const uint32_t beyond = __ballot_sync(0xFFFFFFFFu, at >= left ? true : offsets[1 + lo + at] > i);
        if (!beyond) return lo + left;
        const int skip = (__ffs(beyond) - 1) * step;
        lo += skip;
        left = min(step - 1, left - skip);
    }
    return lo;
}

__global__ void __launch_bounds__(kAppendWarps * 32)
paged_append_kernel(const AppendArgs a) {
    grid_dep_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, S_cap = a.d.S_cap();
    const long long item = blockIdx.x ? (long long)(blockIdx.x - 1) * kAppendWarps + warp : 0;
    const int i = (int)(item / a.parts), part = (int)(item - (long long)i * a.parts);
    // Up to 32 sequences with offsets: every warp looks at all of them at once, a lane each.  Beyond that the CTA looks whether any descend,
    // and the warps search.  (Steps in a graph, with the check and before there was one: 16 sequences 3.1 and 3.3 us, 40 sequences 4.1 and 3.8;
    // 300 sequences of 200 rows 49.5 and 47.6.)
    const bool few = a.offsets && a.d.n_seqs <= 32;
    NewRows r = {i, i, i + 1, 0}, mine = {lane, 0, 0, 0};
    bool none = false;
    if (few) {
        if (lane < a.d.n_seqs) mine = {lane, a.offsets[lane], a.offsets[lane + 1], a.kv_len[lane]};
        none = __any_sync(0xFFFFFFFFu, mine.hi < mine.lo);
    } else if (a.offsets) {
        int down = 0;
        for (int s = threadIdx.x; s < a.d.n_seqs; s += kAppendWarps * 32) down |= a.offsets[s + 1] < a.offsets[s];
        none = __syncthreads_or(down);
    }
    auto of_few = [&](int b) { return NewRows{b, __shfl_sync(0xFFFFFFFFu, mine.lo, b), __shfl_sync(0xFFFFFFFFu, mine.hi, b), __shfl_sync(0xFFFFFFFFu, mine.len, b)}; };
    auto of_many = [&](int b) { return NewRows{b, a.offsets ? a.offsets[b] : b, a.offsets ? a.offsets[b + 1] : b + 1, a.kv_len[b]}; };
    if (blockIdx.x == 0) {                             // the first CTA checks the sequences and writes their lengths
        int bad = 0;
        for (int b = warp; b < a.d.n_seqs; b += kAppendWarps) {
            r = few ? of_few(b) : of_many(b);
            const int len = r.len, lo = r.lo, hi = r.hi;
            bool ok = !none && lo >= 0 && hi <= a.n_new && len >= 0 && len <= S_cap && hi - lo <= S_cap - len;
            if (ok && hi > lo) {
                const int p1 = (len + hi - lo - 1) >> a.d.page_shift;
                bool there = true;
                for (int p = (len >> a.d.page_shift) + lane; p <= p1; p += 32) {
                    const int page = a.block_table[(size_t)b * a.d.max_pages + p];
                    there &= page >= 0 && page < a.d.n_pages;
                }
                ok = __all_sync(0xFFFFFFFFu, there);
            }
            if (lane == 0) a.new_len[b] = ok ? len + hi - lo : len;
            bad |= !ok;
        }
        bad = __syncthreads_or(bad);
        if (threadIdx.x == 0) *a.status = bad ? METOK_ERR_INVALID_ARG : METOK_OK;
        return;
    }
    if (none || i >= a.n_new) return;
    if (few) r = of_few(__popc(__ballot_sync(0xFFFFFFFFu, lane < a.d.n_seqs - 1 && mine.hi <= i)));
    else r = of_many(a.offsets ? sequence_of(a.offsets, a.d.n_seqs, i, lane) : i);
    const int b = r.b, lo = r.lo, hi = r.hi, len = r.len;
    // the row is the sequence's, and the sequence has room
    if (i < lo || i >= hi || lo < 0 || hi > a.n_new || len < 0 || len > S_cap || hi - lo > S_cap - len) return;
    const int row = len + (i - lo);
    const int page = a.block_table[(size_t)b * a.d.max_pages + (row >> a.d.page_shift)];
    if (page < 0 || page >= a.d.n_pages) return;
    const int cpr = a.d.row_chunks, half = a.d.Hkv * cpr;
    uint4* to[kAppendChunks];
    uint4 v[kAppendChunks];
#pragma unroll
    for (int u = 0; u < kAppendChunks; ++u) {
        int e = part * (32 * kAppendChunks) + u * 32 + lane;
        to[u] = nullptr;
        if (e >= 2 * half) continue;
        const bool is_v = e >= half;
        if (is_v) e -= half;
        const int h = e / cpr, c = e - h * cpr;
        to[u] = (is_v ? a.v_pool : a.k_pool) + paged_chunk(a.d, page, h, row) + c;
        v[u] = __ldg(is_v ? a.v_new + h * a.v_head + i * a.v_row + c : a.k_new + h * a.k_head + i * a.k_row + c);
    }
#pragma unroll
    for (int u = 0; u < kAppendChunks; ++u)
        if (to[u]) *to[u] = v[u];
    if (part == 0 && lane == 0) {
        if (a.positions) {
            int32_t* pos = a.positions + (size_t)b * S_cap;
            pos[row] = a.pos_new ? a.pos_new[i] : (len > 0 ? pos[len - 1] + 1 : 0) + (i - lo);
        }
        if (a.mass) a.mass[(size_t)b * S_cap + row] = a.mass_new ? a.mass_new[i] : 0.f;
    }
}

// ---- evict --------------------------------------------------------------------------
// Two kernels.  select: a CTA per (layer, sequence) checks the sequence's pages against those of all others, finds the rows that
// stay, pairs the holes below the new length with the kept rows behind it, and moves their positions and mass.  move: K and V
// rows of the pairs, and the call's status.  Sources lie at or beyond the new length and places below it, so no order is needed
// between them.  28 layers of 4 sequences of 1734 to 4736 rows, 1263 kept: 85 us, in which rows of 256 bytes move at 5.6 TB/s (from cold
// caches, one kernel after the other: 19 us and 64 us).
struct EvictArgs {
    PagedDims d;
    int L, budget, n_sink, n_recent;
    int claimed;                                       // the pages were claimed by a kernel of their own: bad[] is there already
    int keys_fit;                                      // all keys of a sequence fit into the select kernel's shared memory
    const int32_t *block_table, *kv_len;
    int32_t* positions;
    float* mass;
    int32_t *keep_idx, *new_len, *status;
    int32_t *claim, *bad;                              // [n_pages] and [n_seqs]
    int32_t *from, *to, *n_moved;                      // [L][n_seqs][budget] twice, [L][n_seqs]
};

// Whether a sequence may be touched: its length and pages are in range, no page is its own twice or another's.  A bit per page in
// shared memory marks the sequence's own; then every other sequence's pages are looked up, in every layer.  Beyond so many pages (32 KB of
// bits) or sequences a kernel before it claims the pages for all layers, which with its clearing costs two launches more.  Calls in a graph, 80
// pages a sequence, this way and by claims: 6 layers of 12 sequences 11.3 and 16.2 us, of 24 11.7 and 13.2, of 48 22.8 and 20.9, of 256 149
// and 90; 28 layers of 12 28.7 and 30.6, of 24 46.9 and 43.7, of 256 641 and 381; one layer of 24 11.2 and 13.0, of 48 12.1 and 13.0, of 256
// 33 and 21.
constexpr int kEvictBitPages = 1 << 18, kEvictBitSeqs = 32;
__device__ __forceinline__ bool evict_sound(const EvictArgs& a, int b, uint32_t* s_bits) {
    const int tid = threadIdx.x, nthr = blockDim.x, len = a.kv_len[b], page_rows = 1 << a.d.page_shift;
    if (len < 0 || len > a.d.S_cap()) return false;    // uniform
    const int used = (len + page_rows - 1) >> a.d.page_shift;
    for (int w = tid; w < (a.d.n_pages + 31) / 32; w += nthr) s_bits[w] = 0u;
    __syncthreads();
    int bad = 0;
    for (int p = tid; p < used; p += nthr) {
        const int page = a.block_table[(size_t)b * a.d.max_pages + p];
        if (page < 0 || page >= a.d.n_pages) bad = 1;
        else if (atomicOr(&s_bits[page >> 5], 1u << (page & 31)) >> (page & 31) & 1u) bad = 1;
    }
    bad = __syncthreads_or(bad);
    if (bad) return false;
    // other sequences: a warp each
    for (int s = tid >> 5; s < a.d.n_seqs; s += nthr >> 5) {
        const int other = a.kv_len[s];
        if (s == b || other <= 0 || other > a.d.S_cap()) continue;
        const int n = (other + page_rows - 1) >> a.d.page_shift;
        for (int p = tid & 31; p < n; p += 32) {
            const int page = a.block_table[(size_t)s * a.d.max_pages + p];
            if (page >= 0 && page < a.d.n_pages && (s_bits[page >> 5] >> (page & 31) & 1u)) bad = 1;
        }
    }
    return !__syncthreads_or(bad);
}

// The same by claims in global memory: who meets a page claimed already marks both sequences.
__global__ void __launch_bounds__(256)
evict_claim_kernel(const EvictArgs a) {
    const int b = blockIdx.x, len = a.kv_len[b];
    if (len < 0 || len > a.d.S_cap()) {
        if (threadIdx.x == 0) a.bad[b] = 1;
        return;
    }
    const int used = (len + (1 << a.d.page_shift) - 1) >> a.d.page_shift;
    for (int p = threadIdx.x; p < used; p += 256) {
        const int page = a.block_table[(size_t)b * a.d.max_pages + p];
        if (page < 0 || page >= a.d.n_pages) {
            a.bad[b] = 1;
            continue;
        }
        const int before = atomicExch(&a.claim[page], b + 1);   // every meeting is seen by whoever comes second
        if (before) a.bad[b] = a.bad[before - 1] = 1;
    }
}

// Sum over the threads before this one, and over all: `total`.
__device__ __forceinline__ int block_scan(int v, int* s_warp, int* total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, nwarps = blockDim.x >> 5;
    int incl = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int x = __shfl_up_sync(0xFFFFFFFFu, incl, o);
        if (lane >= o) incl += x;
    }
    if (lane == 31) s_warp[warp] = incl;
    __syncthreads();
    int w = lane < nwarps ? s_warp[lane] : 0;
    const int mine = w;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int x = __shfl_up_sync(0xFFFFFFFFu, w, o);
        if (lane >= o) w += x;
    }
    *total = __shfl_sync(0xFFFFFFFFu, w, 31);
    const int before = __shfl_sync(0xFFFFFFFFu, w - mine, warp);
    __syncthreads();                                   // s_warp may be written again
    return before + incl - v;
}

// Rank key of a row: larger ranks higher.  Protected rows above everything, a NaN above every number.
__device__ __forceinline__ uint32_t evict_key(float mass, int pos, int n_sink, long long recent_from) {
    if (pos < n_sink || (long long)pos > recent_from) return 0xFFFFFFFFu;
    return mass != mass ? 0xFFFFFFFEu : float_key(mass);
}

constexpr int kEvictBuckets = 2048;
constexpr int kEvictKeys = 40960;                      // keys of a sequence that are kept in shared memory (160 KB)

__global__ void __launch_bounds__(1024)
evict_select_kernel(const EvictArgs a) {
    grid_dep_wait();
    extern __shared__ uint32_t s_dyn[];                // the pages' bits, then the keys
    __shared__ uint32_t s_hist[kEvictBuckets];
    __shared__ int s_warp[32];
    __shared__ uint32_t s_prefix;
    __shared__ int s_need, s_all;
    const int b = blockIdx.x, layer = blockIdx.y, S_cap = a.d.S_cap(), tid = threadIdx.x, nthr = blockDim.x;
    const size_t prob = (size_t)layer * a.d.n_seqs + b;
    const int len = a.kv_len[b], n = min(len, a.budget);
    const bool bad = a.claimed ? a.bad[b] != 0 : !evict_sound(a, b, s_dyn);
    int32_t* keep = a.keep_idx + prob * a.budget;
    if (layer == 0 && tid == 0) {
        a.new_len[b] = bad ? len : n;
        a.bad[b] = bad;
    }
    if (bad || len <= a.budget) {
        for (int i = tid; i < a.budget; i += nthr) keep[i] = !bad && i < n ? i : -1;
        if (tid == 0) a.n_moved[prob] = 0;
        return;
    }
    int32_t* pos = a.positions + prob * S_cap;
    float* mass = a.mass + prob * S_cap;
    const long long recent_from = (long long)pos[len - 1] - a.n_recent;
    __syncthreads();                                   // the bits are done with
    if (a.keys_fit)
        for (int i = tid; i < len; i += nthr) s_dyn[i] = evict_key(mass[i], pos[i], a.n_sink, recent_from);
    auto key_of = [&](int i) { return a.keys_fit ? s_dyn[i] : evict_key(mass[i], pos[i], a.n_sink, recent_from); };

    // the n-th highest key, digit by digit from the top
    uint32_t prefix = 0u;                              // its digits so far
    int need = n, done = 0;                            // rows still to take among those with these digits; bits decided
#pragma unroll 1
    while (done < 32) {
        const int bits = done < 22 ? 11 : 10, shift = 32 - done - bits;
        for (int i = tid; i < kEvictBuckets; i += nthr) s_hist[i] = 0u;
        __syncthreads();
        for (int i = tid; i < len; i += nthr) {
            const uint32_t k = key_of(i);
            if (done == 0 || (k >> (32 - done)) == prefix) atomicAdd(&s_hist[(k >> shift) & ((1u << bits) - 1u)], 1u);
        }
        __syncthreads();
        // buckets from the top, a run of them per thread
        const int per = (kEvictBuckets + nthr - 1) / nthr, first = kEvictBuckets - 1 - tid * per;
        int sum = 0, total;
        for (int j = 0; j < per; ++j)
            if (first - j >= 0) sum += (int)s_hist[first - j];
        const int before = block_scan(sum, s_warp, &total);
        if (before < need && need <= before + sum) {   // exactly one thread
            int left = need - before;
            for (int j = 0; j < per; ++j) {
                const int c = (int)s_hist[first - j];
                if (left <= c) {
                    s_prefix = (prefix << bits) | (uint32_t)(first - j);
                    s_need = left;
                    s_all = left == c;
                    break;
                }
                left -= c;
            }
        }
        __syncthreads();
        prefix = s_prefix;
        need = s_need;
        done += bits;
        if (s_all) break;                              // all rows with these digits stay
        __syncthreads();
    }
    // keys of at least `prefix` with zeros behind it stay; where not all equal ones do, the first `need` of them
    if (done < 32) prefix <<= 32 - done;
    const bool by_order = done == 32 && !s_all;

    // rows in order, kRun of them per thread: above the threshold, or among the first `need` equal to it, they stay
    constexpr int kRun = 4;
    int32_t *from = a.from + prob * a.budget, *to = a.to + prob * a.budget;
    int equal = 0, holes = 0, movers = 0;              // so far
#pragma unroll 1
    for (int base = 0; base < len; base += nthr * kRun) {
        const int i0 = base + tid * kRun;
        uint32_t k[kRun];
        int total, eq_before = 0, x = 0;
        bool stay[kRun];
#pragma unroll
        for (int u = 0; u < kRun; ++u) k[u] = i0 + u < len ? key_of(i0 + u) : 0u;
        if (by_order) {
            int eq = 0;
#pragma unroll
            for (int u = 0; u < kRun; ++u) eq += i0 + u < len && k[u] == prefix;
            eq_before = equal + block_scan(eq, s_warp, &total);
            equal += total;
        }
#pragma unroll
        for (int u = 0; u < kRun; ++u) {
            const bool in = i0 + u < len, eq = in && k[u] == prefix;
            stay[u] = in && (k[u] > prefix || (eq && (!by_order || eq_before < need)));
            eq_before += eq;
            x += i0 + u < n ? !stay[u] : stay[u] ? 1 << 16 : 0;           // holes below, movers above: at most 4096 of each
        }
        x = block_scan(x, s_warp, &total);
        int hole = holes + (x & 0xFFFF), mover = movers + (x >> 16);
#pragma unroll
        for (int u = 0; u < kRun; ++u) {
            const int i = i0 + u;
            if (i < n) {
                if (stay[u]) keep[i] = i;
                else to[hole++] = i;
            } else if (stay[u]) {
                from[mover++] = i;
            }
        }
        holes += total & 0xFFFF;
        movers += total >> 16;
    }
    __syncthreads();
    for (int i = n + tid; i < a.budget; i += nthr) keep[i] = -1;
    for (int r = tid; r < movers; r += nthr) {
        const int src = from[r], dst = to[r];
        keep[dst] = src;
        pos[dst] = pos[src];
        mass[dst] = mass[src];
    }
    __syncthreads();
    for (int i = n + tid; i < len; i += nthr) mass[i] = 0.f;
    if (tid == 0) a.n_moved[prob] = movers;
}

constexpr int kEvictPtrLayers = 64;                    // layers per launch of the move
struct EvictPools {
    uint4 *k[kEvictPtrLayers], *v[kEvictPtrLayers];
};
// A thread moves one 16-byte chunk of a pair's row in kMoveHeads of the 2 Hkv heads of K and V: where the rows lie is worked out once for them.
// (One chunk after another, each with divisions of its own, kept the issue slots busy 75 % of the time: 28 layers 98.8 -> 84.7 us the call.)
constexpr int kMoveThreads = 256, kMoveHeads = 8, kMoveMostCtas = 1 << 15;

__global__ void __launch_bounds__(kMoveThreads)
evict_move_kernel(const EvictArgs a, const EvictPools pools, int layer0) {
    grid_dep_wait();
    const int ll = blockIdx.y / a.d.n_seqs, b = blockIdx.y - ll * a.d.n_seqs;
    if (layer0 == 0 && blockIdx.x == 0 && blockIdx.y == 0) {             // the call's status
        int any = 0;
        for (int s = threadIdx.x; s < a.d.n_seqs; s += kMoveThreads) any |= a.bad[s];
        any = __syncthreads_or(any);
        if (threadIdx.x == 0) *a.status = any ? METOK_ERR_INVALID_ARG : METOK_OK;
    }
    const size_t prob = (size_t)(layer0 + ll) * a.d.n_seqs + b;
    const int n = a.n_moved[prob], cpr = a.d.row_chunks, heads = 2 * a.d.Hkv, groups = (heads + kMoveHeads - 1) / kMoveHeads;
    const int32_t *from = a.from + prob * a.budget, *to = a.to + prob * a.budget, *table = a.block_table + (size_t)b * a.d.max_pages;
    const int rows_cta = kMoveThreads / cpr, r0 = threadIdx.x / cpr, c = threadIdx.x - r0 * cpr;      // (8, 16 or 32 chunks a row)
    const size_t head = (size_t)cpr << a.d.page_shift;                   // chunks from head to head of a page
    const long long units = (long long)((n + rows_cta - 1) / rows_cta) * groups;
    for (long long unit = blockIdx.x; unit < units; unit += gridDim.x) {
        const int blk = (int)(unit / groups), h0 = (int)(unit - (long long)blk * groups) * kMoveHeads, r = blk * rows_cta + r0;
        if (r >= n) continue;
        const int s = from[r], t = to[r];
        const size_t src = paged_chunk(a.d, table[s >> a.d.page_shift], 0, s) + c, dst = paged_chunk(a.d, table[t >> a.d.page_shift], 0, t) + c;
        uint4 v[kMoveHeads];
#pragma unroll
        for (int u = 0; u < kMoveHeads; ++u) {
            const int h = h0 + u;
            if (h < heads) v[u] = h < a.d.Hkv ? pools.k[ll][src + h * head] : pools.v[ll][src + (h - a.d.Hkv) * head];
        }
#pragma unroll
        for (int u = 0; u < kMoveHeads; ++u) {
            const int h = h0 + u;
            if (h < heads) (h < a.d.Hkv ? pools.k[ll][dst + h * head] : pools.v[ll][dst + (h - a.d.Hkv) * head]) = v[u];
        }
    }
}

// The same over a cache held in 4 bits: of a row of one head there are dh / 32 chunks of codes and a piece of scales, each a thread's.
__global__ void __launch_bounds__(kMoveThreads)
evict_move_q4_kernel(const EvictArgs a, const EvictPools pools, int layer0) {
    grid_dep_wait();
    const int ll = blockIdx.y / a.d.n_seqs, b = blockIdx.y - ll * a.d.n_seqs;
    if (layer0 == 0 && blockIdx.x == 0 && blockIdx.y == 0) {             // the call's status
        int any = 0;
        for (int s = threadIdx.x; s < a.d.n_seqs; s += kMoveThreads) any |= a.bad[s];
        any = __syncthreads_or(any);
        if (threadIdx.x == 0) *a.status = any ? METOK_ERR_INVALID_ARG : METOK_OK;
    }
    const size_t prob = (size_t)(layer0 + ll) * a.d.n_seqs + b;
    const int dh = a.d.dh, chunks = dh / 32, heads = 2 * a.d.Hkv, groups = (heads + kMoveHeads - 1) / kMoveHeads, n = a.n_moved[prob];
    const int32_t *from = a.from + prob * a.budget, *to = a.to + prob * a.budget, *table = a.block_table + (size_t)b * a.d.max_pages;
    const int rows_cta = kMoveThreads / (chunks + 1), r0 = threadIdx.x / (chunks + 1), c = threadIdx.x - r0 * (chunks + 1);
    const size_t head = (size_t)q4_piece(dh) << (a.d.page_shift - 4);    // bytes from head to head of a page
    const long long units = (long long)((n + rows_cta - 1) / rows_cta) * groups;
    if (r0 >= rows_cta) return;                        // (the CTA's last threads: no row is whole there)
    for (long long unit = blockIdx.x; unit < units; unit += gridDim.x) {
        const int blk = (int)(unit / groups), h0 = (int)(unit - (long long)blk * groups) * kMoveHeads, r = blk * rows_cta + r0;
        if (r >= n) continue;
        const int s = from[r], t = to[r];
        auto place = [&](int row) {
            const size_t piece = q4_piece_of(a.d, table[row >> a.d.page_shift], 0, row) * q4_piece(dh);
            return piece + (c < chunks ? (row & 15) * (dh / 2) + c * 16 : 8 * dh + (row & 15) * (dh / 16));
        };
        const size_t src = place(s), dst = place(t);
        auto pool = [&](int h) { return reinterpret_cast<uint8_t*>(h < a.d.Hkv ? pools.k[ll] : pools.v[ll]) + (h < a.d.Hkv ? h : h - a.d.Hkv) * head; };
        if (c < chunks) {
            uint4 v[kMoveHeads];
#pragma unroll
            for (int u = 0; u < kMoveHeads; ++u)
                if (h0 + u < heads) v[u] = *reinterpret_cast<const uint4*>(pool(h0 + u) + src);
#pragma unroll
            for (int u = 0; u < kMoveHeads; ++u)
                if (h0 + u < heads) *reinterpret_cast<uint4*>(pool(h0 + u) + dst) = v[u];
        } else {
            uint32_t v[kMoveHeads][2];
#pragma unroll
            for (int u = 0; u < kMoveHeads; ++u)
                if (h0 + u < heads) {
                    v[u][0] = *reinterpret_cast<const uint32_t*>(pool(h0 + u) + src);
                    if (dh == 128) v[u][1] = *reinterpret_cast<const uint32_t*>(pool(h0 + u) + src + 4);
                }
#pragma unroll
            for (int u = 0; u < kMoveHeads; ++u)
                if (h0 + u < heads) {
                    *reinterpret_cast<uint32_t*>(pool(h0 + u) + dst) = v[u][0];
                    if (dh == 128) *reinterpret_cast<uint32_t*>(pool(h0 + u) + dst + 4) = v[u][1];
                }
        }
    }
}

}  // namespace
}  // namespace metok

using namespace metok;

extern "C" int metok_paged_append(int dtype, const metok_paged_cache* c, const void* k_new, const void* v_new, int64_t k_head,
                                  int64_t k_row, int64_t v_head, int64_t v_row, int n_new, const int32_t* new_offsets,
                                  int32_t* positions, const int32_t* pos_new, float* mass, const float* mass_new, int32_t* new_len,
                                  int32_t* status, void* stream) {
    PagedDims d;
    const int rc = paged_dims(dtype, c, &d);
    if (rc != METOK_OK) return rc;
    if (!c->k_pool || !c->v_pool || !c->block_table || !c->kv_len || !new_len || !status || n_new < 0) return METOK_ERR_INVALID_ARG;
    if (n_new > 0 && (!k_new || !v_new)) return METOK_ERR_INVALID_ARG;
    if (!aligned16(c->k_pool) || !aligned16(c->v_pool) || !aligned16(k_new) || !aligned16(v_new)) return METOK_ERR_INVALID_ARG;
    if (!aligned4(c->block_table) || !aligned4(c->kv_len) || !aligned4(new_offsets) || !aligned4(positions) || !aligned4(pos_new) ||
        !aligned4(mass) || !aligned4(mass_new) || !aligned4(new_len) || !aligned4(status))
        return METOK_ERR_INVALID_ARG;
    if ((pos_new && !positions) || (mass_new && !mass) || (!new_offsets && n_new != c->n_seqs)) return METOK_ERR_INVALID_ARG;
    if (overlap(new_len, (size_t)c->n_seqs * 4, c->kv_len, (size_t)c->n_seqs * 4)) return METOK_ERR_INVALID_ARG;
    const int per = 16 / (dtype == METOK_F32 ? 4 : 2);                  // elements of a chunk
    if (k_head < 0 || v_head < 0 || k_row < c->dh || v_row < c->dh || (k_head | k_row | v_head | v_row) % per) return METOK_ERR_INVALID_ARG;
    AppendArgs a;
    a.d = d;
    a.k_new = (const uint4*)k_new; a.v_new = (const uint4*)v_new;
    a.k_pool = (uint4*)c->k_pool; a.v_pool = (uint4*)c->v_pool;
    a.k_head = k_head / per; a.k_row = k_row / per; a.v_head = v_head / per; a.v_row = v_row / per;
    a.n_new = n_new;
    a.parts = ceil_div(2 * d.Hkv * d.row_chunks, 32 * kAppendChunks);
    a.block_table = c->block_table; a.kv_len = c->kv_len; a.offsets = new_offsets; a.pos_new = pos_new;
    a.positions = positions; a.mass = mass; a.mass_new = mass_new; a.new_len = new_len; a.status = status;
    const long long blocks = 1 + ((long long)n_new * a.parts + kAppendWarps - 1) / kAppendWarps;
    if (blocks > 0x7FFFFFFFLL) return METOK_ERR_UNSUPPORTED;
    cudaStream_t st = (cudaStream_t)stream;
    {
        METOK_TIMED("paged_append", st);
        launch_chained(paged_append_kernel, dim3((unsigned)blocks), dim3(kAppendWarps * 32), 0, st, a);
    }
    METOK_LAUNCH_CHECK();
    return METOK_OK;
}

namespace {
void evict_carve(Carver& cv, const PagedDims& d, int L, int budget, EvictArgs* a) {
    a->claim = cv.take<int32_t>((size_t)d.n_pages + d.n_seqs);          // one piece: cleared together
    a->bad = a->claim ? a->claim + d.n_pages : nullptr;
    const size_t lists = (size_t)L * d.n_seqs * budget;
    a->from = cv.take<int32_t>(lists);
    a->to = cv.take<int32_t>(lists);
    a->n_moved = cv.take<int32_t>((size_t)L * d.n_seqs);
}
}  // namespace

extern "C" size_t metok_paged_evict_workspace_bytes(const metok_paged_cache* c, int L, int budget) {
    PagedDims d;
    if (paged_dims(METOK_F32, c, &d) != METOK_OK || L < 1 || budget < 1) return 0;
    EvictArgs a;
    Carver cv(nullptr);
    evict_carve(cv, d, L, budget, &a);
    return cv.total();
}

extern "C" int metok_paged_evict(int dtype, const metok_paged_cache* c, void* const* k_layers, void* const* v_layers, int L, int budget,
                                 int n_sink, int n_recent, int32_t* positions, float* mass, int32_t* keep_idx, int32_t* new_len,
                                 int32_t* status, void* ws, size_t ws_bytes, void* stream) {
    PagedDims d;
    const bool q4 = dtype == METOK_Q4;
    const int rc = q4 ? paged_dims_q4(c, &d) : paged_dims(dtype, c, &d);
    if (rc != METOK_OK) return rc;
    if (!c->block_table || !c->kv_len || !k_layers || !v_layers || !positions || !mass || !keep_idx || !new_len || !status)
        return METOK_ERR_INVALID_ARG;
    if (L < 1 || budget < 1 || budget > d.S_cap() || n_sink < 0 || n_recent < 1) return METOK_ERR_INVALID_ARG;
    if (!aligned4(c->block_table) || !aligned4(c->kv_len) || !aligned4(positions) || !aligned4(mass) || !aligned4(keep_idx) ||
        !aligned4(new_len) || !aligned4(status))
        return METOK_ERR_INVALID_ARG;
    if (L > 1024 || (long long)L * c->n_seqs > 65535) return METOK_ERR_UNSUPPORTED;
    uintptr_t at[2 * 1024];
    for (int l = 0; l < L; ++l) {
        if (!k_layers[l] || !v_layers[l] || !aligned16(k_layers[l]) || !aligned16(v_layers[l])) return METOK_ERR_INVALID_ARG;
        at[2 * l] = reinterpret_cast<uintptr_t>(k_layers[l]);
        at[2 * l + 1] = reinterpret_cast<uintptr_t>(v_layers[l]);
    }
    std::sort(at, at + 2 * L);
    const size_t pool = q4 ? ((size_t)d.n_pages * d.Hkv << (d.page_shift - 4)) * q4_piece(d.dh) : ((size_t)d.n_pages * d.Hkv << d.page_shift) * d.row_chunks * 16;
    for (int i = 1; i < 2 * L; ++i)                                     // moved twice, a row would be lost
        if (at[i] - at[i - 1] < pool) return METOK_ERR_INVALID_ARG;
    if (overlap(new_len, (size_t)c->n_seqs * 4, c->kv_len, (size_t)c->n_seqs * 4)) return METOK_ERR_INVALID_ARG;
    if (!ws || !aligned16(ws) || ws_bytes < metok_paged_evict_workspace_bytes(c, L, budget)) return METOK_ERR_WORKSPACE;
    EvictArgs a;
    a.d = d;
    a.L = L; a.budget = budget; a.n_sink = n_sink; a.n_recent = n_recent;
    a.block_table = c->block_table; a.kv_len = c->kv_len; a.positions = positions; a.mass = mass;
    a.keep_idx = keep_idx; a.new_len = new_len; a.status = status;
    Carver cv(ws);
    evict_carve(cv, d, L, budget, &a);
    cudaStream_t st = (cudaStream_t)stream;
    a.claimed = d.n_pages > kEvictBitPages || d.n_seqs > kEvictBitSeqs;
    a.keys_fit = d.S_cap() <= kEvictKeys;
    if (a.claimed) {
        METOK_CUDA_TRY(cudaMemsetAsync(a.claim, 0, ((size_t)d.n_pages + d.n_seqs) * sizeof(int32_t), st));
        METOK_TIMED("evict_claim", st);
        evict_claim_kernel<<<d.n_seqs, 256, 0, st>>>(a);
        METOK_LAUNCH_CHECK();
    }
    {
        const size_t smem = std::max(a.claimed ? 0 : (size_t)(d.n_pages + 31) / 32 * 4, a.keys_fit ? (size_t)d.S_cap() * 4 : 0);
        METOK_ALLOW_SMEM(evict_select_kernel, smem);
        METOK_TIMED("evict_select", st);
        const int threads = std::min(1024, std::max(128, ceil_div(d.S_cap(), 32) * 32));
        launch_chained(evict_select_kernel, dim3(d.n_seqs, L), dim3(threads), smem, st, a);
    }
    METOK_LAUNCH_CHECK();
    // A CTA per 32 KB of the most pairs that a problem can have (the rows behind the new length, or the places below it): how many there
    // are is known on the device alone, and what has no work ends at once.  (A fixed share of the SMs per problem left them idle beside the
    // longest: 28 layers of 4 sequences of 1734 to 4736 rows 113 us the call, 1263 kept.)
    const int rows_cta = kMoveThreads / (q4 ? d.dh / 32 + 1 : d.row_chunks);
    const long long most = (long long)ceil_div(std::min(budget, d.S_cap() - budget), rows_cta) * ceil_div(2 * d.Hkv, kMoveHeads);
    const long long blocks = std::max(1LL, std::min(most, (long long)kMoveMostCtas / (std::min(L, kEvictPtrLayers) * d.n_seqs)));
    for (int l0 = 0; l0 < L; l0 += kEvictPtrLayers) {
        const int nl = std::min(kEvictPtrLayers, L - l0);
        EvictPools pools = {};
        for (int l = 0; l < nl; ++l) {
            pools.k[l] = (uint4*)k_layers[l0 + l];
            pools.v[l] = (uint4*)v_layers[l0 + l];
        }
        METOK_TIMED("evict_move", st);
        launch_chained(q4 ? evict_move_q4_kernel : evict_move_kernel, dim3((unsigned)blocks, nl * d.n_seqs), dim3(kMoveThreads), 0, st, a, pools, l0);
        METOK_LAUNCH_CHECK();
    }
    return METOK_OK;
}
