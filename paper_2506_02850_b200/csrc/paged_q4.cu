// metok_paged_append_q4 and metok_paged_read_q4: rows into a paged K/V cache held in 4 bits, and what they stand for back out of it.
//
// A CTA takes up to 32 new (packed) rows: its first warp finds where each of them lies in the cache, a lane each, then a thread takes a block of
// 16 elements (words of eight) of its row in head after head, so that what it works out about the row serves all of them.
// 53 653 rows of 4 heads of 128: in 35 us, 141 MB (20.7 M instructions at 2.5 a clock and SM; a copy of as many bytes takes 26), out 32 us.
// 18 496 rows out: 13 us, 9.9 where outputs stay in L2, 14 from cold caches.  With places worked out for every item 24 M instructions either way and 40 us in; of 64 or more rows a CTA
// takes longer to begin and they go out in 40 to 57 us.
#include "launchers.h"
#include "paged.cuh"
#include "q4.cuh"

namespace metok {

namespace {

constexpr int kThreads = 256, kMostRows = 32, kFewSeqs = 32;
static_assert(kMostRows >= 32, "whole warps find the rows");

struct RowsArgs {
    PagedDims d;
    uint8_t *k_pool, *v_pool;
    char *k_rows, *v_rows;                             // new rows, or outputs
    long long k_head, k_row, v_head, v_row;            // bytes
    int n_rows, rows_shift;                            // rows of all sequences; of a CTA
    const int32_t *block_table, *kv_len, *offsets, *first_row;
    int32_t* positions;                                // of the cache
    const int32_t* pos_new;
    float* mass;
    const float* mass_new;
    int32_t *new_len, *pos_out, *status;
};

// A sequence's share of the packed rows, and the cache's row where it begins.
struct Share {
    int lo, hi, first, len;
    // kAppend: the rows go behind those that are there; else they are there
    template <bool kAppend>
    __device__ __forceinline__ void load(const RowsArgs& a, int b) {
        lo = a.offsets ? a.offsets[b] : b;
        hi = a.offsets ? a.offsets[b + 1] : b + 1;
        len = a.kv_len[b];
        first = kAppend ? len : a.first_row ? a.first_row[b] : 0;
    }
    template <bool kAppend>
    __device__ __forceinline__ bool sound(const RowsArgs& a) const {
        const int S_cap = a.d.S_cap();
        return lo >= 0 && hi <= a.n_rows && len >= 0 && len <= S_cap && first >= 0 && first <= len && hi - lo <= (kAppend ? S_cap : len) - first;
    }
};

// The first CTA checks the sequences: whole CTA.
template <bool kAppend>
__device__ __forceinline__ void check_sequences(const RowsArgs& a, bool none) {
    const int lane = threadIdx.x & 31;
    int bad = none;
    for (int b = threadIdx.x >> 5; b < a.d.n_seqs; b += kThreads / 32) {
        Share r;
        r.load<kAppend>(a, b);
        bool ok = !none && r.sound<kAppend>(a);
        if (ok && r.hi > r.lo) {
            const int p1 = (r.first + r.hi - r.lo - 1) >> a.d.page_shift;
            bool there = true;
            for (int p = (r.first >> a.d.page_shift) + lane; p <= p1; p += 32) {
                const int page = a.block_table[(size_t)b * a.d.max_pages + p];
                there &= page >= 0 && page < a.d.n_pages;
            }
            ok = __all_sync(0xFFFFFFFFu, there);
        }
        if (kAppend && lane == 0) a.new_len[b] = ok ? r.len + r.hi - r.lo : r.len;
        bad |= !ok;
    }
    bad = __syncthreads_or(bad);
    if (threadIdx.x == 0) *a.status = bad ? METOK_ERR_INVALID_ARG : METOK_OK;
}

// Where the CTA's rows lie: page (-1: nowhere) and row of the sequence.  Whole CTA; offsets that descend anywhere leave no row a place.
template <bool kAppend>
__device__ __forceinline__ void find_rows(const RowsArgs& a, int i0, int (&s_page)[kMostRows], int (&s_row)[kMostRows]) {
    const int tid = threadIdx.x, lane = tid & 31, n = a.d.n_seqs, i = i0 + tid;
    const bool mine = tid < (1 << a.rows_shift) && i < a.n_rows, few = a.offsets && n <= kFewSeqs;
    bool none = false;
    if (a.offsets && !few) {
        int down = 0;
        for (int s = tid; s < n; s += kThreads) down |= a.offsets[s + 1] < a.offsets[s];
        none = __syncthreads_or(down);
    }
    if (blockIdx.x == 0) {
        if (few) none = __any_sync(0xFFFFFFFFu, lane < n && a.offsets[lane + 1] < a.offsets[lane]);
        check_sequences<kAppend>(a, none);
        return;
    }
    if (tid < max(32, 1 << a.rows_shift)) {            // whole warps
        Share r = {0, 0, 0, 0};
        int b = 0;
        if (few) {                                     // a sequence per lane
            Share held = {0, 0, 0, 0};
            if (lane < n) held.load<kAppend>(a, lane);
            none = __any_sync(0xFFFFFFFFu, held.hi < held.lo);
            for (int s = 0; s < n; ++s) b += __shfl_sync(0xFFFFFFFFu, held.hi, s) <= i;
            const int at = min(b, n - 1);
            r = {__shfl_sync(0xFFFFFFFFu, held.lo, at), __shfl_sync(0xFFFFFFFFu, held.hi, at), __shfl_sync(0xFFFFFFFFu, held.first, at),
                 __shfl_sync(0xFFFFFFFFu, held.len, at)};
        } else if (mine) {
            b = i;
            if (a.offsets) {                           // the number of offsets[1 .. n] that are <= i: the row's sequence, n for none
                int hi = n;
                b = 0;
                while (b < hi) {
                    const int mid = (b + hi) >> 1;
                    if (a.offsets[1 + mid] <= i) b = mid + 1;
                    else hi = mid;
                }
            }
            if (b < n) r.load<kAppend>(a, b);
        }
        int page = -1, row = 0;
        if (mine && !none && b < n && i >= r.lo && r.sound<kAppend>(a)) {
            row = r.first + (i - r.lo);
            page = a.block_table[(size_t)b * a.d.max_pages + (row >> a.d.page_shift)];
            if (page < 0 || page >= a.d.n_pages) page = -1;
            const size_t at = (size_t)b * a.d.S_cap();
            if (page < 0) {
            } else if (kAppend) {
                if (a.positions)
                    a.positions[at + row] = a.pos_new ? a.pos_new[i] : (r.len > 0 ? a.positions[at + r.len - 1] + 1 : 0) + (i - r.lo);
                if (a.mass) a.mass[at + row] = a.mass_new ? a.mass_new[i] : 0.f;
            } else if (a.pos_out) {
                a.pos_out[i] = a.positions[at + row];
            }
        }
        s_page[tid] = page;
        s_row[tid] = row;
    }
    __syncthreads();
}

// A thread keeps its place in the rows, a block of 16 elements (append) or words of eight (read), and goes over the heads of K and of V.  Of an
// append the next head's elements are on their way, the first ones already while its warps find out where they belong; of a read kReadHeads heads'
// codes at a time.  Where the rows are few, groups of threads share the heads.
constexpr int kReadHeads = 4;

template <typename T, bool kAppend>
__global__ void __launch_bounds__(kThreads)
paged_rows_q4_kernel(const RowsArgs a) {
    constexpr int kOf = kAppend ? 16 : 8, kChunks = kOf * (int)sizeof(T) / 16;       // elements of an item, 16-byte chunks of them
    __shared__ int s_page[kMostRows], s_row[kMostRows];
    grid_dep_wait();
    const int i0 = ((int)blockIdx.x - 1) << a.rows_shift;
    const int dh = a.d.dh, shift = (dh == 128 ? 3 : 2) + (kAppend ? 0 : 1), place_shift = shift + a.rows_shift;
    const int groups = max(1, kThreads >> place_shift), group = (int)threadIdx.x >> place_shift;          // (powers of two)
    const int kv0 = groups > 1 ? group & 1 : 0, kvs = groups > 1 ? kv0 + 1 : 2, h0 = groups > 1 ? group >> 1 : 0, h_step = groups > 1 ? groups >> 1 : 1;
    const long long head = (long long)q4_piece(dh) << (a.d.page_shift - 4);          // bytes from head to head of a page
    const int i = threadIdx.x & ((1 << shift) - 1);
    auto rows_at = [&](int r, int kv) {
        return (kv ? a.v_rows + (i0 + r) * a.v_row + h0 * a.v_head : a.k_rows + (i0 + r) * a.k_row + h0 * a.k_head) + i * (kChunks * 16);
    };
    int place = threadIdx.x & ((1 << place_shift) - 1);
    uint4 x[kChunks];                                  // of an append
    auto fetch = [&](const char* from) {
#pragma unroll
        for (int j = 0; j < kChunks; ++j) x[j] = __ldg(reinterpret_cast<const uint4*>(from) + j);
    };
    if constexpr (kAppend) {
        if (blockIdx.x && i0 + (place >> shift) < a.n_rows && h0 < a.d.Hkv) fetch(rows_at(place >> shift, kv0));
    }
    find_rows<kAppend>(a, i0, s_page, s_row);
    if (blockIdx.x == 0 || h0 >= a.d.Hkv) return;
    for (; place < 1 << place_shift; place += kThreads) {                // (one turn of an append)
        const int r = place >> shift, page = s_page[r], at = s_row[r] & 15;
        if (page < 0) continue;
        const size_t codes = q4_piece_of(a.d, page, 0, s_row[r]) * q4_piece(dh) + at * (dh / 2) + i * (kOf / 2) + h0 * head;
        const int scale = 8 * dh + at * (dh / 16) + (kAppend ? i : i >> 1) - (at * (dh / 2) + i * (kOf / 2));
        const long long code_step = h_step * head;
        for (int kv = kv0; kv < kvs; ++kv) {
            uint8_t* code = (kv ? a.v_pool : a.k_pool) + codes;
            char* row = rows_at(r, kv);
            const long long row_step = h_step * (kv ? a.v_head : a.k_head);
            if constexpr (kAppend) {
                if (kv > kv0) fetch(row);
                for (int h = h0; h < a.d.Hkv; h += h_step) {
                    float v[16];
                    q4_widen<T>(x, v);
                    row += row_step;
                    if (h + h_step < a.d.Hkv) fetch(row);
                    uint32_t c[2];
                    code[scale] = (uint8_t)q4_hold(v, c);
                    *reinterpret_cast<uint2*>(code) = make_uint2(c[0], c[1]);
                    code += code_step;
                }
            } else {
                for (int h = h0; h < a.d.Hkv; h += h_step * kReadHeads) {
                    uint32_t c[kReadHeads], e[kReadHeads];
#pragma unroll
                    for (int u = 0; u < kReadHeads; ++u) {
                        if (h + u * h_step < a.d.Hkv) {
                            c[u] = __ldg(reinterpret_cast<const uint32_t*>(code));
                            e[u] = __ldg(code + scale);
                        }
                        code += code_step;
                    }
#pragma unroll
                    for (int u = 0; u < kReadHeads; ++u) {
                        if (h + u * h_step < a.d.Hkv) {
                            uint4 v[kChunks];
                            q4_stands_for<T>(c[u], e[u], v);
#pragma unroll
                            for (int j = 0; j < kChunks; ++j) reinterpret_cast<uint4*>(row)[j] = v[j];
                        }
                        row += row_step;
                    }
                }
            }
        }
    }
}

// Few rows: few to a CTA, so that they fill the SMs.
int rows_shift_of(int n_rows) {
    int shift = 5;
    while (shift > 0 && (n_rows >> shift) < 4 * kNumSMs) --shift;
    return shift;
}

}  // namespace
}  // namespace metok

using namespace metok;

extern "C" int metok_paged_append_q4(int new_dtype, const metok_paged_cache* c, const void* k_new, const void* v_new, int64_t k_head,
                                     int64_t k_row, int64_t v_head, int64_t v_row, int n_new, const int32_t* new_offsets,
                                     int32_t* positions, const int32_t* pos_new, float* mass, const float* mass_new, int32_t* new_len,
                                     int32_t* status, void* stream) {
    PagedDims d;
    if (new_dtype != METOK_F32 && new_dtype != METOK_BF16) return METOK_ERR_INVALID_ARG;
    const int rc = paged_dims_q4(c, &d);
    if (rc != METOK_OK) return rc;
    if (!c->k_pool || !c->v_pool || !c->block_table || !c->kv_len || !new_len || !status || n_new < 0) return METOK_ERR_INVALID_ARG;
    if (n_new > 0 && (!k_new || !v_new)) return METOK_ERR_INVALID_ARG;
    if (!aligned16(c->k_pool) || !aligned16(c->v_pool) || !aligned16(k_new) || !aligned16(v_new)) return METOK_ERR_INVALID_ARG;
    if (!aligned4(c->block_table) || !aligned4(c->kv_len) || !aligned4(new_offsets) || !aligned4(positions) || !aligned4(pos_new) ||
        !aligned4(mass) || !aligned4(mass_new) || !aligned4(new_len) || !aligned4(status))
        return METOK_ERR_INVALID_ARG;
    if ((pos_new && !positions) || (mass_new && !mass) || (!new_offsets && n_new != c->n_seqs)) return METOK_ERR_INVALID_ARG;
    if (overlap(new_len, (size_t)c->n_seqs * 4, c->kv_len, (size_t)c->n_seqs * 4)) return METOK_ERR_INVALID_ARG;
    const int esize = new_dtype == METOK_F32 ? 4 : 2, per = 16 / esize;
    if (k_head < 0 || v_head < 0 || k_row < c->dh || v_row < c->dh || (k_head | k_row | v_head | v_row) % per) return METOK_ERR_INVALID_ARG;
    RowsArgs a = {};
    a.d = d;
    a.k_pool = (uint8_t*)c->k_pool; a.v_pool = (uint8_t*)c->v_pool;
    a.k_rows = (char*)const_cast<void*>(k_new); a.v_rows = (char*)const_cast<void*>(v_new);
    a.k_head = k_head * esize; a.k_row = k_row * esize; a.v_head = v_head * esize; a.v_row = v_row * esize;
    a.n_rows = n_new; a.rows_shift = rows_shift_of(n_new);
    a.block_table = c->block_table; a.kv_len = c->kv_len; a.offsets = new_offsets; a.pos_new = pos_new;
    a.positions = positions; a.mass = mass; a.mass_new = mass_new; a.new_len = new_len; a.status = status;
    cudaStream_t st = (cudaStream_t)stream;
    {
        METOK_TIMED("paged_append_q4", st);
        const dim3 grid(1 + (unsigned)(((long long)n_new + (1 << a.rows_shift) - 1) >> a.rows_shift));
        if (new_dtype == METOK_F32) launch_chained(paged_rows_q4_kernel<float, true>, grid, dim3(kThreads), 0, st, a);
        else launch_chained(paged_rows_q4_kernel<__nv_bfloat16, true>, grid, dim3(kThreads), 0, st, a);
    }
    METOK_LAUNCH_CHECK();
    return METOK_OK;
}

extern "C" int metok_paged_read_q4(int out_dtype, const metok_paged_cache* c, const int32_t* offsets, const int32_t* first_row, int n_rows,
                                   void* k_out, void* v_out, int64_t k_head, int64_t k_row, int64_t v_head, int64_t v_row,
                                   const int32_t* positions, int32_t* pos_out, int32_t* status, void* stream) {
    PagedDims d;
    if (out_dtype != METOK_F32 && out_dtype != METOK_BF16) return METOK_ERR_INVALID_ARG;
    const int rc = paged_dims_q4(c, &d);
    if (rc != METOK_OK) return rc;
    if (!c->k_pool || !c->v_pool || !c->block_table || !c->kv_len || !offsets || !status || n_rows < 0) return METOK_ERR_INVALID_ARG;
    if (n_rows > 0 && (!k_out || !v_out)) return METOK_ERR_INVALID_ARG;
    if (!aligned16(c->k_pool) || !aligned16(c->v_pool) || !aligned16(k_out) || !aligned16(v_out)) return METOK_ERR_INVALID_ARG;
    if (!aligned4(c->block_table) || !aligned4(c->kv_len) || !aligned4(offsets) || !aligned4(first_row) || !aligned4(positions) ||
        !aligned4(pos_out) || !aligned4(status))
        return METOK_ERR_INVALID_ARG;
    if (pos_out && !positions) return METOK_ERR_INVALID_ARG;
    const int esize = out_dtype == METOK_F32 ? 4 : 2, per = 16 / esize;
    if (k_head < 0 || v_head < 0 || k_row < 0 || v_row < 0 || (k_head | k_row | v_head | v_row) % per) return METOK_ERR_INVALID_ARG;
    if (!rows_apart(d.Hkv, k_head, n_rows, k_row, d.dh) || !rows_apart(d.Hkv, v_head, n_rows, v_row, d.dh)) return METOK_ERR_INVALID_ARG;
    if (n_rows > 0) {
        const Extent k = extent_of(k_out, d.Hkv, k_head, n_rows, k_row, d.dh, esize), v = extent_of(v_out, d.Hkv, v_head, n_rows, v_row, d.dh, esize);
        if (!apart(k, v)) return METOK_ERR_INVALID_ARG;
    }
    RowsArgs a = {};
    a.d = d;
    a.k_pool = (uint8_t*)c->k_pool; a.v_pool = (uint8_t*)c->v_pool;
    a.k_rows = (char*)k_out; a.v_rows = (char*)v_out;
    a.k_head = k_head * esize; a.k_row = k_row * esize; a.v_head = v_head * esize; a.v_row = v_row * esize;
    a.n_rows = n_rows; a.rows_shift = rows_shift_of(n_rows);
    a.block_table = c->block_table; a.kv_len = c->kv_len; a.offsets = offsets; a.first_row = first_row;
    a.positions = const_cast<int32_t*>(positions); a.pos_out = pos_out; a.status = status;
    cudaStream_t st = (cudaStream_t)stream;
    {
        METOK_TIMED("paged_read_q4", st);
        const dim3 grid(1 + (unsigned)(((long long)n_rows + (1 << a.rows_shift) - 1) >> a.rows_shift));
        if (out_dtype == METOK_F32) launch_chained(paged_rows_q4_kernel<float, false>, grid, dim3(kThreads), 0, st, a);
        else launch_chained(paged_rows_q4_kernel<__nv_bfloat16, false>, grid, dim3(kThreads), 0, st, a);
    }
    METOK_LAUNCH_CHECK();
    return METOK_OK;
}
