// What the attention kernels over a paged cache share (paged_attn.cu, paged_attn_q4.cu): the call's arguments, the line of tiles that is
// cut into equal pieces, the kernel that joins the pieces' partial results, and the checks on the host.
#pragma once

#include <algorithm>

#include "launchers.h"
#include "paged.cuh"
#include "sm100.cuh"

namespace metok {

namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kLow = -3.0e38f;                       // below every logit: keeps differences free of inf - inf

struct PagedAttnArgs {
    PagedDims d;
    int Hq, G, NC, heads;                              // heads per K/V head, units per (sequence, K/V head), heads of a unit at most
    int grid, tile_shift;                              // CTAs of the first kernel; rows of a tile
    const void* q;
    long long q_seq, q_head, out_seq, out_head;
    const int32_t *block_table, *kv_len, *positions;
    const float* slopes;
    float scale_log2, cap_scale, cap_log2;             // softcap > 0: x = cap_log2 * tanh(dot * cap_scale); else cap_log2 is 0
    float* mass;
    void* out;
    float *lse, *part_o, *part_ml, *logits;
    long long* line;                                   // [n_seqs + 1]: tiles of the sequences before each, per unit; then of all
    int32_t* status;
    int withhold;                                      // debug builds: the copies to leave out
};

// Tiles of sequence b's one unit (0 for a length out of range, which the second kernel reports).
__device__ __forceinline__ int unit_tiles(const PagedAttnArgs& a, int b) {
    const int len = a.kv_len[b];
    return len > 0 && len <= a.d.S_cap() ? (len + (1 << a.tile_shift) - 1) >> a.tile_shift : 0;
}

// Tiles of all sequences, per unit; whole CTA.  Up to 32 sequences every warp finds out by itself: no barrier.
__device__ __forceinline__ long long line_tiles(const PagedAttnArgs& a, long long* s_sum) {
    if (a.d.n_seqs <= 32) {
        const int lane = threadIdx.x & 31;
        return (long long)__reduce_add_sync(0xFFFFFFFFu, lane < a.d.n_seqs ? unit_tiles(a, lane) : 0);
    }
    long long all = 0;
    for (int i = threadIdx.x; i < a.d.n_seqs; i += blockDim.x) all += unit_tiles(a, i);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) all += __shfl_xor_sync(0xFFFFFFFFu, all, o);
    if ((threadIdx.x & 31) == 0) s_sum[threadIdx.x >> 5] = all;
    __syncthreads();
    all = 0;
    for (int w = 0; w < (int)(blockDim.x >> 5); ++w) all += s_sum[w];
    return all;
}

// The line for the second kernel: one warp, 32 sequences at a time.
__device__ __forceinline__ void write_line(const PagedAttnArgs& a) {
    const int lane = threadIdx.x & 31;
    long long before = 0;
    for (int b0 = 0; b0 < a.d.n_seqs; b0 += 32) {
        const int b = b0 + lane, mine = b < a.d.n_seqs ? unit_tiles(a, b) : 0;
        int incl = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int x = __shfl_up_sync(0xFFFFFFFFu, incl, o);
            if (lane >= o) incl += x;
        }
        if (b < a.d.n_seqs) a.line[b] = before + incl - mine;
        before += __shfl_sync(0xFFFFFFFFu, incl, 31);
    }
    if (lane == 0) a.line[a.d.n_seqs] = before;
}

// CTAs that have tiles: each of them at least one.
__device__ __forceinline__ long long busy_ctas(const PagedAttnArgs& a, long long tiles) { return min((long long)a.grid, tiles); }

// Where a CTA is in the line: the unit, its tiles, and the tile.
struct Place {
    int b, sub, nt, t;                                 // sub: (K/V head, head chunk) of sequence b
    long long left;                                    // tiles still to do
};
__device__ __forceinline__ void next_tile(const PagedAttnArgs& a, Place& p, int subs) {
    --p.left;
    if (++p.t < p.nt) return;
    p.t = 0;
    if (++p.sub < subs) return;
    p.sub = 0;
    if (p.left > 0) {
        do { ++p.b; p.nt = unit_tiles(a, p.b); } while (p.nt == 0 && p.b + 1 < a.d.n_seqs);   // tiles are left: it finds them
    }
}

// a / b of numbers that mostly have 32 bits.
__device__ __forceinline__ long long quotient(long long a, long long b) {
    return ((unsigned long long)(a | b) >> 32) == 0 ? (long long)((uint32_t)a / (uint32_t)b) : a / b;
}

// The tiles of up to 256 sequences, per unit, as a warp's lanes hold them: lane l those of sequences l, l + 32 and so on.
constexpr int kHeldSeqs = 256;
struct HeldTiles {
    uint32_t n[kHeldSeqs / 32], all;
    __device__ __forceinline__ void load(const PagedAttnArgs& a) {
        const int lane = threadIdx.x & 31;
        uint32_t sum = 0;
#pragma unroll
        for (int i = 0; i < kHeldSeqs / 32; ++i) {
            n[i] = 32 * i + lane < a.d.n_seqs ? unit_tiles(a, 32 * i + lane) : 0;
            sum += n[i];
        }
        all = __reduce_add_sync(0xFFFFFFFFu, sum);     // (sequences of 2^24 rows in tiles of 32 at least)
    }
    // The place of tile t_lo of the line, which has less than 2^31 of them.
    __device__ __forceinline__ Place find(int subs, uint32_t t_lo, uint32_t t_hi) const {
        const int lane = threadIdx.x & 31;
        Place p;
        uint32_t at = 0;
#pragma unroll
        for (int i = 0; i < kHeldSeqs / 32; ++i) {
            uint32_t incl = n[i];
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const uint32_t x = __shfl_up_sync(0xFFFFFFFFu, incl, o);
                if (lane >= o) incl += x;
            }
            const uint32_t any = __ballot_sync(0xFFFFFFFFu, (at + incl) * subs > t_lo);
            if (any) {
                const int l = __ffs(any) - 1;
                const uint32_t start = (at + __shfl_sync(0xFFFFFFFFu, incl - n[i], l)) * subs;
                p.b = 32 * i + l;
                p.nt = (int)__shfl_sync(0xFFFFFFFFu, n[i], l);
                p.sub = (int)((t_lo - start) / p.nt);
                p.t = (int)(t_lo - start - (uint32_t)p.sub * p.nt);
                p.left = t_hi - t_lo;
                return p;
            }
            at += __shfl_sync(0xFFFFFFFFu, incl, 31);
        }
        return {0, 0, 0, 0, 0};
    }
};

// The sequence that has tile t_lo, and the tiles before it: looked for 32 sequences at a time.  Whole warp.  N: a type that holds all tiles.
template <typename N>
__device__ __forceinline__ int find_sequence(const PagedAttnArgs& a, int subs, N t_lo, N* start) {
    const int lane = threadIdx.x & 31;
    N at = 0;                                          // tiles before sequence b0
    for (int b0 = 0; b0 < a.d.n_seqs; b0 += 32) {
        const int b = b0 + lane;
        N mine = b < a.d.n_seqs ? (N)unit_tiles(a, b) * subs : 0, incl = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const N x = __shfl_up_sync(0xFFFFFFFFu, incl, o);
            if (lane >= o) incl += x;
        }
        const uint32_t any = __ballot_sync(0xFFFFFFFFu, at + incl > t_lo);
        if (any) {
            const int l = __ffs(any) - 1;
            *start = at + __shfl_sync(0xFFFFFFFFu, incl - mine, l);
            return b0 + l;
        }
        at += __shfl_sync(0xFFFFFFFFu, incl, 31);
    }
    *start = 0;
    return 0;
}
__device__ __forceinline__ Place place_in(const PagedAttnArgs& a, int b, long long start, long long t_lo, long long t_hi) {
    Place p;
    p.b = b;
    p.nt = unit_tiles(a, b);
    const long long in = t_lo - start;
    p.sub = (int)quotient(in, p.nt);
    p.t = (int)(in - (long long)p.sub * p.nt);
    p.left = t_hi - t_lo;
    return p;
}
// The place of tile t_lo of T_all, for a warp.
__device__ __forceinline__ Place find_tile(const PagedAttnArgs& a, int subs, long long T_all, long long t_lo, long long t_hi) {
    if (T_all <= 0x7FFFFFFF) {
        int start;
        const int b = find_sequence<int>(a, subs, (int)t_lo, &start);
        return place_in(a, b, start, t_lo, t_hi);
    }
    long long start;
    const int b = find_sequence<long long>(a, subs, t_lo, &start);
    return place_in(a, b, start, t_lo, t_hi);
}
// The same for a whole CTA: up to 32 sequences every warp looks for itself.
__device__ __forceinline__ Place find_place(const PagedAttnArgs& a, int subs, long long t_lo, long long t_hi, int* s_b, long long* s_start) {
    Place p;
    long long start = 0;
    p.b = 0;
    const int warp = __shfl_sync(0xFFFFFFFFu, (int)threadIdx.x >> 5, 0);           // the same for all lanes, to the compiler too (0.3 us)
    if (warp == 0 || a.d.n_seqs <= 32) p.b = find_sequence<long long>(a, subs, t_lo, &start);
    if (a.d.n_seqs > 32 && threadIdx.x == 0) {
        *s_b = p.b;
        *s_start = start;
    }
    __syncthreads();
    if (a.d.n_seqs > 32) {
        p.b = *s_b;
        start = *s_start;
    }
    p.nt = unit_tiles(a, p.b);
    const long long in = t_lo - start;
    p.sub = (int)(in / p.nt);                          // (64 bits: the caller has just divided so, and the instructions are there)
    p.t = (int)(in - (long long)p.sub * p.nt);
    p.left = t_hi - t_lo;
    return p;
}

// Logit in log2 units of a raw product: scaled, capped, less the distance's share.
__device__ __forceinline__ float logit2(const PagedAttnArgs& a, float dot, float slope2, float far) {
    if (a.cap_log2 > 0.f) dot = a.cap_log2 * tanhf(dot * a.cap_scale);
    else dot *= a.scale_log2;
    return fmaf(-slope2, far, dot);
}

// The partials of a unit: CTAs c0 .. c1, of which CTA c's lies at slot unit + c.
struct Slots { long long first; int n; };
__device__ __forceinline__ Slots unit_slots(const PagedAttnArgs& a, long long all, long long unit, long long f0, int nt) {
    // the CTA that has tile f is the last one with floor(all * c / ctas) <= f
    const long long ctas = busy_ctas(a, all), c0 = ((f0 + 1) * ctas - 1) / all, c1 = ((f0 + nt) * ctas - 1) / all;
    return {unit + c0, (int)(c1 - c0) + 1};
}

// Joins the partials.  The first CTAs: one head's output and lse each, or (kUnits: few partials) those of a unit; the others: the weights of 128
// rows of a sequence.  NT: threads.  kMarked: the first kernel has marked partials that met a bad page, by a sum below 0; else the pages are looked
// up here.
constexpr int kMassRows = 128;                         // rows of a CTA of the second kernel
template <typename T, int DH, int NT, bool kUnits, bool kMarked>
__global__ void __launch_bounds__(NT)
paged_join_kernel(const PagedAttnArgs a) {
    constexpr int kJoinThreads = NT, kShares = NT / kMassRows;           // kShares threads have a row's heads
    // Up to the wait: what needs only the call's inputs, which were complete when the first kernel was let go.
    __shared__ __align__(16) float s_acc[kJoinThreads][4];
    __shared__ float2 s_ml[kJoinThreads];
    extern __shared__ __align__(16) uint8_t s_dyn[];
    const int tid = threadIdx.x, lane = tid & 31;
    const int outs = a.d.n_seqs * (kUnits ? a.d.Hkv * a.NC : a.Hq);
    const bool weights = (int)blockIdx.x >= outs;
    const int chunks = (a.d.S_cap() + kMassRows - 1) / kMassRows;
    const int b = weights ? ((int)blockIdx.x - outs) / chunks : (int)blockIdx.x / (kUnits ? a.d.Hkv * a.NC : a.Hq);
    const int len = a.kv_len[b], subs = a.d.Hkv * a.NC;
    const int row0 = weights ? (((int)blockIdx.x - outs) - b * chunks) * kMassRows : 0;
    // the sequence is sound: only then anything is written for it
    bool ok = len >= 0 && len <= a.d.S_cap();
    if (ok && !kMarked) {
        const int used = (len + (1 << a.d.page_shift) - 1) >> a.d.page_shift;
        bool there = true;
        for (int p = tid; p < used; p += kJoinThreads) {
            const int page = a.block_table[(size_t)b * a.d.max_pages + p];
            there &= page >= 0 && page < a.d.n_pages;
        }
        ok = __syncthreads_and(there);
    }
    const int nt = unit_tiles(a, b);
    long long all = 0, base = 0;                       // tiles of the line, and of the sequences before b
    const bool few = a.d.n_seqs <= (kMarked ? kHeldSeqs : 32);           // a look at all lengths; else the line that the first kernel wrote
    if (few && kMarked) {
        uint32_t sum = 0, before = 0;
        for (int i = lane; i < a.d.n_seqs; i += 32) {
            const uint32_t mine = unit_tiles(a, i);
            sum += mine;
            before += i < b ? mine : 0;
        }
        all = (long long)__reduce_add_sync(0xFFFFFFFFu, sum) * subs;
        base = (long long)__reduce_add_sync(0xFFFFFFFFu, before) * subs;
    } else if (few) {
        const int mine = lane < a.d.n_seqs ? unit_tiles(a, lane) : 0;
        all = (long long)__reduce_add_sync(0xFFFFFFFFu, mine) * subs;
        base = (long long)__reduce_add_sync(0xFFFFFFFFu, lane < b ? mine : 0) * subs;
    } else {
        grid_dep_wait();
        all = a.line[a.d.n_seqs] * subs;
        base = a.line[b] * subs;
    }

    const auto sound = [&] {
        if (few) grid_dep_wait();
        if (!ok && tid == 0) *a.status = METOK_ERR_INVALID_ARG;
        return ok;
    };

    if constexpr (kUnits) {
        if (!weights) {
            // a thread has four elements of a head, of all partials
            constexpr int kLanes = DH / 4, kAhead = 6;
            const int sub = (int)blockIdx.x - b * subs, hk = sub / a.NC, ch = sub - hk * a.NC, nh = min(a.heads, a.G - ch * a.heads);
            const Slots sl = nt ? unit_slots(a, all, (long long)b * subs + sub, base + (long long)sub * nt, nt) : Slots{0, 0};
            if (!sound()) return;
            const int col = tid % kLanes;
            for (int hl = tid / kLanes; hl < nh; hl += NT / kLanes) {
                const int h = hk * a.G + ch * a.heads + hl;
                float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
                float M = kLow, L = 0.f;
                bool bad = false;
                for (int i0 = 0; i0 < sl.n; i0 += kAhead) {
                    float2 ml[kAhead];
                    float4 o[kAhead];
#pragma unroll
                    for (int u = 0; u < kAhead; ++u) {
                        const size_t at = (size_t)(sl.first + i0 + u) * a.heads + hl;
                        const bool in = i0 + u < sl.n;
                        ml[u] = in ? *reinterpret_cast<const float2*>(a.part_ml + at * 2) : make_float2(kLow, 0.f);
                        o[u] = in ? reinterpret_cast<const float4*>(a.part_o + at * DH)[col] : make_float4(0.f, 0.f, 0.f, 0.f);
                    }
                    float top = M;
#pragma unroll
                    for (int u = 0; u < kAhead; ++u) {
                        top = fmaxf(top, ml[u].x);
                        bad |= kMarked && ml[u].y < 0.f;
                    }
                    const float less = sm100::fast_exp2(M - top);
                    M = top;
                    L *= less;
                    acc.x *= less; acc.y *= less; acc.z *= less; acc.w *= less;
#pragma unroll
                    for (int u = 0; u < kAhead; ++u) {
                        const float f = sm100::fast_exp2(ml[u].x - M);
                        L += f * ml[u].y;
                        acc.x += f * o[u].x; acc.y += f * o[u].y; acc.z += f * o[u].z; acc.w += f * o[u].w;
                    }
                }
                if (bad) {
                    *a.status = METOK_ERR_INVALID_ARG;
                    continue;
                }
                T* out = reinterpret_cast<T*>(a.out) + b * a.out_seq + h * a.out_head + col * 4;
                const float inv = L == 0.f ? 0.f : 1.f / L;              // 0: no rows, or every logit is -infinity
                from_float(out[0], acc.x * inv);
                from_float(out[1], acc.y * inv);
                from_float(out[2], acc.z * inv);
                from_float(out[3], acc.w * inv);
                if (col == 0 && a.lse) a.lse[(size_t)b * a.Hq + h] = nt ? kLn2 * (M + log2f(L)) : __int_as_float(0xFF800000);
            }
            return;
        }
    } else if (!weights) {
        const int h = (int)blockIdx.x - b * a.Hq, hk = h / a.G, g = h - hk * a.G, ch = g / a.heads, hl = g - ch * a.heads;
        T* out = reinterpret_cast<T*>(a.out) + b * a.out_seq + h * a.out_head;
        const int sub = hk * a.NC + ch;
        const Slots sl = nt ? unit_slots(a, all, (long long)b * subs + sub, base + (long long)sub * nt, nt) : Slots{0, 0};
        if (!sound()) return;
        if (nt == 0) {
            for (int i = tid; i < DH; i += kJoinThreads) from_float(out[i], 0.f);
            if (tid == 0 && a.lse) a.lse[(size_t)b * a.Hq + h] = __int_as_float(0xFF800000);
            return;
        }
        // DH / 4 threads side by side, kRuns slots at a time, each run with a maximum of its own
        constexpr int kLanes = DH / 4, kRuns = kJoinThreads / kLanes;
        const int col = tid % kLanes, run = tid / kLanes;
        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
        float M = kLow, L = 0.f;
        bool bad = false;
        constexpr int kAhead = 6;                      // slots whose loads are on their way
        for (int i0 = run; i0 < sl.n; i0 += kRuns * kAhead) {
            float2 ml[kAhead];
            float4 o[kAhead];
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const size_t at = (size_t)(sl.first + i0 + u * kRuns) * a.heads + hl;
                const bool in = i0 + u * kRuns < sl.n;
                ml[u] = in ? *reinterpret_cast<const float2*>(a.part_ml + at * 2) : make_float2(kLow, 0.f);
                o[u] = in ? reinterpret_cast<const float4*>(a.part_o + at * DH)[col] : make_float4(0.f, 0.f, 0.f, 0.f);
            }
            float top = M;
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                top = fmaxf(top, ml[u].x);
                bad |= kMarked && ml[u].y < 0.f;
            }
            const float less = sm100::fast_exp2(M - top);
            M = top;
            L *= less;
            acc.x *= less; acc.y *= less; acc.z *= less; acc.w *= less;
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const float f = sm100::fast_exp2(ml[u].x - M);
                L += f * ml[u].y;
                acc.x += f * o[u].x; acc.y += f * o[u].y; acc.z += f * o[u].z; acc.w += f * o[u].w;
            }
        }
        *reinterpret_cast<float4*>(s_acc[tid]) = acc;
        s_ml[tid] = make_float2(M, L);
        if constexpr (kMarked) {
            if (__syncthreads_or(bad)) {
                if (tid == 0) *a.status = METOK_ERR_INVALID_ARG;
                return;
            }
        } else {
            __syncthreads();
        }
        if (run == 0) {
#pragma unroll
            for (int r = 1; r < kRuns; ++r) M = fmaxf(M, s_ml[r * kLanes + col].x);
            L = 0.f;
            acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int r = 0; r < kRuns; ++r) {
                const float4 o = *reinterpret_cast<const float4*>(s_acc[r * kLanes + col]);
                const float2 ml = s_ml[r * kLanes + col];
                const float f = sm100::fast_exp2(ml.x - M);
                acc.x += f * o.x; acc.y += f * o.y; acc.z += f * o.z; acc.w += f * o.w;
                L += f * ml.y;
            }
            const float inv = L == 0.f ? 0.f : 1.f / L;                  // 0: every logit is -infinity
            from_float(out[col * 4], acc.x * inv);
            from_float(out[col * 4 + 1], acc.y * inv);
            from_float(out[col * 4 + 2], acc.z * inv);
            from_float(out[col * 4 + 3], acc.w * inv);
            if (col == 0 && a.lse) a.lse[(size_t)b * a.Hq + h] = kLn2 * (M + log2f(L));
        }
        return;
    }

    // weights: where every unit's partials and every head's logits lie, then the heads' normalisers: eight threads per head, a running
    // (maximum, sum) each with kAhead loads on their way; the first heads' logits come meanwhile
    long long* s_first = reinterpret_cast<long long*>(s_dyn);            // [subs]
    int* s_n = reinterpret_cast<int*>(s_first + subs);                   // [subs]
    float* s_lse = reinterpret_cast<float*>(s_n + subs);                 // [Hq]: log2 of the sum
    long long* s_off = reinterpret_cast<long long*>(s_dyn + ((size_t)subs * 12 + (size_t)a.Hq * 4 + 7) / 8 * 8);   // [Hq]: the head's logits of the sequence
    for (int sub = tid; sub < subs && nt; sub += kJoinThreads) {
        const Slots sl = unit_slots(a, all, (long long)b * subs + sub, base + (long long)sub * nt, nt);
        s_first[sub] = sl.first;
        s_n[sub] = sl.n;
    }
    for (int h = tid; h < a.Hq; h += kJoinThreads) {
        const int hk = h / a.G, g = h - hk * a.G, ch = g / a.heads;
        s_off[h] = ((long long)(hk * a.NC + ch) * nt * a.heads + (g - ch * a.heads)) << a.tile_shift;
    }
    __syncthreads();
    if (!sound() || row0 >= len) return;
    const int share = tid / kMassRows, row = min(row0 + tid % kMassRows, len - 1), tile = row >> a.tile_shift, off = row & ((1 << a.tile_shift) - 1), rows_tile = 1 << a.tile_shift;
    const float* x = a.logits + (size_t)(base + tile) * a.heads * rows_tile + off;
    constexpr int kHeads = 16, kAhead = 10;
    float v[kHeads];
    auto logits_of = [&](int h0) {
#pragma unroll
        for (int u = 0; u < kHeads; ++u) v[u] = h0 + u < a.Hq ? x[s_off[h0 + u]] : kLow;
    };
    logits_of(share * kHeads);
    bool bad = false;
    for (int h0 = 0; h0 < a.Hq; h0 += kJoinThreads / 8) {
        const int h = h0 + (tid >> 3), part = tid & 7;
        float M = kLow, L = 0.f;
        if (h < a.Hq) {
            const int hk = h / a.G, g = h - hk * a.G, ch = g / a.heads, hl = g - ch * a.heads, sub = hk * a.NC + ch;
            const Slots sl = {s_first[sub], s_n[sub]};
            const float2* ml = reinterpret_cast<const float2*>(a.part_ml) + sl.first * a.heads + hl;
            for (int i0 = part; i0 < sl.n; i0 += 8 * kAhead) {
                float2 p[kAhead];
                float top = M;
#pragma unroll
                for (int u = 0; u < kAhead; ++u) p[u] = i0 + 8 * u < sl.n ? ml[(size_t)(i0 + 8 * u) * a.heads] : make_float2(kLow, 0.f);
#pragma unroll
                for (int u = 0; u < kAhead; ++u) {
                    top = fmaxf(top, p[u].x);
                    bad |= kMarked && p[u].y < 0.f;
                }
                L *= sm100::fast_exp2(M - top);
#pragma unroll
                for (int u = 0; u < kAhead; ++u) L += sm100::fast_exp2(p[u].x - top) * p[u].y;
                M = top;
            }
        }
#pragma unroll
        for (int o = 4; o > 0; o >>= 1) {
            const float m2 = __shfl_xor_sync(0xFFFFFFFFu, M, o), l2 = __shfl_xor_sync(0xFFFFFFFFu, L, o), top = fmaxf(M, m2);
            L = L * sm100::fast_exp2(M - top) + l2 * sm100::fast_exp2(m2 - top);
            M = top;
        }
        if (h < a.Hq && part == 0) s_lse[h] = L == 0.f ? 0.f : M + log2f(L);       // (every logit -infinity: weights of 0)
    }
    if constexpr (kMarked) {
        if (__syncthreads_or(bad)) return;             // (the outputs' part reports it)
    } else {
        __syncthreads();
    }
    if (kShares == 1 && row0 + tid >= len) return;
    float sum = 0.f;
    for (int h = share * kHeads; h < a.Hq; h += kShares * kHeads) {      // kHeads loads on their way (a loop of single ones would wait for each)
        if (h != share * kHeads) logits_of(h);
#pragma unroll
        for (int u = 0; u < kHeads; ++u) sum += h + u < a.Hq ? sm100::fast_exp2(v[u] - s_lse[h + u]) : 0.f;
    }
    if constexpr (kShares > 1) {
        s_ml[tid].x = sum;
        __syncthreads();
        if (share) return;
        for (int i = 1; i < kShares; ++i) sum += s_ml[tid + i * kMassRows].x;
    }
    if (row0 + tid < len) a.mass[(size_t)b * a.d.S_cap() + row] += sum / (float)a.Hq;
}


// How the heads of a K/V head are dealt to units, and the line to CTAs.
struct PagedPlan {
    int G, heads, NC, grid, tile_shift;
    size_t slots, tiles;
};
// `heads` of a unit, tiles of 2^tile_shift rows, at most `ctas` CTAs.
inline PagedPlan paged_plan_of(const PagedDims& d, int Hq, int heads, int tile_shift, int ctas) {
    PagedPlan p;
    p.G = Hq / d.Hkv;
    p.heads = heads;
    p.NC = ceil_div(p.G, p.heads);
    p.tile_shift = tile_shift;
    const size_t units = (size_t)d.n_seqs * d.Hkv * p.NC;
    p.tiles = units * (size_t)((d.S_cap() + (1 << p.tile_shift) - 1) >> p.tile_shift);
    p.grid = (int)std::min<size_t>(p.tiles, (size_t)ctas);
    p.slots = units + p.grid;
    return p;
}
inline void paged_carve(Carver& cv, const PagedPlan& p, const PagedDims& d, bool mass, PagedAttnArgs* a) {
    a->part_o = cv.take<float>(p.slots * p.heads * d.dh);
    a->part_ml = cv.take<float>(p.slots * p.heads * 2);
    a->line = cv.take<long long>((size_t)d.n_seqs + 1);
    a->logits = mass ? cv.take<float>(p.tiles * p.heads << p.tile_shift) : nullptr;
}


// Checks what both calls check after the cache's sizes, and fills `a` but for the workspace's pieces.
inline int paged_attention_args(int dtype, const PagedDims& d, const metok_paged_cache* c, const PagedPlan& p, const void* q, int64_t q_seq,
                                int64_t q_head, int Hq, float softmax_scale, float softcap, const float* slopes, const int32_t* positions,
                                float* mass, void* out, int64_t out_seq, int64_t out_head, float* lse, int32_t* status, PagedAttnArgs* a) {
    if (!aligned16(c->k_pool) || !aligned16(c->v_pool) || !aligned16(q) || !aligned16(out)) return METOK_ERR_INVALID_ARG;
    if (!aligned4(c->block_table) || !aligned4(c->kv_len) || !aligned4(slopes) || !aligned4(positions) || !aligned4(mass) ||
        !aligned4(lse) || !aligned4(status))
        return METOK_ERR_INVALID_ARG;
    const int per = 16 / (dtype == METOK_F32 ? 4 : 2);
    if (q_seq < 0 || q_head < 0 || out_seq < 0 || out_head < 0 || (q_seq | q_head | out_seq | out_head) % per) return METOK_ERR_INVALID_ARG;
    // outputs of different heads and sequences do not overlap
    if (!rows_apart(d.n_seqs, out_seq, Hq, out_head, d.dh) || !softmax_numbers(softmax_scale, softcap)) return METOK_ERR_INVALID_ARG;
    const long long join = (long long)d.n_seqs * Hq + (mass ? (long long)d.n_seqs * ((d.S_cap() + kMassRows - 1) / kMassRows) : 0);
    if (join > 0x7FFFFFFFLL) return METOK_ERR_UNSUPPORTED;
    a->d = d;
    a->Hq = Hq; a->G = p.G; a->NC = p.NC; a->heads = p.heads; a->grid = p.grid; a->tile_shift = p.tile_shift;
    a->q = q; a->q_seq = q_seq; a->q_head = q_head; a->out = out; a->out_seq = out_seq; a->out_head = out_head;
    a->block_table = c->block_table; a->kv_len = c->kv_len; a->positions = positions; a->slopes = slopes;
    a->scale_log2 = softmax_scale * kLog2e;
    a->cap_scale = softcap > 0.f ? softmax_scale / softcap : 0.f;
    a->cap_log2 = softcap * kLog2e;
    a->mass = mass; a->lse = lse; a->status = status;
    a->withhold = debug_withheld();
    return METOK_OK;
}
// What has to hold before a plan can be made.
inline int paged_attention_heads(const PagedDims& d, const metok_paged_cache* c, const void* q, const void* out, const int32_t* status, int Hq) {
    if (!c->k_pool || !c->v_pool || !c->block_table || !c->kv_len || !q || !out || !status) return METOK_ERR_INVALID_ARG;
    if (Hq < 1 || Hq % d.Hkv) return METOK_ERR_INVALID_ARG;
    return Hq > 2048 ? METOK_ERR_UNSUPPORTED : METOK_OK;
}
// spread: the first kernel has whole SMs to its CTAs.  The SMs that it leaves first would take all of the second kernel's CTAs, eight or more of them,
// so these ask for as much shared memory as lets them share the SMs evenly (120 + 120 CTAs on 30 SMs: 10.5 us instead of 6).
template <typename T, int DH, int NT, bool kUnits, bool kMarked>
int launch_paged_join(const PagedAttnArgs& a, cudaStream_t st, bool spread = false) {
    {
        METOK_TIMED("paged_join", st);
        const long long blocks = (long long)a.d.n_seqs * (kUnits ? a.d.Hkv * a.NC : a.Hq) + (a.mass ? (long long)a.d.n_seqs * ((a.d.S_cap() + kMassRows - 1) / kMassRows) : 0);
        size_t smem = a.mass ? ((size_t)a.d.Hkv * a.NC * 12 + (size_t)a.Hq * 4 + 7) / 8 * 8 + (size_t)a.Hq * 8 : 0;
        if (spread) {
            const long long share = 224 * 1024 / ((blocks + kNumSMs - 1) / kNumSMs) - 8 * 1024;         // (6 KB are static, 1 KB the system's)
            smem = std::max(smem, (size_t)std::max(share, 0LL));
        }
        METOK_ALLOW_SMEM((paged_join_kernel<T, DH, NT, kUnits, kMarked>), smem);
        launch_chained(paged_join_kernel<T, DH, NT, kUnits, kMarked>, dim3((unsigned)blocks), dim3(NT), smem, st, a);
    }
    METOK_LAUNCH_CHECK();
    return METOK_OK;
}

}  // namespace
}  // namespace metok
