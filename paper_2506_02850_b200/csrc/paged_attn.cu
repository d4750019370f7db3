// metok_paged_attention: attention of one new token per sequence over its paged K/V cache.
//
// A unit is (sequence, K/V head, up to 8 or 16 query heads of its group); its rows are cut into tiles.  The tiles of all
// units form one line, and every CTA takes an equal piece of it, whatever the lengths: a batch of one long and many short
// sequences keeps all SMs busy to the end.  A CTA leaves, per unit that it met, the running maximum m, sum l and
// unnormalised output o of its rows (a partial); the second kernel joins a unit's partials,
//   M = max m_i,  L = sum 2^(m_i - M) l_i,  out = sum 2^(m_i - M) o_i / L,  lse = ln 2 * (M + log2 L),
// and, where the rows' weights are wanted, turns the logits that the first kernel left into sum_h 2^(x - lse_h) / Hq.
//
// What bounds it is reading K and V once.  One warp brings tiles by TMA (a page's rows of a head are contiguous) through a
// ring of shared memory, four warps compute; every warp has rows of its own of each tile and a running softmax of its own,
// so that the warps meet only where a unit ends.
//   bf16: a warp takes 16 rows of a tile.  x^T = K Q^T (rows x heads) and o^T += V^T P^T by mma.sync m16n8k16: eight heads
//     are a whole side of the product, where the tensor memory path would pad them to 128 (the products are a few per cent of
//     either's rate).  P is split into two bf16 parts, so its rounding is 2^-17: fp32-like sums at no cost in bytes.
//     48 sequences of up to 9001 rows, 28 / 4 heads of 128, capped: 99.7 us, 5.6 TB/s; one of 18 496 rows with weights 17.5 us, of which its 38 MB
//     are 5.8: two launches, filling the ring and the joins' chain of loads are the rest.
//   fp32: eight lanes share a row, four rows at a time; the lanes' partial dot products of several heads are reduced and
//     dealt out in one butterfly.
#include <algorithm>

#include "launchers.h"
#include "paged.cuh"
#include "sm100.cuh"

namespace metok {

namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kLow = -3.0e38f;                       // below every logit: keeps differences free of inf - inf
constexpr int kWarps = 4, kThreads = (kWarps + 1) * 32;

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

// Logit in log2 units of a raw product: scaled, capped, less the distance's share.
__device__ __forceinline__ float logit2(const PagedAttnArgs& a, float dot, float slope2, float far) {
    if (a.cap_log2 > 0.f) dot = a.cap_log2 * tanhf(dot * a.cap_scale);
    else dot *= a.scale_log2;
    return fmaf(-slope2, far, dot);
}

template <typename T, int DH>
struct PagedShape {
    static constexpr bool kBf16 = sizeof(T) == 2;
    static constexpr int kTile = kBf16 ? 64 : 32;      // rows of a tile
    static constexpr int kCols = 128 / sizeof(T);      // elements of a 128-byte swizzled row
    static constexpr int KB = DH / kCols;              // such pieces of a row
    static constexpr uint32_t kBlk = kTile * 128;      // bytes of a piece of all rows
    static constexpr uint32_t kHalf = KB * kBlk;       // K, or V
    static constexpr uint32_t kStage = 2 * kHalf;
    static constexpr int kStages = kStage >= 32768 ? 3 : 6;
    static constexpr size_t kRing = (size_t)kStages * kStage + 1024;
};

// Rows of a unit's running softmax, heads and outputs as the two types hold them, in registers.
// bf16: NG groups of eight heads; lane l holds the logits of rows l / 4 and l / 4 + 8 of the warp's 16 and of heads 2 (l % 4), + 1.
template <int DH, int NG>
struct Bf16Unit {
    uint32_t q[NG][DH / 16][2];
    float m[NG][2], l[NG][2], o[NG][DH / 16][4], slope[NG][2];

    __device__ __forceinline__ void start(const PagedAttnArgs& a, int b, int h0, int nh) {
        const int lane = threadIdx.x & 31;
#pragma unroll
        for (int n = 0; n < NG; ++n) {
            const int h = n * 8 + (lane >> 2);
            const __nv_bfloat16* src = reinterpret_cast<const __nv_bfloat16*>(a.q) + b * a.q_seq + (long long)(h0 + h) * a.q_head + 2 * (lane & 3);
#pragma unroll
            for (int k = 0; k < DH / 16; ++k) {
                q[n][k][0] = h < nh ? *reinterpret_cast<const uint32_t*>(src + k * 16) : 0u;
                q[n][k][1] = h < nh ? *reinterpret_cast<const uint32_t*>(src + k * 16 + 8) : 0u;
            }
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int hc = n * 8 + 2 * (lane & 3) + e;
                m[n][e] = kLow;
                l[n][e] = 0.f;
                slope[n][e] = a.slopes && hc < nh ? a.slopes[h0 + hc] * kLog2e : 0.f;
            }
#pragma unroll
            for (int k = 0; k < DH / 16; ++k)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[n][k][e] = 0.f;
        }
    }
};

__device__ __forceinline__ void ldmatrix4(uint32_t addr, uint32_t (&r)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldmatrix4_trans(uint32_t addr, uint32_t (&r)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t v) {
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
    return r;
}
__device__ __forceinline__ void mma_bf16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

// One tile of 64 rows, of which `rows` are there; `far`: distances of the lane's two rows; `logits`: [head][64] of the tile or null.
template <int DH, int NG>
__device__ __forceinline__ void bf16_tile(Bf16Unit<DH, NG>& u, const PagedAttnArgs& a, uint32_t k_smem, uint32_t v_smem, int rows,
                                          const float (&far)[2], float* logits, int nh) {
    using S = PagedShape<__nv_bfloat16, DH>;
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    float x[NG][4];
#pragma unroll
    for (int n = 0; n < NG; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) x[n][e] = 0.f;
    {
        const int row = w * 16 + ((lane >> 3) & 1) * 8 + (lane & 7);
        const uint32_t base = k_smem + row * 128;
#pragma unroll
        for (int k = 0; k < DH / 16; ++k) {
            uint32_t f[4];
            const int chunk = (k & 3) * 2 + (lane >> 4);
            ldmatrix4(base + (k >> 2) * S::kBlk + ((chunk ^ (row & 7)) << 4), f);
#pragma unroll
            for (int n = 0; n < NG; ++n) mma_bf16(x[n], f, u.q[n][k][0], u.q[n][k][1]);
        }
    }
    const int r0 = w * 16 + (lane >> 2);
    const bool in0 = r0 < rows, in1 = r0 + 8 < rows;
    uint32_t hi[NG][2], lo[NG][2];
#pragma unroll
    for (int n = 0; n < NG; ++n) {
#pragma unroll
        for (int e = 0; e < 4; ++e) x[n][e] = logit2(a, x[n][e], u.slope[n][e & 1], far[e >> 1]);
        if (logits) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int h = n * 8 + 2 * (lane & 3) + (e & 1);
                if (h < nh && (e < 2 ? in0 : in1)) logits[h * S::kTile + r0 + (e >> 1) * 8] = x[n][e];
            }
        }
        float top[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            top[e] = fmaxf(in0 ? x[n][e] : kLow, in1 ? x[n][e + 2] : kLow);
#pragma unroll
            for (int s = 4; s < 32; s <<= 1) top[e] = fmaxf(top[e], __shfl_xor_sync(0xFFFFFFFFu, top[e], s));
            top[e] = fmaxf(top[e], u.m[n][e]);
        }
        if (__any_sync(0xFFFFFFFFu, top[0] > u.m[n][0] || top[1] > u.m[n][1])) {
            const float f0 = sm100::fast_exp2(u.m[n][0] - top[0]), f1 = sm100::fast_exp2(u.m[n][1] - top[1]);
            u.l[n][0] *= f0;
            u.l[n][1] *= f1;
#pragma unroll
            for (int k = 0; k < DH / 16; ++k) {
                u.o[n][k][0] *= f0;
                u.o[n][k][1] *= f1;
                u.o[n][k][2] *= f0;
                u.o[n][k][3] *= f1;
            }
            u.m[n][0] = top[0];
            u.m[n][1] = top[1];
        }
        float p[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) p[e] = (e < 2 ? in0 : in1) ? sm100::fast_exp2(x[n][e] - u.m[n][e & 1]) : 0.f;
        u.l[n][0] += p[0] + p[2];
        u.l[n][1] += p[1] + p[3];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const uint32_t h = pack_bf16(p[2 * e], p[2 * e + 1]);
            const uint32_t r = pack_bf16(p[2 * e] - __uint_as_float(h << 16), p[2 * e + 1] - __uint_as_float(h & 0xFFFF0000u));
            hi[n][e] = transpose8x8(h);
            lo[n][e] = transpose8x8(r);
        }
    }
    // V^T: rows that are not there count as zeros, whatever the page holds
    const int kr = w * 16 + 2 * (lane & 3);
    uint32_t mask0 = 0xFFFFFFFFu, mask1 = 0xFFFFFFFFu;
    if (rows < S::kTile) {
        mask0 = (kr < rows ? 0xFFFFu : 0u) | (kr + 1 < rows ? 0xFFFF0000u : 0u);
        mask1 = (kr + 8 < rows ? 0xFFFFu : 0u) | (kr + 9 < rows ? 0xFFFF0000u : 0u);
    }
    {
        const int row = w * 16 + ((lane >> 4) & 1) * 8 + (lane & 7);
        const uint32_t base = v_smem + row * 128;
#pragma unroll
        for (int k = 0; k < DH / 16; ++k) {
            uint32_t f[4];
            const int chunk = (k & 3) * 2 + ((lane >> 3) & 1);
            ldmatrix4_trans(base + (k >> 2) * S::kBlk + ((chunk ^ (row & 7)) << 4), f);
            f[0] &= mask0;
            f[1] &= mask0;
            f[2] &= mask1;
            f[3] &= mask1;
#pragma unroll
            for (int n = 0; n < NG; ++n) {
                mma_bf16(u.o[n][k], f, hi[n][0], hi[n][1]);
                mma_bf16(u.o[n][k], f, lo[n][0], lo[n][1]);
            }
        }
    }
}

// A unit's warps meet in shared memory, o [head][DH], m and l [head]: close() adds up the lanes' sums, store() writes the warp's part,
// merge() takes another warp's part in.
template <int DH, int NG>
__device__ __forceinline__ void unit_close(Bf16Unit<DH, NG>& u) {
#pragma unroll
    for (int n = 0; n < NG; ++n)
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
            for (int s = 4; s < 32; s <<= 1) u.l[n][e] += __shfl_xor_sync(0xFFFFFFFFu, u.l[n][e], s);
}
template <int DH, int NG>
__device__ __forceinline__ void unit_merge(Bf16Unit<DH, NG>& u, const float* s_o, const float* s_ml) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int n = 0; n < NG; ++n) {
        const int h = n * 8 + 2 * (lane & 3);
        float f[2], g[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const float m = s_ml[2 * (h + e)], M = fmaxf(m, u.m[n][e]);
            f[e] = sm100::fast_exp2(u.m[n][e] - M);
            g[e] = sm100::fast_exp2(m - M);
            u.l[n][e] = u.l[n][e] * f[e] + s_ml[2 * (h + e) + 1] * g[e];
            u.m[n][e] = M;
        }
#pragma unroll
        for (int k = 0; k < DH / 16; ++k)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                u.o[n][k][e] = u.o[n][k][e] * f[e & 1] + s_o[(h + (e & 1)) * DH + k * 16 + (lane >> 2) + (e >> 1) * 8] * g[e & 1];
    }
}
template <int DH, int NG>
__device__ __forceinline__ void unit_store(Bf16Unit<DH, NG>& u, float* s_o, float* s_ml) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int n = 0; n < NG; ++n) {
        const int h = n * 8 + 2 * (lane & 3);
        if (lane < 4) {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                s_ml[2 * (h + e)] = u.m[n][e];
                s_ml[2 * (h + e) + 1] = u.l[n][e];
            }
        }
#pragma unroll
        for (int k = 0; k < DH / 16; ++k)
#pragma unroll
            for (int e = 0; e < 4; ++e) s_o[(h + (e & 1)) * DH + k * 16 + (lane >> 2) + (e >> 1) * 8] = u.o[n][k][e];
    }
}

// fp32: the warp takes HW heads (from `hb` on) and NR rows of every tile; lane l holds elements (l % 8) * 4 + 32 j,
// j < DH / 32, of q, and of o for the rows that are l / 8 modulo 4.
template <int DH, int HW>
struct F32Unit {
    float q[HW][DH / 8], o[HW][DH / 8];
    float m, l, slope;                                 // of head (lane & 7) * HW / 8: the one whose logits the lane gets
    int hb;

    __device__ __forceinline__ void start(const PagedAttnArgs& a, int b, int h0, int nh) {
        const int sub = threadIdx.x & 7;
#pragma unroll
        for (int h = 0; h < HW; ++h) {
            const float* src = reinterpret_cast<const float*>(a.q) + b * a.q_seq + (long long)(h0 + hb + h) * a.q_head + sub * 4;
#pragma unroll
            for (int j = 0; j < DH / 32; ++j) {
                const float4 v = hb + h < nh ? *reinterpret_cast<const float4*>(src + 32 * j) : make_float4(0.f, 0.f, 0.f, 0.f);
                q[h][4 * j] = v.x; q[h][4 * j + 1] = v.y; q[h][4 * j + 2] = v.z; q[h][4 * j + 3] = v.w;
            }
#pragma unroll
            for (int j = 0; j < DH / 8; ++j) o[h][j] = 0.f;
        }
        m = kLow;
        l = 0.f;
        const int h = hb + sub * HW / 8;
        slope = a.slopes && h < nh ? a.slopes[h0 + h] * kLog2e : 0.f;
    }
};

template <int DH, int HW, int NR>                      // NR: rows of the tile that are this warp's, from row r_lo on
__device__ __forceinline__ void f32_tile(F32Unit<DH, HW>& u, const PagedAttnArgs& a, const uint8_t* k_smem, const uint8_t* v_smem, int r_lo, int rows,
                                         float far_lane, float* logits, int nh) {
    using S = PagedShape<float, DH>;
    constexpr int P = NR / 4;                          // passes of four rows
    const int lane = threadIdx.x & 31, sub = lane & 7, kg = lane >> 3;
    float x[P];
#pragma unroll
    for (int p = 0; p < P; ++p) {
        const int r = r_lo + p * 4 + kg;
        float acc[HW];
#pragma unroll
        for (int h = 0; h < HW; ++h) acc[h] = 0.f;
#pragma unroll
        for (int j = 0; j < DH / 32; ++j) {
            const float4 v = *reinterpret_cast<const float4*>(k_smem + j * S::kBlk + r * 128 + ((sub ^ (r & 7)) << 4));
#pragma unroll
            for (int h = 0; h < HW; ++h)
                acc[h] = fmaf(u.q[h][4 * j + 3], v.w, fmaf(u.q[h][4 * j + 2], v.z, fmaf(u.q[h][4 * j + 1], v.y, fmaf(u.q[h][4 * j], v.x, acc[h]))));
        }
        // eight lanes' sums of HW heads: a lane gives away the heads of the other half until it has one
        if constexpr (HW == 4) {
            const bool up = sub & 4;
            const float g0 = __shfl_xor_sync(0xFFFFFFFFu, up ? acc[0] : acc[2], 4), g1 = __shfl_xor_sync(0xFFFFFFFFu, up ? acc[1] : acc[3], 4);
            acc[0] = (up ? acc[2] : acc[0]) + g0;
            acc[1] = (up ? acc[3] : acc[1]) + g1;
        }
        if constexpr (HW >= 2) {
            constexpr int kStep = HW == 4 ? 2 : 4;
            const bool up = sub & kStep;
            const float g0 = __shfl_xor_sync(0xFFFFFFFFu, up ? acc[0] : acc[1], kStep);
            acc[0] = (up ? acc[1] : acc[0]) + g0;
        }
#pragma unroll
        for (int s = 4 / HW; s >= 1; s >>= 1) acc[0] += __shfl_xor_sync(0xFFFFFFFFu, acc[0], s);
        x[p] = logit2(a, acc[0], u.slope, __shfl_sync(0xFFFFFFFFu, far_lane, r));
    }
    const int head = u.hb + sub * HW / 8;
    if (logits && (sub & (8 / HW - 1)) == 0 && head < nh) {
#pragma unroll
        for (int p = 0; p < P; ++p) {
            const int r = r_lo + p * 4 + kg;
            if (r < rows) logits[head * S::kTile + r] = x[p];
        }
    }
    float top = u.m;
#pragma unroll
    for (int p = 0; p < P; ++p)
        if (r_lo + p * 4 + kg < rows) top = fmaxf(top, x[p]);
    top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 8));
    top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 16));
    if (__any_sync(0xFFFFFFFFu, top > u.m)) {
        const float f = sm100::fast_exp2(u.m - top);
        u.m = top;
        u.l *= f;
#pragma unroll
        for (int h = 0; h < HW; ++h) {
            const float fh = __shfl_sync(0xFFFFFFFFu, f, h * (8 / HW));
#pragma unroll
            for (int j = 0; j < DH / 8; ++j) u.o[h][j] *= fh;
        }
    }
#pragma unroll
    for (int p = 0; p < P; ++p) {
        const int r = r_lo + p * 4 + kg;
        const bool in = r < rows;
        const float w = in ? sm100::fast_exp2(x[p] - u.m) : 0.f;
        u.l += w;
        float wh[HW];
#pragma unroll
        for (int h = 0; h < HW; ++h) wh[h] = __shfl_sync(0xFFFFFFFFu, w, (lane & 24) + h * (8 / HW));
#pragma unroll
        for (int j = 0; j < DH / 32; ++j) {
            float4 v = *reinterpret_cast<const float4*>(v_smem + j * S::kBlk + r * 128 + ((sub ^ (r & 7)) << 4));
            if (!in) v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int h = 0; h < HW; ++h) {
                u.o[h][4 * j] = fmaf(wh[h], v.x, u.o[h][4 * j]);
                u.o[h][4 * j + 1] = fmaf(wh[h], v.y, u.o[h][4 * j + 1]);
                u.o[h][4 * j + 2] = fmaf(wh[h], v.z, u.o[h][4 * j + 2]);
                u.o[h][4 * j + 3] = fmaf(wh[h], v.w, u.o[h][4 * j + 3]);
            }
        }
    }
}

template <int DH, int HW>
__device__ __forceinline__ void unit_close(F32Unit<DH, HW>& u) {
    u.l += __shfl_xor_sync(0xFFFFFFFFu, u.l, 8);
    u.l += __shfl_xor_sync(0xFFFFFFFFu, u.l, 16);
#pragma unroll
    for (int h = 0; h < HW; ++h)
#pragma unroll
        for (int j = 0; j < DH / 8; ++j) {
            u.o[h][j] += __shfl_xor_sync(0xFFFFFFFFu, u.o[h][j], 8);
            u.o[h][j] += __shfl_xor_sync(0xFFFFFFFFu, u.o[h][j], 16);
        }
}
template <int DH, int HW>
__device__ __forceinline__ void unit_merge(F32Unit<DH, HW>& u, const float* s_o, const float* s_ml) {
    const int sub = threadIdx.x & 7, head = u.hb + sub * HW / 8;
    const float m = s_ml[2 * head], M = fmaxf(m, u.m), f = sm100::fast_exp2(u.m - M), g = sm100::fast_exp2(m - M);
    u.l = u.l * f + s_ml[2 * head + 1] * g;
    u.m = M;
#pragma unroll
    for (int h = 0; h < HW; ++h) {
        const float fh = __shfl_sync(0xFFFFFFFFu, f, h * (8 / HW)), gh = __shfl_sync(0xFFFFFFFFu, g, h * (8 / HW));
#pragma unroll
        for (int j = 0; j < DH / 32; ++j) {
            const float4 x = *reinterpret_cast<const float4*>(s_o + (u.hb + h) * DH + sub * 4 + 32 * j);
            u.o[h][4 * j] = u.o[h][4 * j] * fh + x.x * gh;
            u.o[h][4 * j + 1] = u.o[h][4 * j + 1] * fh + x.y * gh;
            u.o[h][4 * j + 2] = u.o[h][4 * j + 2] * fh + x.z * gh;
            u.o[h][4 * j + 3] = u.o[h][4 * j + 3] * fh + x.w * gh;
        }
    }
}
template <int DH, int HW>
__device__ __forceinline__ void unit_store(F32Unit<DH, HW>& u, float* s_o, float* s_ml) {
    const int lane = threadIdx.x & 31, sub = lane & 7;
    if (lane < 8) {
        if ((sub & (8 / HW - 1)) == 0) {
            const int h = u.hb + sub * HW / 8;
            s_ml[2 * h] = u.m;
            s_ml[2 * h + 1] = u.l;
        }
#pragma unroll
        for (int h = 0; h < HW; ++h)
#pragma unroll
            for (int j = 0; j < DH / 32; ++j)
                *reinterpret_cast<float4*>(s_o + (u.hb + h) * DH + sub * 4 + 32 * j) = make_float4(u.o[h][4 * j], u.o[h][4 * j + 1], u.o[h][4 * j + 2], u.o[h][4 * j + 3]);
    }
}

// HX: bf16: groups of eight heads of a unit; fp32: heads per warp (with 8 of a unit: two warps share the heads, two the rows).
template <typename T, int DH, int HX, int kUnitHeads>
__global__ void __launch_bounds__(kThreads)
paged_attn_kernel(const PagedAttnArgs a, const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v) {
    using namespace sm100;
    using S = PagedShape<T, DH>;
    extern __shared__ uint8_t smem_dyn[];
    __shared__ __align__(8) uint64_t full_bar[S::kStages], empty_bar[S::kStages];
    __shared__ __align__(16) float s_o[2][kUnitHeads * DH];
    __shared__ float s_ml[2][kUnitHeads * 2];
    __shared__ long long s_sum[kWarps + 1];
    __shared__ long long s_start;
    __shared__ int s_b;
    __shared__ int s_abort;
    const int warp = __shfl_sync(0xFFFFFFFFu, (int)threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    const uint32_t ring = (smem_u32(smem_dyn) + 1023u) & ~1023u;
    const int subs = a.d.Hkv * a.NC;
    if (threadIdx.x == 0) {
        prefetch_tmap(&tm_k);
        prefetch_tmap(&tm_v);
        for (int s = 0; s < S::kStages; ++s) { mbar_init(smem_u32(&full_bar[s]), 1); mbar_init(smem_u32(&empty_bar[s]), kWarps); }
        s_abort = 0;
        mbar_fence_init();
    }
    grid_dep_wait();
    if (blockIdx.x == a.grid) {                        // one CTA more than pieces
        if (warp == 0) write_line(a);
        return;
    }
    if (blockIdx.x == 0 && threadIdx.x == 0) *a.status = METOK_OK;       // a wait that gives up writes it, seconds later
    const long long T_all = line_tiles(a, s_sum) * subs, ctas = busy_ctas(a, T_all);
    if (blockIdx.x >= ctas) return;                    // uniform
    const long long t_lo = T_all * blockIdx.x / ctas, t_hi = T_all * (blockIdx.x + 1) / ctas;
    // the sequence that holds tile t_lo, 32 at a time: by every warp for itself where there are no more
    Place p;
    long long start = 0;
    p.b = 0;
    if (warp == 0 || a.d.n_seqs <= 32) {
        long long at = 0;                              // tiles before sequence b0
        for (int b0 = 0; b0 < a.d.n_seqs; b0 += 32) {
            const int b = b0 + lane;
            long long mine = b < a.d.n_seqs ? (long long)unit_tiles(a, b) * subs : 0, incl = mine;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const long long x = __shfl_up_sync(0xFFFFFFFFu, incl, o);
                if (lane >= o) incl += x;
            }
            const uint32_t any = __ballot_sync(0xFFFFFFFFu, at + incl > t_lo);
            if (any) {
                const int l = __ffs(any) - 1;
                p.b = b0 + l;
                start = at + __shfl_sync(0xFFFFFFFFu, incl - mine, l);
                break;
            }
            at += __shfl_sync(0xFFFFFFFFu, incl, 31);
        }
    }
    if (a.d.n_seqs > 32 && threadIdx.x == 0) {
        s_b = p.b;
        s_start = start;
    }
    __syncthreads();
    if (a.d.n_seqs > 32) {
        p.b = s_b;
        start = s_start;
    }
    p.nt = unit_tiles(a, p.b);
    const long long in = t_lo - start;
    p.sub = (int)(in / p.nt);
    p.t = (int)(in - (long long)p.sub * p.nt);
    p.left = t_hi - t_lo;
    volatile int* abort_flag = &s_abort;

    if (warp == kWarps) {                              // brings the tiles
        const int page_rows = 1 << a.d.page_shift, piece = min(page_rows, S::kTile), per_tile = S::kTile / piece;
        const uint32_t piece_bytes = (uint32_t)piece * 128u;
        int it = 0;
        for (; p.left > 0; ++it) {
            const int s = it % S::kStages;
            if (!mbar_wait_warp(smem_u32(&empty_bar[s]), ((uint32_t)(it / S::kStages) & 1u) ^ 1u, abort_flag)) break;
            const int r0 = p.t * S::kTile, rows = min(S::kTile, a.kv_len[p.b] - r0);
            const int pieces = (rows + piece - 1) / piece, copies = pieces * 2 * S::KB;
            const uint32_t fb = smem_u32(&full_bar[s]);
            if (lane == 0) mbar_arrive_expect_tx(fb, (uint32_t)copies * piece_bytes);
            __syncwarp();
            for (int c = lane; c < per_tile * 2 * S::KB; c += 32) {
                const int pc = c / (2 * S::KB), e = c - pc * (2 * S::KB), kb = e >> 1;
                if (pc >= pieces) continue;
                if (dbg_held(a.withhold, kDbgPagedAttn) && blockIdx.x == 0 && it == 0 && c == 0) continue;   // debug builds: one copy never sent
                const int row = r0 + pc * piece;
                int page = a.block_table[(size_t)p.b * a.d.max_pages + (row >> a.d.page_shift)];
                if (page < 0 || page >= a.d.n_pages) page = 0;          // the second kernel drops the sequence
                const int y = (int)((((long long)page * a.d.Hkv + p.sub / a.NC) << a.d.page_shift) + (row & (page_rows - 1)));
                const uint32_t dst = ring + s * S::kStage + (e & 1) * S::kHalf + kb * S::kBlk + pc * piece_bytes;
                tma_load_2d(dst, (e & 1) ? &tm_v : &tm_k, kb * S::kCols, y, fb);
            }
            __syncwarp();
            next_tile(a, p, subs);
        }
        // all copies have landed before the shared memory goes away
        for (int back = 1; back <= S::kStages && back <= it; ++back) {
            const int j = it - back;
            mbar_wait_warp(smem_u32(&full_bar[j % S::kStages]), (uint32_t)(j / S::kStages) & 1u, abort_flag);
        }
    } else {
        constexpr int kHeadWarps = S::kBf16 ? 1 : kUnitHeads / HX;      // fp32: warps that share the heads
        constexpr int kRowsWarp = S::kBf16 ? 16 : S::kTile * kHeadWarps / kWarps;
        int it = 0;
        bool ok = true, fresh = true;
        auto run = [&](auto& u) {
            int newest = 0;
            while (p.left > 0) {
                const int hk = p.sub / a.NC, ch = p.sub - hk * a.NC, h0 = hk * a.G + ch * a.heads, nh = min(a.heads, a.G - ch * a.heads);
                const int len = a.kv_len[p.b], r0 = p.t * S::kTile, rows = min(S::kTile, len - r0);
                const int32_t* pos = a.positions ? a.positions + (size_t)p.b * a.d.S_cap() : nullptr;
                if (fresh) {
                    u.start(a, p.b, h0, nh);
                    newest = a.slopes ? (pos ? pos[len - 1] : len - 1) : 0;
                    fresh = false;
                }
                const int s = it % S::kStages;
                // distances of the rows that this lane's logits are of
                float far[2] = {0.f, 0.f};
                if (a.slopes) {
                    auto distance = [&](int r) { r = min(r0 + r, len - 1); return fabsf((float)newest - (float)(pos ? pos[r] : r)); };
                    if constexpr (S::kBf16) {
                        far[0] = distance(warp * 16 + (lane >> 2));
                        far[1] = distance(warp * 16 + (lane >> 2) + 8);
                    } else {
                        far[0] = distance(lane);
                    }
                }
                float* logits = nullptr;
                if (a.mass) logits = a.logits + (size_t)(t_hi - p.left) * a.heads * S::kTile;
                if (ok && !mbar_wait_warp(smem_u32(&full_bar[s]), (uint32_t)(it / S::kStages) & 1u, abort_flag)) ok = false;
                if (ok) {
                    if constexpr (S::kBf16) {
                        const uint32_t k = ring + s * S::kStage;
                        bf16_tile<DH, HX>(u, a, k, k + S::kHalf, rows, far, logits, nh);
                    } else {
                        const uint8_t* base = smem_dyn + (ring - smem_u32(smem_dyn)) + s * S::kStage;
                        f32_tile<DH, HX, kRowsWarp>(u, a, base, base + S::kHalf, (warp / kHeadWarps) * kRowsWarp, rows, far[0], logits, nh);
                    }
                    __syncwarp();
                    if (lane == 0) mbar_arrive(smem_u32(&empty_bar[s]));
                }
                const long long unit = (long long)p.b * subs + p.sub;
                const bool ends = p.t + 1 == p.nt || p.left == 1;
                ++it;
                next_tile(a, p, subs);
                if (ends) {
                    fresh = true;
                    // warps 2 and 3 give their rows to warps 0 and 1 (of the same heads); what those have is joined on the way out
                    unit_close(u);
                    if (warp >= 2) unit_store(u, s_o[warp - 2], s_ml[warp - 2]);
                    named_bar_sync(1, kWarps * 32);
                    if (warp < 2) unit_merge(u, s_o[warp], s_ml[warp]);
                    __syncwarp();
                    if (warp < 2) unit_store(u, s_o[warp], s_ml[warp]);
                    named_bar_sync(1, kWarps * 32);
                    const size_t slot = (size_t)(unit + blockIdx.x);
                    for (int i = threadIdx.x; i < nh * (DH / 4); i += kWarps * 32) {
                        const int h = i / (DH / 4);
                        float M, L;
                        float4 o;
                        if constexpr (kHeadWarps == 1) {       // both have the head
                            const float m0 = s_ml[0][2 * h], m1 = s_ml[1][2 * h];
                            M = fmaxf(m0, m1);
                            const float f = sm100::fast_exp2(m0 - M), g = sm100::fast_exp2(m1 - M);
                            L = f * s_ml[0][2 * h + 1] + g * s_ml[1][2 * h + 1];
                            const float4 x = reinterpret_cast<const float4*>(s_o[0])[i], y = reinterpret_cast<const float4*>(s_o[1])[i];
                            o = make_float4(f * x.x + g * y.x, f * x.y + g * y.y, f * x.z + g * y.z, f * x.w + g * y.w);
                        } else {
                            M = s_ml[h / HX][2 * h];
                            L = s_ml[h / HX][2 * h + 1];
                            o = reinterpret_cast<const float4*>(s_o[h / HX])[i];
                        }
                        reinterpret_cast<float4*>(a.part_o + slot * a.heads * DH)[i] = o;
                        if (i % (DH / 4) == 0) reinterpret_cast<float2*>(a.part_ml + slot * a.heads * 2)[h] = make_float2(M, L);
                    }
                    named_bar_sync(1, kWarps * 32);
                }
            }
        };
        if constexpr (S::kBf16) {
            Bf16Unit<DH, HX> u;
            run(u);
        } else {
            F32Unit<DH, HX> u;
            u.hb = (warp % kHeadWarps) * HX;
            run(u);
        }
    }
    __syncthreads();
    if (threadIdx.x == 0 && s_abort) *a.status = METOK_ERR_TIMEOUT;
}

// The partials of a unit: CTAs c0 .. c1, of which CTA c's lies at slot unit + c.
struct Slots { long long first; int n; };
__device__ __forceinline__ Slots unit_slots(const PagedAttnArgs& a, long long all, long long unit, long long f0, int nt) {
    // the CTA that has tile f is the last one with floor(all * c / ctas) <= f
    const long long ctas = busy_ctas(a, all), c0 = ((f0 + 1) * ctas - 1) / all, c1 = ((f0 + nt) * ctas - 1) / all;
    return {unit + c0, (int)(c1 - c0) + 1};
}

// Joins the partials.  CTAs [0, n_seqs * Hq): one head's output and lse; the others: the weights of kMassRows rows of a sequence.
constexpr int kJoinThreads = 128, kMassRows = 128;
template <typename T, int DH>
__global__ void __launch_bounds__(kJoinThreads)
paged_join_kernel(const PagedAttnArgs a) {
    // Up to the wait: what needs only the call's inputs, which were complete when the first kernel was let go.
    __shared__ __align__(16) float s_acc[kJoinThreads][4];
    __shared__ float2 s_ml[kJoinThreads];
    extern __shared__ __align__(16) uint8_t s_dyn[];
    const int tid = threadIdx.x, lane = tid & 31;
    const int outs = a.d.n_seqs * a.Hq;
    const bool weights = (int)blockIdx.x >= outs;
    const int chunks = (a.d.S_cap() + kMassRows - 1) / kMassRows;
    const int b = weights ? ((int)blockIdx.x - outs) / chunks : (int)blockIdx.x / a.Hq;
    const int len = a.kv_len[b], subs = a.d.Hkv * a.NC;
    const int row0 = weights ? (((int)blockIdx.x - outs) - b * chunks) * kMassRows : 0;
    // the sequence is sound: only then anything is written for it
    bool ok = len >= 0 && len <= a.d.S_cap();
    if (ok) {
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
    const bool few = a.d.n_seqs <= 32;                 // one look at all lengths; else the line that the first kernel wrote
    if (few) {
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

    if (!weights) {
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
            for (int u = 0; u < kAhead; ++u) top = fmaxf(top, ml[u].x);
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
        __syncthreads();
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
    const int row = min(row0 + tid, len - 1), tile = row >> a.tile_shift, off = row & ((1 << a.tile_shift) - 1), rows_tile = 1 << a.tile_shift;
    const float* x = a.logits + (size_t)(base + tile) * a.heads * rows_tile + off;
    constexpr int kHeads = 16, kAhead = 10;
    float v[kHeads];
    auto logits_of = [&](int h0) {
#pragma unroll
        for (int u = 0; u < kHeads; ++u) v[u] = h0 + u < a.Hq ? x[s_off[h0 + u]] : kLow;
    };
    logits_of(0);
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
                for (int u = 0; u < kAhead; ++u) top = fmaxf(top, p[u].x);
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
    __syncthreads();
    if (row0 + tid >= len) return;
    float sum = 0.f;
    for (int h = 0; h < a.Hq; h += kHeads) {           // kHeads loads on their way (a loop of single ones would wait for each)
        if (h) logits_of(h);
#pragma unroll
        for (int u = 0; u < kHeads; ++u) sum += h + u < a.Hq ? sm100::fast_exp2(v[u] - s_lse[h + u]) : 0.f;
    }
    a.mass[(size_t)b * a.d.S_cap() + row] += sum / (float)a.Hq;
}

// How the heads of a K/V head are dealt to units, and the line to CTAs.
struct PagedPlan {
    int G, heads, NC, grid, tile_shift;
    size_t slots, tiles;
};
PagedPlan paged_plan(int dtype, const PagedDims& d, int Hq) {
    PagedPlan p;
    p.G = Hq / d.Hkv;
    const int most = dtype == METOK_BF16 ? 16 : 8;     // heads of a unit
    const int per = ceil_div(p.G, ceil_div(p.G, most));
    if (dtype == METOK_BF16) p.heads = per <= 8 ? 8 : 16;
    else p.heads = per <= 1 ? 1 : per <= 2 ? 2 : per <= 4 ? 4 : 8;
    p.NC = ceil_div(p.G, p.heads);
    p.tile_shift = dtype == METOK_BF16 ? 6 : 5;
    const size_t units = (size_t)d.n_seqs * d.Hkv * p.NC;
    p.tiles = units * (size_t)((d.S_cap() + (1 << p.tile_shift) - 1) >> p.tile_shift);
    p.grid = (int)std::min<size_t>(p.tiles, 2 * kNumSMs);
    p.slots = units + p.grid;
    return p;
}
void paged_carve(Carver& cv, const PagedPlan& p, const PagedDims& d, bool mass, PagedAttnArgs* a) {
    a->part_o = cv.take<float>(p.slots * p.heads * d.dh);
    a->part_ml = cv.take<float>(p.slots * p.heads * 2);
    a->line = cv.take<long long>((size_t)d.n_seqs + 1);
    a->logits = mass ? cv.take<float>(p.tiles * p.heads << p.tile_shift) : nullptr;
}

template <typename T, int DH, int HX, int kUnitHeads>
int launch_paged(const PagedAttnArgs& a, const CUtensorMap& tk, const CUtensorMap& tv, cudaStream_t st) {
    using S = PagedShape<T, DH>;
    auto kern = paged_attn_kernel<T, DH, HX, kUnitHeads>;
    METOK_ALLOW_SMEM(kern, S::kRing);
    {
        METOK_TIMED("paged_attn", st);
        launch_chained(kern, dim3(a.grid + 1), dim3(kThreads), S::kRing, st, a, tk, tv);
    }
    METOK_LAUNCH_CHECK();
    {
        METOK_TIMED("paged_join", st);
        const long long blocks = (long long)a.d.n_seqs * a.Hq + (a.mass ? (long long)a.d.n_seqs * ((a.d.S_cap() + kMassRows - 1) / kMassRows) : 0);
        const size_t smem = a.mass ? ((size_t)a.d.Hkv * a.NC * 12 + (size_t)a.Hq * 4 + 7) / 8 * 8 + (size_t)a.Hq * 8 : 0;
        METOK_ALLOW_SMEM((paged_join_kernel<T, DH>), smem);
        launch_chained(paged_join_kernel<T, DH>, dim3((unsigned)blocks), dim3(kJoinThreads), smem, st, a);
    }
    METOK_LAUNCH_CHECK();
    return METOK_OK;
}
template <int DH>
int launch_paged_dh(int dtype, const PagedAttnArgs& a, const CUtensorMap& tk, const CUtensorMap& tv, cudaStream_t st) {
    if (dtype == METOK_BF16) {
        if (a.heads == 8) return launch_paged<__nv_bfloat16, DH, 1, 8>(a, tk, tv, st);
        return launch_paged<__nv_bfloat16, DH, 2, 16>(a, tk, tv, st);
    }
    if (a.heads == 1) return launch_paged<float, DH, 1, 1>(a, tk, tv, st);
    if (a.heads == 2) return launch_paged<float, DH, 2, 2>(a, tk, tv, st);
    if (a.heads == 4) return launch_paged<float, DH, 4, 4>(a, tk, tv, st);
    return launch_paged<float, DH, 4, 8>(a, tk, tv, st);
}

}  // namespace
}  // namespace metok

using namespace metok;

extern "C" size_t metok_paged_attention_workspace_bytes(int dtype, const metok_paged_cache* c, int Hq, int with_mass) {
    PagedDims d;
    if (paged_dims(dtype, c, &d) != METOK_OK || Hq < 1 || Hq % d.Hkv) return 0;
    PagedAttnArgs a;
    Carver cv(nullptr);
    paged_carve(cv, paged_plan(dtype, d, Hq), d, with_mass != 0, &a);
    return cv.total();
}

extern "C" int metok_paged_attention(int dtype, const metok_paged_cache* c, const void* q, int64_t q_seq, int64_t q_head, int Hq,
                                     float softmax_scale, float softcap, const float* slopes, const int32_t* positions, float* mass,
                                     void* out, int64_t out_seq, int64_t out_head, float* lse, int32_t* status, void* ws,
                                     size_t ws_bytes, void* stream) {
    PagedDims d;
    int rc = paged_dims(dtype, c, &d);
    if (rc != METOK_OK) return rc;
    if (!c->k_pool || !c->v_pool || !c->block_table || !c->kv_len || !q || !out || !status) return METOK_ERR_INVALID_ARG;
    if (Hq < 1 || Hq % d.Hkv) return METOK_ERR_INVALID_ARG;
    if (Hq > 2048) return METOK_ERR_UNSUPPORTED;
    if (!aligned16(c->k_pool) || !aligned16(c->v_pool) || !aligned16(q) || !aligned16(out)) return METOK_ERR_INVALID_ARG;
    if (!aligned4(c->block_table) || !aligned4(c->kv_len) || !aligned4(slopes) || !aligned4(positions) || !aligned4(mass) ||
        !aligned4(lse) || !aligned4(status))
        return METOK_ERR_INVALID_ARG;
    const int per = 16 / (dtype == METOK_F32 ? 4 : 2);
    if (q_seq < 0 || q_head < 0 || out_seq < 0 || out_head < 0 || (q_seq | q_head | out_seq | out_head) % per) return METOK_ERR_INVALID_ARG;
    // outputs of different heads and sequences do not overlap
    if (!rows_apart(d.n_seqs, out_seq, Hq, out_head, d.dh) || !softmax_numbers(softmax_scale, softcap)) return METOK_ERR_INVALID_ARG;
    const PagedPlan p = paged_plan(dtype, d, Hq);
    const long long join = (long long)d.n_seqs * Hq + (mass ? (long long)d.n_seqs * ((d.S_cap() + kMassRows - 1) / kMassRows) : 0);
    if (join > 0x7FFFFFFFLL) return METOK_ERR_UNSUPPORTED;
    if (!ws || !aligned16(ws) || ws_bytes < metok_paged_attention_workspace_bytes(dtype, c, Hq, mass != nullptr)) return METOK_ERR_WORKSPACE;
    PagedAttnArgs a;
    a.d = d;
    a.Hq = Hq; a.G = p.G; a.NC = p.NC; a.heads = p.heads; a.grid = p.grid; a.tile_shift = p.tile_shift;
    a.q = q; a.q_seq = q_seq; a.q_head = q_head; a.out = out; a.out_seq = out_seq; a.out_head = out_head;
    a.block_table = c->block_table; a.kv_len = c->kv_len; a.positions = positions; a.slopes = slopes;
    a.scale_log2 = softmax_scale * kLog2e;
    a.cap_scale = softcap > 0.f ? softmax_scale / softcap : 0.f;
    a.cap_log2 = softcap * kLog2e;
    a.mass = mass; a.lse = lse; a.status = status;
    a.withhold = debug_withheld();
    Carver cv(ws);
    paged_carve(cv, p, d, mass != nullptr, &a);
    const uint64_t rows = (uint64_t)d.n_pages * d.Hkv << d.page_shift;
    const uint32_t box = (uint32_t)std::min(1 << d.page_shift, 1 << p.tile_shift);
    CUtensorMap tk, tv;
    rc = make_tmap_rows(&tk, dtype, c->k_pool, rows, d.dh, box);
    if (rc == METOK_OK) rc = make_tmap_rows(&tv, dtype, c->v_pool, rows, d.dh, box);
    if (rc != METOK_OK) return rc;
    cudaStream_t st = (cudaStream_t)stream;
    return d.dh == 64 ? launch_paged_dh<64>(dtype, a, tk, tv, st) : launch_paged_dh<128>(dtype, a, tk, tv, st);
}
