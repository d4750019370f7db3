// metok_paged_attention_q4: attention of one new token per sequence over its paged K/V cache held in 4 bits.
//
// The line of tiles, the partials and the join are those of the attention over a cache of numbers (paged_attn.cuh).  A tile is four pieces
// of 16 rows, which one warp brings by bulk copies through a ring of shared memory; four warps take a piece each.
//
// A row is 4.5 bits per element, so that what would bound the kernel next to reading is turning codes into numbers.  It costs two
// operations for a pair and a half of a shift: a nibble c of one row and the one 16 bits above it are masked into the fractions of two fp16
// numbers, 1024 + c or 1024 + 16 c, and one multiply-add with constants of the block, (1024 + c) e - 1032 e or (1024 + 16 c) e/16 - 72 e,
// gives (c - 8) e.  e has three significant bits, so that all constants and results are exact (q4.cuh).
//   x^T = K Q^T: a thread holds the nibbles of whole blocks, a quarter of two rows, so it needs these blocks' constants alone; the
//     elements of Q are dealt out in the order in which the nibbles come.
//   o^T += V^T P^T: a thread holds an eighth of four rows; two rows' words are interleaved by 16 bits first, since a pair of the product
//     is a pair of rows.
//   The rows that a thread takes for its places in the products are permuted, r -> r ^ (r >> 2 & 1), which no sum notices: so the reads of V
//   meet two banks at a time at most (and those of K none).
// Q takes part as fp16 numbers of the head's largest element's scale: bf16's eight bits are in one; fp32's are in two to 2^-22.  The weights
// are 2^14 times exp2(x - max) and take part as one fp16 number for bf16 outputs (off by 2^-12 of a weight, beside 2^-9 of the output's own rounding), as two
// for fp32.  Logits, their sums, and outputs up to their end are fp32.
#include "paged_attn.cuh"
#include "q4.cuh"

namespace metok {

namespace {

constexpr int kWarps = 4, kThreads = (kWarps + 1) * 32;
constexpr float kLift = 14.f;                          // weights are relative to 2^-14 of the largest

template <int DH>
struct Q4Shape {
    static constexpr int kTile = kQ4Rows * kWarps;
    static constexpr uint32_t kPiece = q4_piece(DH), kHalf = kWarps * kPiece, kStage = 2 * kHalf;      // K, then V
    static constexpr int kStages = DH == 128 ? 6 : 12;
    static constexpr size_t kRing = (size_t)kStages * kStage + 128;
};
constexpr int q4_ctas(int groups) { return groups == 1 ? 3 : 2; }        // CTAs of an SM

__device__ __forceinline__ uint32_t as_u32(__half2 h) { return *reinterpret_cast<uint32_t*>(&h); }
__device__ __forceinline__ __half2 as_half2(uint32_t u) { return *reinterpret_cast<__half2*>(&u); }
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) { return as_u32(__floats2half2_rn(lo, hi)); }
__device__ __forceinline__ uint32_t transpose8x8(uint32_t v) {
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
    return r;
}
__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// The constants of two scales (as fp16: their bytes in the upper halves).
struct Q4Block {
    __half2 e, e16, c0, c1;
    __device__ __forceinline__ explicit Q4Block(uint32_t scales) {
        e = as_half2(scales);
        e16 = __hmul2(e, __float2half2_rn(0.0625f));
        c0 = __hmul2(e, __float2half2_rn(-1032.f));
        c1 = __hmul2(e, __float2half2_rn(-72.f));
    }
    // Nibbles j and j + 4 of `w`, j = 0 .. 3.
    __device__ __forceinline__ void pairs(uint32_t w, uint32_t (&r)[4]) const {
#pragma unroll
        for (int j = 0; j < 4; j += 2) {
            r[j] = as_u32(__hfma2(as_half2((w & 0x000F000Fu) | 0x64006400u), e, c0));
            r[j + 1] = as_u32(__hfma2(as_half2((w & 0x00F000F0u) | 0x64006400u), e16, c1));
            w >>= 8;
        }
    }
};

// A unit's running softmax.  NG groups of eight heads, QP fp16 numbers per element of Q (and per weight).  Lane l holds the logits of rows
// pi(l / 4) and pi(l / 4) + 8 of the warp's 16 and of heads 2 (l % 4), + 1; of o the DH / 8 elements from DH / 8 * (l / 4) on.
template <int DH, int NG, int QP>
struct Q4Unit {
    uint32_t q[QP][NG][DH / 16][2];
    float m[NG][2], l[NG][2], o[NG][DH / 16][4], slope[NG][2], lift[NG][2];      // lift: what the head's q was divided by, and the scales' unit

    template <typename T>
    __device__ __forceinline__ void start(const PagedAttnArgs& a, int b, int h0, int nh) {
        const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
#pragma unroll
        for (int n = 0; n < NG; ++n) {
            const int h = n * 8 + g;
            const T* src = reinterpret_cast<const T*>(a.q) + b * a.q_seq + (long long)(h0 + h) * a.q_head + t * (DH / 4);
            float x[DH / 4], top = 0.f;
#pragma unroll
            for (int i = 0; i < DH / 64; ++i) {
                uint4 v[sizeof(T)];
#pragma unroll
                for (int j = 0; j < (int)sizeof(T); ++j) v[j] = h < nh ? reinterpret_cast<const uint4*>(src + 16 * i)[j] : make_uint4(0u, 0u, 0u, 0u);
                float w[16];
                q4_widen<T>(v, w);
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    x[16 * i + j] = w[j];
                    top = fmaxf(top, fabsf(w[j]));
                }
            }
            top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
            top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
            // the largest element comes to lie in [2^13, 2^14): 2^-ex times it
            const int ex = max((int)(__float_as_uint(top) >> 23) - 127, -100) - 13;
            const float down = __uint_as_float((uint32_t)(127 - ex) << 23), up = __uint_as_float((uint32_t)(127 + ex) << 23) * kQ4Unit;
#pragma unroll
            for (int i = 0; i < DH / 32; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) {          // pair e of word i: elements 8 i + e and + 4
                    const float x0 = x[8 * i + e] * down, x1 = x[8 * i + e + 4] * down;
                    const __half2 hi = __floats2half2_rn(x0, x1);
                    q[0][n][2 * i + (e >> 1)][e & 1] = as_u32(hi);
                    if constexpr (QP == 2) q[1][n][2 * i + (e >> 1)][e & 1] = pack_f16(x0 - __low2float(hi), x1 - __high2float(hi));
                }
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int hc = n * 8 + 2 * t + e;
                lift[n][e] = __shfl_sync(0xFFFFFFFFu, up, (2 * t + e) * 4);
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

__device__ __forceinline__ int row_at(int r) { return r ^ (r >> 2 & 1); }          // pi: the row at place r of eight

// The warp's piece of a tile, of whose rows `rows` are there (<= 0: none); `far`: distances of the lane's two rows; `logits`: those of the
// piece's rows, [head][kTile], or null.
template <int DH, int NG, int QP>
__device__ __forceinline__ void q4_tile(Q4Unit<DH, NG, QP>& u, const PagedAttnArgs& a, const uint8_t* kp, const uint8_t* vp, int rows,
                                        const float (&far)[2], float* logits, int nh) {
    using S = Q4Shape<DH>;
    const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3, r0 = row_at(g);
    float x[NG][4], y[NG][4];                          // two chains of products
#pragma unroll
    for (int n = 0; n < NG; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) x[n][e] = y[n][e] = 0.f;
    {
        uint32_t w[2][DH / 32], sc[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int row = r0 + 8 * i;
            if constexpr (DH == 128) {
                const uint4 v = *reinterpret_cast<const uint4*>(kp + row * 64 + t * 16);
                w[i][0] = v.x; w[i][1] = v.y; w[i][2] = v.z; w[i][3] = v.w;
                sc[i] = *reinterpret_cast<const uint16_t*>(kp + 8 * DH + row * 8 + 2 * t);
            } else {
                const uint2 v = *reinterpret_cast<const uint2*>(kp + row * 32 + t * 8);
                w[i][0] = v.x; w[i][1] = v.y;
                sc[i] = kp[8 * DH + row * 4 + t];
            }
        }
#pragma unroll
        for (int b = 0; b < DH / 64; ++b) {
            // byte b of the scales into the upper bytes of both halves
            const Q4Block b0(__byte_perm(sc[0], 0u, b ? 0x1414 : 0x0404)), b1(__byte_perm(sc[1], 0u, b ? 0x1414 : 0x0404));
#pragma unroll
            for (int i = 2 * b; i < 2 * b + 2; ++i) {
                uint32_t f0[4], f1[4];
                b0.pairs(w[0][i], f0);
                b1.pairs(w[1][i], f1);
#pragma unroll
                for (int n = 0; n < NG; ++n)
#pragma unroll
                    for (int z = 0; z < QP; ++z) {
                        mma_f16(x[n], f0[0], f1[0], f0[1], f1[1], u.q[z][n][2 * i][0], u.q[z][n][2 * i][1]);
                        mma_f16(y[n], f0[2], f1[2], f0[3], f1[3], u.q[z][n][2 * i + 1][0], u.q[z][n][2 * i + 1][1]);
                    }
            }
        }
    }
    const bool in0 = r0 < rows, in1 = r0 + 8 < rows;
    uint32_t p16[QP][NG][2];
#pragma unroll
    for (int n = 0; n < NG; ++n) {
#pragma unroll
        for (int e = 0; e < 4; ++e) x[n][e] = logit2(a, (x[n][e] + y[n][e]) * u.lift[n][e & 1], u.slope[n][e & 1], far[e >> 1]);
        if (logits) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int h = n * 8 + 2 * t + (e & 1);
                if (h < nh && (e < 2 ? in0 : in1)) logits[h * S::kTile + r0 + (e >> 1) * 8] = x[n][e];
            }
        }
        float top[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            top[e] = fmaxf(in0 ? x[n][e] : kLow, in1 ? x[n][e + 2] : kLow);
#pragma unroll
            for (int s = 4; s < 32; s <<= 1) top[e] = fmaxf(top[e], __shfl_xor_sync(0xFFFFFFFFu, top[e], s));
            top[e] = fmaxf(top[e] - kLift, u.m[n][e]);
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
            const __half2 hi = __floats2half2_rn(p[2 * e], p[2 * e + 1]);
            p16[0][n][e] = transpose8x8(as_u32(hi));
            if constexpr (QP == 2) p16[1][n][e] = transpose8x8(pack_f16(p[2 * e] - __low2float(hi), p[2 * e + 1] - __high2float(hi)));
        }
    }
    {
        // places 2 t + e + 8 f: words of both rows of a pair, interleaved; scales of rows that are not there are zeros
        uint32_t w[2][DH / 64][2], sc[2];
#pragma unroll
        for (int f = 0; f < 2; ++f) {
            const int ra = row_at(2 * t) + 8 * f, rb = row_at(2 * t + 1) + 8 * f;
            uint32_t va[DH / 64], vb[DH / 64], sa, sb;
            if constexpr (DH == 128) {
                const uint2 x0 = *reinterpret_cast<const uint2*>(vp + ra * 64 + g * 8), x1 = *reinterpret_cast<const uint2*>(vp + rb * 64 + g * 8);
                va[0] = x0.x; va[1] = x0.y; vb[0] = x1.x; vb[1] = x1.y;
                sa = vp[8 * DH + ra * 8 + g];
                sb = vp[8 * DH + rb * 8 + g];
            } else {
                va[0] = *reinterpret_cast<const uint32_t*>(vp + ra * 32 + g * 4);
                vb[0] = *reinterpret_cast<const uint32_t*>(vp + rb * 32 + g * 4);
                sa = vp[8 * DH + ra * 4 + (g >> 1)];
                sb = vp[8 * DH + rb * 4 + (g >> 1)];
            }
            sc[f] = (ra < rows ? sa << 8 : 0u) | (rb < rows ? sb << 24 : 0u);
#pragma unroll
            for (int i = 0; i < DH / 64; ++i) {
                w[f][i][0] = __byte_perm(va[i], vb[i], 0x5410);
                w[f][i][1] = __byte_perm(va[i], vb[i], 0x7632);
            }
        }
        const Q4Block b0(sc[0]), b1(sc[1]);
#pragma unroll
        for (int i = 0; i < DH / 64; ++i)
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                uint32_t f0[4], f1[4];
                b0.pairs(w[0][i][half], f0);
                b1.pairs(w[1][i][half], f1);
                const int k = 4 * i + 2 * half;
#pragma unroll
                for (int n = 0; n < NG; ++n)
#pragma unroll
                    for (int z = 0; z < QP; ++z) {
                        mma_f16(u.o[n][k], f0[0], f0[1], f1[0], f1[1], p16[z][n][0], p16[z][n][1]);
                        mma_f16(u.o[n][k + 1], f0[2], f0[3], f1[2], f1[3], p16[z][n][0], p16[z][n][1]);
                    }
            }
    }
}

// A unit's warps meet in shared memory, o [head][DH], m and l [head]: close() adds up the lanes' sums, store() writes the warp's part,
// merge() takes another warp's part in.
template <int DH, int NG, int QP>
__device__ __forceinline__ void unit_close(Q4Unit<DH, NG, QP>& u) {
#pragma unroll
    for (int n = 0; n < NG; ++n)
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
            for (int s = 4; s < 32; s <<= 1) u.l[n][e] += __shfl_xor_sync(0xFFFFFFFFu, u.l[n][e], s);
}
template <int DH, int NG, int QP>
__device__ __forceinline__ void unit_merge(Q4Unit<DH, NG, QP>& u, const float* s_o, const float* s_ml) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int n = 0; n < NG; ++n) {
        const int h = n * 8 + 2 * (lane & 3);
        float f[2], w[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const float m = s_ml[2 * (h + e)], M = fmaxf(m, u.m[n][e]);
            f[e] = sm100::fast_exp2(u.m[n][e] - M);
            w[e] = sm100::fast_exp2(m - M);
            u.l[n][e] = u.l[n][e] * f[e] + s_ml[2 * (h + e) + 1] * w[e];
            u.m[n][e] = M;
        }
#pragma unroll
        for (int k = 0; k < DH / 16; ++k)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const float2 x = *reinterpret_cast<const float2*>(s_o + (h + e) * DH + DH / 8 * (lane >> 2) + 2 * k);
                u.o[n][k][e] = u.o[n][k][e] * f[e] + x.x * w[e];
                u.o[n][k][e + 2] = u.o[n][k][e + 2] * f[e] + x.y * w[e];
            }
    }
}
template <int DH, int NG, int QP>
__device__ __forceinline__ void unit_store(Q4Unit<DH, NG, QP>& u, float* s_o, float* s_ml) {
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
            for (int e = 0; e < 2; ++e)
                *reinterpret_cast<float2*>(s_o + (h + e) * DH + DH / 8 * (lane >> 2) + 2 * k) = make_float2(u.o[n][k][e], u.o[n][k][e + 2]);
    }
}

template <typename T, int DH, int NG>
__global__ void __launch_bounds__(kThreads, q4_ctas(NG))
paged_attn_q4_kernel(const PagedAttnArgs a, const uint8_t* __restrict__ k_pool, const uint8_t* __restrict__ v_pool) {
    using namespace sm100;
    using S = Q4Shape<DH>;
    constexpr int QP = sizeof(T) == 4 ? 2 : 1;
    extern __shared__ uint8_t smem_dyn[];
    __shared__ __align__(8) uint64_t full_bar[S::kStages], empty_bar[S::kStages];
    __shared__ __align__(16) float s_o[2][NG * 8 * DH];
    __shared__ float s_ml[2][NG * 16];
    __shared__ long long s_sum[kWarps + 1];
    __shared__ long long s_start;
    __shared__ int s_b;
    __shared__ int s_abort;
    const int warp = __shfl_sync(0xFFFFFFFFu, (int)threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    uint8_t* const ring = smem_dyn + (((smem_u32(smem_dyn) + 127u) & ~127u) - smem_u32(smem_dyn));
    const int subs = a.d.Hkv * a.NC;
    if (threadIdx.x == 0) {
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
    Place p = find_place(a, subs, t_lo, t_hi, &s_b, &s_start);
    volatile int* abort_flag = &s_abort;

    if (warp == kWarps) {                              // brings the tiles
        const int per_page = 1 << (a.d.page_shift - 4), run = min(per_page, kWarps);       // pieces of a page that are a copy
        int it = 0;
        for (; p.left > 0; ++it) {
            const int s = it % S::kStages;
            if (!mbar_wait_warp(smem_u32(&empty_bar[s]), ((uint32_t)(it / S::kStages) & 1u) ^ 1u, abort_flag)) break;
            const int r0 = p.t * S::kTile, rows = min(S::kTile, a.kv_len[p.b] - r0), pieces = (rows + kQ4Rows - 1) / kQ4Rows;
            const uint32_t fb = smem_u32(&full_bar[s]);
            if (lane == 0) mbar_arrive_expect_tx(fb, 2u * pieces * S::kPiece);
            __syncwarp();
            const int pc = (lane >> 1) * run, n = min(run, pieces - pc);
            // (debug builds: one copy never sent)
            if (n > 0 && !(dbg_held(a.withhold, kDbgPagedAttn) && blockIdx.x == 0 && it == 0 && lane == 0)) {
                const int row = r0 + pc * kQ4Rows;
                int page = a.block_table[(size_t)p.b * a.d.max_pages + (row >> a.d.page_shift)];
                if (page < 0 || page >= a.d.n_pages) page = 0;          // the second kernel drops the sequence
                const size_t at = q4_piece_of(a.d, page, p.sub / a.NC, row) * S::kPiece;
                bulk_load(smem_u32(ring) + s * S::kStage + (lane & 1) * S::kHalf + pc * S::kPiece, ((lane & 1) ? v_pool : k_pool) + at,
                          (uint32_t)n * S::kPiece, fb);
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
        int it = 0, newest = 0;
        bool ok = true, fresh = true;
        Q4Unit<DH, NG, QP> u;
        while (p.left > 0) {
            const int hk = p.sub / a.NC, ch = p.sub - hk * a.NC, h0 = hk * a.G + ch * a.heads, nh = min(a.heads, a.G - ch * a.heads);
            const int len = a.kv_len[p.b], r0 = p.t * S::kTile + warp * kQ4Rows, rows = len - r0;
            const int32_t* pos = a.positions ? a.positions + (size_t)p.b * a.d.S_cap() : nullptr;
            if (fresh) {
                u.template start<T>(a, p.b, h0, nh);
                newest = a.slopes ? (pos ? pos[len - 1] : len - 1) : 0;
                fresh = false;
            }
            const int s = it % S::kStages;
            // distances of the rows that this lane's logits are of
            float far[2] = {0.f, 0.f};
            if (a.slopes) {
                auto distance = [&](int r) { r = min(r0 + r, len - 1); return fabsf((float)newest - (float)(pos ? pos[r] : r)); };
                far[0] = distance(row_at(lane >> 2));
                far[1] = distance(row_at(lane >> 2) + 8);
            }
            float* logits = nullptr;
            if (a.mass) logits = a.logits + (size_t)(t_hi - p.left) * a.heads * S::kTile + warp * kQ4Rows;
            if (ok && !mbar_wait_warp(smem_u32(&full_bar[s]), (uint32_t)(it / S::kStages) & 1u, abort_flag)) ok = false;
            if (ok) {
                const uint8_t* k = ring + s * S::kStage + warp * S::kPiece;
                if (rows > 0) q4_tile<DH, NG, QP>(u, a, k, k + S::kHalf, rows, far, logits, nh);
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&empty_bar[s]));
            }
            const long long unit = (long long)p.b * subs + p.sub;
            const bool ends = p.t + 1 == p.nt || p.left == 1;
            ++it;
            next_tile(a, p, subs);
            if (ends) {
                fresh = true;
                // warps 2 and 3 give their rows to warps 0 and 1; what those have is joined on the way out
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
                    const float m0 = s_ml[0][2 * h], m1 = s_ml[1][2 * h], M = fmaxf(m0, m1);
                    const float f = fast_exp2(m0 - M), w = fast_exp2(m1 - M), L = f * s_ml[0][2 * h + 1] + w * s_ml[1][2 * h + 1];
                    const float4 x = reinterpret_cast<const float4*>(s_o[0])[i], y = reinterpret_cast<const float4*>(s_o[1])[i];
                    reinterpret_cast<float4*>(a.part_o + slot * a.heads * DH)[i] =
                        make_float4(kQ4Unit * (f * x.x + w * y.x), kQ4Unit * (f * x.y + w * y.y), kQ4Unit * (f * x.z + w * y.z), kQ4Unit * (f * x.w + w * y.w));
                    if (i % (DH / 4) == 0) reinterpret_cast<float2*>(a.part_ml + slot * a.heads * 2)[h] = make_float2(M, L);
                }
                named_bar_sync(1, kWarps * 32);
            }
        }
    }
    __syncthreads();
    if (threadIdx.x == 0 && s_abort) *a.status = METOK_ERR_TIMEOUT;
}

PagedPlan q4_plan(const PagedDims& d, int Hq) {
    const int G = Hq / d.Hkv, per = ceil_div(G, ceil_div(G, 16)), heads = per <= 8 ? 8 : 16;
    return paged_plan_of(d, Hq, heads, 6, q4_ctas(heads / 8) * kNumSMs);
}

template <typename T, int DH, int NG>
int launch_q4(const PagedAttnArgs& a, const void* k_pool, const void* v_pool, cudaStream_t st) {
    using S = Q4Shape<DH>;
    auto kern = paged_attn_q4_kernel<T, DH, NG>;
    METOK_ALLOW_SMEM(kern, S::kRing);
    {
        METOK_TIMED("paged_attn_q4", st);
        launch_chained(kern, dim3(a.grid + 1), dim3(kThreads), S::kRing, st, a, (const uint8_t*)k_pool, (const uint8_t*)v_pool);
    }
    METOK_LAUNCH_CHECK();
    return launch_paged_join<T, DH>(a, st);
}
template <typename T>
int launch_q4_type(const PagedAttnArgs& a, const void* k, const void* v, cudaStream_t st) {
    if (a.d.dh == 64) return a.heads == 8 ? launch_q4<T, 64, 1>(a, k, v, st) : launch_q4<T, 64, 2>(a, k, v, st);
    return a.heads == 8 ? launch_q4<T, 128, 1>(a, k, v, st) : launch_q4<T, 128, 2>(a, k, v, st);
}

}  // namespace
}  // namespace metok

using namespace metok;

extern "C" size_t metok_paged_attention_q4_workspace_bytes(int dtype, const metok_paged_cache* c, int Hq, int with_mass) {
    PagedDims d;
    if ((dtype != METOK_F32 && dtype != METOK_BF16) || paged_dims_q4(c, &d) != METOK_OK || Hq < 1 || Hq % d.Hkv) return 0;
    PagedAttnArgs a;
    Carver cv(nullptr);
    paged_carve(cv, q4_plan(d, Hq), d, with_mass != 0, &a);
    return cv.total();
}

extern "C" int metok_paged_attention_q4(int dtype, const metok_paged_cache* c, const void* q, int64_t q_seq, int64_t q_head, int Hq,
                                        float softmax_scale, float softcap, const float* slopes, const int32_t* positions, float* mass,
                                        void* out, int64_t out_seq, int64_t out_head, float* lse, int32_t* status, void* ws,
                                        size_t ws_bytes, void* stream) {
    PagedDims d;
    if (dtype != METOK_F32 && dtype != METOK_BF16) return METOK_ERR_INVALID_ARG;
    int rc = paged_dims_q4(c, &d);
    if (rc == METOK_OK) rc = paged_attention_heads(d, c, q, out, status, Hq);
    if (rc != METOK_OK) return rc;
    const PagedPlan p = q4_plan(d, Hq);
    PagedAttnArgs a;
    rc = paged_attention_args(dtype, d, c, p, q, q_seq, q_head, Hq, softmax_scale, softcap, slopes, positions, mass, out, out_seq, out_head, lse,
                              status, &a);
    if (rc != METOK_OK) return rc;
    if (!ws || !aligned16(ws) || ws_bytes < metok_paged_attention_q4_workspace_bytes(dtype, c, Hq, mass != nullptr)) return METOK_ERR_WORKSPACE;
    Carver cv(ws);
    paged_carve(cv, p, d, mass != nullptr, &a);
    cudaStream_t st = (cudaStream_t)stream;
    return dtype == METOK_F32 ? launch_q4_type<float>(a, c->k_pool, c->v_pool, st) : launch_q4_type<__nv_bfloat16>(a, c->k_pool, c->v_pool, st);
}
