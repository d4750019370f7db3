// metok_paged_attention_q4: attention of one new token per sequence over its paged K/V cache held in 4 bits.
//
// The line of tiles, the partials and the join are those of the attention over a cache of numbers (paged_attn.cuh).  A tile is eight pieces
// of 16 rows, which one warp brings by bulk copies through a ring of shared memory; four warps take two pieces each.
//
// A row is 4.5 bits per element, so that what bounds the kernel is no longer reading but turning codes into numbers.  It costs two
// operations and a quarter of a shift for a pair: a nibble c of one element and that of the element four behind it, or of another row's, are masked into
// the fractions of two fp16 numbers, 1024 + c or 1024 + 16 c, and one multiply-add with constants of the block, (1024 + c) e - 1032 e or
// (1024 + 16 c) e/16 - 72 e, gives (c - 8) e.  e has three significant bits, so that all constants and results are exact (q4.cuh).
//   x^T = K Q^T (mma.sync m16n8k16, rows x heads): a thread holds the nibbles of whole blocks, a quarter of two rows, so it needs these
//     blocks' constants alone; the elements of Q are dealt out in the order in which the nibbles come.
//   o^T += V^T P^T: a thread holds an eighth of four rows; two rows' words are interleaved by 16 bits first, since a pair of the product
//     is a pair of rows.
//   The rows that a thread takes for its places in the products are permuted, r -> r ^ (r >> 2 & 1), which no sum notices: so the reads of V
//   meet two banks at a time at most (and those of K none).
// The tensor memory path would take one side of 128 for eight heads, and 4-bit operands of another format whose scales go along the sum, which V's
// rows do not.
// Q takes part as fp16 numbers relative to the head's largest element: bf16's eight bits are in one; fp32's are in two to 2^-22.  The weights
// are 2^12 to 2^15.5 times those relative to the largest and take part as two fp16 numbers, to 2^-22: as one (off by 2^-11) they moved one bf16
// output in twelve to forty to another step, and small sums of large terms by several, for 2 to 5 % of the time.  Logits, their sums, and outputs up to
// their end are fp32.
//
// 48 sequences of up to 9001 rows, 28 / 4 heads of 128, capped: 47.4 us with the join, of which reading 157 MB would be 24.  Three sequences of up to
// 6313 rows, 40 heads of their own, biased, with weights: 34 us (reading: 13).
#include "paged_attn.cuh"
#include "q4.cuh"

namespace metok {

namespace {

// A head's weights are exp2(x - m) with a reference m that was 2^12 below the largest when it was taken; it is taken anew where a weight passes 2^15.5
// (fp16 ends at 2^16).
constexpr float kLift = 12.f, kMostWeight = 15.5f;

// A CTA has an SM to itself: kGroups groups of kWarps warps, each with a piece of the line, a ring and a warp that fills it.  (As CTAs of their
// own the groups of an SM end at different times, since its schedulers prefer some warps to others: here no ring may be filled further ahead of
// the others than by a tile.)  RP: pieces of 16 rows of a tile that are one warp's.
constexpr int kWarps = 4;
template <int DH, int NG, int RP>
struct Q4Shape {
    static constexpr int kGroups = NG == 1 ? 3 : 2, kThreads = kGroups * (kWarps + 1) * 32;
    static constexpr int kPieces = kWarps * RP, kTile = kQ4Rows * kPieces;
    static constexpr uint32_t kPiece = q4_piece(DH), kHalf = kPieces * kPiece, kStage = 2 * kHalf;     // K, then V
    static constexpr int kStages = 55296 / kStage;
    static constexpr uint32_t kRing = kStages * kStage;
};

__device__ __forceinline__ uint32_t as_u32(__half2 h) { return *reinterpret_cast<uint32_t*>(&h); }
__device__ __forceinline__ __half2 as_half2(uint32_t u) { return *reinterpret_cast<__half2*>(&u); }
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) { return as_u32(__floats2half2_rn(lo, hi)); }
__device__ __forceinline__ uint32_t transpose8x8(uint32_t v) {
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
    return r;
}
__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// The first product of a sum.
__device__ __forceinline__ void mma_f16_first(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
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
    // Nibbles j and j + 4 of `w`, j = 0 .. 3.  (One operation masks and sets the exponents only where one of the constants is in a register.)
    __device__ __forceinline__ void pairs(uint32_t w, uint32_t (&r)[4]) const {
#pragma unroll
        for (int j = 0; j < 4; j += 2) {
            r[j] = as_u32(__hfma2(as_half2(mask_or(w, 0x000F000Fu)), e, c0));
            r[j + 1] = as_u32(__hfma2(as_half2(mask_or(w, 0x00F000F0u)), e16, c1));
            w >>= 8;
        }
    }
    static __device__ __forceinline__ uint32_t mask_or(uint32_t w, uint32_t mask) {
        uint32_t r;
        asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(r) : "r"(w), "r"(mask), "r"(0x64006400u));
        return r;
    }
};

// A unit's running softmax.  NG groups of eight heads, QP fp16 numbers per element of Q.  Lane l holds the logits of rows
// pi(l / 4) and pi(l / 4) + 8 of the warp's 16 and of heads 2 (l % 4), + 1; of o the DH / 8 elements from DH / 8 * (l / 4) on.
template <int DH, int NG, int QP>
struct Q4Unit {
    uint32_t q[QP][NG][DH / 16][2];
    float m[NG][2], l[NG][2], o[NG][DH / 16][4], slope[NG][2], scale[NG][2];     // scale: from products to logits, or to those of whole q where they are capped

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
                    // what is left of an infinite element is nothing (inf - inf would make a NaN of its logits)
                    const auto rest = [](float x, float h) { return isinf(h) ? 0.f : x - h; };
                    if constexpr (QP == 2) q[1][n][2 * i + (e >> 1)][e & 1] = pack_f16(rest(x0, __low2float(hi)), rest(x1, __high2float(hi)));
                }
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int hc = n * 8 + 2 * t + e;
                scale[n][e] = __shfl_sync(0xFFFFFFFFu, up, (2 * t + e) * 4);
                if (!(a.cap_log2 > 0.f)) scale[n][e] = fmaxf(scale[n][e] * a.scale_log2, 1.2e-38f);      // (never 0: rows that are not there count as -infinity)
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

// tanh(y) of logits in units of the cap, |y| <= 1: y P(y^2), P the polynomial of degree 6 of least largest relative error (7e-8 with coefficients in
// fp32; 1.6e-7 worked out in fp32).
__device__ __forceinline__ uint64_t tanh_near(uint64_t y) {
    using namespace sm100;
    const auto both = [](float c) { return pair(c, c); };
    const uint64_t u = mul_pair(y, y);
    uint64_t t = both(0.0010410226f);
    t = fma_pair(t, u, both(-0.00620337902f));
    t = fma_pair(t, u, both(0.0202899799f));
    t = fma_pair(t, u, both(-0.0534570292f));
    t = fma_pair(t, u, both(0.13325204f));
    t = fma_pair(t, u, both(-0.333328396f));
    t = fma_pair(t, u, both(0.99999994f));
    return mul_pair(y, t);
}

// The warp's RP pieces of a tile, of whose rows `rows` are there (kPart: not all; >= 1).  kBent: logits are capped or biased; `pos`: positions of the
// lane's rows, for the bias.  kMass: `logits` of the warp's rows, [head][kTile], are left for the second kernel.
template <int DH, int NG, int QP, int RP, bool kBent, bool kMass, bool kPart>
__device__ __forceinline__ void q4_tile(Q4Unit<DH, NG, QP>& u, const PagedAttnArgs& a, const uint8_t* kp, const uint8_t* vp, int rows,
                                        float newest, const int (&pos)[2 * RP], float* logits, int nh) {
    using S = Q4Shape<DH, NG, RP>;
    const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3, r0 = row_at(g);
    using namespace sm100;
    float x[RP][NG][4];                                // products, or logits (kBent)
    const auto two = [](const float* v) { return pair(v[0], v[1]); };    // the lane's two heads
    uint64_t low[NG];
    auto less = [&](int r, int n, int i, float (&d)[2]) {                // logits of row i less their references
        const uint64_t v = two(&x[r][n][2 * i]);
        unpair(kBent ? add_pair(v, low[n]) : fma_pair(v, two(u.scale[n]), low[n]), d[0], d[1]);
    };
#pragma unroll
    for (int r = 0; r < RP; ++r) {
        const uint8_t* const piece = kp + r * S::kPiece;
        float y[NG][4];                                // two chains of products
        uint32_t w[2][DH / 32], sc[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int row = r0 + 8 * i;
            if constexpr (DH == 128) {
                const uint4 v = *reinterpret_cast<const uint4*>(piece + row * 64 + t * 16);
                w[i][0] = v.x; w[i][1] = v.y; w[i][2] = v.z; w[i][3] = v.w;
                sc[i] = *reinterpret_cast<const uint16_t*>(piece + 8 * DH + row * 8 + 2 * t);
            } else {
                const uint2 v = *reinterpret_cast<const uint2*>(piece + row * 32 + t * 8);
                w[i][0] = v.x; w[i][1] = v.y;
                sc[i] = piece[8 * DH + row * 4 + t];
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
                        if (i == 0 && z == 0) {
                            mma_f16_first(x[r][n], f0[0], f1[0], f0[1], f1[1], u.q[z][n][2 * i][0], u.q[z][n][2 * i][1]);
                            mma_f16_first(y[n], f0[2], f1[2], f0[3], f1[3], u.q[z][n][2 * i + 1][0], u.q[z][n][2 * i + 1][1]);
                        } else {
                            mma_f16(x[r][n], f0[0], f1[0], f0[1], f1[1], u.q[z][n][2 * i][0], u.q[z][n][2 * i][1]);
                            mma_f16(y[n], f0[2], f1[2], f0[3], f1[3], u.q[z][n][2 * i + 1][0], u.q[z][n][2 * i + 1][1]);
                        }
                    }
            }
        }
#pragma unroll
        for (int n = 0; n < NG; ++n)
#pragma unroll
            for (int i = 0; i < 4; i += 2) {
                uint64_t v = add_pair(two(&x[r][n][i]), two(&y[n][i]));
                if constexpr (kBent) v = mul_pair(v, two(u.scale[n]));
                unpair(v, x[r][n][i], x[r][n][i + 1]);
            }
    }
    if constexpr (kBent) {
        if (a.cap_log2 > 0.f) {
            float most = 0.f;
#pragma unroll
            for (int r = 0; r < RP; ++r)
#pragma unroll
                for (int n = 0; n < NG; ++n)
#pragma unroll
                    for (int i = 0; i < 4; i += 2) {   // in units of the cap
                        unpair(mul_pair(two(&x[r][n][i]), pair(a.cap_scale, a.cap_scale)), x[r][n][i], x[r][n][i + 1]);
                        // rows that are not there have no say in how the others are capped
                        if (kPart && r0 + 16 * r + 4 * i >= rows) x[r][n][i] = x[r][n][i + 1] = 0.f;
                        most = fmaxf(most, fmaxf(fabsf(x[r][n][i]), fabsf(x[r][n][i + 1])));
                    }
            if (__any_sync(0xFFFFFFFFu, !(most <= 1.f))) {
#pragma unroll
                for (int r = 0; r < RP; ++r)
#pragma unroll
                    for (int n = 0; n < NG; ++n)
#pragma unroll
                        for (int e = 0; e < 4; ++e) x[r][n][e] = a.cap_log2 * tanhf(x[r][n][e]);
            } else {                                   // (a NaN comes out as one here, too)
#pragma unroll
                for (int r = 0; r < RP; ++r)
#pragma unroll
                    for (int n = 0; n < NG; ++n)
#pragma unroll
                        for (int i = 0; i < 4; i += 2)
                            unpair(mul_pair(tanh_near(two(&x[r][n][i])), pair(a.cap_log2, a.cap_log2)), x[r][n][i], x[r][n][i + 1]);
            }
        }
        if (a.slopes) {
#pragma unroll
            for (int r = 0; r < RP; ++r)
#pragma unroll
                for (int n = 0; n < NG; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[r][n][e] = fmaf(-u.slope[n][e & 1], fabsf(newest - (float)pos[2 * r + (e >> 1)]), x[r][n][e]);
        }
    }
    if constexpr (kMass) {
#pragma unroll
        for (int r = 0; r < RP; ++r)
#pragma unroll
            for (int n = 0; n < NG; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int h = n * 8 + 2 * t + (e & 1), row = r0 + 16 * r + 8 * (e >> 1);
                    if (h < nh && (!kPart || row < rows)) logits[h * S::kTile + row] = kBent ? x[r][n][e] : x[r][n][e] * u.scale[n][e & 1];
                }
    }
    float more = kLow;
#pragma unroll
    for (int n = 0; n < NG; ++n) low[n] = pair(-u.m[n][0], -u.m[n][1]);
#pragma unroll
    for (int r = 0; r < RP; ++r)
#pragma unroll
        for (int n = 0; n < NG; ++n)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                // rows that are not there have no weight
                if (kPart && r0 + 16 * r + 8 * i >= rows) x[r][n][2 * i] = x[r][n][2 * i + 1] = __int_as_float(0xFF800000);
                float d[2];
                less(r, n, i, d);
                more = fmaxf(more, fmaxf(d[0], d[1]));
            }
    if (__any_sync(0xFFFFFFFFu, more > kMostWeight)) {
#pragma unroll
        for (int n = 0; n < NG; ++n) {
            float f[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float top = kLow;
#pragma unroll
                for (int r = 0; r < RP; ++r) top = fmaxf(top, fmaxf(x[r][n][e], x[r][n][e + 2]));
#pragma unroll
                for (int s = 4; s < 32; s <<= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, s));
                if (!kBent) top *= u.scale[n][e];              // (> 0)
                top = fmaxf(top - kLift, u.m[n][e]);
                f[e] = sm100::fast_exp2(u.m[n][e] - top);
                u.l[n][e] *= f[e];
                u.m[n][e] = top;
            }
#pragma unroll
            for (int k = 0; k < DH / 16; ++k)
#pragma unroll
                for (int e = 0; e < 4; ++e) u.o[n][k][e] *= f[e & 1];
            low[n] = pair(-u.m[n][0], -u.m[n][1]);
        }
    }
    uint32_t p16[RP][2][NG][2];                        // weights: a number and what it leaves
#pragma unroll
    for (int r = 0; r < RP; ++r)
#pragma unroll
        for (int n = 0; n < NG; ++n) {
            float p[4];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                float d[2];
                less(r, n, i, d);
                p[2 * i] = fast_exp2(d[0]);
                p[2 * i + 1] = fast_exp2(d[1]);
            }
            unpair(add_pair(two(u.l[n]), add_pair(two(p), two(p + 2))), u.l[n][0], u.l[n][1]);
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const __half2 hi = __floats2half2_rn(p[2 * e], p[2 * e + 1]);
                p16[r][0][n][e] = transpose8x8(as_u32(hi));
                p16[r][1][n][e] = transpose8x8(pack_f16(p[2 * e] - __low2float(hi), p[2 * e + 1] - __high2float(hi)));
            }
        }
#pragma unroll
    for (int r = 0; r < RP; ++r) {
        const uint8_t* const piece = vp + r * S::kPiece;
        // places 2 t + e + 8 f: words of both rows of a pair, interleaved; scales of rows that are not there are zeros
        uint32_t w[2][DH / 64][2], sc[2];
#pragma unroll
        for (int f = 0; f < 2; ++f) {
            const int ra = row_at(2 * t) + 8 * f, rb = row_at(2 * t + 1) + 8 * f;
            uint32_t va[DH / 64], vb[DH / 64], sa, sb;
            if constexpr (DH == 128) {
                const uint2 x0 = *reinterpret_cast<const uint2*>(piece + ra * 64 + g * 8), x1 = *reinterpret_cast<const uint2*>(piece + rb * 64 + g * 8);
                va[0] = x0.x; va[1] = x0.y; vb[0] = x1.x; vb[1] = x1.y;
                sa = piece[8 * DH + ra * 8 + g];
                sb = piece[8 * DH + rb * 8 + g];
            } else {
                va[0] = *reinterpret_cast<const uint32_t*>(piece + ra * 32 + g * 4);
                vb[0] = *reinterpret_cast<const uint32_t*>(piece + rb * 32 + g * 4);
                sa = piece[8 * DH + ra * 4 + (g >> 1)];
                sb = piece[8 * DH + rb * 4 + (g >> 1)];
            }
            sc[f] = __byte_perm(sa, sb, 0x4101);       // the bytes into the upper bytes of the halves
            if (kPart) sc[f] &= (ra + 16 * r < rows ? 0xFFFFu : 0u) | (rb + 16 * r < rows ? 0xFFFF0000u : 0u);
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
                    for (int z = 0; z < 2; ++z) {
                        mma_f16(u.o[n][k], f0[0], f0[1], f1[0], f1[1], p16[r][z][n][0], p16[r][z][n][1]);
                        mma_f16(u.o[n][k + 1], f0[2], f0[3], f1[2], f1[3], p16[r][z][n][0], p16[r][z][n][1]);
                    }
            }
    }
}

// A unit's end: the warps leave o in shared memory as their lanes hold it, and m and l by head; then each warp joins a quarter of o.
template <int DH, int NG>
struct Q4Join {
    float2 o[kWarps][NG][DH / 16][2][32];              // elements 2 k, 2 k + 1 of the lane's of heads 2 t, 2 t + 1
    float2 ml[kWarps][NG * 8];
};
template <int DH, int NG, int QP>
__device__ __forceinline__ void unit_end(Q4Unit<DH, NG, QP>& u, Q4Join<DH, NG>& j, int group, int bad, int nh, float* part_o, float2* part_ml) {
    const int warp = (threadIdx.x >> 5) % kWarps, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
#pragma unroll
    for (int n = 0; n < NG; ++n) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
#pragma unroll
            for (int s = 4; s < 32; s <<= 1) u.l[n][e] += __shfl_xor_sync(0xFFFFFFFFu, u.l[n][e], s);
            if (lane < 4) j.ml[warp][n * 8 + 2 * t + e] = make_float2(u.m[n][e], u.l[n][e]);
#pragma unroll
            for (int k = 0; k < DH / 16; ++k) j.o[warp][n][k][e][lane] = make_float2(u.o[n][k][e], u.o[n][k][e + 2]);
        }
    }
    sm100::named_bar_sync(1 + group, kWarps * 32);
    constexpr int kMine = DH / 16 / kWarps;            // k that are this warp's: 2 kMine elements in a row
#pragma unroll
    for (int n = 0; n < NG; ++n)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int h = n * 8 + 2 * t + e;
            float2 ml[kWarps];
            float M = kLow, L = 0.f;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) {
                ml[w] = j.ml[w][h];
                M = fmaxf(M, ml[w].x);
            }
            float2 o[kMine];
#pragma unroll
            for (int k = 0; k < kMine; ++k) o[k] = make_float2(0.f, 0.f);
#pragma unroll
            for (int w = 0; w < kWarps; ++w) {
                const float f = sm100::fast_exp2(ml[w].x - M);
                L += f * ml[w].y;
#pragma unroll
                for (int k = 0; k < kMine; ++k) {
                    const float2 x = j.o[w][n][warp * kMine + k][e][lane];
                    o[k].x = fmaf(f * kQ4Unit, x.x, o[k].x);
                    o[k].y = fmaf(f * kQ4Unit, x.y, o[k].y);
                }
            }
            if (h < nh) {
                float* dst = part_o + h * DH + DH / 8 * g + 2 * kMine * warp;
                if constexpr (kMine == 2) *reinterpret_cast<float4*>(dst) = make_float4(o[0].x, o[0].y, o[1].x, o[1].y);
                else *reinterpret_cast<float2*>(dst) = o[0];
                if (warp == 0 && g == 0) part_ml[h] = make_float2(M, bad ? -1.f : L);
            }
        }
    sm100::named_bar_sync(1 + group, kWarps * 32);
}

template <typename T, int DH, int NG, int RP, bool kBent, bool kMass>
__global__ void __launch_bounds__((Q4Shape<DH, NG, RP>::kThreads), 1)
paged_attn_q4_kernel(const PagedAttnArgs a, const uint8_t* __restrict__ k_pool, const uint8_t* __restrict__ v_pool) {
    using namespace sm100;
    using S = Q4Shape<DH, NG, RP>;
    constexpr int QP = sizeof(T) == 4 ? 2 : 1, kGroups = S::kGroups;
    extern __shared__ uint8_t smem_dyn[];
    __shared__ __align__(8) uint64_t full_bar[kGroups][S::kStages], empty_bar[kGroups][S::kStages];
    __shared__ long long s_sum[kGroups * (kWarps + 1)];
    __shared__ volatile int s_filled[kGroups];
    __shared__ int s_bad[kGroups][S::kStages];
    __shared__ int s_abort;
    const int warp = __shfl_sync(0xFFFFFFFFu, (int)threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    const bool fills = warp >= kGroups * kWarps;
    const int group = fills ? warp - kGroups * kWarps : warp / kWarps;
    const int subs = a.d.Hkv * a.NC;
    uint8_t* const base = smem_dyn + (((smem_u32(smem_dyn) + 127u) & ~127u) - smem_u32(smem_dyn));
    uint8_t* const ring = base + group * S::kRing;
    if (fills && lane == 0) {
        for (int s = 0; s < S::kStages; ++s) { mbar_init(smem_u32(&full_bar[group][s]), 1); mbar_init(smem_u32(&empty_bar[group][s]), kWarps); }
        s_filled[group] = 0;
        s_abort = 0;
        mbar_fence_init();
    }
    grid_dep_wait();
    if (blockIdx.x == 0 && threadIdx.x == 0) *a.status = METOK_OK;       // a wait that gives up writes it, seconds later
    // pieces of the line go to the CTAs first, then to their groups
    const int piece = group * gridDim.x + blockIdx.x;
    long long t_hi = 0;
    Place p;
    p.left = 0;
    const auto cut = [&](long long T_all) {            // false: the whole CTA has nothing to do
        const long long busy = busy_ctas(a, T_all);
        if (blockIdx.x >= busy) {
            if (blockIdx.x == 0 && warp == 0) write_line(a);
            return false;
        }
        if (piece < busy) {
            const long long t_lo = quotient(T_all * piece, busy);
            t_hi = quotient(T_all * (piece + 1), busy);
            p.left = t_hi - t_lo;
        } else if (fills && lane == 0) {
            s_filled[group] = 0x7FFFFFFF;
        }
        return true;
    };
    if (a.d.n_seqs <= kHeldSeqs) {
        HeldTiles held;
        held.load(a);
        const long long T_all = (long long)held.all * subs;
        if (!cut(T_all)) return;
        if (p.left > 0) p = T_all <= 0x7FFFFFFF ? held.find(subs, (uint32_t)(t_hi - p.left), (uint32_t)t_hi) : find_tile(a, subs, T_all, t_hi - p.left, t_hi);
    } else {
        const long long T_all = line_tiles(a, s_sum) * subs;
        if (!cut(T_all)) return;
        if (p.left > 0) p = find_tile(a, subs, T_all, t_hi - p.left, t_hi);
    }
    __syncthreads();
    volatile int* abort_flag = &s_abort;

    if (fills) {
        const int per_page = 1 << (a.d.page_shift - 4), run = min(per_page, S::kPieces);   // pieces of a page that are a copy
        int it = 0;
        for (; p.left > 0; ++it) {
            const int s = it % S::kStages, r0 = p.t * S::kTile, rows = min(S::kTile, a.kv_len[p.b] - r0), pieces = (rows + kQ4Rows - 1) / kQ4Rows;
            const int pc = (lane >> 1) * run, n = min(run, pieces - pc), row = r0 + pc * kQ4Rows;
            int page = n > 0 ? a.block_table[(size_t)p.b * a.d.max_pages + (row >> a.d.page_shift)] : 0;
            if (!mbar_wait_warp(smem_u32(&empty_bar[group][s]), ((uint32_t)(it / S::kStages) & 1u) ^ 1u, abort_flag)) break;
            uint32_t polls = 0;
            for (int g = 0; g < kGroups; ++g)
                while (s_filled[g] < it - 1 && polls < kWaitLimit && !((++polls & 255u) == 0 && *abort_flag)) {}
            const uint32_t fb = smem_u32(&full_bar[group][s]);
            // (debug builds: one copy never sent)
            const bool bad = __any_sync(0xFFFFFFFFu, n > 0 && (page < 0 || page >= a.d.n_pages));
            if (lane == 0) s_bad[group][s] = bad;      // the tile's partial is marked, and the second kernel drops the sequence
            __syncwarp();
            if (lane == 0) mbar_arrive_expect_tx(fb, 2u * pieces * S::kPiece);
            __syncwarp();
            if (n > 0 && !(dbg_held(a.withhold, kDbgPagedAttn) && blockIdx.x == 0 && group == 0 && it == 0 && lane == 0)) {
                if (bad) page = 0;
                const size_t at = q4_piece_of(a.d, page, p.sub / a.NC, row) * S::kPiece;
                bulk_load(smem_u32(ring) + s * S::kStage + (lane & 1) * S::kHalf + pc * S::kPiece, ((lane & 1) ? v_pool : k_pool) + at,
                          (uint32_t)n * S::kPiece, fb);
            }
            __syncwarp();
            if (lane == 0) s_filled[group] = it + 1;
            next_tile(a, p, subs);
        }
        if (lane == 0) s_filled[group] = 0x7FFFFFFF;
        if (blockIdx.x == 0 && group == 0 && a.d.n_seqs > kHeldSeqs) write_line(a);
        // all copies have landed before the shared memory goes away
        for (int back = 1; back <= S::kStages && back <= it; ++back) {
            const int j = it - back;
            mbar_wait_warp(smem_u32(&full_bar[group][j % S::kStages]), (uint32_t)(j / S::kStages) & 1u, abort_flag);
        }
    } else {
        const int mine = warp % kWarps * RP * kQ4Rows;
        Q4Join<DH, NG>& join = reinterpret_cast<Q4Join<DH, NG>*>(base + kGroups * S::kRing)[group];
        int stage = 0;
        uint32_t phase = 0;
        bool ok = true;
        Q4Unit<DH, NG, QP> u;
        while (p.left > 0) {                           // units
            const int hk = p.sub / a.NC, ch = p.sub - hk * a.NC, h0 = hk * a.G + ch * a.heads, nh = min(a.heads, a.G - ch * a.heads);
            const int len = a.kv_len[p.b], tiles = (int)min((long long)(p.nt - p.t), p.left);
            const int32_t* pos = a.positions ? a.positions + (size_t)p.b * a.d.S_cap() : nullptr;
            const float newest = kBent && a.slopes ? (float)(pos ? pos[len - 1] : len - 1) : 0.f;
            float* logits = kMass ? a.logits + (size_t)(t_hi - p.left) * a.heads * S::kTile + mine : nullptr;
            u.template start<T>(a, p.b, h0, nh);
            int first = p.t * S::kTile + mine, bad = 0;    // the warp's first row of the tile
            for (int n = 0; n < tiles; ++n) {
                // positions of the rows that this lane's logits are of: they are not wanted before the products are there
                int at[2 * RP] = {};
                if (kBent && a.slopes) {
#pragma unroll
                    for (int i = 0; i < 2 * RP; ++i) {
                        at[i] = min(first + row_at(lane >> 2) + 8 * i, len - 1);
                        if (pos) at[i] = pos[at[i]];
                    }
                }
                if (ok && !mbar_wait_warp(smem_u32(&full_bar[group][stage]), phase, abort_flag)) ok = false;
                if (ok) {
                    const uint8_t* k = ring + stage * S::kStage + warp % kWarps * RP * S::kPiece;
                    bad |= s_bad[group][stage];
                    if (first + kQ4Rows * RP <= len) q4_tile<DH, NG, QP, RP, kBent, kMass, false>(u, a, k, k + S::kHalf, 0, newest, at, logits, nh);
                    else if (first < len) q4_tile<DH, NG, QP, RP, kBent, kMass, true>(u, a, k, k + S::kHalf, len - first, newest, at, logits, nh);
                    __syncwarp();
                    if (lane == 0) mbar_arrive(smem_u32(&empty_bar[group][stage]));
                }
                if (++stage == S::kStages) {
                    stage = 0;
                    phase ^= 1u;
                }
                first += S::kTile;
                if (kMass) logits += a.heads * S::kTile;
            }
            const long long unit = (long long)p.b * subs + p.sub;
            p.t += tiles - 1;
            p.left -= tiles - 1;
            next_tile(a, p, subs);
            const size_t slot = (size_t)(unit + piece) * a.heads;
            unit_end(u, join, group, bad, nh, a.part_o + slot * DH, reinterpret_cast<float2*>(a.part_ml) + slot);
        }
    }
    __syncthreads();
    if (threadIdx.x == 0 && s_abort) *a.status = METOK_ERR_TIMEOUT;
}

constexpr int kRP = 2, kTileShift = 7;                 // (one piece a warp at a time: a sixth slower)
static_assert(Q4Shape<64, 1, kRP>::kTile == 1 << kTileShift, "rows of a tile");
// A unit has as many heads as are dealt to it, and so has its room in the workspace; the kernel works on eight or sixteen of them.
PagedPlan q4_plan(const PagedDims& d, int Hq) {
    const int G = Hq / d.Hkv, heads = ceil_div(G, ceil_div(G, 16));
    return paged_plan_of(d, Hq, heads, kTileShift, (heads <= 8 ? Q4Shape<64, 1, kRP>::kGroups : Q4Shape<64, 2, kRP>::kGroups) * kNumSMs);
}

template <typename T, int DH, int NG, bool kBent, bool kMass>
int launch_q4(const PagedAttnArgs& a, const void* k_pool, const void* v_pool, cudaStream_t st) {
    using S = Q4Shape<DH, NG, kRP>;
    auto kern = paged_attn_q4_kernel<T, DH, NG, kRP, kBent, kMass>;
    constexpr size_t smem = S::kGroups * (S::kRing + sizeof(Q4Join<DH, NG>)) + 128;
    static_assert(smem <= 226 * 1024, "shared memory of an SM");
    METOK_ALLOW_SMEM(kern, smem);
    {
        METOK_TIMED("paged_attn_q4", st);
        launch_chained(kern, dim3(std::min(a.grid, kNumSMs)), dim3(S::kThreads), smem, st, a, (const uint8_t*)k_pool, (const uint8_t*)v_pool);
    }
    METOK_LAUNCH_CHECK();
    // A unit's partials are few where the units are many: a CTA joins all of its heads (192 units 42.8 us the call, a head at a time 48.6; 80 18.2 and 19.4; 56
    // 15.3 and 15.0; 28 15.3 and 13.4; with weights units lose 1 to 26 us from 80 units on, but
    // outputs are to be the same as without).
    // Where the line is short, small CTAs (30 short sequences 8.3 us, of 256 threads 10.6; one of 300 rows 6.0 and 6.3).
    if (a.grid < kNumSMs) return launch_paged_join<T, DH, 128, false, true>(a, st);
    const bool few = (long long)a.d.n_seqs * a.d.Hkv * a.NC * 8 >= a.grid;
    return few ? launch_paged_join<T, DH, 256, true, true>(a, st, true) : launch_paged_join<T, DH, 256, false, true>(a, st, true);
}
template <typename T, int DH>
int launch_q4_dh(const PagedAttnArgs& a, const void* k, const void* v, cudaStream_t st) {
    const bool bent = a.cap_log2 > 0.f || a.slopes, mass = a.mass != nullptr;
    // (sixteen heads have no kernels of their own for calls without cap and bias: 66 us instead of 68 for 48 sequences of 36 / 4 heads, fp32 87 instead of 91)
    if (a.heads > 8) return mass ? launch_q4<T, DH, 2, true, true>(a, k, v, st) : launch_q4<T, DH, 2, true, false>(a, k, v, st);
    if (bent) return mass ? launch_q4<T, DH, 1, true, true>(a, k, v, st) : launch_q4<T, DH, 1, true, false>(a, k, v, st);
    return mass ? launch_q4<T, DH, 1, false, true>(a, k, v, st) : launch_q4<T, DH, 1, false, false>(a, k, v, st);
}
template <typename T>
int launch_q4_type(const PagedAttnArgs& a, const void* k, const void* v, cudaStream_t st) {
    return a.d.dh == 64 ? launch_q4_dh<T, 64>(a, k, v, st) : launch_q4_dh<T, 128>(a, k, v, st);
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
