// metok_rotate_heads: norms of the heads of Q and K and their rotary positions, one pass over both.
//
// A group of dh / 16 lanes has a head of a row, 16 elements a lane that hold both halves of eight pairs; a warp has 8 (dh 64) or 4
// (dh 128) heads at a time and goes over the heads of its row, so that the row's sines and cosines stay in registers.  Each lane works
// out one or two of the pairs' angles and the groups exchange them: t = position * inv_freq / 2 pi in 64 bits, of which the distance to
// the nearest integer is exact enough for any int32 position, and sincospi of that in 32.  Elements are worked on two at a time.
//
// What bounds it is reading and writing Q and K once: the next four turns' elements are on their way to a ring in shared memory, 96 KB (fp32:
// 192) for the 24 warps of an SM, that costs no registers (of two turns' in registers, for which there were 16 warps, 76 us).  18 496 rows of 28 + 4 heads of
// 128: 52 us, 5.8 TB/s, as a copy of as many bytes (56 in passes that go on for long); some 230 operations a turn of a warp, with pointers that are worked out for every turn 56 us.
#include <math.h>

#include "launchers.h"
#include "common.cuh"
#include "sm100.cuh"

namespace metok {

namespace {

constexpr int kWarps = 8, kMaxAxes = 4, kMaxPairs = 64;
constexpr int kDepth = 4;                              // turns whose elements are on their way
constexpr float kSmall = 1.2621774483536189e-29f;      // 2^-96: mean squares above it lose next to nothing below fp32's smallest numbers

struct RotateRows {
    const void* x;
    void* out;
    long long head, row, out_head, out_row;            // elements
    const float* weight;
    int H, passes;                                     // passes: turns of a warp over all heads
};
struct RotateArgs {
    RotateRows q, k;
    int n, split, rotary, interleaved, norm;           // split: warps of a row
    float eps;
    const float* inv_freq;
    const int32_t* positions;
    uint64_t axis[kMaxPairs / 32];                     // two bits per pair
};

template <typename T> struct Raw { uint4 v[sizeof(T)]; };              // 16 elements: two chunks of eight

// Elements 2 i, 2 i + 1 side by side.
template <typename T>
__device__ __forceinline__ void widen(const Raw<T>& r, uint64_t (&x)[8]) {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T); ++i) {
        const uint32_t w[4] = {r.v[i].x, r.v[i].y, r.v[i].z, r.v[i].w};
        if constexpr (sizeof(T) == 4) {
            x[2 * i] = sm100::pair(__uint_as_float(w[0]), __uint_as_float(w[1]));
            x[2 * i + 1] = sm100::pair(__uint_as_float(w[2]), __uint_as_float(w[3]));
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) x[4 * i + j] = sm100::pair(__uint_as_float(w[j] << 16), __uint_as_float(w[j] & 0xFFFF0000u));
        }
    }
}
template <typename T>
__device__ __forceinline__ Raw<T> narrow(const uint64_t (&x)[8]) {
    Raw<T> r;
    uint32_t w[4 * sizeof(T)];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        float lo, hi;
        sm100::unpair(x[i], lo, hi);
        if constexpr (sizeof(T) == 4) {
            w[2 * i] = __float_as_uint(lo);
            w[2 * i + 1] = __float_as_uint(hi);
        } else {
            asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w[i]) : "f"(hi), "f"(lo));
        }
    }
#pragma unroll
    for (int i = 0; i < (int)sizeof(T); ++i) r.v[i] = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
    return r;
}

__device__ __forceinline__ void copy16(uint32_t dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copies_close() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int kPending>
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(kPending) : "memory"); }

template <typename T, int DH>
__global__ void __launch_bounds__(kWarps * 32, 3)
rotate_kernel(const RotateArgs a) {
    using namespace sm100;
    constexpr int L = DH / 16, G = 32 / L, kMine = 8 / G;                // lanes of a head, heads at a time, angles of a lane
    constexpr int kHalf = sizeof(T) / 2;                                 // 16-byte pieces of a chunk
    extern __shared__ uint4 s_ring[];                  // [warp][turn][piece][lane]: each lane reads what it has copied
    const int lane = threadIdx.x & 31, s = lane % L, g = lane / L;
    const uint32_t item = blockIdx.x * kWarps + (threadIdx.x >> 5);
    const int row = (int)(item / (uint32_t)a.split), part = (int)(item - (uint32_t)row * a.split), passes = a.q.passes + a.k.passes;
    // the lane's two chunks of eight elements
    const int slots = a.rotary / 16;                   // lanes of a head whose elements turn
    const int c0 = a.interleaved || s >= slots ? 16 * s : 8 * s, c1 = a.interleaved || s >= slots ? 16 * s + 8 : a.rotary / 2 + 8 * s;
    // the row's turns: as many for every warp, one more for the first ones (products of turns and warps would pass 32 bits)
    const int each = (int)((uint32_t)passes / (uint32_t)a.split), over = passes - each * a.split;
    const int p0 = part * each + min(part, over), p1 = p0 + each + (part < over);
    grid_dep_wait();
    if (row >= a.n) return;                            // uniform in the warp
    // The warp's way over the heads, to be fetched and to be turned: a lane's head, in a turn, and its first element there.
    struct Way {
        int p, h;
        char* at;
    };
    auto set = [&](Way& w, bool out) {                 // at the first turn, and where K's begin
        const bool is_k = w.p >= a.q.passes;
        const RotateRows& o = is_k ? a.k : a.q;
        w.h = (is_k ? w.p - a.q.passes : w.p) * G + g;
        w.at = out ? reinterpret_cast<char*>(reinterpret_cast<T*>(o.out) + row * o.out_row + w.h * o.out_head)
                   : reinterpret_cast<char*>(const_cast<T*>(reinterpret_cast<const T*>(o.x) + row * o.row + w.h * o.head));
    };
    auto next = [&](Way& w, bool out) {
        if (++w.p == a.q.passes) {
            set(w, out);
            return;
        }
        const RotateRows& o = w.p >= a.q.passes ? a.k : a.q;
        w.h += G;
        w.at += (out ? o.out_head : o.head) * (long long)(G * sizeof(T));
    };
    const uint4* const mine = s_ring + (threadIdx.x >> 5) * (kDepth * (int)sizeof(T) * 32) + lane;
    const uint32_t mine_at = smem_u32(mine);
    Way in = {p0, 0, nullptr}, out = {p0, 0, nullptr};
    set(in, false);
    set(out, true);
    const int b0 = c0 * (int)sizeof(T), b1 = c1 * (int)sizeof(T);
    uint32_t slot = 0;                                 // of the next to be fetched, and of the one at hand
    auto fetch = [&]() {
        if (in.p < p1) {
            if (in.h < (in.p >= a.q.passes ? a.k.H : a.q.H)) {
                const uint32_t dst = mine_at + slot;
#pragma unroll
                for (int i = 0; i < kHalf; ++i) {
                    copy16(dst + i * 512, in.at + b0 + i * 16);
                    copy16(dst + (kHalf + i) * 512, in.at + b1 + i * 16);
                }
            }
            next(in, false);
        }
        copies_close();
        slot = slot + (uint32_t)sizeof(T) * 512 == kDepth * (uint32_t)sizeof(T) * 512 ? 0 : slot + (uint32_t)sizeof(T) * 512;
    };
    for (int u = 0; u < kDepth; ++u) fetch();

    // sines and cosines of pairs 8 s .. 8 s + 7, side by side
    uint64_t cs[4], sn[4];
    if (slots > 0) {
        float mc[kMine], ms[kMine];
#pragma unroll
        for (int u = 0; u < kMine; ++u) {
            const int at = 8 * s + g * kMine + u;
            float x = 0.f;
            if (s < slots) {
                const int axis = (int)(a.axis[at >> 5] >> (2 * (at & 31))) & 3;
                const int pos = a.positions ? a.positions[(long long)axis * a.n + row] : row;
                const double t = (double)pos * ((double)a.inv_freq[at] * 0.15915494309189533577);     // turns
                x = (float)(2.0 * (t - rint(t)));
            }
            sincospif(x, &ms[u], &mc[u]);
        }
        float c[8], d[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            c[j] = __shfl_sync(0xFFFFFFFFu, mc[j % kMine], (j / kMine) * L + s);
            d[j] = __shfl_sync(0xFFFFFFFFu, ms[j % kMine], (j / kMine) * L + s);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            cs[j] = pair(c[2 * j], c[2 * j + 1]);
            sn[j] = pair(d[2 * j], d[2 * j + 1]);
        }
    }

    uint64_t w[8];
    auto weights = [&](const float* src) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int at = i < 4 ? c0 + 2 * i : c1 + 2 * (i - 4);
            w[i] = src ? pair(src[at], src[at + 1]) : pair(1.f, 1.f);
        }
    };
    for (; out.p < p1; next(out, true)) {
        const bool is_k = out.p >= a.q.passes;
        uint64_t x[8];
        copies_wait<kDepth - 1>();
        {
            Raw<T> raw;
            const uint4* from = mine + slot / 16;
#pragma unroll
            for (int i = 0; i < (int)sizeof(T); ++i) raw.v[i] = from[i * 32];
            widen<T>(raw, x);
        }
        fetch();
        if (a.norm) {
            if (out.p == p0 || out.p == a.q.passes) weights(is_k ? a.k.weight : a.q.weight);
            const auto squares = [&](uint32_t lanes) {
                uint64_t sum = mul_pair(x[0], x[0]);
#pragma unroll
                for (int i = 1; i < 8; ++i) sum = fma_pair(x[i], x[i], sum);
                float ss, odd;
                unpair(sum, ss, odd);
                ss += odd;
#pragma unroll
                for (int m = 1; m < L; m <<= 1) ss += __shfl_xor_sync(lanes, ss, m);
                return ss;
            };
            float mean = fmaf(squares(0xFFFFFFFFu), 1.f / DH, a.eps);
            if (mean < kSmall) {                       // few heads: squares that fp32 does not hold.  The same for all lanes of a head
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = mul_pair(x[i], pair(1.f / kSmall, 1.f / kSmall));
                mean = fmaf(squares(((1u << L) - 1u) << (lane & -L)), 1.f / DH, a.eps * (1.f / kSmall) * (1.f / kSmall));
            }
            const float f = rsqrtf(mean);
            const uint64_t f2 = pair(f, f);
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = mul_pair(x[i], mul_pair(f2, w[i]));
        }
        if (s < slots) {
            if (a.interleaved) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    float u, v, c, d;
                    unpair(x[j], u, v);
                    if (j & 1) {
                        float skip;
                        unpair(cs[j / 2], skip, c);
                        unpair(sn[j / 2], skip, d);
                    } else {
                        float skip;
                        unpair(cs[j / 2], c, skip);
                        unpair(sn[j / 2], d, skip);
                    }
                    x[j] = pair(fmaf(u, c, -v * d), fmaf(v, c, u * d));
                }
            } else {
                const uint64_t minus = pair(-1.f, -1.f);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint64_t u = x[j], v = x[4 + j];
                    x[j] = fma_pair(u, cs[j], mul_pair(mul_pair(v, minus), sn[j]));
                    x[4 + j] = fma_pair(v, cs[j], mul_pair(u, sn[j]));
                }
            }
        }
        if (out.h < (is_k ? a.k.H : a.q.H)) {
            const Raw<T> r = narrow<T>(x);
#pragma unroll
            for (int i = 0; i < kHalf; ++i) {
                *reinterpret_cast<uint4*>(out.at + b0 + i * 16) = r.v[i];
                *reinterpret_cast<uint4*>(out.at + b1 + i * 16) = r.v[kHalf + i];
            }
        }
    }
    copies_wait<0>();
}

template <typename T>
int launch_rotate(int dh, const RotateArgs& a, unsigned blocks, cudaStream_t st) {
    constexpr size_t smem = (size_t)kWarps * kDepth * sizeof(T) * 512;
    if (dh == 64) {
        METOK_ALLOW_SMEM((rotate_kernel<T, 64>), smem);
        METOK_TIMED("rotate_heads", st);
        launch_chained(rotate_kernel<T, 64>, dim3(blocks), dim3(kWarps * 32), smem, st, a);
    } else {
        METOK_ALLOW_SMEM((rotate_kernel<T, 128>), smem);
        METOK_TIMED("rotate_heads", st);
        launch_chained(rotate_kernel<T, 128>, dim3(blocks), dim3(kWarps * 32), smem, st, a);
    }
    METOK_LAUNCH_CHECK();
    return METOK_OK;
}

}  // namespace
}  // namespace metok

using namespace metok;

extern "C" int metok_rotate_heads(int dtype, const metok_rotate_params* p, void* stream) {
    if (!p || (dtype != METOK_F32 && dtype != METOK_BF16)) return METOK_ERR_INVALID_ARG;
    if (p->n < 0 || p->Hq < 1 || p->Hkv < 0 || p->dh < 1) return METOK_ERR_INVALID_ARG;
    if (p->dh != 64 && p->dh != 128) return METOK_ERR_UNSUPPORTED;
    if (p->rotary_dim < 0 || p->rotary_dim > p->dh || p->rotary_dim % 16 || p->n_axes < 1 || p->n_axes > kMaxAxes) return METOK_ERR_INVALID_ARG;
    if (!(p->eps >= 0.f) || p->eps > 3.0e38f) return METOK_ERR_INVALID_ARG;
    if (p->rotary_dim > 0 && (!p->inv_freq || (!p->positions && p->n_axes > 1 && p->n > 0))) return METOK_ERR_INVALID_ARG;
    if (!aligned4(p->inv_freq) || !aligned4(p->positions) || !aligned4(p->q_weight) || !aligned4(p->k_weight)) return METOK_ERR_INVALID_ARG;
    const int esize = dtype == METOK_F32 ? 4 : 2, per = 16 / esize;
    RotateArgs a = {};
    Extent in[2], out[2];
    const int sides = p->Hkv > 0 ? 2 : 1;
    for (int i = 0; i < sides; ++i) {
        const void* x = i ? p->k : p->q;
        void* o = i ? p->k_out : p->q_out;
        const int64_t head = i ? p->k_head : p->q_head, row = i ? p->k_row : p->q_row, ohead = i ? p->ko_head : p->qo_head,
                      orow = i ? p->ko_row : p->qo_row;
        const int H = i ? p->Hkv : p->Hq;
        if ((p->n > 0 && (!x || !o)) || !aligned16(x) || !aligned16(o)) return METOK_ERR_INVALID_ARG;
        if (head < 0 || row < 0 || ohead < 0 || orow < 0 || (head | row | ohead | orow) % per) return METOK_ERR_INVALID_ARG;
        if ((H > 1 && head < p->dh) || (p->n > 1 && row < p->dh) || !rows_apart(H, ohead, p->n, orow, p->dh)) return METOK_ERR_INVALID_ARG;
        in[i] = extent_of(x, H, head, p->n, row, p->dh, esize);
        out[i] = extent_of(o, H, ohead, p->n, orow, p->dh, esize);
        RotateRows& r = i ? a.k : a.q;
        r = {x, o, head, row, ohead, orow, i ? p->k_weight : p->q_weight, H, ceil_div(H, 32 / (p->dh / 16))};
    }
    a.axis[0] = a.axis[1] = 0;
    if (p->pair_axis)
        for (int i = 0; i < p->rotary_dim / 2; ++i) {
            const int axis = p->pair_axis[i];
            if (axis < 0 || axis >= p->n_axes) return METOK_ERR_INVALID_ARG;
            a.axis[i >> 5] |= (uint64_t)axis << (2 * (i & 31));
        }
    if (p->n == 0) return METOK_OK;
    for (int i = 0; i < sides; ++i) {
        const bool same = in[i].at == out[i].at && in[i].head == out[i].head && in[i].row == out[i].row;
        for (int j = 0; j < sides; ++j)
            if (!(j == i && same) && !apart(out[i], in[j])) return METOK_ERR_INVALID_ARG;
    }
    if (sides == 2 && !apart(out[0], out[1])) return METOK_ERR_INVALID_ARG;
    a.n = p->n; a.rotary = p->rotary_dim; a.interleaved = p->interleaved != 0; a.norm = p->norm != 0;
    a.eps = p->eps; a.inv_freq = p->inv_freq; a.positions = p->positions;
    // few rows: a row's heads are dealt to 32 warps for every SM, which holds 24 (with 24: 600 rows of 28 + 4 heads 5.5 us instead of 5.3, 2000 of 14 + 2
    // 5.5 instead of 5.1, 1000 of 28 + 4 6.3 instead of 6.5; others alike)
    const int passes = a.q.passes + a.k.passes;
    a.split = std::max(1, std::min(passes, (int)std::min<long long>(passes, (32LL * kNumSMs + p->n - 1) / p->n)));
    const long long blocks = ((long long)p->n * a.split + kWarps - 1) / kWarps;
    if (blocks > 0x7FFFFFFFLL / kWarps) return METOK_ERR_UNSUPPORTED;
    cudaStream_t st = (cudaStream_t)stream;
    return dtype == METOK_F32 ? launch_rotate<float>(p->dh, a, (unsigned)blocks, st) : launch_rotate<__nv_bfloat16>(p->dh, a, (unsigned)blocks, st);
}
