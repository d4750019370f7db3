// metok_rotate_heads: norms of the heads of Q and K and their rotary positions, one pass over both.
//
// A group of dh / 16 lanes has a head of a row, 16 elements a lane that hold both halves of eight pairs; a warp has 8 (dh 64) or 4
// (dh 128) heads at a time and goes over the heads of its row, so that the row's sines and cosines stay in registers.  Each lane works
// out one or two of a pair's angles and the groups exchange them: t = position * inv_freq / 2 pi in 64 bits, of which the distance to
// the nearest integer is exact enough for any int32 position, and sincospif of that in 32.  The sum of squares is the lanes' 16, added by
// shuffles.  The next heads' elements are on their way while these are turned.
//
// What bounds it is reading and writing Q and K once.
#include <math.h>

#include "launchers.h"
#include "paged.cuh"

namespace metok {

namespace {

constexpr int kWarps = 8, kMaxAxes = 4, kMaxPairs = 64;

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

template <typename T>
__device__ __forceinline__ void widen(const Raw<T>& r, float (&x)[16]) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[4 * i] = __uint_as_float(r.v[i].x); x[4 * i + 1] = __uint_as_float(r.v[i].y);
            x[4 * i + 2] = __uint_as_float(r.v[i].z); x[4 * i + 3] = __uint_as_float(r.v[i].w);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint32_t w[4] = {r.v[i].x, r.v[i].y, r.v[i].z, r.v[i].w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                x[8 * i + 2 * j] = __uint_as_float(w[j] << 16);
                x[8 * i + 2 * j + 1] = __uint_as_float(w[j] & 0xFFFF0000u);
            }
        }
    }
}
__device__ __forceinline__ uint32_t two_bf16(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
template <typename T>
__device__ __forceinline__ Raw<T> narrow(const float (&x)[16]) {
    Raw<T> r;
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            r.v[i] = make_uint4(__float_as_uint(x[4 * i]), __float_as_uint(x[4 * i + 1]), __float_as_uint(x[4 * i + 2]), __float_as_uint(x[4 * i + 3]));
    } else {
#pragma unroll
        for (int i = 0; i < 2; ++i)
            r.v[i] = make_uint4(two_bf16(x[8 * i], x[8 * i + 1]), two_bf16(x[8 * i + 2], x[8 * i + 3]), two_bf16(x[8 * i + 4], x[8 * i + 5]),
                                two_bf16(x[8 * i + 6], x[8 * i + 7]));
    }
    return r;
}

template <typename T, int DH>
__global__ void __launch_bounds__(kWarps * 32)
rotate_kernel(const RotateArgs a) {
    constexpr int L = DH / 16, G = 32 / L, kMine = 8 / G;                // lanes of a head, heads at a time, angles of a lane
    constexpr int kHalf = sizeof(T) / 2;                                 // 16-byte pieces of a chunk
    const int lane = threadIdx.x & 31, s = lane % L, g = lane / L;
    const long long item = (long long)blockIdx.x * kWarps + (threadIdx.x >> 5);
    const long long row = item / a.split;
    const int part = (int)(item - row * a.split), passes = a.q.passes + a.k.passes;
    grid_dep_wait();
    if (row >= a.n) return;                            // uniform in the warp
    const int p0 = passes * part / a.split, p1 = passes * (part + 1) / a.split;
    // the lane's two chunks of eight elements
    const int slots = a.rotary / 16;                   // lanes of a head whose elements turn
    const int c0 = a.interleaved || s >= slots ? 16 * s : 8 * s, c1 = a.interleaved || s >= slots ? 16 * s + 8 : a.rotary / 2 + 8 * s;

    auto fetch = [&](int p, Raw<T>& r) {
        const RotateRows& x = p < a.q.passes ? a.q : a.k;
        const int h = (p < a.q.passes ? p : p - a.q.passes) * G + g;
        if (p >= p1 || h >= x.H) return;
        const T* src = reinterpret_cast<const T*>(x.x) + h * x.head + row * x.row;
#pragma unroll
        for (int i = 0; i < kHalf; ++i) {
            r.v[i] = reinterpret_cast<const uint4*>(src + c0)[i];
            r.v[kHalf + i] = reinterpret_cast<const uint4*>(src + c1)[i];
        }
    };
    Raw<T> next = {};
    fetch(p0, next);

    // sines and cosines of pairs 8 s .. 8 s + 7
    float cs[8], sn[8];
    if (slots > 0) {
        float mc[kMine], ms[kMine];
#pragma unroll
        for (int u = 0; u < kMine; ++u) {
            const int pair = 8 * s + g * kMine + u;
            float x = 0.f;
            if (s < slots) {
                const int axis = (int)(a.axis[pair >> 5] >> (2 * (pair & 31))) & 3;
                const int pos = a.positions ? a.positions[(long long)axis * a.n + row] : (int)row;
                const double t = (double)pos * ((double)a.inv_freq[pair] * 0.15915494309189533577);   // turns
                x = (float)(2.0 * (t - rint(t)));
            }
            sincospif(x, &ms[u], &mc[u]);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            cs[j] = __shfl_sync(0xFFFFFFFFu, mc[j % kMine], (j / kMine) * L + s);
            sn[j] = __shfl_sync(0xFFFFFFFFu, ms[j % kMine], (j / kMine) * L + s);
        }
    }

    float w[16];
    bool weights_of_k = false;
    auto weights = [&](const float* src) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float* at = src + (i < 2 ? c0 + 4 * i : c1 + 4 * (i - 2));
#pragma unroll
            for (int j = 0; j < 4; ++j) w[4 * i + j] = src ? at[j] : 1.f;
        }
    };
    for (int p = p0; p < p1; ++p) {
        const bool is_k = p >= a.q.passes;
        const RotateRows& o = is_k ? a.k : a.q;
        const int h = (is_k ? p - a.q.passes : p) * G + g;
        float x[16];
        widen<T>(next, x);
        fetch(p + 1, next);
        if (a.norm) {
            if (p == p0 || is_k != weights_of_k) {
                weights(o.weight);
                weights_of_k = is_k;
            }
            float ss = 0.f;
#pragma unroll
            for (int i = 0; i < 16; ++i) ss = fmaf(x[i], x[i], ss);
#pragma unroll
            for (int m = 1; m < L; m <<= 1) ss += __shfl_xor_sync(0xFFFFFFFFu, ss, m);
            const float f = 1.f / sqrtf(ss * (1.f / DH) + a.eps);
#pragma unroll
            for (int i = 0; i < 16; ++i) x[i] *= f * w[i];
        }
        if (s < slots) {
            if (a.interleaved) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float u = x[2 * j], v = x[2 * j + 1];
                    x[2 * j] = fmaf(u, cs[j], -v * sn[j]);
                    x[2 * j + 1] = fmaf(v, cs[j], u * sn[j]);
                }
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float u = x[j], v = x[8 + j];
                    x[j] = fmaf(u, cs[j], -v * sn[j]);
                    x[8 + j] = fmaf(v, cs[j], u * sn[j]);
                }
            }
        }
        if (h < o.H) {
            const Raw<T> r = narrow<T>(x);
            T* dst = reinterpret_cast<T*>(o.out) + h * o.out_head + row * o.out_row;
#pragma unroll
            for (int i = 0; i < kHalf; ++i) {
                reinterpret_cast<uint4*>(dst + c0)[i] = r.v[i];
                reinterpret_cast<uint4*>(dst + c1)[i] = r.v[kHalf + i];
            }
        }
    }
}

template <typename T>
void launch_rotate(int dh, const RotateArgs& a, unsigned blocks, cudaStream_t st) {
    METOK_TIMED("rotate_heads", st);
    if (dh == 64) launch_chained(rotate_kernel<T, 64>, dim3(blocks), dim3(kWarps * 32), 0, st, a);
    else launch_chained(rotate_kernel<T, 128>, dim3(blocks), dim3(kWarps * 32), 0, st, a);
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
    if (p->rotary_dim > 0 && (!p->inv_freq || (!p->positions && p->n_axes > 1))) return METOK_ERR_INVALID_ARG;
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
    // few rows: a row's heads are dealt to as many warps as keep 32 of them on every SM
    const int passes = a.q.passes + a.k.passes;
    a.split = std::max(1, std::min(passes, (int)std::min<long long>(passes, (32LL * kNumSMs + p->n - 1) / p->n)));
    const long long blocks = ((long long)p->n * a.split + kWarps - 1) / kWarps;
    if (blocks > 0x7FFFFFFFLL) return METOK_ERR_UNSUPPORTED;
    cudaStream_t st = (cudaStream_t)stream;
    if (dtype == METOK_F32) launch_rotate<float>(p->dh, a, (unsigned)blocks, st);
    else launch_rotate<__nv_bfloat16>(p->dh, a, (unsigned)blocks, st);
    METOK_LAUNCH_CHECK();
    return METOK_OK;
}
