// metok_prefill_attention on the tensor cores (bf16).
//
// A CTA works on two tiles of 128 query rows of one K/V head: the tiles of a document's query heads of the group are dealt
// out in pairs (tile by tile, head by head), so that both use the same K and V tiles, and for few rows the heads of a group
// share a read of the keys.  Per tile of 128 keys and query tile x:
//   S_x = Q_x K^T        tcgen05.mma, both operands in shared memory, fp32 in tensor memory (128 columns)
//   P_x = 2^(logit - m)  one thread per row; bf16, written over S_x in tensor memory (64 columns)
//   O_x += P_x V         tcgen05.mma, P_x from tensor memory, V as it lies (keys x dh: the second operand's other order)
// S_0, S_1, O_0 and O_1 fill the 512 columns.  While one tile's rows are in their exponentials the other's products run.
//
// Key tiles are taken from the last one down.  A row's reference m is the maximum of the first tile that it sees; later tiles' weights are taken against it with no maximum of their own,
// since any m within the range of the exponent gives the same result.  Where the sum of 64 weights leaves that range they are
// made again against their own maximum, and O_x and the sum are scaled: by the row's own thread, when the products
// before on O_x are complete (one thread issues all of them, in order).
//
// Warps 0-3 and 4-7: the rows of tiles 0 and 1; warp 8: TMA; warp 9: products.  Every wait is bounded.  A row's 128 logits are read
// from tensor memory 32 at a time: held in registers they spill.
#include <algorithm>

#include "launchers.h"
#include "prefill_attn.cuh"
#include "sm100.cuh"

namespace metok {

namespace {

constexpr int kM = 128, kN = 128, kThreads = 320;
constexpr float kMost = 1.0e18f, kRoom = 32.f;         // sum of 64 weights beyond which a row's reference grows, and by how many octaves above their maximum

template <int DH>
struct MmaShape {
    static constexpr int KB = DH / 64;                 // 128-byte pieces of a row
    static constexpr uint32_t kBlk = 128 * 128;        // bytes of a piece of a tile's 128 rows
    static constexpr uint32_t kTile = KB * kBlk;
    static constexpr int kStages = DH == 128 ? 4 : 8;  // K and V tiles on their way
    static constexpr size_t kSmem = (size_t)(2 + kStages) * kTile + 1024;
};

// 32 registers of this thread's lane to 32 tensor-memory columns.
__device__ __forceinline__ void tmem_st32(uint32_t taddr, const uint32_t (&r)[32]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31};"
        ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
          "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]),
          "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]),
          "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31]),
          "r"(taddr)
        : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// D[tmem] (+)= A[tmem] * B[smem], issued by ONE thread.
__device__ __forceinline__ void umma_bf16_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
        ::"r"(d_tmem), "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate)
        : "memory");
}
// Descriptor of V as the second operand in its other order: a tile lies as rows (keys) of 128 swizzled bytes = 64 columns of
// the product; the next 64 columns follow kBlk bytes on (leading offset), the next eight keys 1024 bytes on (stride).
__device__ __forceinline__ uint64_t desc_v(uint32_t smem_addr, uint32_t blk_bytes) {
    uint64_t d = 0;
    d |= (uint64_t)((smem_addr & 0x3FFFFu) >> 4);
    d |= (uint64_t)(blk_bytes >> 4) << 16;
    d |= (uint64_t)(1024 >> 4) << 32;
    d |= (uint64_t)1 << 46;
    d |= (uint64_t)2 << 61;
    return d;
}
__device__ __forceinline__ void tma_load_3d(uint32_t dst_smem, const CUtensorMap* m, int x, int y, int z, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
        ::"r"(dst_smem), "l"(reinterpret_cast<uint64_t>(m)), "r"(bar), "r"(x), "r"(y), "r"(z)
        : "memory");
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

struct MmaMaps {
    CUtensorMap q, k, v;
    int q_step, k_step, v_step;                        // 1, or 0 where all heads are the same rows
};

template <int DH, bool kCap, bool kBias>
__global__ void __launch_bounds__(kThreads, 1)
prompt_attn_mma_kernel(const PromptArgs a, const __grid_constant__ MmaMaps maps) {
    using namespace sm100;
    using S = MmaShape<DH>;
    grid_dep_wait();
    extern __shared__ uint8_t smem_dyn[];
    __shared__ __align__(8) uint64_t q_bar, full_bar[S::kStages], empty_bar[S::kStages], s_bar[2], p_bar[2][2], h_bar[2], o_bar[2], drain_bar;
    __shared__ uint32_t s_tmem_base;
    __shared__ int s_abort;
    __shared__ __align__(16) float s_pos[2][2][kN];    // [tile][buffer]: positions of the keys
    const int warp = __shfl_sync(0xFFFFFFFFu, (int)threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    const int g = blockIdx.x % a.Hkv;
    const int G = a.G;
    const PromptDoc d = prompt_tile(a, blockIdx.x / a.Hkv, [G](int Lq) { return (int)(((long long)((Lq + kM - 1) / kM) * G + 1) / 2); });
    if (d.tile < 0) return;                            // uniform

    // the pair's items: 2 t and 2 t + 1 of the document's (tile, head) pairs
    const int n_items = (d.Lq + kM - 1) / kM * G;
    int i0[2], head[2], rows[2], lo = 0, n[2] = {0, 0};   // first row, query head, rows, key tiles of each item
    int hi = 0;
#pragma unroll
    for (int x = 0; x < 2; ++x) {
        const int item = 2 * d.tile + x;
        const bool there = item < n_items;
        const int t = there ? item / G : 0;
        i0[x] = t * kM;
        head[x] = g * G + (there ? item - t * G : 0);
        rows[x] = there ? min(kM, d.Lq - i0[x]) : 0;
        n[x] = there ? (prompt_keys(a, d, i0[x] + rows[x] - 1) + kN - 1) / kN : 0;
        hi = max(hi, n[x]);
    }
    if (a.splits > 1) {
        const int all = hi;
        lo = (int)((long long)all * blockIdx.y / a.splits);
        hi = (int)((long long)all * (blockIdx.y + 1) / a.splits);
    }
#pragma unroll
    for (int x = 0; x < 2; ++x) n[x] = max(0, min(n[x], hi) - lo);
    // key tiles lo + nt - 1 down to lo: the nearest ones first, which a bias makes the largest; item x joins in at step st[x]
    const int nt = max(n[0], n[1]), st[2] = {nt - n[0], nt - n[1]};
    auto tile_key = [&](int j) { return (lo + nt - 1 - j) * kN; };

    const uint32_t smem_base = (smem_u32(smem_dyn) + 1023u) & ~1023u;
    auto q_addr = [&](int x) { return smem_base + (uint32_t)x * S::kTile; };
    auto kv_addr = [&](int s) { return smem_base + (uint32_t)(2 + s) * S::kTile; };
    if (threadIdx.x == 0) {
        mbar_init(smem_u32(&q_bar), 1);
        mbar_init(smem_u32(&drain_bar), 1);
        for (int s = 0; s < S::kStages; ++s) { mbar_init(smem_u32(&full_bar[s]), 1); mbar_init(smem_u32(&empty_bar[s]), 1); }
        for (int x = 0; x < 2; ++x) { mbar_init(smem_u32(&s_bar[x]), 1); mbar_init(smem_u32(&o_bar[x]), 1); mbar_init(smem_u32(&h_bar[x]), 1); for (int p = 0; p < 2; ++p) mbar_init(smem_u32(&p_bar[x][p]), 4); }
        s_abort = 0;
        mbar_fence_init();
    }
    if (warp == 9) {
        tmem_alloc(smem_u32(&s_tmem_base), 512);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = __shfl_sync(0xFFFFFFFFu, s_tmem_base, 0);
    volatile int* abort_flag = &s_abort;

    if (warp == 8) {
        // ---- TMA: Q of both items, then K and V tiles in turn
        int it = 0;
        if (nt > 0) {
            if (elect_one()) {
                prefetch_tmap(&maps.k);
                prefetch_tmap(&maps.v);
                const int both = rows[1] > 0 ? 2 : 1;
                mbar_arrive_expect_tx(smem_u32(&q_bar), (uint32_t)both * S::kTile);
#pragma unroll
                for (int x = 0; x < 2; ++x)
                    if (x < both) {
#pragma unroll
                        for (int kb = 0; kb < S::KB; ++kb)
                            tma_load_3d(q_addr(x) + kb * S::kBlk, &maps.q, kb * 64, d.q0 + i0[x], head[x] * maps.q_step, smem_u32(&q_bar));
                    }
            }
            __syncwarp();
            for (; it < 2 * nt; ++it) {
                const int s = it % S::kStages, row = d.k0 + tile_key(it >> 1);
                if (!mbar_wait_warp(smem_u32(&empty_bar[s]), ((uint32_t)(it / S::kStages) & 1u) ^ 1u, abort_flag)) break;
                if (elect_one()) {
                    const uint32_t fb = smem_u32(&full_bar[s]);
                    mbar_arrive_expect_tx(fb, S::kTile);
#pragma unroll
                    for (int kb = 0; kb < S::KB; ++kb) {
                        if (it & 1) tma_load_3d(kv_addr(s) + kb * S::kBlk, &maps.v, kb * 64, row, g * maps.v_step, fb);
                        else tma_load_3d(kv_addr(s) + kb * S::kBlk, &maps.k, kb * 64, row, g * maps.k_step, fb);
                    }
                }
                __syncwarp();
            }
            // every copy has landed before the shared memory goes away
            mbar_wait_warp(smem_u32(&q_bar), 0u, abort_flag);
            for (int back = 1; back <= S::kStages && back <= it; ++back) {
                const int j = it - back;
                mbar_wait_warp(smem_u32(&full_bar[j % S::kStages]), (uint32_t)(j / S::kStages) & 1u, abort_flag);
            }
        }
    } else if (warp == 9) {
        // ---- products
        constexpr uint32_t idesc_s = make_idesc_bf16(kM, kN), idesc_o = make_idesc_bf16(kM, DH) | (1u << 16);
        bool ok = nt == 0 || mbar_wait_warp(smem_u32(&q_bar), 0u, abort_flag);
        auto wait_full = [&](int it) { return mbar_wait_warp(smem_u32(&full_bar[it % S::kStages]), (uint32_t)(it / S::kStages) & 1u, abort_flag); };
        auto logits = [&](int x, int j) {              // S_x of key tile j
            const uint32_t kb = kv_addr((2 * j) % S::kStages), qb = q_addr(x), dst = tmem + (uint32_t)x * kN;
            if (elect_one()) {
#pragma unroll
                for (int kk = 0; kk < DH / 16; ++kk)
                    umma_bf16(dst, make_desc_k128(qb + (kk >> 2) * S::kBlk + (kk & 3) * 32), make_desc_k128(kb + (kk >> 2) * S::kBlk + (kk & 3) * 32),
                              idesc_s, kk != 0 ? 1u : 0u);
                umma_commit(smem_u32(&s_bar[x]));
            }
            __syncwarp();
        };
        auto values = [&](int x, int j, int half) {    // O_x += P_x V of 64 keys of tile j
            const int vs = (2 * j + 1) % S::kStages, jx = j - st[x];
            if (!mbar_wait_warp(smem_u32(&p_bar[x][half]), (uint32_t)jx & 1u, abort_flag)) return false;
            tc_fence_after();
            if (elect_one()) {
#pragma unroll
                for (int kk = 0; kk < 4; ++kk)
                    umma_bf16_ts(tmem + 2 * kN + (uint32_t)x * DH, tmem + (uint32_t)x * kN + half * 32 + kk * 8, desc_v(kv_addr(vs) + (half * 4 + kk) * 2048, S::kBlk), idesc_o,
                                 jx > 0 || half || kk > 0 ? 1u : 0u);
                if (!half) umma_commit(smem_u32(&h_bar[x]));
                else if (j + 1 == nt) umma_commit(smem_u32(&o_bar[x]));
            }
            __syncwarp();
            return true;
        };
        auto release = [&](int it) {
            if (elect_one()) umma_commit(smem_u32(&empty_bar[it % S::kStages]));
            __syncwarp();
        };
        // One item's second half and next logits lie between the other's halves, so that the products go on while either's weights
        // are made: per step  O_0 first half | O_1 second half of the step before, S_1 | O_0 second half, next S_0 | O_1 first half.
        if (ok && nt > 0 && (ok = wait_full(0))) {
            tc_fence_after();
            for (int x = 0; x < 2; ++x)
                if (st[x] == 0) logits(x, 0);
        }
        for (int j = 0; ok && j < nt; ++j) {
            const int vi = 2 * j + 1, vs = vi % S::kStages;
            if (!(ok = wait_full(vi))) break;
            const int left = d.Lk - tile_key(j);       // rows of the document in this tile
            if (left < kN) {                           // those behind count as zeros, whatever they hold
                for (int c = lane; c < (kN - left) * S::KB * 8; c += 32) {
                    const int r = left + c / (S::KB * 8), e = c % (S::KB * 8);
                    asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(kv_addr(vs) + (uint32_t)(e >> 3) * S::kBlk + (uint32_t)r * 128u + (uint32_t)(e & 7) * 16u), "r"(0) : "memory");
                }
                fence_proxy_async();
                __syncwarp();
            }
            if (j >= st[0] && !(ok = values(0, j, 0))) break;
            if (j > 0) {
                if (j > st[1] && !(ok = values(1, j - 1, 1))) break;
                if (j >= st[1]) logits(1, j);
                release(vi - 2);
            }
            release(2 * j);                            // (S_1's, or S_0's in the first step)
            if (j >= st[0] && !(ok = values(0, j, 1))) break;
            if (j + 1 < nt) {
                if (!(ok = wait_full(2 * j + 2))) break;
                if (j + 1 >= st[0]) logits(0, j + 1);
            }
            if (j >= st[1] && !(ok = values(1, j, 0))) break;
        }
        if (ok && n[1] > 0) ok = values(1, nt - 1, 1);
        if (!ok) {                                     // whatever was issued has retired before the tensor memory goes
            if (elect_one()) umma_commit(smem_u32(&drain_bar));
            __syncwarp();
            mbar_wait_warp(smem_u32(&drain_bar), 0u, abort_flag);
        }
    } else {
        // ---- rows
        const int x = warp >> 2, quad = warp & 3, r = quad * 32 + lane;
        const int my_n = x ? n[1] : n[0], my_rows = x ? rows[1] : rows[0], my_i0 = x ? i0[1] : i0[0], my_head = x ? head[1] : head[0];
        const uint32_t lane_base = (uint32_t)(quad * 32) << 16;
        const uint32_t t_s = tmem + lane_base + (uint32_t)x * kN, t_o = tmem + lane_base + 2 * kN + (uint32_t)x * DH;
        const float ninf = __int_as_float(0xFF800000);
        const int keys = r < my_rows ? prompt_keys(a, d, my_i0 + r) : 0;
        const int sure = my_rows > 0 ? prompt_keys(a, d, my_i0) : 0;    // keys that all rows of the tile see
        float m = ninf, l = 0.f;
        bool ok = true;
        float slope = 0.f, my_pos = 0.f, next_pos = 0.f;
        if (kBias && my_n > 0) {
            slope = a.slopes[my_head] * kAttnLog2e;
            my_pos = prompt_position(a, d, d.Lk - d.Lq + my_i0 + r);
            next_pos = prompt_position(a, d, (lo + my_n - 1) * kN + r);
        }
        for (int j = 0; j < my_n; ++j) {
            const int k0 = (lo + my_n - 1 - j) * kN;
            if constexpr (kBias) {                     // (two buffers: who writes one again has met the others since it was read)
                s_pos[x][j & 1][r] = next_pos;
                next_pos = prompt_position(a, d, k0 - kN + r);
                named_bar_sync(1 + x, 128);
            }
            if (ok && !mbar_wait(smem_u32(&s_bar[x]), (uint32_t)j & 1u, abort_flag)) ok = false;
            ok = __all_sync(0xFFFFFFFFu, ok);
            if (!ok) {
                if constexpr (kBias) continue;         // keeps meeting the tile's other warps
                break;
            }
            tc_fence_after();
            const bool masked = k0 + kN > sure;
            // Logits of columns 32 c .. in log2 units less `base`; those of keys that the row does not see are -infinity.
            auto logit = [&](const uint32_t (&raw)[32], int c, float base, float (&v)[32]) {
                if constexpr (kCap) {
#pragma unroll
                    for (int i = 0; i < 32; ++i)
                        v[i] = (a.cap_log2 - base) - __fdividef(2.f * a.cap_log2, 1.f + fast_exp2(fminf(__uint_as_float(raw[i]) * (2.f * kAttnLog2e * a.cap_scale), 80.f)));
                } else {
#pragma unroll
                    for (int i = 0; i < 32; i += 2)
                        unpair(fma_pair(pair(__uint_as_float(raw[i]), __uint_as_float(raw[i + 1])), pair(a.scale_log2, a.scale_log2), pair(-base, -base)), v[i], v[i + 1]);
                }
                if constexpr (kBias) {
#pragma unroll
                    for (int i = 0; i < 32; i += 4) {
                        const float4 p = *reinterpret_cast<const float4*>(&s_pos[x][j & 1][c * 32 + i]);
                        v[i] = fmaf(-slope, fabsf(my_pos - p.x), v[i]);
                        v[i + 1] = fmaf(-slope, fabsf(my_pos - p.y), v[i + 1]);
                        v[i + 2] = fmaf(-slope, fabsf(my_pos - p.z), v[i + 2]);
                        v[i + 3] = fmaf(-slope, fabsf(my_pos - p.w), v[i + 3]);
                    }
                }
                if (masked) {
#pragma unroll
                    for (int i = 0; i < 32; ++i) v[i] = k0 + c * 32 + i < keys ? v[i] : ninf;
                }
            };
            // the largest of columns [32 c0, 32 c1)
            auto largest = [&](int c0, int c1) {
                float mx = ninf;
#pragma unroll 1
                for (int c = c0; c < c1; ++c) {
                    uint32_t raw[32];
                    float v[32];
                    tmem_ld32_issue(t_s + c * 32, raw);
                    tmem_ld32_wait(raw);
                    logit(raw, c, 0.f, v);
                    float t8[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) t8[i] = fmaxf(fmaxf(v[i], v[i + 8]), fmaxf(v[i + 16], v[i + 24]));
                    mx = fmaxf(mx, fmaxf(fmaxf(fmaxf(t8[0], t8[1]), fmaxf(t8[2], t8[3])), fmaxf(fmaxf(t8[4], t8[5]), fmaxf(t8[6], t8[7]))));
                }
                return mx;
            };
            // 32 weights of the row, and their sum
            auto weights = [&](const uint32_t (&raw)[32], int c, uint32_t* p) {
                float v[32];
                logit(raw, c, m == ninf ? 0.f : m, v);
                uint64_t sum0 = 0ull, sum1 = 0ull;
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const float w0 = fast_exp2(v[2 * i]), w1 = fast_exp2(v[2 * i + 1]);
                    if (i & 1) sum1 = add_pair(sum1, pair(w0, w1));
                    else sum0 = add_pair(sum0, pair(w0, w1));
                    p[i] = pack_bf16(w0, w1);
                }
                float s0, s1;
                unpair(add_pair(sum0, sum1), s0, s1);
                return s0 + s1;
            };
            const bool first = m == ninf && keys > k0; // the first tile of which the row sees something
            if (__any_sync(0xFFFFFFFFu, first)) {
                const float mx = largest(0, 4);
                if (first) m = mx;
            }
            uint32_t raw[2][32];
            tmem_ld32_issue(t_s, raw[0]);
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                uint32_t p[32];
                tmem_ld32_wait(raw[0]);
                tmem_ld32_issue(t_s + half * 64 + 32, raw[1]);
                float sum = weights(raw[0], half * 2, p);
                tmem_ld32_wait(raw[1]);
                if (!half) tmem_ld32_issue(t_s + 64, raw[0]);
                sum += weights(raw[1], half * 2 + 1, p + 16);
                const bool far = !(sum < kMost);
                if (__any_sync(0xFFFFFFFFu, far)) {    // again, against the maximum of these
                    if (!half) tmem_ld32_wait(raw[0]); // (in order: nothing is on its way while registers are short)
                    const float mx = largest(half * 2, half * 2 + 2);
                    const bool grow = far && mx > m;
                    const float f = grow ? fast_exp2(m - (mx + kRoom)) : 1.f;
                    if (grow) m = mx + kRoom;
                    l *= f;
                    // the product before this one on O_x is complete: that of the tile before since S_x is there, that of the first half when its barrier says so
                    if (half && ok && !mbar_wait(smem_u32(&h_bar[x]), (uint32_t)j & 1u, abort_flag)) ok = false;
                    ok = __all_sync(0xFFFFFFFFu, ok);
                    tc_fence_after();
                    if (j > 0 || half) {
#pragma unroll 1
                        for (int c = 0; c < DH / 32; ++c) {
                            uint32_t o[32];
                            tmem_ld32_issue(t_o + c * 32, o);
                            tmem_ld32_wait(o);
#pragma unroll
                            for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
                            tmem_st32(t_o + c * 32, o);
                        }
                    }
                    sum = 0.f;
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        uint32_t again[32];
                        tmem_ld32_issue(t_s + half * 64 + c * 32, again);
                        tmem_ld32_wait(again);
                        sum += weights(again, half * 2 + c, p + c * 16);
                    }
                }
                l += sum;
                tmem_st32(t_s + half * 32, p);         // 64 keys' weights: their product may begin
                tmem_st_wait();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&p_bar[x][half]));
            }
        }
        if (my_n > 0 && ok && !mbar_wait(smem_u32(&o_bar[x]), 0u, abort_flag)) ok = false;
        ok = __all_sync(0xFFFFFFFFu, ok);
        tc_fence_after();
        const bool mine = r < my_rows;
        const long long row = d.q0 + my_i0 + r;
        const long long at = ((long long)blockIdx.y * a.Hq + my_head) * a.n_q + row;
        const float scale = a.splits > 1 ? 1.f : l > 0.f ? 1.f / l : 0.f;
        __nv_bfloat16* out = reinterpret_cast<__nv_bfloat16*>(a.out) + my_head * a.out_head + row * a.out_row;
        if (ok) {
#pragma unroll
            for (int c = 0; c < DH / 32; ++c) {
                float o[32];
                if (my_n > 0) {
                    tmem_ld32(t_o + c * 32, o);
                } else {
#pragma unroll
                    for (int i = 0; i < 32; ++i) o[i] = 0.f;
                }
                if (mine && a.splits > 1) {
                    if (my_n > 0) {
#pragma unroll
                        for (int i = 0; i < 32; i += 4) *reinterpret_cast<float4*>(a.part_o + at * DH + c * 32 + i) = make_float4(o[i], o[i + 1], o[i + 2], o[i + 3]);
                    }
                } else if (mine) {
#pragma unroll
                    for (int i = 0; i < 32; i += 8)
                        *reinterpret_cast<uint4*>(out + c * 32 + i) = make_uint4(pack_bf16(o[i] * scale, o[i + 1] * scale), pack_bf16(o[i + 2] * scale, o[i + 3] * scale),
                                                                                 pack_bf16(o[i + 4] * scale, o[i + 5] * scale), pack_bf16(o[i + 6] * scale, o[i + 7] * scale));
                }
            }
            if (mine && a.splits > 1) *reinterpret_cast<float2*>(a.part_ml + at * 2) = make_float2(l > 0.f ? m : ninf, l);
            else if (mine && a.lse) a.lse[(long long)my_head * a.n_q + row] = kAttnLn2 * (m + log2f(l));
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 9) tmem_dealloc(tmem, 512);
    if (threadIdx.x == 0 && s_abort) *a.status = METOK_ERR_TIMEOUT;
}

template <int DH, bool kCap, bool kBias>
int launch(const PromptArgs& a, long long ctas, const MmaMaps& maps, cudaStream_t st) {
    auto kern = prompt_attn_mma_kernel<DH, kCap, kBias>;
    METOK_ALLOW_SMEM(kern, MmaShape<DH>::kSmem);
    METOK_TIMED("prompt_attn_mma", st);
    launch_chained(kern, dim3((unsigned)ctas, a.splits), dim3(kThreads), MmaShape<DH>::kSmem, st, a, maps);
    METOK_LAUNCH_CHECK();
    return METOK_OK;
}
template <int DH>
int launch_dh(const PromptArgs& a, long long ctas, const MmaMaps& maps, cudaStream_t st) {
    if (a.cap_log2 > 0.f) return a.slopes ? launch<DH, true, true>(a, ctas, maps, st) : launch<DH, true, false>(a, ctas, maps, st);
    return a.slopes ? launch<DH, false, true>(a, ctas, maps, st) : launch<DH, false, false>(a, ctas, maps, st);
}

}  // namespace

// CTAs for the pairs of items of all documents, at most: one document has ceil(n_q / 128) G items, several at most a started tile more each.
long long prompt_mma_ctas(int Hkv, int G, int n_q, int n_seq) {
    const long long docs = std::min(n_seq, n_q), tiles = n_seq == 1 ? ceil_div(n_q, kM) : n_q / kM + docs;
    return std::max(1LL, (tiles * G + docs) / 2) * Hkv;
}

int launch_prompt_attn_mma(const PromptArgs& a, int dh, long long ctas, cudaStream_t st) {
    MmaMaps maps = {};
    maps.q_step = a.Hq > 1 && a.q_head > 0;
    maps.k_step = a.Hkv > 1 && a.k_head > 0;
    maps.v_step = a.Hkv > 1 && a.v_head > 0;
    if (a.n_q > 0) {
        int rc = make_tmap_heads(&maps.q, a.q, a.n_q, dh, maps.q_step ? a.Hq : 1, a.q_row, a.q_head, kM);
        // where there are no keys no tile of them is asked for, and any rows will do
        if (rc == METOK_OK) rc = a.n_k ? make_tmap_heads(&maps.k, a.k, a.n_k, dh, maps.k_step ? a.Hkv : 1, a.k_row, a.k_head, kN) : (maps.k = maps.q, METOK_OK);
        if (rc == METOK_OK) rc = a.n_k ? make_tmap_heads(&maps.v, a.v, a.n_k, dh, maps.v_step ? a.Hkv : 1, a.v_row, a.v_head, kN) : (maps.v = maps.q, METOK_OK);
        if (rc != METOK_OK) return rc;
    }
    return dh == 64 ? launch_dh<64>(a, ctas, maps, st) : launch_dh<128>(a, ctas, maps, st);
}

}  // namespace metok
