// metok_prefill_attention: the C entry, the fp32 kernel, and the join of split keys.  (bf16: prefill_attn_mma.cu.)
//
// fp32, on the CUDA cores: a CTA of 256 threads takes a tile of 16 R query rows (consecutive rows of a document, each with all query heads
// of one K/V head, so that few rows fill a tile too) and walks their keys in tiles of 64, of which the next one is on its way while
// one is worked on.  Thread (ty, tx) holds the logits of rows R ty + i and keys tx + 16 j, and the outputs of the same rows; a row's
// running maximum and sum are shared by the sixteen threads of its ty by shuffles.  A row sees the keys [0, n) with n not falling
// from row to row, so only tiles that reach beyond the first row's n are masked, by comparing indices.
// R = 4 feeds the multiply-adds best (five of them per shared-memory wavefront, 1.8 with R = 1); R = 2 and 1 are for calls of few rows, and
// those that leave most SMs without a tile, where a tile's own latency counts: 132 rows of one head, capped: 21 us with R = 4, 12.8 with 1 (13.2 with its loops unrolled half as far).
#include <algorithm>

#include "launchers.h"
#include "prefill_attn.cuh"
#include "sm100.cuh"

namespace metok {

namespace {

constexpr int kSN = 64, kSThreads = 256;

template <int DH, int R>
struct SimtAttnSmem {
    float q[16 * R][DH + 4], k[2][kSN][DH + 4], v[2][kSN][DH], p[16 * R][kSN + 4];
    float pos[2][kSN];
};

template <int DH, int R>
__global__ void __launch_bounds__(kSThreads)
prompt_attn_simt_kernel(const PromptArgs a) {
    constexpr int kSM = 16 * R;
    grid_dep_wait();
    extern __shared__ __align__(16) uint8_t smem_raw[];
    SimtAttnSmem<DH, R>& sm = *reinterpret_cast<SimtAttnSmem<DH, R>*>(smem_raw);
    const int g = blockIdx.x % a.Hkv, tid = threadIdx.x, ty = tid >> 4, tx = tid & 15;
    const PromptDoc d = prompt_tile(a, blockIdx.x / a.Hkv, [&](int Lq) { return (Lq + a.rows_item - 1) / a.rows_item * a.head_chunks; });
    if (d.tile < 0) return;
    const int blk = d.tile / a.head_chunks, h0 = (d.tile - blk * a.head_chunks) * a.heads_item, i0 = blk * a.rows_item;
    const int nr = min(a.rows_item, d.Lq - i0), heads = min(a.heads_item, a.G - h0);
    const int first_keys = prompt_keys(a, d, i0), all_keys = prompt_keys(a, d, i0 + nr - 1);
    const int nt = (all_keys + kSN - 1) / kSN, t_lo = (int)((long long)nt * blockIdx.y / a.splits), t_hi = (int)((long long)nt * (blockIdx.y + 1) / a.splits);
    // row r of the tile: document row i0 + r / heads_item, head h0 + r % heads_item of the K/V head's; -1 if it is none
    auto row_of = [&](int r) { const int i = r / a.heads_item; return i < nr && r - i * a.heads_item < heads ? i0 + i : -1; };
    auto head_of = [&](int r) { return g * a.G + h0 + r % a.heads_item; };
    const float* k = reinterpret_cast<const float*>(a.k) + g * a.k_head + (long long)d.k0 * a.k_row;
    const float* v = reinterpret_cast<const float*>(a.v) + g * a.v_head + (long long)d.k0 * a.v_row;
    constexpr int CPR = DH / 4;                        // 16-byte pieces of a row
    auto fetch = [&](int t) {                          // rows behind the document's keys count as zeros
        const int b = t & 1, j0 = t * kSN;
        for (int c = tid; c < kSN * CPR; c += kSThreads) {
            const int r = c / CPR, e = (c - r * CPR) * 4;
            const uint32_t bytes = j0 + r < d.Lk ? 16u : 0u;
            const long long row = bytes ? j0 + r : 0;
            sm100::cp_async16_zfill(sm100::smem_u32(&sm.k[b][r][e]), k + row * a.k_row + e, bytes);
            sm100::cp_async16_zfill(sm100::smem_u32(&sm.v[b][r][e]), v + row * a.v_row + e, bytes);
        }
        if (a.slopes && tid < kSN) sm.pos[b][tid] = prompt_position(a, d.k0, d.Lk, j0 + tid);
        sm100::cp_async_commit();
    };
    if (t_lo < t_hi) fetch(t_lo);
    for (int c = tid; c < kSM * CPR; c += kSThreads) {
        const int r = c / CPR, e = (c - r * CPR) * 4;
        float x[4];
        const int i = row_of(r);
        if (i >= 0) Vec16<float>::load(reinterpret_cast<const float*>(a.q) + head_of(r) * a.q_head + (long long)(d.q0 + i) * a.q_row + e, x);
        else Vec16<float>::zero(x);
        *reinterpret_cast<float4*>(&sm.q[r][e]) = make_float4(x[0], x[1], x[2], x[3]);
    }
    int keys[R];
    float my_pos[R], slope[R], m[R], l[R], o[R][DH / 16];
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const int r = ty * R + i, row = row_of(r);
        keys[i] = row >= 0 ? prompt_keys(a, d, row) : 0;
        my_pos[i] = a.slopes ? prompt_position(a, d.k0, d.Lk, d.Lk - d.Lq + row) : 0.f;
        slope[i] = a.slopes && row >= 0 ? a.slopes[head_of(r)] * kAttnLog2e : 0.f;
        m[i] = __int_as_float(0xFF800000);
        l[i] = 0.f;
#pragma unroll
        for (int c = 0; c < DH / 16; ++c) o[i][c] = 0.f;
    }
    for (int t = t_lo; t < t_hi; ++t) {
        const int j0 = t * kSN, b = t & 1;
        __syncthreads();                               // everybody is done with the tile before, whose place the next one takes
        if (t + 1 < t_hi) {
            fetch(t + 1);
            sm100::cp_async_wait<1>();
        } else {
            sm100::cp_async_wait<0>();
        }
        __syncthreads();
        float s[R][4];
#pragma unroll
        for (int i = 0; i < R; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) s[i][j] = 0.f;
#pragma unroll (R == 1 ? 8 : 4)
        for (int e = 0; e < DH; e += 4) {
            float4 x[R], y[4];
#pragma unroll
            for (int i = 0; i < R; ++i) x[i] = *reinterpret_cast<const float4*>(&sm.q[ty * R + i][e]);
#pragma unroll
            for (int j = 0; j < 4; ++j) y[j] = *reinterpret_cast<const float4*>(&sm.k[b][tx + 16 * j][e]);
#pragma unroll
            for (int i = 0; i < R; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    s[i][j] = fmaf(x[i].w, y[j].w, fmaf(x[i].z, y[j].z, fmaf(x[i].y, y[j].y, fmaf(x[i].x, y[j].x, s[i][j]))));
        }
        const bool masked = j0 + kSN > first_keys;
#pragma unroll
        for (int i = 0; i < R; ++i) {
            float top = m[i];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                float x = a.cap_log2 > 0.f ? a.cap_log2 * tanhf(s[i][j] * a.cap_scale) : s[i][j] * a.scale_log2;
                if (a.slopes) x = fmaf(-slope[i], fabsf(my_pos[i] - sm.pos[b][tx + 16 * j]), x);
                if (masked && j0 + tx + 16 * j >= keys[i]) x = __int_as_float(0xFF800000);
                s[i][j] = x;
                top = fmaxf(top, x);
            }
#pragma unroll
            for (int w = 8; w >= 1; w >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, w));
            const float base = top == __int_as_float(0xFF800000) ? 0.f : top;    // no key so far: weights of 0, not of inf - inf
            const float f = exp2f(m[i] - base);
            m[i] = top;
            float sum = 0.f;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                s[i][j] = exp2f(s[i][j] - base);
                sum += s[i][j];
                sm.p[ty * R + i][tx + 16 * j] = s[i][j];
            }
            l[i] = l[i] * f + sum;
#pragma unroll
            for (int c = 0; c < DH / 16; ++c) o[i][c] *= f;
        }
        __syncwarp();                                  // a row's weights are written and read by one half of a warp
#pragma unroll (R == 1 ? 4 : 2)
        for (int j = 0; j < kSN; j += 4) {
            float4 p[R];
#pragma unroll
            for (int i = 0; i < R; ++i) p[i] = *reinterpret_cast<const float4*>(&sm.p[ty * R + i][j]);
#pragma unroll
            for (int jj = 0; jj < 4; ++jj)
#pragma unroll
                for (int c = 0; c < DH / 64; ++c) {
                    const float4 x = *reinterpret_cast<const float4*>(&sm.v[b][j + jj][tx * 4 + 64 * c]);
#pragma unroll
                    for (int i = 0; i < R; ++i) {
                        const float w = jj == 0 ? p[i].x : jj == 1 ? p[i].y : jj == 2 ? p[i].z : p[i].w;
                        o[i][4 * c] = fmaf(w, x.x, o[i][4 * c]);
                        o[i][4 * c + 1] = fmaf(w, x.y, o[i][4 * c + 1]);
                        o[i][4 * c + 2] = fmaf(w, x.z, o[i][4 * c + 2]);
                        o[i][4 * c + 3] = fmaf(w, x.w, o[i][4 * c + 3]);
                    }
                }
        }
    }
#pragma unroll
    for (int i = 0; i < R; ++i) {
#pragma unroll
        for (int w = 8; w >= 1; w >>= 1) l[i] += __shfl_xor_sync(0xFFFFFFFFu, l[i], w);
        const int r = ty * R + i, in_doc = row_of(r);
        if (in_doc < 0) continue;
        const int h = head_of(r);
        const long long row = d.q0 + in_doc;
        const bool part = a.splits > 1;
        const float inv = part ? 1.f : l[i] == 0.f ? 0.f : 1.f / l[i];
        const long long at = ((long long)blockIdx.y * a.Hq + h) * a.n_q + row;
        float* out = part ? a.part_o + at * DH : reinterpret_cast<float*>(a.out) + h * a.out_head + row * a.out_row;
#pragma unroll
        for (int c = 0; c < DH / 64; ++c)
            *reinterpret_cast<float4*>(out + tx * 4 + 64 * c) = make_float4(o[i][4 * c] * inv, o[i][4 * c + 1] * inv, o[i][4 * c + 2] * inv, o[i][4 * c + 3] * inv);
        if (tx != 0) continue;
        if (part) *reinterpret_cast<float2*>(a.part_ml + at * 2) = make_float2(m[i], l[i]);
        else if (a.lse) a.lse[(long long)h * a.n_q + row] = kAttnLn2 * (m[i] + log2f(l[i]));
    }
}

// Joins the parts of split keys: a warp per row of a head.
constexpr int kJoinWarps = 8;
template <int DH>
__global__ void __launch_bounds__(kJoinWarps * 32)
prompt_join_kernel(const PromptArgs a) {
    grid_dep_wait();
    if (*a.status != METOK_OK) return;                 // offsets out of order: no row is anybody's
    const int lane = threadIdx.x & 31, h = blockIdx.y;
    const long long row = (long long)blockIdx.x * kJoinWarps + (threadIdx.x >> 5);
    const int lo = a.seq_q ? a.seq_q[0] : 0, hi = a.seq_q ? a.seq_q[a.n_seq] : a.n_q;
    if (row < lo || row >= hi) return;
    float M = __int_as_float(0xFF800000);
    for (int s = lane; s < a.splits; s += 32) M = fmaxf(M, a.part_ml[(((long long)s * a.Hq + h) * a.n_q + row) * 2]);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor_sync(0xFFFFFFFFu, M, o));
    constexpr int E = DH / 32;
    float acc[E], L = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] = 0.f;
#pragma unroll 4
    for (int s = 0; s < a.splits; ++s) {
        const long long at = ((long long)s * a.Hq + h) * a.n_q + row;
        const float2 ml = *reinterpret_cast<const float2*>(a.part_ml + at * 2);
        if (ml.y == 0.f) continue;                     // a part of no keys (M may be -infinity too); one of NaN counts
        const float f = exp2f(ml.x - M);
        L += f * ml.y;
#pragma unroll
        for (int e = 0; e < E; ++e) acc[e] += f * a.part_o[at * DH + lane * E + e];
    }
    const float inv = L == 0.f ? 0.f : 1.f / L;
    float* out = reinterpret_cast<float*>(a.out) + h * a.out_head + row * a.out_row;
#pragma unroll
    for (int e = 0; e < E; ++e) out[lane * E + e] = acc[e] * inv;
    if (lane == 0 && a.lse) a.lse[(long long)h * a.n_q + row] = kAttnLn2 * (M + log2f(L));
}

// fp32: rows of a tile, how heads and rows make one, CTAs without splits, and splits of the keys.
struct PromptPlan {
    int rows, heads_item, head_chunks, rows_item;
    long long ctas;
    int splits;
};
PromptPlan prompt_plan(const metok_attention_params* p) {
    PromptPlan pl;
    const int G = p->Hq / p->Hkv;
    for (int rows : {64, 32, 16}) {
        pl.rows = rows;
        pl.heads_item = std::min(G, rows);
        pl.head_chunks = ceil_div(G, pl.heads_item);
        pl.rows_item = rows / pl.heads_item;
        // several documents: at most a started tile more each than whole ones fit into n_q
        const long long tiles = p->n_seq == 1 ? ceil_div(p->n_q, pl.rows_item) : (long long)p->n_q / pl.rows_item + std::min(p->n_seq, p->n_q);
        pl.ctas = std::max(1LL, tiles * pl.head_chunks) * p->Hkv;
        // few rows: the keys are cut until every SM has work (documents of different lengths: several parts), no part shorter than two tiles
        const long long most = std::max(1LL, std::min((long long)p->n_k / (2 * kSN), 64LL));
        // (no rows: nothing to join)
        pl.splits = p->n_q == 0 ? 1 : (int)std::max(1LL, std::min(most, (p->n_seq == 1 ? kNumSMs : 4 * kNumSMs) / pl.ctas));
        // the largest tile that the average document fills by three quarters and that leaves a CTA for every SM
        if (pl.ctas * most >= kNumSMs && 4LL * p->n_q * pl.heads_item >= 3LL * rows * p->n_seq) break;
    }
    return pl;
}
void prompt_carve(Carver& cv, int dtype, const metok_attention_params* p, PromptArgs* a) {
    if (dtype == METOK_BF16) return prompt_mma_carve(cv, p, a);
    const int splits = prompt_plan(p).splits;
    if (splits == 1) return;
    const size_t rows = (size_t)splits * p->Hq * p->n_q;
    a->part_o = cv.take<float>(rows * p->dh);
    a->part_ml = cv.take<float>(rows * 2);
}

template <int DH, int R>
int launch_prompt_simt(const PromptArgs& a, const PromptPlan& pl, cudaStream_t st) {
    auto kern = prompt_attn_simt_kernel<DH, R>;
    METOK_ALLOW_SMEM(kern, sizeof(SimtAttnSmem<DH, R>));
    {
        METOK_TIMED("prompt_attn_simt", st);
        launch_chained(kern, dim3((unsigned)pl.ctas, pl.splits), dim3(kSThreads), sizeof(SimtAttnSmem<DH, R>), st, a);
    }
    METOK_LAUNCH_CHECK();
    if (pl.splits > 1) {
        METOK_TIMED("prompt_join", st);
        launch_chained(prompt_join_kernel<DH>, dim3(ceil_div(a.n_q, kJoinWarps), a.Hq), dim3(kJoinWarps * 32), 0, st, a);
        METOK_LAUNCH_CHECK();
    }
    return METOK_OK;
}

int prompt_check(int dtype, const metok_attention_params* p) {
    if (!p || (dtype != METOK_F32 && dtype != METOK_BF16)) return METOK_ERR_INVALID_ARG;
    if (p->Hq < 1 || p->Hkv < 1 || p->Hq % p->Hkv || p->dh < 1 || p->n_q < 0 || p->n_k < 0 || p->n_seq < 1) return METOK_ERR_INVALID_ARG;
    if (!p->seq_q != !p->seq_k || (!p->seq_q && p->n_seq != 1)) return METOK_ERR_INVALID_ARG;
    if (p->dh != 64 && p->dh != 128) return METOK_ERR_UNSUPPORTED;
    if (p->n_q > (1 << 24) || p->n_k > (1 << 24) || p->n_seq > kPromptDocs || p->Hq > 65535) return METOK_ERR_UNSUPPORTED;
    if (dtype == METOK_F32 && prompt_plan(p).ctas > 0x7FFFFFFFLL) return METOK_ERR_UNSUPPORTED;
    // (bf16: items of a K/V head)
    const int G = p->Hq / p->Hkv;
    if (((long long)p->n_q + p->n_seq) * ceil_div(G, 128) > (1LL << 30)) return METOK_ERR_UNSUPPORTED;
    return METOK_OK;
}

}  // namespace
}  // namespace metok

using namespace metok;

extern "C" size_t metok_prefill_attention_workspace_bytes(int dtype, const metok_attention_params* p) {
    if (prompt_check(dtype, p) != METOK_OK) return 0;
    PromptArgs a;
    Carver cv(nullptr);
    prompt_carve(cv, dtype, p, &a);
    return cv.total();
}

extern "C" int metok_prefill_attention(int dtype, const metok_attention_params* p, int32_t* status, void* ws, size_t ws_bytes, void* stream) {
    int rc = prompt_check(dtype, p);
    if (rc != METOK_OK) return rc;
    if ((p->n_q > 0 && (!p->q || !p->out)) || (p->n_k > 0 && (!p->k || !p->v)) || !status) return METOK_ERR_INVALID_ARG;
    if (!aligned16(p->q) || !aligned16(p->k) || !aligned16(p->v) || !aligned16(p->out)) return METOK_ERR_INVALID_ARG;
    if (!aligned4(p->lse) || !aligned4(p->seq_q) || !aligned4(p->seq_k) || !aligned4(p->prefix_len) || !aligned4(p->positions) ||
        !aligned4(p->slopes) || !aligned4(status))
        return METOK_ERR_INVALID_ARG;
    const int per = 16 / (dtype == METOK_F32 ? 4 : 2);
    if (p->q_head < 0 || p->k_head < 0 || p->v_head < 0 || p->out_head < 0) return METOK_ERR_INVALID_ARG;
    if (p->q_row < p->dh || p->k_row < p->dh || p->v_row < p->dh || p->out_row < p->dh) return METOK_ERR_INVALID_ARG;
    if ((p->Hq > 1 && p->q_head < p->dh) || !rows_apart(p->Hq, p->out_head, p->n_q, p->out_row, p->dh)) return METOK_ERR_INVALID_ARG;
    if ((p->q_head | p->k_head | p->v_head | p->out_head | p->q_row | p->k_row | p->v_row | p->out_row) % per) return METOK_ERR_INVALID_ARG;
    if (!softmax_numbers(p->softmax_scale, p->softcap)) return METOK_ERR_INVALID_ARG;
    const size_t need = metok_prefill_attention_workspace_bytes(dtype, p);
    if (need > 0 && (!ws || !aligned16(ws) || ws_bytes < need)) return METOK_ERR_WORKSPACE;
    PromptArgs a = {};
    a.q = p->q; a.k = p->k; a.v = p->v; a.out = p->out; a.lse = p->lse;
    a.q_head = p->q_head; a.q_row = p->q_row; a.k_head = p->k_head; a.k_row = p->k_row;
    a.v_head = p->v_head; a.v_row = p->v_row; a.out_head = p->out_head; a.out_row = p->out_row;
    a.Hq = p->Hq; a.Hkv = p->Hkv; a.G = p->Hq / p->Hkv; a.n_q = p->n_q; a.n_k = p->n_k; a.n_seq = p->n_seq;
    a.seq_q = p->seq_q; a.seq_k = p->seq_k; a.prefix_len = p->prefix_len; a.positions = p->positions; a.slopes = p->slopes;
    a.scale_log2 = p->softmax_scale * kAttnLog2e;
    a.cap_scale = p->softcap > 0.f ? p->softmax_scale / p->softcap : 0.f;
    a.cap_log2 = p->softcap * kAttnLog2e;
    a.causal = p->causal != 0;
    a.status = status;
    a.withhold = debug_withheld();
    Carver cv(ws);
    prompt_carve(cv, dtype, p, &a);
    cudaStream_t st = (cudaStream_t)stream;
    if (dtype == METOK_BF16) return launch_prompt_attn_mma(a, p->dh, st);
    const PromptPlan pl = prompt_plan(p);
    a.splits = pl.splits;
    a.heads_item = pl.heads_item; a.head_chunks = pl.head_chunks; a.rows_item = pl.rows_item;
    if (pl.rows == 32) return p->dh == 64 ? launch_prompt_simt<64, 2>(a, pl, st) : launch_prompt_simt<128, 2>(a, pl, st);
    if (pl.rows == 16) return p->dh == 64 ? launch_prompt_simt<64, 1>(a, pl, st) : launch_prompt_simt<128, 1>(a, pl, st);
    return p->dh == 64 ? launch_prompt_simt<64, 4>(a, pl, st) : launch_prompt_simt<128, 4>(a, pl, st);
}
