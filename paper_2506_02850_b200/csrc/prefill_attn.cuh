// What the kernels of metok_prefill_attention share: arguments, the documents' tiles, the range of keys of a query.
#pragma once

#include "common.cuh"

namespace metok {

constexpr float kAttnLog2e = 1.4426950408889634f, kAttnLn2 = 0.6931471805599453f;

struct PromptArgs {
    const void *q, *k, *v;
    void* out;
    float* lse;
    long long q_head, q_row, k_head, k_row, v_head, v_row, out_head, out_row;   // elements
    int Hq, Hkv, G, n_q, n_k, n_seq;
    const int32_t *seq_q, *seq_k, *prefix_len, *positions;
    const float* slopes;
    float scale_log2, cap_scale, cap_log2;     // softcap > 0: x = cap_log2 * tanh(dot * cap_scale); else cap_log2 is 0 (log2 units)
    float cap_poly[7];                         // bf16: cap_log2 * tanh(y) / y in powers of y^2, y = dot * cap_scale
    int causal;
    int splits;                                // fp32: parts that a tile's keys are cut into; above 1 the parts are joined by another kernel
    int heads_item, head_chunks, rows_item;    // query heads of a tile of rows, such tiles for all heads of a K/V head, document rows of a tile
    uint32_t rows_magic;                       // bf16: ceil(2^32 / rows_item)
    int pair_cost;                             // bf16: what a pair costs beside its key tiles, in tiles
    float *part_o, *part_ml;                   // unnormalised outputs and (maximum, sum) of the parts; fp32: [splits][Hq][n_q]
    void* cuts;                                // bf16: what the second kernel joins
    int32_t* status;
    int withhold;                              // debug builds: the copies to leave out
};

constexpr int kPromptDocs = 8192;              // documents at most

// The tensor-core kernels (bf16): their workspace, and the launch.
void prompt_mma_carve(Carver& cv, const metok_attention_params* p, PromptArgs* a);
int launch_prompt_attn_mma(PromptArgs a, int dh, cudaStream_t st);

struct PromptDoc {
    int q0, k0, Lq, Lk, prefix;
    int tile;                                  // of the document's tiles, longest keys first; -1: there is none
};

// Keys that the document's query i sees: [0, result).
__device__ __forceinline__ int prompt_keys(const PromptArgs& a, const PromptDoc& d, int i) {
    if (!a.causal) return d.Lk;
    return max(0, min(d.Lk, max(d.Lk - d.Lq + i + 1, d.prefix)));
}

// Document and tile of the CTA's place `at` in the line of all documents' tiles, tiles(Lq) of each; whole CTA.  Checks all offsets:
// where one is out of order every CTA finds no tile, and the first one says so in the status word.
template <typename Tiles>
__device__ __forceinline__ PromptDoc prompt_tile(const PromptArgs& a, int at, Tiles tiles) {
    PromptDoc d = {0, 0, a.n_q, a.n_k, 0, -1};
    if (!a.seq_q) {
        if (blockIdx.x == 0 && threadIdx.x == 0) *a.status = METOK_OK;
        const int n = tiles(a.n_q);
        if (at < n) d.tile = n - 1 - at;
        d.prefix = a.prefix_len ? a.prefix_len[0] : 0;
        return d;
    }
    __shared__ int s_doc, s_tile;
    int bad = 0;
    for (int s = threadIdx.x; s < a.n_seq; s += blockDim.x) {
        const int q0 = a.seq_q[s], q1 = a.seq_q[s + 1], k0 = a.seq_k[s], k1 = a.seq_k[s + 1];
        bad |= q0 < 0 || q1 < q0 || q1 > a.n_q || k0 < 0 || k1 < k0 || k1 > a.n_k;
    }
    bad = __syncthreads_or(bad);
    if (blockIdx.x == 0 && threadIdx.x == 0) *a.status = bad ? METOK_ERR_INVALID_ARG : METOK_OK;
    if (bad) return d;
    if (threadIdx.x < 32) {
        const int lane = threadIdx.x;
        if (lane == 0) s_doc = -1;
        __syncwarp();
        long long before = 0;                  // tiles of the documents before s0
        for (int s0 = 0; s0 < a.n_seq; s0 += 32) {
            const int s = s0 + lane;
            const long long mine = s < a.n_seq ? tiles(a.seq_q[s + 1] - a.seq_q[s]) : 0;
            long long incl = mine;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const long long x = __shfl_up_sync(0xFFFFFFFFu, incl, o);
                if (lane >= o) incl += x;
            }
            const uint32_t any = __ballot_sync(0xFFFFFFFFu, before + incl > at);
            if (any) {
                if (lane == __ffs(any) - 1) {
                    s_doc = s;
                    s_tile = (int)(before + incl - 1 - at);              // the last tile first
                }
                break;
            }
            before += __shfl_sync(0xFFFFFFFFu, incl, 31);
        }
    }
    __syncthreads();
    const int s = s_doc;
    if (s < 0) return d;
    d.q0 = a.seq_q[s];
    d.k0 = a.seq_k[s];
    d.Lq = a.seq_q[s + 1] - d.q0;
    d.Lk = a.seq_k[s + 1] - d.k0;
    d.prefix = a.prefix_len ? a.prefix_len[s] : 0;
    d.tile = s_tile;
    return d;
}

// Position of key j of the document whose Lk keys begin at k0 (or of the query that sits there).
__device__ __forceinline__ float prompt_position(const PromptArgs& a, int k0, int Lk, int j) {
    if (Lk < 1) return 0.f;                    // (there may be no key at k0)
    j = max(0, min(j, Lk - 1));
    return (float)(a.positions ? a.positions[k0 + j] : j);
}

}  // namespace metok
