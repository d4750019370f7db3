// metok_prefill_attention on the tensor cores (bf16).
//
// An item is a tile of 128 query rows: 128 / G consecutive rows of a document with all G query heads of one K/V head, so that
// few rows fill a tile too, and a tile's rows end at nearly the same key.  A CTA works on two items side by side (a pair: neighbours
// in the document), which use the same K and V tiles.  Per tile of 128 keys and item x:
//   S_x = Q_x K^T        tcgen05.mma, both operands in shared memory, fp32 in tensor memory
//   P_x = 2^(logit - m)  one thread per row; bf16, written over S_x in tensor memory
//   O_x += P_x V         tcgen05.mma, P_x from tensor memory, V as it lies (keys x dh: the second operand's other order)
// S_0, S_1, O_0 and O_1 fill the 512 columns (128 each).  The halves of S_x, of 64 keys each, go round by themselves: while the rows make one
// half's weights, the other's are multiplied with V and the next tile's logits take its place, so that the rows never wait for
// a product.  (S_x whole, the rows waited for two products a tile: 28 heads of 128, 4624 rows, 340 us instead of 298 when this was changed.)
//
// The key tiles of all pairs of all documents and K/V heads form one line, and every CTA (one per SM) takes an equal piece of it:
// a piece may begin and end inside a pair, whose parts are then joined by a second kernel.  So a batch of documents of any lengths,
// few rows over many keys and a number of pairs that is no multiple of the SMs all keep every SM busy to the end.  Every CTA finds its
// piece by itself, from the documents' offsets.
//
// Key tiles of a pair are taken from the last one down (a bias makes the nearest ones the largest).  A row's reference m is the maximum of
// the first 64 keys that it sees; later weights are taken against it with no maximum of their own, since any m within the range of the
// exponent gives the same result.  Where a row's sum leaves that range 64 weights are made again against a higher reference, and O_x
// and the row's sum are scaled: by the row's own thread, when the product before on O_x is complete.
//
// What bounds it: with heads of 128 the products (2.05 us per 128 keys of a pair, 1.54 at the 1.62 PFLOP/s of a large library product; 9472 rows
// of four heads over 12 800 keys run at 1.22 PFLOP/s); with heads of 64, which halve the products and not the exponentials, the rows' arithmetic (14 heads,
// 2664 x 12 800: 0.65 PFLOP/s, 3300 clocks per 128 keys; with a cap, whose polynomial costs seven multiply-adds more, 5600).  A bias adds 1250 clocks: sixteen 16-byte
// reads of positions from the shared memory that the products read too, and three operations a weight (as packed pairs they took 40 us more
// of 530).
//
// Warps 0-3 and 4-7: the rows of items 0 and 1; warp 8: TMA; warps 9 and 10: the products of items 0 and 1, each with waits of its
// own (an issuing warp is held up while products run, so one warp's waits for both items lie open).  Every wait is bounded.  A row's 128 logits are read
// from tensor memory 32 at a time: held in registers they spill.
#include <algorithm>

#include "launchers.h"
#include "prefill_attn.cuh"
#include "sm100.cuh"

namespace metok {

namespace {

constexpr int kM = 128, kN = 128, kThreads = 352;
// A row's reference grows where 64 weights add up to kMost (one of them has passed it by 18 octaves then), and where the row's sum has: by kGrow
// octaves, or to the maximum of the 64 keys at hand where that is higher.  So the row's sum, looked at before every tile, stays below 2^26 however many keys
// there are, and that of weight * V within fp32 for V up to 2^100.  With at most 2^24 keys, a sum of 2^24 takes a weight of 1 or more: the reference is at most 16
// octaves above the maximum, and what underflows is below 2^-109 of it.
constexpr float kMost = 0x1p24f, kGrow = 16.f;
// Caps above this have a kernel of their own (kCap = 2).  1 - 2 / (1 + e^2y) is off by some 2^-21 of 1 however small y is, so a capped logit
// by 2^-21 of the cap: up to here at most 2^-13, a thirty-second of what a weight's rounding to bf16 takes.  Beyond, rows that hold a logit past the cap
// take the polynomial for their others.  (With that in all capped calls: 4624 rows of 28 heads, cap 20, 293 -> 340 us, cap 50 242 -> 252.)
constexpr float kWideCap = 256.f;
constexpr __device__ bool kShare(int i) { return (i & 3) == 3; }     // pairs of exponentials that go to the FMA pipe

template <int DH>
struct MmaShape {
    static constexpr int KB = DH / 64;                 // 128-byte pieces of a row
    static constexpr uint32_t kBlk = 128 * 128;        // bytes of a piece of a tile's 128 rows
    static constexpr uint32_t kTile = KB * kBlk;
    static constexpr int kStages = DH == 128 ? 4 : 8;  // K and V tiles on their way
    static constexpr uint32_t kStagePad = 2048;        // a rows' warp turns 32 columns of its output round in this
    static constexpr size_t kSmem = (size_t)(2 + kStages) * kTile + 8 * kStagePad + 1024;
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

// D[tmem] (+)= A[tmem] * B[smem], issued by ONE thread; the descriptor's upper word is that of umma_bf16_words.
__device__ __forceinline__ void umma_bf16_ts(uint32_t d_tmem, uint32_t a_tmem, uint32_t b_lo, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 db;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "mov.b64 db, {%2, %5};\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], db, %3, p;\n\t}"
        ::"r"(d_tmem), "r"(a_tmem), "r"(b_lo), "r"(idesc), "r"(accumulate), "r"(sm100::desc_k128_hi())
        : "memory");
}
// Lower word of V's descriptor as the second operand in its other order: a tile lies as rows (keys) of 128 swizzled bytes = 64 columns of
// the product; the next 64 columns follow blk_bytes on (leading offset), the next eight keys 1024 bytes on (stride, as in K's).
__device__ __forceinline__ uint32_t desc_v_lo(uint32_t smem_addr, uint32_t blk_bytes) { return ((smem_addr & 0x3FFFFu) >> 4) | ((blk_bytes >> 4) << 16); }
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

// 2^x on the FMA pipe (exp2_fma_pair): arguments outside [-125, 128] are held there.  2^-125 is taken off (rounded away beside what
// counts), so that a hidden key's weight is 0 and its V, however large, adds nothing.  At 128 the exponent's bits are those of +infinity:
// a NaN is held there too (a minimum takes the number of the two), and a sum of weights that is not finite is a row's sign of one.
__device__ __forceinline__ uint64_t exp2_held_pair(uint64_t x) {
    float a, b;
    sm100::unpair(x, a, b);
    a = fmaxf(fminf(a, 128.f), -125.f);
    b = fmaxf(fminf(b, 128.f), -125.f);
    return sm100::add_pair(sm100::exp2_fma_core(sm100::pair(a, b)), sm100::pair(-0x1p-125f, -0x1p-125f));
}
// The lesser of the two; NaN if one is.
__device__ __forceinline__ float min_nan(float a, float b) {
    float r;
    asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
// 16 registers of this thread's lane to 16 tensor-memory columns.
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};"
        ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
          "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(taddr)
        : "memory");
}

struct MmaMaps {
    CUtensorMap q, k, v;
    int k_step, v_step;                                // 1, or 0 where all K/V heads are the same rows
};

// x / rows_item for x up to 2^25 - 1 (rows_item <= 128: the host's reciprocal is exact there).
__device__ __forceinline__ int div_rows(const PromptArgs& a, int x) { return a.rows_item == 1 ? x : (int)__umulhi((uint32_t)x, a.rows_magic); }
// Item -> (block of rows, chunk of heads).
__device__ __forceinline__ int item_block(const PromptArgs& a, int item) { return a.head_chunks == 1 ? item : item / a.head_chunks; }

// A pair's place in its document, and what its items need.
struct Pair {
    int i0[2], h0[2], rows[2], n[2];                   // first row, first head (of the K/V head's), rows of the tile in use, key tiles
    int nt;                                            // key tiles of the pair
};
__device__ __forceinline__ int doc_items(const PromptArgs& a, int Lq) { return div_rows(a, Lq + a.rows_item - 1) * a.head_chunks; }
__device__ __forceinline__ Pair pair_of(const PromptArgs& a, const PromptDoc& d, int t) {
    Pair p;
    const int r = a.rows_item, items = doc_items(a, d.Lq);
    p.nt = 0;
#pragma unroll
    for (int x = 0; x < 2; ++x) {
        const int item = 2 * t + x;
        const bool there = item < items;
        const int blk = there ? item_block(a, item) : 0, ch = there ? item - blk * a.head_chunks : 0;
        p.i0[x] = blk * r;
        p.h0[x] = ch * a.heads_item;
        const int nr = there ? min(r, d.Lq - p.i0[x]) : 0;
        p.rows[x] = nr * a.heads_item;
        p.n[x] = there ? (prompt_keys(a, d, p.i0[x] + nr - 1) + kN - 1) / kN : 0;
        p.nt = max(p.nt, p.n[x]);
    }
    return p;
}
// Steps of a pair in the line: what it costs beside its key tiles (first, without work of their own), then the tiles; one at least.
__device__ __forceinline__ int pair_steps(const PromptArgs& a, const PromptDoc& d, int t) {
    const int last = item_block(a, min(2 * t + 1, doc_items(a, d.Lq) - 1)), r = a.rows_item;
    return max(1, a.pair_cost + (prompt_keys(a, d, min(d.Lq, (last + 1) * r) - 1) + kN - 1) / kN);
}
__device__ __forceinline__ int doc_pairs(const PromptArgs& a, int Lq) { return (doc_items(a, Lq) + 1) / 2; }

// A CTA's way along the line, pair by pair; the same in every warp.
struct Walk {
    PromptDoc d;
    int doc, g, t, pairs;                              // document, K/V head, pair, pairs of the document
    int e0;                                            // first step of the pair that is this CTA's
    long long left;                                    // steps still to do
};
__device__ __forceinline__ PromptDoc doc_of(const PromptArgs& a, int s) {
    PromptDoc d = {0, 0, a.n_q, a.n_k, a.prefix_len ? a.prefix_len[s] : 0, 0};
    if (a.seq_q) {
        d.q0 = a.seq_q[s];
        d.k0 = a.seq_k[s];
        d.Lq = a.seq_q[s + 1] - d.q0;
        d.Lk = a.seq_k[s + 1] - d.k0;
    }
    return d;
}
// Past the `steps` steps of this CTA's piece of the pair.
__device__ __forceinline__ void walk_on(const PromptArgs& a, Walk& w, int steps) {
    w.left -= steps;
    w.e0 = 0;
    if (w.left <= 0 || ++w.t < w.pairs) return;
    w.t = 0;
    do {                                               // steps are left: a document with rows comes
        if (++w.doc == a.n_seq) { w.doc = 0; ++w.g; }
        w.d = doc_of(a, w.doc);
        w.pairs = doc_pairs(a, w.d.Lq);
    } while (w.pairs == 0 && w.g < a.Hkv);
}

// The line of `all` steps in `ctas` pieces that differ by one step at most: the longer ones first.
struct Line {
    long long piece;
    int ctas, longer;
    __device__ __forceinline__ Line(long long all, int n) {
        ctas = (int)max(1LL, min((long long)n, all));
        piece = all < (1LL << 31) ? (long long)((uint32_t)all / (uint32_t)ctas) : all / ctas;
        longer = (int)(all - piece * ctas);
    }
    __device__ __forceinline__ long long begin(int c) const { return piece * c + min(c, longer); }
    __device__ __forceinline__ int holder(long long step) const {      // the CTA whose piece has the step
        const long long edge = (piece + 1) * longer;
        return step < edge ? (int)(step / (piece + 1)) : longer + (int)((step - edge) / piece);
    }
};

// What the second kernel joins: the parts of the pair that CTAs c0 .. c1 share, noted by CTA c0 + 1.
struct Cut {
    int c0, c1, first_slot;                            // c1 < 0: nothing; slot of CTA c0's part (the others' are their first ones)
    int q0, g, Lq, i0[2], h0[2], rows[2];
};

template <int DH, int kCap, bool kBias>
__global__ void __launch_bounds__(kThreads, 1)
prompt_attn_mma_kernel(const PromptArgs a, const __grid_constant__ MmaMaps maps) {
    using namespace sm100;
    using S = MmaShape<DH>;
    grid_dep_wait();
    extern __shared__ uint8_t smem_dyn[];
    __shared__ __align__(8) uint64_t q_bar, q_free_bar, full_bar[S::kStages], empty_bar[S::kStages], s_bar[2][2], p_bar[2][2], h_bar[2], o_bar[2], o_free_bar[2], drain_bar[2];
    __shared__ uint32_t s_tmem_base;
    __shared__ int s_abort;
    __shared__ __align__(16) float s_pos[2][2][kN];    // [item][buffer]: positions of the keys
    __shared__ Walk s_walk[8];                         // the rows' warps keep their way along the line here: in registers it would cost spills
    __shared__ int s_at[5];
    const int warp = __shfl_sync(0xFFFFFFFFu, (int)threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    const uint32_t smem_base = (smem_u32(smem_dyn) + 1023u) & ~1023u;
    auto q_addr = [&](int x) { return smem_base + (uint32_t)x * S::kTile; };
    auto kv_addr = [&](int s) { return smem_base + (uint32_t)(2 + s) * S::kTile; };
    Cut* cuts = reinterpret_cast<Cut*>(a.cuts);

    // ---- the line: steps of the documents before each (the tiles' memory serves for it), then this CTA's piece
    long long* s_pre = reinterpret_cast<long long*>(smem_dyn + (kv_addr(0) - smem_u32(smem_dyn)));
    int bad = 0;
    for (int s = threadIdx.x; a.seq_q && s < a.n_seq; s += kThreads) {
        const int q0 = a.seq_q[s], q1 = a.seq_q[s + 1], k0 = a.seq_k[s], k1 = a.seq_k[s + 1];
        bad |= q0 < 0 || q1 < q0 || q1 > a.n_q || k0 < 0 || k1 < k0 || k1 > a.n_k;
    }
    if (a.seq_q) bad = __syncthreads_or(bad);
    if (threadIdx.x == 0) {
        if (blockIdx.x == 0) *a.status = bad ? METOK_ERR_INVALID_ARG : METOK_OK;
        cuts[blockIdx.x].c1 = -1;
    }
    if (bad) return;
    for (int s = warp; s < a.n_seq; s += kThreads / 32) {
        const PromptDoc d = doc_of(a, s);
        const int pairs = doc_pairs(a, d.Lq);
        long long sum = 0;
        for (int t = lane; t < pairs; t += 32) sum += pair_steps(a, d, t);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
        if (lane == 0) s_pre[s + 1] = sum;
    }
    if (threadIdx.x == 0) s_pre[0] = 0;
    __syncthreads();
    if (warp == 0 && a.n_seq > 1) {                    // running sums, a run of documents per lane
        const int per = (a.n_seq + 31) / 32, s0 = lane * per, s1 = min(a.n_seq, s0 + per);
        long long sum = 0;
        for (int s = s0; s < s1; ++s) sum += s_pre[s + 1];
        long long incl = sum;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long x = __shfl_up_sync(0xFFFFFFFFu, incl, o);
            if (lane >= o) incl += x;
        }
        long long run = incl - sum;
        for (int s = s0; s < s1; ++s) {
            run += s_pre[s + 1];
            s_pre[s + 1] = run;
        }
    }
    __syncthreads();
    const long long per_head = s_pre[a.n_seq], all = per_head * a.Hkv;
    if (all == 0) return;                              // uniform, as below
    const Line line(all, gridDim.x);
    if (blockIdx.x >= line.ctas) return;
    const long long begin = line.begin(blockIdx.x), end = line.begin(blockIdx.x + 1);
    if (warp < 2) {                                    // the pair where it begins (0), and where it ends (1)
        const long long edge = warp ? end : begin;
        int g = 0;
        if (a.Hkv > 1) g = all < (1LL << 31) ? (int)((uint32_t)edge / (uint32_t)per_head) : (int)(edge / per_head);
        const long long at = warp && edge == all ? 0 : edge - g * per_head;
        int lo = 0, hi = a.n_seq;                      // the document: s_pre[lo] <= at < s_pre[hi]
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (s_pre[mid] <= at) lo = mid;
            else hi = mid;
        }
        const PromptDoc d = doc_of(a, lo);
        const int pairs = doc_pairs(a, d.Lq);
        int rest = 0;
        long long before = s_pre[lo];
        int t0 = 0;
        for (; t0 < pairs; t0 += 32) {
            const int mine = t0 + lane < pairs ? pair_steps(a, d, t0 + lane) : 0;
            int incl = mine;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int x = __shfl_up_sync(0xFFFFFFFFu, incl, o);
                if (lane >= o) incl += x;
            }
            const uint32_t any = __ballot_sync(0xFFFFFFFFu, before + incl > at);
            if (any) {
                const int l = __ffs(any) - 1;
                rest = (int)(at - before) - __shfl_sync(0xFFFFFFFFu, incl - mine, l);
                t0 += l;
                break;
            }
            before += __shfl_sync(0xFFFFFFFFu, incl, 31);
        }
        if (lane == 0 && warp) {
            s_at[4] = rest;
        } else if (lane == 0) {
            s_at[0] = g;
            s_at[1] = lo;
            s_at[2] = t0;
            s_at[3] = rest;
        }
    }
    fence_proxy_async();                               // what was written here by threads, before copies write it
    __syncthreads();
    Walk walk;
    walk.g = s_at[0];
    walk.doc = s_at[1];
    walk.t = s_at[2];
    walk.e0 = s_at[3];
    walk.d = doc_of(a, walk.doc);
    walk.pairs = doc_pairs(a, walk.d.Lq);
    // A pair is not cut within its cost (a part without tiles would be no help, and pairs of one tile stay whole): such a cut is moved to the
    // pair's first step.
    walk.left = end - begin + (walk.e0 <= a.pair_cost ? walk.e0 : 0) - (s_at[4] <= a.pair_cost ? s_at[4] : 0);
    if (walk.e0 <= a.pair_cost) walk.e0 = 0;

    if (threadIdx.x == 0) {
        mbar_init(smem_u32(&q_bar), 1);
        mbar_init(smem_u32(&q_free_bar), 2);
        mbar_init(smem_u32(&drain_bar[0]), 1);
        mbar_init(smem_u32(&drain_bar[1]), 1);
        for (int s = 0; s < S::kStages; ++s) { mbar_init(smem_u32(&full_bar[s]), 1); mbar_init(smem_u32(&empty_bar[s]), 2); }
        for (int x = 0; x < 2; ++x) {
            mbar_init(smem_u32(&o_bar[x]), 1);
            mbar_init(smem_u32(&h_bar[x]), 1);
            mbar_init(smem_u32(&o_free_bar[x]), 4);
            for (int p = 0; p < 2; ++p) { mbar_init(smem_u32(&s_bar[x][p]), 1); mbar_init(smem_u32(&p_bar[x][p]), 4); }
        }
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

    // this CTA's part of the walk's pair: steps e0 .. e1 - 1, with key tiles lo + nt - 1 down to lo; item x joins in at tile st[x] of them
    struct Part {
        Pair p;
        int steps, lo, nt, st[2];
        bool whole;
    };
    auto part_of = [&](const Walk& w) {
        Part q;
        q.p = pair_of(a, w.d, w.t);
        const int steps = max(1, q.p.nt + a.pair_cost);
        q.steps = (int)min((long long)(steps - w.e0), w.left);
        q.whole = q.steps == steps;
        const int t0 = max(0, w.e0 - a.pair_cost), t1 = max(0, w.e0 + q.steps - a.pair_cost);
        q.lo = max(0, q.p.nt - t1);
        q.nt = q.p.nt ? t1 - t0 : 0;
#pragma unroll
        for (int x = 0; x < 2; ++x) q.st[x] = q.nt - max(0, min(q.p.n[x] - q.lo, q.nt));
        return q;
    };
    auto tile_key = [](int top, int j) { return (top - j) * kN; };       // `top`: the part's highest key tile
    // (into the warp's uniform registers, which a product's descriptors are made in)
    auto uniform = [](int v) { return __reduce_max_sync(0xFFFFFFFFu, v); };

    if (warp == 8) {
        // ---- TMA: per part Q of both items, then K and V tiles in turn
        int it = 0, np = 0;
        bool ok = true;
        if (elect_one()) { prefetch_tmap(&maps.q); prefetch_tmap(&maps.k); prefetch_tmap(&maps.v); }
        __syncwarp();
        while (ok && walk.left > 0) {
            const Part q = part_of(walk);
            const int nt = uniform(q.nt), top = uniform(q.lo + q.nt - 1), k0 = uniform(walk.d.k0), gk = uniform(walk.g * maps.k_step), gv = uniform(walk.g * maps.v_step);
            if (nt > 0) {
                if (!mbar_wait_warp(smem_u32(&q_free_bar), (uint32_t)(np & 1) ^ 1u, abort_flag)) { ok = false; break; }
                if (elect_one()) {
                    const int both = q.p.rows[1] > 0 ? 2 : 1;
                    mbar_arrive_expect_tx(smem_u32(&q_bar), (uint32_t)both * S::KB * (uint32_t)(a.rows_item * a.heads_item) * 128u);
#pragma unroll
                    for (int x = 0; x < 2; ++x)
                        if (x < both) {
#pragma unroll
                            for (int kb = 0; kb < S::KB; ++kb)
                                tma_load_3d(q_addr(x) + kb * S::kBlk, &maps.q, kb * 64, walk.g * a.G + q.p.h0[x], walk.d.q0 + q.p.i0[x], smem_u32(&q_bar));
                        }
                }
                __syncwarp();
                ++np;
                for (int j = 0; ok && j < 2 * nt; ++j, ++it) {
                    const int s = it % S::kStages, row = k0 + tile_key(top, j >> 1);
                    if (!mbar_wait_warp(smem_u32(&empty_bar[s]), ((uint32_t)(it / S::kStages) & 1u) ^ 1u, abort_flag)) { ok = false; break; }
                    if (elect_one()) {
                        const uint32_t fb = smem_u32(&full_bar[s]);
                        mbar_arrive_expect_tx(fb, S::kTile);
                        const bool held = dbg_held(a.withhold, kDbgPromptAttn) && blockIdx.x == 0 && it == 0;       // debug builds: one copy never sent
#pragma unroll
                        for (int kb = 0; kb < S::KB && !held; ++kb) {
                            if (j & 1) tma_load_3d(kv_addr(s) + kb * S::kBlk, &maps.v, kb * 64, row, gv, fb);
                            else tma_load_3d(kv_addr(s) + kb * S::kBlk, &maps.k, kb * 64, row, gk, fb);
                        }
                    }
                    __syncwarp();
                }
            }
            walk_on(a, walk, q.steps);
        }
        // every copy has landed before the shared memory goes away
        if (np > 0) mbar_wait_warp(smem_u32(&q_bar), (uint32_t)(np - 1) & 1u, abort_flag);
        for (int back = 1; back <= S::kStages && back <= it; ++back) {
            const int j = it - back;
            mbar_wait_warp(smem_u32(&full_bar[j % S::kStages]), (uint32_t)(j / S::kStages) & 1u, abort_flag);
        }
    } else if (warp >= 9) {
        // ---- products of item x
        constexpr uint32_t idesc_s = make_idesc_bf16(kM, kN / 2), idesc_o = make_idesc_bf16(kM, DH) | (1u << 16);
        const int x = warp - 9;
        const uint32_t t_s = tmem + (uint32_t)x * kN, t_o = tmem + 2 * kN + (uint32_t)x * DH;
        const uint32_t q_lo = desc_k128_lo(q_addr(x)), k_lo0 = desc_k128_lo(kv_addr(0)), v_lo0 = desc_v_lo(kv_addr(0), S::kBlk);
        bool ok = true;
        int it0 = 0, np = 0, tiles = 0, outs = 0;      // key and value tiles, parts, the item's tiles and outputs so far
        auto wait_full = [&](int it) { return mbar_wait_warp(smem_u32(&full_bar[it % S::kStages]), (uint32_t)(it / S::kStages) & 1u, abort_flag); };
        while (ok && walk.left > 0) {
            const Part q = part_of(walk);
            const int nt = uniform(q.nt), top = uniform(q.lo + q.nt - 1), st = uniform(x ? q.st[1] : q.st[0]), Lk = uniform(walk.d.Lk);
            auto logits = [&](int it, int half) {      // S of 64 keys of the tile at `it`
                const uint32_t k_lo = k_lo0 + (uint32_t)(it % S::kStages) * (S::kTile >> 4) + (uint32_t)half * 512u;
                if (elect_one()) {
#pragma unroll
                    for (int kk = 0; kk < DH / 16; ++kk) {
                        constexpr uint32_t kNext = S::kBlk >> 4;
                        umma_bf16_words(t_s + half * 64, q_lo + (kk >> 2) * kNext + (kk & 3) * 2, k_lo + (kk >> 2) * kNext + (kk & 3) * 2, idesc_s, kk != 0 ? 1u : 0u);
                    }
                    umma_commit(smem_u32(&s_bar[x][half]));
                    if (half) umma_commit(smem_u32(&empty_bar[it % S::kStages]));
                }
                __syncwarp();
            };
            // a tile that the item does not take part in: the other one does
            auto pass = [&](int it) {
                if (!wait_full(it)) return false;
                if (lane == 0) mbar_arrive(smem_u32(&empty_bar[it % S::kStages]));
                __syncwarp();
                return true;
            };
            if (nt > 0) {
                for (int j = 0; ok && j < 2 * min(st, nt); ++j) ok = pass(it0 + j);
                if (ok && st < nt) {
                    ok = mbar_wait_warp(smem_u32(&q_bar), (uint32_t)np & 1u, abort_flag) && wait_full(it0 + 2 * st);
                    if (ok) {
                        tc_fence_after();
                        logits(it0 + 2 * st, 0);
                        logits(it0 + 2 * st, 1);
                    }
                }
                for (int j = st; ok && j < nt; ++j) {
                    const int vi = it0 + 2 * j + 1, vs = vi % S::kStages, seen = tiles + j - st;
                    if (!(ok = wait_full(vi))) break;
                    const int left = Lk - tile_key(top, j);        // rows of the document in this tile
                    if (left < kN) {                   // those behind count as zeros, whatever they hold (both items' warps write them)
                        for (int c = lane; c < (kN - left) * S::KB * 8; c += 32) {
                            const int r = left + c / (S::KB * 8), e = c % (S::KB * 8);
                            asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(kv_addr(vs) + (uint32_t)(e >> 3) * S::kBlk + (uint32_t)r * 128u + (uint32_t)(e & 7) * 16u), "r"(0) : "memory");
                        }
                        fence_proxy_async();
                        __syncwarp();
                    }
                    // the rows have taken the output of the part before
                    if (j == st && !(ok = mbar_wait_warp(smem_u32(&o_free_bar[x]), (uint32_t)(outs & 1) ^ 1u, abort_flag))) break;
                    const uint32_t v_lo = v_lo0 + (uint32_t)vs * (S::kTile >> 4);
#pragma unroll
                    for (int half = 0; half < 2; ++half) {         // O += P V of 64 keys; then the next tile's logits go to their place
                        if (!(ok = mbar_wait_warp(smem_u32(&p_bar[x][half]), (uint32_t)seen & 1u, abort_flag))) break;
                        tc_fence_after();
                        if (elect_one()) {
#pragma unroll
                            for (int kk = 0; kk < 4; ++kk)
                                umma_bf16_ts(t_o, t_s + half * 64 + kk * 8, v_lo + (half * 4 + kk) * 128, idesc_o, half || kk > 0 || j > st ? 1u : 0u);
                            umma_commit(smem_u32(&h_bar[x]));
                            if (half) umma_commit(smem_u32(&empty_bar[vs]));
                            if (half && j + 1 == nt) umma_commit(smem_u32(&o_bar[x]));
                        }
                        __syncwarp();
                        if (j + 1 < nt) {
                            if (!half && !(ok = wait_full(vi + 1))) break;
                            logits(vi + 1, half);
                        }
                    }
                }
                // Q has been read, or was not wanted
                if (ok) {
                    if (st < nt) {
                        if (elect_one()) umma_commit(smem_u32(&q_free_bar));
                    } else if (mbar_wait_warp(smem_u32(&q_bar), (uint32_t)np & 1u, abort_flag)) {
                        if (lane == 0) mbar_arrive(smem_u32(&q_free_bar));
                    } else {
                        ok = false;
                    }
                    __syncwarp();
                }
                ++np;
                it0 += 2 * nt;
                tiles += max(0, nt - st);
                outs += st < nt;
            }
            walk_on(a, walk, q.steps);
        }
        if (!ok) {                                     // whatever was issued has retired before the tensor memory goes
            if (elect_one()) umma_commit(smem_u32(&drain_bar[x]));
            __syncwarp();
            mbar_wait_warp(smem_u32(&drain_bar[x]), 0u, abort_flag);
        }
    } else {
        // ---- rows
        const int x = warp >> 2, quad = warp & 3, r = quad * 32 + lane;
        const uint32_t lane_base = (uint32_t)(quad * 32) << 16;
        const uint32_t t_s = tmem + lane_base + (uint32_t)x * kN, t_o = tmem + lane_base + 2 * kN + (uint32_t)x * DH;
        const float ninf = __int_as_float(0xFF800000);
        const int my_i = r / a.heads_item, my_h = r - my_i * a.heads_item;      // row and head of the tile
        bool ok = true, first_part = true;
        int seen = 0, outs = 0;                        // tiles and outputs of this item so far
        Walk* my_walk = &s_walk[warp];
        if (lane == 0) *my_walk = walk;
        __syncwarp();
        while (my_walk->left > 0) {
        // what the tiles' loop needs; the rest is worked out again behind it
        int my_n, my_lo, keys, sure, k_first, k_rows;  // tiles, the lowest of them, keys that the row and that all rows of the item see; the document's keys
        float slope = 0.f, my_pos = 0.f, next_pos = 0.f;
        {
            const PromptDoc d = my_walk->d;
            const Part q = part_of(*my_walk);
            const int i0 = x ? q.p.i0[1] : q.p.i0[0], h0 = x ? q.p.h0[1] : q.p.h0[0], rows = x ? q.p.rows[1] : q.p.rows[0];
            my_n = q.nt - (x ? q.st[1] : q.st[0]);
            my_lo = q.lo;
            const bool mine = r < rows && h0 + my_h < a.G;
            keys = mine ? prompt_keys(a, d, i0 + my_i) : 0;
            sure = rows > 0 ? prompt_keys(a, d, i0) : 0;
            k_first = d.k0;
            k_rows = d.Lk;
            if (kBias && my_n > 0) {
                slope = mine ? a.slopes[my_walk->g * a.G + h0 + my_h] * kAttnLog2e : 0.f;
                my_pos = prompt_position(a, d.k0, d.Lk, d.Lk - d.Lq + i0 + my_i);
                next_pos = prompt_position(a, k_first, k_rows, (my_lo + my_n - 1) * kN + r);
            }
        }
        float m = ninf, l = 0.f;
        for (int j = 0; j < my_n; ++j, ++seen) {
            const int k0 = (my_lo + my_n - 1 - j) * kN;
            if constexpr (kBias) {                     // (two buffers: who writes one again has met the others since it was read)
                s_pos[x][seen & 1][r] = next_pos;
                next_pos = prompt_position(a, k_first, k_rows, k0 - kN + r);
                named_bar_sync(1 + x, 128);
            }
            const bool masked = k0 + kN > sure;
            const bool full = __any_sync(0xFFFFFFFFu, keys > 0 && l >= kMost);       // (looked up while the logits are on their way)
#pragma unroll 1                                       // (one copy of the code: the instruction cache is short)
            for (int half = 0; half < 2; ++half) {     // 64 keys
                if (ok && !mbar_wait(smem_u32(&s_bar[x][half]), (uint32_t)seen & 1u, abort_flag)) ok = false;
                ok = __all_sync(0xFFFFFFFFu, ok);
                if (!ok) continue;                     // (keeps meeting the item's other warps where they meet)
                tc_fence_after();
                // whether a reference is wanted: at the first keys that a row sees, and where the weights came out too large for the one there is
                bool check = full || __any_sync(0xFFFFFFFFu, m == ninf && keys > k0 + half * 64), again = false;
                uint32_t p[32];
                float sum;
#pragma unroll 1
                for (;;) {
                    const float base = m == ninf || again ? 0.f : m;     // (again: a reference far from the logits would cost them digits)
                    uint32_t raw[2][32];
                    tmem_ld32_issue(t_s + half * 64, raw[0]);
                    tmem_ld32_issue(t_s + half * 64 + 32, raw[1]);
                    tmem_ld32_wait(raw[0]);
                    tmem_ld32_wait(raw[1]);
                    uint64_t v[32];                    // logits in log2 units less the reference, in pairs
#pragma unroll
                    for (int i = 0; i < 32; ++i) v[i] = pair(__uint_as_float(raw[i >> 4][2 * (i & 15)]), __uint_as_float(raw[i >> 4][2 * (i & 15) + 1]));
                    const uint64_t low = pair(-base, -base);
                    if constexpr (kCap) {
                        // y = product * scale / cap.  Up to |y| = 1 tanh(y) = y P(y^2), P the polynomial of degree 6 of least largest error (2e-8; 1e-7 in
                        // fp32), with the cap in its coefficients; where a warp has one beyond, 1 - 2 / (1 + e^2y), of which every part costs the
                        // special-function unit a step.
                        auto near = [&](uint64_t y) {
                            const uint64_t u = mul_pair(y, y);
                            uint64_t t = pair(a.cap_poly[6], a.cap_poly[6]);
#pragma unroll
                            for (int c = 5; c >= 0; --c) t = fma_pair(t, u, pair(a.cap_poly[c], a.cap_poly[c]));
                            return fma_pair(y, t, low);
                        };
                        float most = 0.f;
#pragma unroll
                        for (int i = 0; i < 32; ++i) {
                            v[i] = mul_pair(v[i], pair(a.cap_scale, a.cap_scale));
                            float y0, y1;
                            unpair(v[i], y0, y1);
                            most = fmaxf(most, fmaxf(fabsf(y0), fabsf(y1)));
                        }
                        if (__any_sync(0xFFFFFFFFu, !(most <= 1.f))) {
#pragma unroll
                            for (int i = 0; i < 32; ++i) {
                                float y0, y1, near0, near1;
                                unpair(v[i], y0, y1);
                                const bool far0 = !(fabsf(y0) <= 1.f), far1 = !(fabsf(y1) <= 1.f);
                                if constexpr (kCap == 2) unpair(near(v[i]), near0, near1);
                                y0 = (a.cap_log2 - base) - __fdividef(2.f * a.cap_log2, 1.f + fast_exp2(min_nan(y0 * (2.f * kAttnLog2e), 80.f)));
                                y1 = (a.cap_log2 - base) - __fdividef(2.f * a.cap_log2, 1.f + fast_exp2(min_nan(y1 * (2.f * kAttnLog2e), 80.f)));
                                v[i] = kCap == 1 ? pair(y0, y1) : pair(far0 ? y0 : near0, far1 ? y1 : near1);
                            }
                        } else {
#pragma unroll
                            for (int i = 0; i < 32; ++i) v[i] = near(v[i]);
                        }
                    } else {
#pragma unroll
                        for (int i = 0; i < 32; ++i) v[i] = fma_pair(v[i], pair(a.scale_log2, a.scale_log2), low);
                    }
                    if constexpr (kBias) {
#pragma unroll
                        for (int i = 0; i < 32; i += 2) {
                            const float4 at = *reinterpret_cast<const float4*>(&s_pos[x][seen & 1][half * 64 + 2 * i]);
                            float v0, v1, v2, v3;
                            unpair(v[i], v0, v1);
                            unpair(v[i + 1], v2, v3);
                            v[i] = pair(fmaf(-slope, fabsf(my_pos - at.x), v0), fmaf(-slope, fabsf(my_pos - at.y), v1));
                            v[i + 1] = pair(fmaf(-slope, fabsf(my_pos - at.z), v2), fmaf(-slope, fabsf(my_pos - at.w), v3));
                        }
                    }
                    if (masked) {                      // keys that the row does not see
                        const int see = keys - k0 - half * 64;
#pragma unroll
                        for (int i = 0; i < 32; ++i) {
                            float v0, v1;
                            unpair(v[i], v0, v1);
                            v[i] = pair(2 * i < see ? v0 : ninf, 2 * i + 1 < see ? v1 : ninf);
                        }
                    }
                    if (check) {
                        float top[4] = {ninf, ninf, ninf, ninf};
#pragma unroll
                        for (int i = 0; i < 32; ++i) {
                            float v0, v1;
                            unpair(v[i], v0, v1);
                            top[i & 3] = fmaxf(top[i & 3], fmaxf(v0, v1));
                        }
                        const float mx = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3])) + base;
                        const bool grow = keys > 0 && (again ? mx > m + kGrow : m == ninf ? mx > ninf : l >= kMost);
                        const float higher = fmaxf(mx, m + kGrow), f = grow ? fast_exp2(m - higher) : 1.f;
                        if (grow) m = higher;
                        l *= f;
                        const float off = m == ninf ? 0.f : base - m;
                        const uint64_t less = pair(off, off);
#pragma unroll
                        for (int i = 0; i < 32; ++i) v[i] = add_pair(v[i], less);
                        if (j > 0 || half) {           // when the product before this one on O_x is complete
                            if (!mbar_wait(smem_u32(&h_bar[x]), (uint32_t)(half ^ 1), abort_flag)) ok = false;
                            ok = __all_sync(0xFFFFFFFFu, ok);
                            tc_fence_after();
#pragma unroll 1
                            for (int c = 0; c < DH / 16; ++c) {
                                float o[16];
                                tmem_ld16(t_o + c * 16, o);
                                uint32_t w[16];
#pragma unroll
                                for (int i = 0; i < 16; ++i) w[i] = __float_as_uint(o[i] * f);
                                tmem_st16(t_o + c * 16, w);
                            }
                        }
                    }
                    // A weight is one bf16 value in the product, the type of V there, while the sum that divides them is of unrounded ones.  Beside
                    // the outputs' own rounding (1.7e-3 of them) this leaves errors of 1.9e-3 to 2.4e-3.  A second part for what is rounded off
                    // would take half as many products again, which bound heads of 128; a sum of the rounded weights was measured: 269 -> 285 us
                    // for errors 1.16 times the outputs' rounding instead of 1.23.
                    uint64_t sum0 = 0ull, sum1 = 0ull;
#pragma unroll
                    for (int i = 0; i < 32; ++i) {
                        // some on the FMA pipe, so that both work
                        const uint64_t w = kShare(i) ? exp2_held_pair(v[i]) : exp2_pair(v[i]);
                        if (i & 1) sum1 = add_pair(sum1, w);
                        else sum0 = add_pair(sum0, w);
                        float w0, w1;
                        unpair(w, w0, w1);
                        p[i] = pack_bf16(w0, w1);
                    }
                    float s0, s1;
                    unpair(add_pair(sum0, sum1), s0, s1);
                    sum = s0 + s1;
                    if (again || !__any_sync(0xFFFFFFFFu, keys > 0 && !(sum < kMost))) break;      // (a tile's unused rows may hold anything)
                    check = again = true;              // once
                }
                l += sum;
                tmem_st32(t_s + half * 64, p);         // their product may begin
                tmem_st_wait();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&p_bar[x][half]));
            }
        }
        // A row that has seen no key has m = -infinity and l = 0.  Weights are finite where logits are, so a sum that is not comes of a NaN or
        // +infinity among them: out and lse become NaN, here or in the join.
        if (!(l < __int_as_float(0x7F800000))) l = __int_as_float(0x7FFFFFFF);
        if (my_n > 0 && ok && !mbar_wait(smem_u32(&o_bar[x]), (uint32_t)outs & 1u, abort_flag)) ok = false;
        ok = __all_sync(0xFFFFFFFFu, ok);
        tc_fence_after();
        const PromptDoc d = my_walk->d;
        const Part part = part_of(*my_walk);
        const int my_i0 = x ? part.p.i0[1] : part.p.i0[0], h0 = x ? part.p.h0[1] : part.p.h0[0], my_head = my_walk->g * a.G + h0 + my_h;
        const bool mine = r < (x ? part.p.rows[1] : part.p.rows[0]) && h0 + my_h < a.G, whole = part.whole;
        const long long row = d.q0 + my_i0 + my_i;
        // partial outputs lie [slot][16-byte piece][row]: a warp's rows side by side
        const long long slot = 2LL * blockIdx.x + (first_part ? 0 : 1), at = slot * (2 * kM) + x * kM + r;
        if (ok && !whole && my_n > 0) {
            float4* part_o = reinterpret_cast<float4*>(a.part_o) + slot * (2 * kM) * (DH / 4) + x * kM + r;
#pragma unroll 1                                       // (code that runs once per part comes from memory: short is fast)
            for (int c = 0; c < DH / 16; ++c) {
                float o[16];
                tmem_ld16(t_o + c * 16, o);
                if (mine) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) part_o[(c * 4 + i) * (2 * kM)] = make_float4(o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]);
                }
            }
        }
        if (ok && whole) {
            // 32 columns at a time through shared memory, so that four lanes write 64 bytes of a row (each lane its own row: a store instruction
            // of 32 lines, 4 us a part)
            const float scale = l == 0.f ? 0.f : 1.f / l;
            const long long to = mine ? (long long)my_head * a.out_head + row * a.out_row : -1;
            const uint32_t pad = smem_base + (2 + S::kStages) * S::kTile + (uint32_t)warp * S::kStagePad;
            long long dst[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) dst[i] = __shfl_sync(0xFFFFFFFFu, to, i * 8 + (lane >> 2));
#pragma unroll 1
            for (int c = 0; c < DH / 32; ++c) {
                float o[32];
                if (my_n > 0) {
                    tmem_ld32(t_o + c * 32, o);
                } else {
#pragma unroll
                    for (int i = 0; i < 32; ++i) o[i] = 0.f;
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float* v = o + 8 * i;
                    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(pad + (uint32_t)(lane * 64 + ((i ^ ((lane >> 1) & 3)) << 4))),
                                 "r"(pack_bf16(v[0] * scale, v[1] * scale)), "r"(pack_bf16(v[2] * scale, v[3] * scale)), "r"(pack_bf16(v[4] * scale, v[5] * scale)),
                                 "r"(pack_bf16(v[6] * scale, v[7] * scale)) : "memory");
                }
                __syncwarp();
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int rr = i * 8 + (lane >> 2), e = lane & 3;
                    uint4 v;
                    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
                                 : "r"(pad + (uint32_t)(rr * 64 + ((e ^ ((rr >> 1) & 3)) << 4))) : "memory");
                    if (dst[i] >= 0) *reinterpret_cast<uint4*>(reinterpret_cast<__nv_bfloat16*>(a.out) + dst[i] + c * 32 + e * 8) = v;
                }
                __syncwarp();
            }
        }
        if (ok) {
            if (mine && !whole) *reinterpret_cast<float2*>(a.part_ml + at * 2) = make_float2(m, l);
            else if (mine && a.lse) a.lse[(long long)my_head * a.n_q + row] = kAttnLn2 * (m + log2f(l));
        }
        if (my_n > 0) {                                // O_x may be written again
            ++outs;
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&o_free_bar[x]));
        }
        // a pair that began in another CTA: the second of those that share it notes what there is to join
        if (threadIdx.x == 0 && first_part && my_walk->e0 > 0) {
            const int steps = max(1, part.p.nt + a.pair_cost);
            const long long f0 = begin - my_walk->e0;  // the pair's place in the line
            const int c0 = line.holder(f0 + a.pair_cost), c1 = line.holder(f0 + steps - 1);
            if (c0 + 1 == blockIdx.x) {
                Cut cut;
                cut.c0 = c0;
                cut.c1 = c1;
                cut.first_slot = 2 * c0 + (line.begin(c0) >= f0 ? 0 : 1);
                cut.q0 = d.q0;
                cut.g = my_walk->g;
                cut.Lq = d.Lq;
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    cut.i0[y] = part.p.i0[y];
                    cut.h0[y] = part.p.h0[y];
                    cut.rows[y] = part.p.rows[y];
                }
                cuts[blockIdx.x] = cut;
            }
        }
        first_part = false;
        __syncwarp();
        if (lane == 0) walk_on(a, *my_walk, part.steps);
        __syncwarp();
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 9) tmem_dealloc(tmem, 512);
    if (threadIdx.x == 0 && s_abort) *a.status = METOK_ERR_TIMEOUT;
}

// Joins the parts of the pairs that were cut: blockIdx.x is the CTA that noted the cut.  A lane per row, a warp for kCutPieces 16-byte
// pieces of 32 rows' outputs, kAhead parts on their way (four pieces and two parts, on half as many CTAs: 28 heads of 64 rows over 18 496 keys,
// which leave 18 parts a pair, 14.7 -> 12.9 us; two pieces with eight parts take 8 us longer where there are many pairs).
constexpr int kCutBlocks = 2 * kM / 32, kCutPieces = 2, kAhead = 4;
template <int DH>
__global__ void __launch_bounds__(256)
prompt_cut_join_kernel(const PromptArgs a) {
    grid_dep_wait();
    const Cut cut = reinterpret_cast<const Cut*>(a.cuts)[blockIdx.x];
    if (cut.c1 < 0) return;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, rr = (blockIdx.y % kCutBlocks) * 32 + lane, x = rr / kM, r = rr - x * kM;
    const int i = r / a.heads_item, h = (x ? cut.h0[1] : cut.h0[0]) + r - i * a.heads_item;
    if (r >= (x ? cut.rows[1] : cut.rows[0]) || h >= a.G) return;
    const int parts = cut.c1 - cut.c0 + 1, head = cut.g * a.G + h;
    const long long row = cut.q0 + (x ? cut.i0[1] : cut.i0[0]) + i;
    auto slot = [&](int p) { return (size_t)(p == 0 ? cut.first_slot : 2 * (cut.c0 + p)); };
    const float ninf = __int_as_float(0xFF800000);
    constexpr int E = kCutPieces;
    const int piece = (blockIdx.y / kCutBlocks * 8 + warp) * E;
    // A part's sum is below 2^26 and there are fewer than 2^8 of them: with a 2^8th of each, their sum * V is in range too.
    constexpr float kLess = 0x1p-8f;
    static_assert(kNumSMs < 256);
    float M = ninf, L = 0.f;
    float4 acc[E];
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int p0 = 0; p0 < parts; p0 += kAhead) {
        float2 ml[kAhead];
        float4 o[kAhead][E];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const bool in = p0 + u < parts;
            ml[u] = in ? *reinterpret_cast<const float2*>(a.part_ml + (slot(p0 + u) * (2 * kM) + rr) * 2) : make_float2(ninf, 0.f);
#pragma unroll
            for (int e = 0; e < E; ++e)
                o[u][e] = in ? reinterpret_cast<const float4*>(a.part_o)[(slot(p0 + u) * (DH / 4) + piece + e) * (2 * kM) + rr] : make_float4(0.f, 0.f, 0.f, 0.f);
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            if (ml[u].y == 0.f) continue;              // a part of no keys has written no output (one of NaN has)
            const float top = fmaxf(M, ml[u].x), f = sm100::fast_exp2(M - top), g = sm100::fast_exp2(ml[u].x - top) * kLess;
            M = top;
            L = L * f + ml[u].y * g;
#pragma unroll
            for (int e = 0; e < E; ++e)
                acc[e] = make_float4(acc[e].x * f + o[u][e].x * g, acc[e].y * f + o[u][e].y * g, acc[e].z * f + o[u][e].z * g, acc[e].w * f + o[u][e].w * g);
        }
    }
    const float inv = L == 0.f ? 0.f : 1.f / L;
    __nv_bfloat16* out = reinterpret_cast<__nv_bfloat16*>(a.out) + (long long)head * a.out_head + row * a.out_row;
#pragma unroll
    for (int e = 0; e < E; e += 2)
        reinterpret_cast<uint4*>(out)[(piece + e) / 2] = make_uint4(pack_bf16(acc[e].x * inv, acc[e].y * inv), pack_bf16(acc[e].z * inv, acc[e].w * inv),
                                                                       pack_bf16(acc[e + 1].x * inv, acc[e + 1].y * inv), pack_bf16(acc[e + 1].z * inv, acc[e + 1].w * inv));
    if (piece == 0 && a.lse) a.lse[(long long)head * a.n_q + row] = kAttnLn2 * (M + log2f(L * (1.f / kLess)));
}

template <int DH, int kCap, bool kBias>
int launch(const PromptArgs& a, const MmaMaps& maps, cudaStream_t st) {
    auto kern = prompt_attn_mma_kernel<DH, kCap, kBias>;
    METOK_ALLOW_SMEM(kern, MmaShape<DH>::kSmem);
    {
        METOK_TIMED("prompt_attn_mma", st);
        launch_chained(kern, dim3(kNumSMs), dim3(kThreads), MmaShape<DH>::kSmem, st, a, maps);
    }
    METOK_LAUNCH_CHECK();
    if (a.n_k > kN) {                                  // (pairs of one step are never cut)
        METOK_TIMED("prompt_cut_join", st);
        launch_chained(prompt_cut_join_kernel<DH>, dim3(kNumSMs, kCutBlocks * (DH / 32 / kCutPieces)), dim3(256), 0, st, a);
        METOK_LAUNCH_CHECK();
    }
    return METOK_OK;
}
template <int DH>
int launch_dh(const PromptArgs& a, const MmaMaps& maps, cudaStream_t st) {
    if (a.cap_log2 > kWideCap * kAttnLog2e) return a.slopes ? launch<DH, 2, true>(a, maps, st) : launch<DH, 2, false>(a, maps, st);
    if (a.cap_log2 > 0.f) return a.slopes ? launch<DH, 1, true>(a, maps, st) : launch<DH, 1, false>(a, maps, st);
    return a.slopes ? launch<DH, 0, true>(a, maps, st) : launch<DH, 0, false>(a, maps, st);
}

}  // namespace

void prompt_mma_carve(Carver& cv, const metok_attention_params* p, PromptArgs* a) {
    a->cuts = cv.take<Cut>(kNumSMs);
    if (p->n_k <= kN) return;                          // pairs of one step are never cut
    a->part_ml = cv.take<float>((size_t)2 * kNumSMs * 2 * kM * 2);
    a->part_o = cv.take<float>((size_t)2 * kNumSMs * 2 * kM * p->dh);
}

int launch_prompt_attn_mma(PromptArgs a, int dh, cudaStream_t st) {
    MmaMaps maps = {};
    a.heads_item = std::min(a.G, kM);
    a.rows_item = kM / a.heads_item;
    // tanh(y) / y in powers of y^2, |y| <= 1: least largest error of y times it
    constexpr double kTanh[7] = {0.999999693, -0.333321293, 0.133195837, -0.0532658353, 0.0199732827, -0.00595128048, 0.000963772187};
    for (int c = 0; c < 7; ++c) a.cap_poly[c] = (float)(kTanh[c] * a.cap_log2);
    a.rows_magic = a.rows_item > 1 ? (uint32_t)((0x100000000ULL + a.rows_item - 1) / a.rows_item) : 0u;
    a.head_chunks = ceil_div(a.G, a.heads_item);
    // A pair costs its first reference, its output and code that the instruction cache does not hold beside its tiles: 5 500 to 6 500 clocks,
    // where a tile takes 3 300 (no cap, no bias) to 5 600.  It counts where every CTA has pairs of its own (where they are cut among CTAs, each
    // has two parts at most): nine documents of 7001 rows, 14 heads of 64, capped 96.2 -> 79.9 us; six of 3500, 28 heads of 128 65.5 -> 50.3.
    a.pair_cost = a.n_k > kN && (long long)ceil_div(a.n_q, a.rows_item) * a.head_chunks * a.Hkv >= 2 * kNumSMs ? (a.cap_log2 > 0.f || a.slopes ? 1 : 2) : 0;
    maps.k_step = a.Hkv > 1 && a.k_head > 0;
    maps.v_step = a.Hkv > 1 && a.v_head > 0;
    if (a.n_q > 0) {
        // Q: heads of a row side by side
        int rc = make_tmap_3d(&maps.q, a.q, dh, a.Hq, a.n_q, a.Hq > 1 ? a.q_head : a.q_row, a.q_row, a.heads_item, a.rows_item);
        // where there are no keys no tile of them is asked for, and any rows will do
        if (rc == METOK_OK) rc = a.n_k ? make_tmap_3d(&maps.k, a.k, dh, a.n_k, maps.k_step ? a.Hkv : 1, a.k_row, maps.k_step ? a.k_head : a.k_row, kN, 1) : (maps.k = maps.q, METOK_OK);
        if (rc == METOK_OK) rc = a.n_k ? make_tmap_3d(&maps.v, a.v, dh, a.n_k, maps.v_step ? a.Hkv : 1, a.v_row, maps.v_step ? a.v_head : a.v_row, kN, 1) : (maps.v = maps.q, METOK_OK);
        if (rc != METOK_OK) return rc;
    }
    return dh == 64 ? launch_dh<64>(a, maps, st) : launch_dh<128>(a, maps, st);
}

}  // namespace metok
