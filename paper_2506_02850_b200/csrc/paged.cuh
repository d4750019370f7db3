// What the kernels on a paged K/V cache share: the sizes of a cache, their checks on the host, and the place of a row.
#pragma once

#include <algorithm>

#include "common.cuh"

namespace metok {

constexpr int kMaxCacheRows = 1 << 24;                 // rows of a sequence: positions are exact in fp32

struct PagedDims {
    int n_pages, Hkv, page_shift, dh, n_seqs, max_pages;
    int row_chunks;                                    // 16-byte chunks of a row of one head
    __host__ __device__ int S_cap() const { return max_pages << page_shift; }
};

// Checks what every call on a cache checks; fills `d`.  Pools are checked by the callers.
inline int paged_dims(int dtype, const metok_paged_cache* c, PagedDims* d) {
    if (!c || (dtype != METOK_F32 && dtype != METOK_BF16)) return METOK_ERR_INVALID_ARG;
    if (c->n_pages < 1 || c->Hkv < 1 || c->page_size < 1 || c->dh < 1 || c->n_seqs < 1 || c->max_pages < 1) return METOK_ERR_INVALID_ARG;
    if (c->dh != 64 && c->dh != 128) return METOK_ERR_UNSUPPORTED;
    int shift = 4;
    while (shift < 8 && (1 << shift) < c->page_size) ++shift;
    if ((1 << shift) != c->page_size) return METOK_ERR_UNSUPPORTED;
    if ((long long)c->n_pages * c->Hkv > (0x7FFFFFFFLL >> shift)) return METOK_ERR_UNSUPPORTED;
    if (((long long)c->max_pages << shift) > kMaxCacheRows) return METOK_ERR_UNSUPPORTED;
    const int esize = dtype == METOK_F32 ? 4 : 2;
    *d = {c->n_pages, c->Hkv, shift, c->dh, c->n_seqs, c->max_pages, c->dh * esize / 16};
    return METOK_OK;
}
// The same for a cache held in 4 bits: its rows lie in pieces of 16, a row_chunks of its own has no meaning.
constexpr int kQ4Rows = 16;                            // rows of a piece
__host__ __device__ constexpr int q4_piece(int dh) { return 9 * dh; }    // bytes of a piece: codes [16][dh / 2], scales [16][dh / 16]
inline int paged_dims_q4(const metok_paged_cache* c, PagedDims* d) {
    const int rc = paged_dims(METOK_BF16, c, d);
    d->row_chunks = 0;
    return rc;
}
// [a, a + an) and [b, b + bn) share an element
inline bool overlap(const void* a, size_t an, const void* b, size_t bn) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return x < y + bn && y < x + an;
}

#ifdef __CUDACC__
// First 16-byte chunk of row `r` (a row of a sequence), head `h`, in the page `page`: pools may pass 2^32 chunks.
__device__ __forceinline__ size_t paged_chunk(const PagedDims& d, int page, int h, int r) {
    const size_t row = (((size_t)page * d.Hkv + h) << d.page_shift) + (r & ((1 << d.page_shift) - 1));
    return row * d.row_chunks;
}
// The piece that has row `r` of head `h` in the page `page` of a cache held in 4 bits, and the row's place in it: r % 16.
__device__ __forceinline__ size_t q4_piece_of(const PagedDims& d, int page, int h, int r) {
    return (((size_t)page * d.Hkv + h) << (d.page_shift - 4)) + ((r & ((1 << d.page_shift) - 1)) >> 4);
}
#endif

}  // namespace metok
