// The cache in pages: where its rows lie, and which tokens of a sequence are new.
#pragma once
#include "window.h"

namespace infllmv2 {

struct Pages {
    Tensor k, v;                                         // sb: from page to page
    const int32_t *table;
    int32_t ld, lg, count;                               // entries per sequence; page size 2^lg; pages
};
struct NewTokens {
    const int32_t *counts;                               // null: `most` of every sequence
    int32_t most;
};
struct Rotation {
    const uint64_t *steps;
    int32_t dim;                                         // 0: nothing rotates
    int32_t interleaved;
    float amplitude, sign;                               // sign -1: back
};

// Rows of a sequence and how many of them are new; a sequence that is shorter than that is skipped: L = 0.
struct Chunk {
    int L, n, before;                                    // before: rows before the new ones
    __device__ __forceinline__ Chunk(const NewTokens &nt, const int32_t *__restrict__ seqlens, int b, int max_seqlen) {
        L = clamp_len(uniform_load(seqlens + b), max_seqlen);
        n = nt.counts ? clamp_len(uniform_load(nt.counts + b), nt.most) : nt.most;
        if (L < n) L = 0;
        before = L - n;
    }
};

// Behind a product whose result is first read beyond a branch.  The wait states that the compiler counts there (the branch and an s_nop, 12 in all for a 32x32x16 product)
// let a maximum read sums without the last product's part; 16 did not in 20 x 32 x 4 calls of 8 units, these are 20.  In one piece of straight code its 12 are enough.
template <typename T>
__device__ __forceinline__ void settle(T &x) { asm volatile("s_nop 7" : "+v"(x)); }

// The page of 16 rows from `row` on (page sizes are multiples of 16), -1: none, and none behind `end`.
__device__ __forceinline__ int page_of(const Pages &pg, const int32_t *__restrict__ table, int row, int end) {
    if (row >= end) return -1;
    const int page = table[row >> pg.lg];
    return (uint32_t)page < (uint32_t)pg.count ? page : -1;
}
// Pages of 64 units of 32 rows, a unit to a lane: asked for at once, so that a walk finds them in registers.
struct UnitPages {
    int lo, hi;                                          // of rows 0 .. 15 of this lane's unit, of rows 16 .. 31
    __device__ __forceinline__ void load(const Pages &pg, const int32_t *__restrict__ table, int row, int end) {
        lo = page_of(pg, table, row, end);
        hi = page_of(pg, table, row + 16, end);
    }
};
// A store of 16 bytes.  kStream: past the caches.  A call that writes more than all L2s hold leaves its first results nowhere near their reader anyway, and its stores then run
// beside the loads at 6 TB/s instead of 4.7 to 5.7 (8000 new tokens, 36 heads: 29.6 -> 23.2 us; 32768 tokens, 34 heads: 99.6 -> 94.9; 144000 evicted rows 80.8 -> 76.2).
constexpr int64_t kAllL2 = 32ll << 20;
template <bool kStream>
__device__ __forceinline__ void store16(char *p, u32x4_t x) {
    if constexpr (kStream) __builtin_nontemporal_store(x, reinterpret_cast<u32x4_t *>(p));
    else *reinterpret_cast<u32x4_t *>(p) = x;
}
// Byte offset of row `row` of a page from the pool's start.
__device__ __forceinline__ int64_t page_bytes(const Tensor &t, int lg, int page, int row) {
    return 2 * ((int64_t)page * t.sb + (int64_t)(row & ((1 << lg) - 1)) * t.st);
}

size_t paged_attn_ws_bytes(const Dims &dm, int max_new);
int launch_paged_attn(const Dims &dm, Tensor q, const Pages &pg, NewTokens nt, const int32_t *seqlens, Tensor out, float *lse, void *ws, hipStream_t stream);
size_t paged_weights_ws_bytes(const Dims &dm, int max_new);
int launch_paged_weights(const Dims &dm, Tensor q, const float *lse, const Pages &pg, NewTokens nt, const int32_t *seqlens, const float *weights, int pitch,
                         float *weights_out, void *ws, hipStream_t stream);
size_t paged_evict_ws_bytes(const Dims &dm);
int launch_paged_evict(const Dims &dm, const float *weights, int pitch, const Pages &from, const int32_t *seqlens, int budget, int first, int recent,
                       const Pages &to, int32_t *kept, float *weights_out, int32_t *seqlens_out, void *ws, hipStream_t stream);
// null pointers: without queries, without keys
int launch_rope(const Dims &dm, const Rotation &rot, const Tensor *q, const Tensor *k, const int32_t *positions, const int32_t *seqlens, const Tensor *q_out,
                const Tensor *k_out, hipStream_t stream);
int launch_paged_append(const Dims &dm, const Rotation &rot, Tensor k_new, Tensor v_new, const Tensor *q, const Pages &pg, const int32_t *positions,
                        NewTokens nt, const int32_t *seqlens, const Tensor *q_out, hipStream_t stream);

}  // namespace infllmv2
