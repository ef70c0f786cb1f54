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
// The sum of lanes 0 .. lane: within rows of sixteen by shifts, then the rows' sums.
__device__ __forceinline__ uint32_t wave_scan(uint32_t x, int lane) {
    int y = (int)x;
    y += __builtin_amdgcn_update_dpp(0, y, 0x111, 0xf, 0xf, true);
    y += __builtin_amdgcn_update_dpp(0, y, 0x112, 0xf, 0xf, true);
    y += __builtin_amdgcn_update_dpp(0, y, 0x114, 0xf, 0xf, true);
    y += __builtin_amdgcn_update_dpp(0, y, 0x118, 0xf, 0xf, true);
    const int r0 = __builtin_amdgcn_readlane(y, 15), r1 = r0 + __builtin_amdgcn_readlane(y, 31), r2 = r1 + __builtin_amdgcn_readlane(y, 47);
    return (uint32_t)(y + (lane < 16 ? 0 : lane < 32 ? r0 : lane < 48 ? r1 : r2));
}

// The units of 32 keys of a batch's sequences, end to end, dealt to workgroups in runs of `per`: workgroup x takes units x per ..; what it has of sequence b is part x + b of
// all, so a sequence's parts lie side by side.  `aim` workgroups, and fewer where a sequence would come to more than `most` parts.  All lanes of a wavefront.
// (Each sequence cut into as many, 64 of 1501 to 32749 rows wait for the longest's parts: 226 us instead of 205.)  Sequences of about one length are cut into as many all the same, so that no
// workgroup has of two: `per` units to a part, `parts` to a sequence, workgroup x part x % parts of sequence x / parts (64 of 5000 rows 64.7 us without).
struct BatchUnits {
    const int32_t *seqlens;
    NewTokens nt;
    int batch, cap, each, per, parts, total, before, mine;      // before, mine: units before this lane's `each` sequences, and of them
    __device__ __forceinline__ int of(int b) const {     // b uniform
        if (each == 1) return __builtin_amdgcn_readlane(mine, b);        // (up to 64 sequences: no further load)
        const int L = clamp_len(uniform_load(seqlens + b), cap), n = nt.counts ? clamp_len(uniform_load(nt.counts + b), nt.most) : nt.most;
        return L < n ? 0 : (L + 31) >> 5;
    }
    __device__ __forceinline__ int of_lane(int b) const {
        if (b >= batch) return 0;
        const int L = clamp_len(seqlens[b], cap), n = nt.counts ? clamp_len(nt.counts[b], nt.most) : nt.most;
        return L < n ? 0 : (L + 31) >> 5;
    }
    __device__ __forceinline__ BatchUnits(const NewTokens &nt, const int32_t *__restrict__ seqlens, int batch, int cap, int aim, int most, int lane)
        : seqlens(seqlens), nt(nt), batch(batch), cap(cap), each((batch + 63) >> 6), mine(0) {
        int longest = 0;
        for (int i = 0; i < each; ++i) {
            const int u = of_lane(lane * each + i);
            mine += u;
            longest = max(longest, u);
        }
        const int upto = (int)wave_scan((uint32_t)mine, lane);
        before = upto - mine;
        total = __builtin_amdgcn_readlane(upto, 63);
        longest = (int)wave_max_u32((uint32_t)longest);
        parts = (float)longest * (float)batch <= 1.125f * (float)total ? min(most, max(1, aim / batch)) : 0;          // 0: by units
        per = max(4, parts ? (longest + parts - 1) / parts : max((total + aim - 1) / aim, (longest + most - 2) / (most - 1)));
    }
    // the sequence of unit g < total, and the units before it
    __device__ __forceinline__ int find(int g, int &start) const {
        const int l = __builtin_ctzll(__ballot(g >= before && g < before + mine));
        start = __builtin_amdgcn_readlane(before, l);
        int b = l * each;
        for (int u; start + (u = of(b)) <= g; ++b) start += u;
        return b;
    }
    // every sequence's first part and how many it has, by lanes
    __device__ __forceinline__ void write_plan(int2 *plan, int lane) const {
        int start = before;
        for (int i = 0; i < each; ++i) {
            const int b = lane * each + i, u = of_lane(b);
            const int from = parts ? b * parts : start / per, to = parts ? from + (u - 1) / per : (start + u - 1) / per;
            if (b < batch) plan[b] = u > 0 ? int2{from + b, to - from + 1} : int2{0, 0};
            start += u;
        }
    }
};
// A store of 16 bytes.  kStream: past the caches, in a call that writes more than all L2s hold: its stores then run beside the loads at 6 TB/s instead of 4.7 to 5.7 (8000 new tokens, 36
// heads: 29.6 -> 23.2 us; 32768 tokens, 34 heads: 99.6 -> 94.9; 144000 evicted rows 80.8 -> 76.2).  What reads them next finds less in the last-level cache: with a token's attention behind it an append of 16 x 1000
// tokens of 48 heads takes 83.4 us against 91.4, of 4 x 8000 of 24 heads 101.1 against 99.1, and the eviction of 144000 rows 107.9 against 104.8.
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

// A launch has fewer than 2^32 threads along a dimension: of more the runtime starts what is left modulo 2^32, without an error.  Workgroups of 256 beyond 2^23 go along another one.
constexpr int kLgGroups = 23;
inline unsigned groups_x(int64_t groups) { return (unsigned)min(groups, (int64_t)1 << kLgGroups); }
inline unsigned groups_beyond(int64_t groups) { return (unsigned)((groups + (1 << kLgGroups) - 1) >> kLgGroups); }

int64_t paged_attn_groups(const Dims &dm, int max_new);
int64_t paged_weights_groups(const Dims &dm);            // at least, of chunks
int64_t rotate_wavefronts(int64_t rows, int64_t heads);  // of a sequence, at most
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
