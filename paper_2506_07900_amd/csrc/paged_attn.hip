// Attention of a sequence's new tokens over its cache in pages, causal among themselves.
//
// Query rows are (token, head of the group) with the heads fastest.  Up to 16 of them (single tokens) are the columns of 16x16x32 products, and a
// workgroup's wavefronts take units of 32 keys in turn; more are taken 128 to a workgroup, 32 to a wavefront, all wavefronts at the same unit.  Keys are split
// over workgroups where rows are few, and a second kernel joins the parts.
//
// Probabilities are 2^(score - m - shift).  m is a whole number near the running maximum, so rescaling by its changes is exact, and it follows only where scores
// exceed it by more than 2^kSlack.  2^shift exceeds the sum of probabilities that a row can have by then, so values up to the largest of their type do not
// overflow in the sums, which are divided at the end.
#include "paged.h"

namespace infllmv2 {

typedef float f32x2_t __attribute__((ext_vector_type(2)));

constexpr int kChunkRows = 128;
constexpr float kSlack = 8.f;

__device__ __forceinline__ int shift_of(int L) { return 32 - __builtin_clz((uint32_t)max(L, 1)) + (int)kSlack; }

// A row's running maximum (a whole number) with a tile's largest score: whether it moves, and by what the sums are multiplied then.
__device__ __forceinline__ float follow(float &m, float mx) {
    const float m_new = fmaxf(m, __builtin_ceilf(mx)), alpha = fast_exp2(m - (m_new == -INFINITY ? 0.f : m_new));
    m = m_new;
    return alpha;
}

// The halves of words that are infinities or NaN taken out; -> whether there were any.
__device__ __forceinline__ bool take_odd_out(bf16x8 &x) {
    u32x4_t y = __builtin_bit_cast(u32x4_t, x);
    bool odd = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const bool low = (y[i] & 0x7f80u) == 0x7f80u, high = (y[i] & 0x7f800000u) == 0x7f800000u;
        y[i] = (low ? 0u : y[i] & 0xffffu) | (high ? 0u : y[i] & 0xffff0000u);
        odd |= low | high;
    }
    x = __builtin_bit_cast(bf16x8, y);
    return odd;
}
// What a value that is not finite adds to a row that sees it.
__device__ __forceinline__ float odd_value(uint2 y, int e, bool sees) {
    const uint32_t w = e < 2 ? y.x : y.y;
    const float z = __uint_as_float(e & 1 ? w & 0xffff0000u : w << 16);
    return sees && !(__builtin_fabsf(z) < INFINITY) ? z : 0.f;
}

// Probabilities rounded to bf16 may add up to 2^-8 more than their sum, and a mean of values near the largest would round to an infinity.
__device__ __forceinline__ float mean(float x) {
    constexpr float most = 3.3895313892515355e38f;       // bf16's largest
    return __builtin_fabsf(x) < INFINITY ? __builtin_amdgcn_fmed3f(x, -most, most) : x;
}

// ---- 128 rows ------------------------------------------------------------------------------------------------------------

// A wavefront's 32 rows: lane 32 hf + c holds row c.
struct ChunkRows {
    float scale, shift;
    int hf, i;                                           // position of the lane's row
    TileReader rd;
    bf16x8 q[8];
    f32x16 o[4];                                         // channels 32 ct + 8 (e / 4) + 4 hf + e % 4
    float m, l;                                          // l: of this lane's keys
    __device__ __forceinline__ explicit ChunkRows(int lane) : hf(lane >> 5), rd(lane), m(-INFINITY), l(0.f) {}

    // A unit's scores to probabilities, in place; rows' sums and, where maxima move, all that was added up follow.
    __device__ __forceinline__ void probabilities(f32x16 &s) {
        float mx = max3(s[0], s[1], s[2]);
#pragma unroll
        for (int e = 3; e < 15; e += 2) mx = max3(mx, s[e], s[e + 1]);
        mx = half_reduce(max3(mx, s[15], s[15]), [](float a, float d) { return fmaxf(a, d); }) * scale;
        if (__any(mx > m + kSlack)) {
            const float alpha = follow(m, mx);
            l *= alpha;
#pragma unroll
            for (int ct = 0; ct < 4; ++ct) o[ct] *= alpha;
        }
        const float base = (m == -INFINITY ? 0.f : m) + shift;
        float sum[2] = {0.f, 0.f};
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            s[e] = fast_exp2(__builtin_fmaf(s[e], scale, -base));
            sum[e & 1] += s[e];
        }
        l += sum[0] + sum[1];
    }
    __device__ __forceinline__ f32x16 scores(const char *k) const {
        f32x16 s = zero16();
#pragma unroll
        for (int ks = 0; ks < 8; ++ks) s = mfma32(rd.rows(k, ks), q[ks], s);
        return s;
    }
    // 32 keys that all of the workgroup's rows see
    __device__ __forceinline__ void take(const KVHalf &cur) {
        f32x16 s = scores(cur.k);
        probabilities(s);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const bf16x8 p = pack8(s, j);                // (bf16: what the matrix cores multiply; the sum is of what they were)
#pragma unroll
            for (int ct = 0; ct < 4; ++ct) o[ct] = mfma32(rd.columns(cur.v, j, ct), p, o[ct]);
        }
    }
    // Keys k0 .. k0 + 31 that not all rows see; pages: bit 0 those of the first 16 have one, bit 1 of the others.  A product multiplies a key that a row does not see by 0, and 0 times an infinity or a NaN reaches the row's sum: such values
    // are left out, and added to the rows that see them.
    __device__ __forceinline__ void take_edge(const KVHalf &cur, int k0, uint32_t pages) {
        f32x16 s = scores(cur.k);
        const int at = i - k0 - 4 * hf, at0 = pages & 1u ? at : -1, at1 = pages & 2u ? at : -1;      // keys up to this one are seen
#pragma unroll
        for (int e = 0; e < 16; ++e) s[e] = 8 * (e >> 2) + (e & 3) <= (e < 8 ? at0 : at1) ? s[e] : -INFINITY;
        probabilities(s);
        bool odd = false;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const bf16x8 p = pack8(s, j);
#pragma unroll
            for (int ct = 0; ct < 4; ++ct) {
                bf16x8 x = rd.columns(cur.v, j, ct);
                odd |= take_odd_out(x);
                o[ct] = mfma32(x, p, o[ct]);
                __builtin_amdgcn_sched_barrier(0);       // (registers)
            }
        }
        if (!__any(odd)) return;
#pragma unroll 1
        for (int t = 0; t < 32; ++t) {
            const bool sees = k0 + t <= i;               // (rows without a page read as zeros)
            const char *row = cur.v + 64 * t + 8 * hf;
#pragma unroll
            for (int ct = 0; ct < 4; ++ct)
#pragma unroll
                for (int e4 = 0; e4 < 4; ++e4) {
                    const uint2 y = *reinterpret_cast<const uint2 *>(row + ct * 2048 + ((e4 ^ ((t >> 2) & 3)) << 4));
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        o[ct][4 * e4 + e] += odd_value(y, e, sees);
                        __builtin_amdgcn_sched_barrier(0);
                    }
                }
        }
    }
};

// Where tiles are few: those that hold new tokens, of all sequences, each with its keys cut into as many parts as there are workgroups for.  Items are numbered by sequence, head, part and
// tile, the last fastest; item x has the 128 partial rows 128 x ..  All lanes of a wavefront.  (As many parts as for `most` tokens of each, 37 and 21 new tokens of 32749 rows, 16 : 2 heads,
// leave 42 of 252 workgroups without work: 40.0 us instead of 36.2.  Where all have as many it costs up to 0.8 us: 8 of 64 tokens, 34.4 / 35.2.)
constexpr int kChunkItems = 256;
struct ChunkTiles {
    const int32_t *seqlens;
    NewTokens nt;
    int batch, cap, lg, each, before, mine, total, parts;       // before, mine: tiles before this lane's `each` sequences, and of them
    __device__ __forceinline__ int of(int b) const {
        if (b >= batch) return 0;
        const int L = clamp_len(seqlens[b], cap), n = nt.counts ? clamp_len(nt.counts[b], nt.most) : nt.most;
        return L < n ? 0 : (int)((((int64_t)n << lg) + kChunkRows - 1) / kChunkRows);
    }
    __device__ __forceinline__ ChunkTiles(const NewTokens &nt, const int32_t *__restrict__ seqlens, int batch, int cap, int lg, int heads, int most, int lane)
        : seqlens(seqlens), nt(nt), batch(batch), cap(cap), lg(lg), each((batch + 63) >> 6), mine(0) {
        for (int i = 0; i < each; ++i) mine += of(lane * each + i);
        const int upto = (int)wave_scan((uint32_t)mine, lane);
        before = upto - mine;
        total = __builtin_amdgcn_readlane(upto, 63);
        parts = max(1, min(most, kChunkItems / max(1, total * heads)));
    }
    // the sequence of tile g < total, the tiles before it and its own
    __device__ __forceinline__ int find(int g, int &start, int &tiles) const {
        const int l = __builtin_ctzll(__ballot(g >= before && g < before + mine));
        start = __builtin_amdgcn_readlane(before, l);
        tiles = __builtin_amdgcn_readlane(mine, l);
        int b = l * each;
        if (each > 1)
            for (; start + (tiles = __builtin_amdgcn_readfirstlane(of(b))) <= g; ++b) start += tiles;
        return b;
    }
    // every sequence's first item, and its tiles (0: of none) and parts, by lanes
    __device__ __forceinline__ void write_plan(int2 *plan, int heads, int lane) const {
        int start = before;
        for (int i = 0; i < each; ++i) {
            const int b = lane * each + i, n = of(b);
            if (b < batch) plan[b] = int2{start * heads * parts, n | parts << 16};
            start += n;
        }
    }
};

// Items: (sequence, head), tile of 128 rows, the last fastest, or (kParts) as ChunkTiles numbers them, n_tiles: most parts.
// kGroups groups of four wavefronts take every kGroups-th unit and are joined in LDS at the end.  Three fill a compute unit as three workgroups of one do, with a third of the parts
// (1000 new tokens of 65000, 16 : 2 heads: 615 -> 527 us; 2 x 2048 of 4096, 8 : 8: 99.9 -> 74.2).  8192 of 65536, 32 : 2: 7.4 to 7.9 ms by card, 1.04 to 1.11 PFLOP/s: matrix cores and vector unit busy
// 57 and 59 % at 1.9 to 1.8 GHz.  A unit's scores ahead, between the exponentials of the one before, takes registers for two wavefronts to a SIMD only: 8.6 ms against 8.2 in turn.
template <int kGroups, bool kParts>
__global__ __launch_bounds__(256 * kGroups, 3) void paged_attn_kernel(Dims dm, Pages pg, NewTokens nt, int lg, int n_tiles, int run, Tensor q,
                                                            const int32_t *__restrict__ seqlens, Tensor out, float *__restrict__ lse,
                                                            float *__restrict__ o_part, float2 *__restrict__ ml_part, int2 *__restrict__ plan) {
    __shared__ KVHalf slots0[kGroups], slots1[kGroups], slots2[kGroups];
    __shared__ float2 ml_s[kGroups][4][64];
    const int item = xcd_item(blockIdx.x, run), lane = threadIdx.x & 63;
    int b, h, ti, split = 0, n_split = 1, slot = 0;      // ti: the last rows, which see most keys, first
    if constexpr (kParts) {
        const ChunkTiles all(nt, seqlens, dm.batch, dm.max_seqlen, lg, dm.Hkv, n_tiles, lane);
        if (blockIdx.x == 0 && threadIdx.x < 64) all.write_plan(plan, dm.Hkv, lane);
        n_split = all.parts;
        if (item >= all.total * dm.Hkv * n_split) return;
        int start, tiles;
        b = all.find(item / (dm.Hkv * n_split), start, tiles);
        const int x = item - start * (dm.Hkv * n_split), hs = x / tiles;
        h = hs / n_split;
        split = hs - h * n_split;
        ti = (hs + 1) * tiles - 1 - x;
        slot = start * (dm.Hkv * n_split) + hs * tiles + ti;
    } else {
        const int bh = item / n_tiles;
        b = bh / dm.Hkv;
        h = bh - b * dm.Hkv;
        ti = (bh + 1) * n_tiles - 1 - item;
        if (b >= dm.batch) return;
    }
    const int id = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wave = id & 3, group = id >> 2;
    KVHalf &slot0 = slots0[group], &slot1 = slots1[group], &slot2 = slots2[group];
    const Chunk ch(nt, seqlens, b, dm.max_seqlen);
    const int t0 = ti * (kChunkRows >> lg), t1 = min(ch.n, t0 + (kChunkRows >> lg));
    ChunkRows r(lane);
    const int row = 32 * wave + (lane & 31), token = t0 + (row >> lg), hq = h * dm.G + (row & (dm.G - 1));
    const int end = ch.L > 0 && t0 < ch.n ? ch.before + t1 : 0;          // keys that the workgroup's rows see
    const int units = (end + 31) >> 5, from = (int)((int64_t)units * split / n_split), all = (int)((int64_t)units * (split + 1) / n_split) - from;
    const int count = (all - group + kGroups - 1) / kGroups;              // this group's units
    auto unit = [&](int x) __attribute__((always_inline)) { return from + group + kGroups * x; };
    if (!kParts && t0 >= ch.n && !dm.fill) return;
    r.scale = dm.scale_log2;
    r.shift = (float)shift_of(ch.L);
    r.i = ch.before + token;
    {
        const __bf16 *qr = q.ptr + b * q.sb + (int64_t)max(0, min(token, ch.n - 1)) * q.st + (int64_t)hq * q.sh + 8 * r.hf;
#pragma unroll
        for (int ks = 0; ks < 8; ++ks) r.q[ks] = load8(qr + 16 * ks);
    }
#pragma unroll
    for (int ct = 0; ct < 4; ++ct) r.o[ct] = zero16();
    const char *k_head = reinterpret_cast<const char *>(pg.k.ptr + h * pg.k.sh) + 64 * wave, *v_head = reinterpret_cast<const char *>(pg.v.ptr + h * pg.v.sh) + 64 * wave;
    const uint32_t k_at = (lane >> 2) * (2 * (uint32_t)pg.k.st) + 16 * copy_piece(lane), v_at = (lane >> 2) * (2 * (uint32_t)pg.v.st) + 16 * copy_piece(lane);
    const int32_t *table = pg.table + (int64_t)b * pg.ld;
    UnitPages up;
    auto look_up = [&](int x) __attribute__((always_inline)) {           // (before the wait for copies: behind it the compiler would wait for all of them)
        if ((x & 63) == 0) up.load(pg, table, 32 * unit(x + lane), x + lane < count ? end : 0);
    };
    // unit x into a slot, four copies of 16 rows each; -> which of its halves have a page.  Those past the last bring zeros.
    auto stage = [&](KVHalf &dst, int x) __attribute__((always_inline)) -> uint32_t {
        uint32_t there = 0u;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int page = __builtin_amdgcn_readlane(j ? up.hi : up.lo, x & 63), first = 32 * unit(x) + 16 * j;
            const bool some = page >= 0, in = some && first + (lane >> 2) < end;
            there |= some ? 1u << j : 0u;
            copy_rows(dst.k + wave * 2048 + j * 1024, k_head + page_bytes(pg.k, pg.lg, max(page, 0), first), in ? k_at : kNoRow, 0);
            copy_rows(dst.v + wave * 2048 + j * 1024, v_head + page_bytes(pg.v, pg.lg, max(page, 0), first), in ? v_at : kNoRow, 0);
        }
        return there;
    };
    // Unit x lies in slot x % 3.  The first `whole` are seen by all rows; from the first of them that has no page on, all are taken as the others are.
    look_up(0);
    __builtin_amdgcn_sched_barrier(0);                   // (queries are asked for before the copies: else each step waits for a unit more)
    uint32_t p0 = stage(slot0, 0), p1 = stage(slot1, 1), p2 = 3u;
    int whole = max(0, min(count, (((ch.before + t0 + 1) >> 5) - from - group + kGroups - 1) / kGroups));
    if (p1 != 3u) whole = min(whole, 1);
    if (p0 != 3u) whole = 0;
    const bool alive = t0 + ((32 * wave) >> lg) < ch.n;  // (of no token: these rows only help to fetch)
    auto arrived = [&]() __attribute__((always_inline)) {
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_waitcnt(0x0f74);              // all copies but the next unit's four
        asm volatile("s_barrier" ::: "memory");          // everyone's, and everyone is past the unit before
        __builtin_amdgcn_sched_barrier(0);
    };
    auto step = [&](const KVHalf &cur, KVHalf &next, uint32_t &pages_next, int x) __attribute__((always_inline)) {
        look_up(x + 2);
        arrived();
        pages_next = stage(next, x + 2);
        whole = pages_next != 3u ? min(whole, x + 2) : whole;
        if (alive) r.take(cur);
    };
    for (int x = 0; x < whole; x += 3) {
        step(slot0, slot2, p2, x);
        if (x + 1 >= whole) break;
        step(slot1, slot0, p0, x + 1);
        if (x + 2 >= whole) break;
        step(slot2, slot1, p1, x + 2);
    }
#pragma unroll 1
    for (int x = whole; x < count; ++x) {
        const int at = x % 3;
        KVHalf *const cur = at == 0 ? &slot0 : at == 1 ? &slot1 : &slot2, *const next = at == 0 ? &slot2 : at == 1 ? &slot0 : &slot1;
        look_up(x + 2);
        arrived();
        const uint32_t there = at == 0 ? p0 : at == 1 ? p1 : p2, then = stage(*next, x + 2);
        p0 = at == 1 ? then : p0;
        p1 = at == 2 ? then : p1;
        p2 = at == 0 ? then : p2;
        if (alive) r.take_edge(*cur, 32 * unit(x), there);
    }
    if (kGroups > 1 && count < (all + kGroups - 1) / kGroups) asm volatile("s_barrier" ::: "memory");   // (the first groups have one unit more)
    __builtin_amdgcn_s_waitcnt(0);                       // (the copies past the last unit have landed)
    __syncthreads();
    char *mine = (wave < 2 ? slots0[0].k : slots1[0].k) + (wave & 1) * kHalfTile;              // 8 KiB of this wavefront's own
    if constexpr (kGroups > 1) {                         // a row's state is in the same lanes of all groups: the others hand theirs to the first
        static_assert(kGroups == 3, "nine slots hold the states of two groups");
        auto block = [&](int g) __attribute__((always_inline)) {
            const int i = 4 * (g - 1) + wave;
            return reinterpret_cast<char *>(i < 3 ? &slots0[i] : i < 6 ? &slots1[i - 3] : &slots2[i - 6]) + 16 * lane;
        };
        if (group > 0) {
            ml_s[group][wave][lane] = float2{r.m, r.l};
            char *at = block(group);
#pragma unroll
            for (int ct = 0; ct < 4; ++ct)
#pragma unroll
                for (int e4 = 0; e4 < 4; ++e4)
                    *reinterpret_cast<f32x4 *>(at + 1024 * (4 * ct + e4)) = f32x4{r.o[ct][4 * e4], r.o[ct][4 * e4 + 1], r.o[ct][4 * e4 + 2], r.o[ct][4 * e4 + 3]};
        }
        __syncthreads();
        if (group > 0) return;
        float M = r.m;
#pragma unroll
        for (int g = 1; g < kGroups; ++g) M = fmaxf(M, ml_s[g][wave][lane].x);
        const float base = M == -INFINITY ? 0.f : M, own = fast_exp2(r.m - base);
        r.m = M;
        r.l *= own;
#pragma unroll
        for (int ct = 0; ct < 4; ++ct) r.o[ct] *= own;
#pragma unroll
        for (int g = 1; g < kGroups; ++g) {
            const float2 other = ml_s[g][wave][lane];
            const float theirs = fast_exp2(other.x - base);
            r.l += other.y * theirs;
            const char *at = block(g);
#pragma unroll
            for (int ct = 0; ct < 4; ++ct) {
#pragma unroll
                for (int e4 = 0; e4 < 4; ++e4) {
                    const f32x4 x = *reinterpret_cast<const f32x4 *>(at + 1024 * (4 * ct + e4));
#pragma unroll
                    for (int e = 0; e < 4; ++e) r.o[ct][4 * e4 + e] += x[e] * theirs;
                }
                asm volatile("" : "+v"(r.o[ct]));        // (here: else the additions move behind the branch below, and all of x is kept for them)
            }
        }
        mine = block(1) - 16 * lane;                     // (read by this wavefront alone)
        reads_done();
    }
    r.l = half_reduce(r.l, [](float a, float d) { return a + d; });
    const bool live = token < ch.n;
    if constexpr (kParts) {
        if (!live) return;
        const int64_t at = (int64_t)slot * kChunkRows + row;
        if (r.hf == 0) ml_part[at] = float2{r.m + r.shift, r.l};
        if (r.l != 0.f) {                                // (a NaN too)
            float *op = o_part + at * kHeadDim + 4 * r.hf;
#pragma unroll
            for (int ct = 0; ct < 4; ++ct)
#pragma unroll
                for (int e4 = 0; e4 < 4; ++e4)
                    *reinterpret_cast<f32x4 *>(op + 32 * ct + 8 * e4) = f32x4{r.o[ct][4 * e4], r.o[ct][4 * e4 + 1], r.o[ct][4 * e4 + 2], r.o[ct][4 * e4 + 3]};
        }
        return;
    }
    // rows that see no key, and those behind the last token where they are written: zeros
    const bool some = live && r.l != 0.f;
    const float inv = some ? 1.f / r.l : 0.f;
    float factor = inv;
    float most = 0.f;
#pragma unroll
    for (int ct = 0; ct < 4; ++ct) {
#pragma unroll
        for (int e = 0; e < 16; e += 2) most = __builtin_elementwise_maximum(most, __builtin_elementwise_maximum(__builtin_fabsf(r.o[ct][e]), __builtin_fabsf(r.o[ct][e + 1])));
    }
    if (__builtin_expect(__any(!(most * inv < 3.3e38f)), 0)) {           // (near the largest, or no number)
#pragma unroll
        for (int ct = 0; ct < 4; ++ct)
#pragma unroll
            for (int e = 0; e < 16; ++e) r.o[ct][e] = some ? mean(r.o[ct][e] * inv) : 0.f;
        factor = 1.f;                                    // (the same products: other rows of the wavefront come out the same)
    }
    store_rows(mine, r.o, factor, lane, [&](int at) __attribute__((always_inline)) -> __bf16 * {
        const int t = t0 + ((32 * wave + at) >> lg);
        return t < nt.most && (t < ch.n || dm.fill) ? out.ptr + b * out.sb + (int64_t)t * out.st + (int64_t)(h * dm.G + ((32 * wave + at) & (dm.G - 1))) * out.sh : nullptr;
    });
    if (r.hf == 0 && token < nt.most && (live || dm.fill))
        lse[((int64_t)b * nt.most + token) * dm.Hq + hq] = !live ? 0.f : some ? lse_of(r.m + r.shift, r.l) : -INFINITY;
}

// ---- up to 16 rows ---------------------------------------------------------------------------------------------------------

// grid (parts of the keys, Hkv, batch), or of a batch dealt by units (workgroups, Hkv): aim and most as in BatchUnits; where a sequence's parts lie goes to `plan`.
// Column c of the products: head c % G of new token c / G.  A wavefront has its keys in the registers of the first product and its values in LDS, the next unit's under way: 32 KiB
// a wavefront, two workgroups to a compute unit.  Bound by traffic where rows are many (64 sequences of 1501 to 32749 rows: 201 us, 5.6 TB/s), by a chain of round trips
// (length, table, keys) where they are few (one of 20011: 7.6 us, and 4.3 to join).
constexpr int kFewWaves = 4;
template <bool kBatch>
__global__ __launch_bounds__(64 * kFewWaves, 2) void paged_attn_few_kernel(Dims dm, Pages pg, NewTokens nt, int lg, Tensor q, const int32_t *__restrict__ seqlens,
                                                                Tensor out, float *__restrict__ lse, float *__restrict__ o_part,
                                                                float2 *__restrict__ ml_part, int2 *__restrict__ plan, int aim, int most) {
    __shared__ __align__(16) char V0[kFewWaves][kHalfTile], V1[kFewWaves][kHalfTile];
    __shared__ float2 ml_s[kFewWaves][16];
    const int h = blockIdx.y;
    // units u_from .. u_to - 1 of sequence b; to part `part`, or (whole) the result itself
    auto attend_part = [&](const int b, const int u_from, const int u_to, const int64_t part, const bool whole) __attribute__((always_inline)) {
        const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 15, g = lane >> 4;
        const Chunk ch(nt, seqlens, b, dm.max_seqlen);
        const int token = n >> lg, hq = h * dm.G + (n & (dm.G - 1));
        bf16x8 bq[4];                                        // channels 32 ks + 8 g ..
        {
            const __bf16 *qr = q.ptr + b * q.sb + (int64_t)max(0, min(token, ch.n - 1)) * q.st + (int64_t)hq * q.sh + 8 * g;
#pragma unroll
            for (int ks = 0; ks < 4; ++ks) bq[ks] = load8(qr + 32 * ks);
        }
        const int end = ch.L, u_end = u_to, u0 = u_from + wave;
        const int count = u0 < u_end ? (u_end - u0 + kFewWaves - 1) / kFewWaves : 0;   // units u0, u0 + kFewWaves, ..
        const char *k_head = reinterpret_cast<const char *>(pg.k.ptr + h * pg.k.sh), *v_head = reinterpret_cast<const char *>(pg.v.ptr + h * pg.v.sh);
        const uint32_t k_at = n * (2 * (uint32_t)pg.k.st) + 16 * g;
        const int32_t *table = pg.table + (int64_t)b * pg.ld;
        struct Unit {
            bf16x8 k[2][4];
            uint32_t there;
            int k0;
        };
        UnitPages up;
        auto fetch = [&](Unit &u, char *vs, int x) __attribute__((always_inline)) {
            if ((x & 63) == 0) up.load(pg, table, 32 * (u0 + kFewWaves * (x + lane)), x + lane < count ? end : 0);
            u.k0 = 32 * (u0 + kFewWaves * x);
            u.there = 0u;
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const int page = __builtin_amdgcn_readlane(t ? up.hi : up.lo, x & 63), first = u.k0 + 16 * t;
                const bool some = page >= 0;
                u.there |= some ? 1u << t : 0u;
                const auto from = __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(k_head + page_bytes(pg.k, pg.lg, max(page, 0), first)), 0, 0xfffffffeu, 0x00027000);
                const uint32_t at = some && first + n < end ? k_at : kNoRow;
#pragma unroll
                for (int ks = 0; ks < 4; ++ks)
                    u.k[t][ks] = __builtin_bit_cast(bf16x8, (u32x4_t)__builtin_amdgcn_raw_buffer_load_b128(from, at, 64 * ks, 0));
                const char *vb = v_head + page_bytes(pg.v, pg.lg, max(page, 0), first);
#pragma unroll
                for (int i = 0; i < 4; ++i) {                // 1 KiB: rows 4 i + lane / 16, whose 16-byte pieces are XORed with what row_swizzle says
                    const int r = 4 * i + g;
                    copy_rows(vs + 4096 * t + 1024 * i, vb, some && first + r < end ? r * (2 * (uint32_t)pg.v.st) + 16 * (n ^ row_swizzle(r)) : kNoRow, 0);
                }
            }
        };
        f32x4 o[8];                                          // o[c][e]: channel 16 c + 4 g + e of column n
        float m = -INFINITY, l = 0.f;
#pragma unroll
        for (int c = 0; c < 8; ++c) o[c] = f32x4{0.f, 0.f, 0.f, 0.f};
        const float shift = (float)shift_of(ch.L);
        const int last = ch.before + min(token, ch.n - 1);   // the last key that this column sees
        auto attend = [&](const Unit &u, const char *vs) __attribute__((always_inline)) {
            f32x4 s[2];
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                s[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int ks = 0; ks < 4; ++ks) s[t] = mfma16(u.k[t][ks], bq[ks], s[t]);
                settle<8>(s[t]);
            }
            float y[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = s[e >> 2][e & 3];             // key 16 (e / 4) + 4 g + e % 4
            const bool whole = u.k0 + 31 <= ch.before && u.there == 3u;
            if (!whole) {
                const int at = last - u.k0 - 4 * g, at0 = u.there & 1u ? at : -1, at1 = u.there & 2u ? at : -1;
#pragma unroll
                for (int e = 0; e < 8; ++e) y[e] = 16 * (e >> 2) + (e & 3) <= (e < 4 ? at0 : at1) ? y[e] : -INFINITY;
            }
            const float mx = xgroup_max(max3(max3(max3(y[0], y[1], y[2]), y[3], y[4]), max3(y[5], y[6], y[7]), y[7])) * dm.scale_log2;
            if (__any(mx > m + kSlack)) {
                const float alpha = follow(m, mx);
                l *= alpha;
#pragma unroll
                for (int c = 0; c < 8; ++c) o[c] *= alpha;
            }
            const float base = (m == -INFINITY ? 0.f : m) + shift;
            float ps = 0.f;
            bf16x8 p;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float e = fast_exp2(__builtin_fmaf(y[j], dm.scale_log2, -base));
                ps += e;
                p[j] = (__bf16)e;
            }
            l += ps;                                         // (this lane's keys only: joined over g at the end)
            const int r = 4 * g + (n >> 2);
            bool odd = false;
#pragma unroll
            for (int c = 0; c < 8; ++c) {                    // A: channel 16 c + n, keys 4 g .. and 16 + 4 g ..
                const char *at = vs + 8 * (n & 1);
                const int piece = 2 * c + ((n & 3) >> 1);
                const s16x4 x0 = lds_read_tr16(at + r * 256 + ((piece ^ row_swizzle(r)) << 4));
                const s16x4 x1 = lds_read_tr16(at + (r + 16) * 256 + ((piece ^ row_swizzle(r)) << 4));
                bf16x8 x = __builtin_bit_cast(bf16x8, __builtin_shufflevector(x0, x1, 0, 1, 2, 3, 4, 5, 6, 7));
                if (!whole) odd |= take_odd_out(x);
                o[c] = mfma16(x, p, o[c]);
            }
            if (whole || !__any(odd)) return;
#pragma unroll 1
            for (int t = 0; t < 32; ++t) {
                const bool sees = u.k0 + t <= last;
#pragma unroll
                for (int c = 0; c < 8; ++c) {
                    const uint2 w = *reinterpret_cast<const uint2 *>(vs + 256 * t + (((2 * c + (g >> 1)) ^ row_swizzle(t)) << 4) + 8 * (g & 1));
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[c][e] += odd_value(w, e, sees);
                }
            }
        };
        {
            Unit a, c;
            char *v0 = V0[wave], *v1 = V1[wave];
            auto step = [&](Unit &cur, Unit &next, char *vc, char *vn, int x) __attribute__((always_inline)) {
                reads_done();
                if (x + 1 < count) fetch(next, vn, x + 1);
                copies_landed(x + 1 < count);
                attend(cur, vc);
            };
            if (count > 0) fetch(a, v0, 0);
            for (int x = 0; x < count; x += 2) {
                step(a, c, v0, v1, x);
                if (x + 1 < count) step(c, a, v1, v0, x + 1);
            }
        }
        reads_done();
        l = xgroup_sum(l);
        // ---- the wavefronts' states into one -----------------------------------------------------------------------------------
        if (g == 0) ml_s[wave][n] = float2{m, l};
        __syncthreads();
        float M = -INFINITY;
#pragma unroll
        for (int i = 0; i < kFewWaves; ++i) M = fmaxf(M, ml_s[i][n].x);
        const float w = fast_exp2(m - (M == -INFINITY ? 0.f : M));
        float *mine = reinterpret_cast<float *>(V0[wave]);   // [column][channel]
#pragma unroll
        for (int c = 0; c < 8; ++c) *reinterpret_cast<f32x4 *>(mine + n * kHeadDim + 16 * (c ^ (n & 7)) + 4 * g) = o[c] * w;
        __syncthreads();
        const int col = tid >> 4, c8 = 8 * (tid & 15), ct = col >> lg;       // a thread joins eight channels of a column
        if (ct >= nt.most || (ct >= ch.n && (!whole || !dm.fill))) return;
        float den = 0.f, Mc = -INFINITY, y[8];
#pragma unroll
        for (int i = 0; i < kFewWaves; ++i) Mc = fmaxf(Mc, ml_s[i][col].x);
        const float bc = Mc == -INFINITY ? 0.f : Mc;
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = 0.f;
#pragma unroll
        for (int i = 0; i < kFewWaves; ++i) {
            den += ml_s[i][col].y * fast_exp2(ml_s[i][col].x - bc);
            const float *from = reinterpret_cast<const float *>(V0[i]) + col * kHeadDim + 16 * ((c8 >> 4) ^ (col & 7)) + (c8 & 15);
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] += from[e];
        }
        const int hc = h * dm.G + (col & (dm.G - 1));
        const int64_t row = ((int64_t)b * nt.most + ct) * dm.Hq + hc;
        if (whole) {
            const bool some = ct < ch.n && den != 0.f;
            bf16x8 z;
#pragma unroll
            for (int e = 0; e < 8; ++e) z[e] = (__bf16)(some ? mean(y[e] / den) : 0.f);
            *reinterpret_cast<uint4 *>(out.ptr + b * out.sb + (int64_t)ct * out.st + (int64_t)hc * out.sh + c8) = __builtin_bit_cast(uint4, z);
            if (c8 == 0) lse[row] = ct >= ch.n ? 0.f : some ? lse_of(bc + shift, den) : -INFINITY;
        } else {
            const int64_t at = kBatch ? part * 16 + col : row * gridDim.x + part;
            if (den != 0.f) {
                float4 *op = reinterpret_cast<float4 *>(o_part + at * kHeadDim + c8);
                op[0] = float4{y[0], y[1], y[2], y[3]};
                op[1] = float4{y[4], y[5], y[6], y[7]};
            }
            if (c8 == 0) ml_part[at] = float2{bc + shift, den};
        }
    };
    if constexpr (kBatch) {
        const int lane = threadIdx.x & 63;
        const BatchUnits all(nt, seqlens, dm.batch, dm.max_seqlen, aim, most, lane);
        if (blockIdx.x == 0 && h == 0 && threadIdx.x < 64) all.write_plan(plan, lane);
        if (all.parts) {
            const int b = blockIdx.x / all.parts, from = (blockIdx.x - b * all.parts) * all.per, units = b < dm.batch ? all.of(b) : 0;
            if (from < units) attend_part(b, from, min(units, from + all.per), (int64_t)h * (gridDim.x + dm.batch) + blockIdx.x + b, false);
            return;
        }
        const int g0 = (int)min((int64_t)all.total, (int64_t)blockIdx.x * all.per), g1 = (int)min((int64_t)all.total, (int64_t)g0 + all.per);
        if (g0 >= g1) return;
        int start, b = all.find(g0, start);
        for (;;) {
            const int units = all.of(b);
            if (units > 0) attend_part(b, max(0, g0 - start), min(units, g1 - start), (int64_t)h * (gridDim.x + dm.batch) + blockIdx.x + b, false);
            start += units;
            if (start >= g1) return;
            ++b;
            __syncthreads();                             // (LDS is free)
        }
    } else {
        const int b = blockIdx.z, split = blockIdx.x, n_split = gridDim.x;
        const int64_t units = (Chunk(nt, seqlens, b, dm.max_seqlen).L + 31) >> 5;
        attend_part(b, (int)(units * split / n_split), (int)(units * (split + 1) / n_split), split, n_split == 1);
    }
}

// ---- joining the parts --------------------------------------------------------------------------------------------------------

// kWaves wavefronts to a row, two channels to a lane, parts wave, wave + kWaves, ..: sums and channels are asked for together, before it is known which parts have any (one whose sum is
// 0 has not, and what lies in its place is not looked at): a row costs one round trip.
template <int kWaves, bool kTiles>
__global__ __launch_bounds__(kWaves == 1 ? 256 : 64 * kWaves) void paged_merge_kernel(Dims dm, NewTokens nt, int n_split, const int2 *__restrict__ plan, int64_t rows, const float *__restrict__ o_part,
                                                          const float2 *__restrict__ ml_part, Tensor out, float *__restrict__ lse) {
    __shared__ f32x2_t joined[kWaves][64];
    const int lane = threadIdx.x & 63, id = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wave = kWaves == 1 ? 0 : id;
    const int64_t row = kWaves == 1 ? (int64_t)blockIdx.x * 4 + id : blockIdx.x;
    if (row >= rows) return;                             // (more than one row to a workgroup: no barrier follows)
    const int64_t bt = row / dm.Hq;
    const int hq = (int)(row - bt * dm.Hq), b = (int)(bt / nt.most), t = (int)(bt - (int64_t)b * nt.most);
    const int n = nt.counts ? clamp_len(uniform_load(nt.counts + b), nt.most) : nt.most;
    if (t >= n && !dm.fill) return;
    f32x2_t y = {0.f, 0.f};
    float M = -INFINITY, den = 0.f;
    int n_parts = n_split;
    if (plan && t < n) n_parts = uniform_load(&plan[b].y);
    const int tiles = n_parts & 0xffff;                  // (kTiles)
    if constexpr (kTiles) n_parts = tiles ? n_parts >> 16 : 0;
    if (t < n && n_parts > 0) {                          // (a skipped sequence has no parts, or parts without sums)
        int64_t base = row * n_split;                    // the row's parts: base, base + step, ..
        int step = 1;
        const int lg = __builtin_ctz(dm.G);
        if constexpr (kTiles) {
            const int at = (t << lg) + (hq & (dm.G - 1));
            base = (int64_t)(uniform_load(&plan[b].x) + (hq >> lg) * n_parts * tiles + at / kChunkRows) * kChunkRows + at % kChunkRows;
            step = tiles * kChunkRows;
        } else if (plan) {                               // (n_split: parts of all sequences)
            base = ((int64_t)(hq >> lg) * n_split + uniform_load(&plan[b].x)) * 16 + (t << lg) + (hq & (dm.G - 1));
            step = 16;
        }
        const float2 ml = lane < n_parts ? ml_part[base + lane * step] : float2{-INFINITY, 0.f};
        const float2 ml2 = kWaves == 8 && 64 + lane < n_parts ? ml_part[base + (64 + lane) * step] : float2{-INFINITY, 0.f};
        const float *o = o_part + base * kHeadDim + 2 * lane;
        constexpr int kStep = 16;                        // (of kWaves = 1: all parts, of 4 up to 64, of 8 up to 128)
        f32x2_t x[kStep];
#pragma unroll
        for (int i = 0; i < kStep; ++i) x[i] = *reinterpret_cast<const f32x2_t *>(o + (int64_t)(min(wave + kWaves * i, n_parts - 1) * step) * kHeadDim);
        const uint64_t have = __ballot(ml.y != 0.f), have2 = kWaves == 8 ? __ballot(ml2.y != 0.f) : 0ull;    // (a NaN too)
        M = fmaxf(ml.y != 0.f ? ml.x : -INFINITY, ml2.y != 0.f ? ml2.x : -INFINITY);
        M = row_reduce(M, [](float a, float d) { return fmaxf(a, d); });
        M = xgroup_max(M);
        const float w = ml.y != 0.f ? fast_exp2(ml.x - M) : 0.f, w2 = ml2.y != 0.f ? fast_exp2(ml2.x - M) : 0.f;
        den = (ml.y != 0.f ? ml.y * w : 0.f) + (ml2.y != 0.f ? ml2.y * w2 : 0.f);
        den = row_reduce(den, [](float a, float d) { return a + d; });
        den = xgroup_sum(den);
#pragma unroll
        for (int i = 0; i < kStep; ++i) {
            const int s = wave + kWaves * i;
            const bool high = kWaves == 8 && i >= 8;     // (a constant: s >= 64)
            if (((high ? have2 : have) >> (s & 63)) & 1ull) y += x[i] * __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(high ? w2 : w), s & 63));
        }
    }
    if constexpr (kWaves > 1) {
        joined[id][lane] = y;
        __syncthreads();
        if (wave > 0) return;
#pragma unroll
        for (int i = 1; i < kWaves; ++i) y += joined[i][lane];
    }
    const bool some = den != 0.f;
    bf16x2_t z;
    z[0] = (__bf16)(some ? mean(y[0] / den) : 0.f);
    z[1] = (__bf16)(some ? mean(y[1] / den) : 0.f);
    *reinterpret_cast<uint32_t *>(out.ptr + b * out.sb + (int64_t)t * out.st + (int64_t)hq * out.sh + 2 * lane) = __builtin_bit_cast(uint32_t, z);
    if (lane == 0) lse[row] = t >= n ? 0.f : some ? lse_of(M, den) : -INFINITY;
}

// ---- host side -------------------------------------------------------------------------------------------------------------
static inline size_t align256(size_t x) { return (x + 255) / 256 * 256; }

constexpr int kMaxParts = 128, kMaxChunkParts = 64;      // what paged_merge_kernel joins; of tiles of 128 rows
// Up to 16 rows: two workgroups to a compute unit run at a time, and the keys are cut into as many parts, those of a batch by the sequences' lengths.  More rows: with more tiles than
// compute units up to three workgroups of one group to each; with fewer, unless the keys are few, workgroups of three groups, and parts of the keys where they are fewer than half.
constexpr int kFewItems = 512;
struct PagedPlan {
    bool few, groups, batch;                             // batch: parts by lengths
    int tiles, parts, most;                              // parts: of an item; of all sequences.  most: of a sequence
    int64_t items;                                       // of one part
};
static int64_t paged_tiles(const Dims &dm, int64_t max_new) {
    const int64_t rows = max_new * dm.G;
    return rows <= 16 ? 1 : (rows + kChunkRows - 1) / kChunkRows;
}
int64_t paged_attn_groups(const Dims &dm, int max_new) { return (int64_t)max_new * dm.G <= 16 ? 0 : (int64_t)dm.batch * dm.Hkv * paged_tiles(dm, max_new); }
static int64_t most_parts(const Dims &dm, bool few) {    // 128 keys and more to a part of few rows, a unit to a wavefront, or 256
    return max((int64_t)1, few ? min((int64_t)kMaxParts, ((int64_t)dm.max_seqlen + 127) / 128) : min((int64_t)kMaxChunkParts, ((int64_t)dm.max_seqlen + 255) / 256));
}
static PagedPlan paged_plan(const Dims &dm, int max_new) {
    PagedPlan p;
    p.few = (int64_t)max_new * dm.G <= 16;
    p.tiles = (int)paged_tiles(dm, max_new);
    p.items = (int64_t)dm.batch * dm.Hkv * p.tiles;
    // (three groups / one: 250 tiles of 2000 rows 37 / 52 us, 304 of 800 40 / 33, of 6000 186 / 185, 504 of 3000 109 / 107, of 6000 202 / 207; 20 new tokens of 100 / 300 / 500 rows
    // 12.8 / 9.5, 15.3 / 14.1, 17.8 / 18.3)
    p.groups = p.items <= kChunkItems && dm.max_seqlen > 448;
    // (of few rows and short caches one launch: 300 tokens 8.6 / 9.2 us, 500 10.3 / 9.3; 64 sequences of 1000 17.2 / 19.4, 32 of 768 12.9 / 12.1)
    // (of tiles: 20 new tokens of 300 / 500 / 700 / 1000 rows, 32 : 2 heads: 15.3 / 17.7 / 20.2 / 24.3 in one launch, 17.2 / 18.4 / 18.7 / 18.8 in parts)
    const bool alone = p.few ? dm.max_seqlen <= 320 || (dm.max_seqlen <= 1024 && p.items >= 128) : dm.max_seqlen <= 512;
    p.most = (int)most_parts(dm, p.few);
    p.parts = alone ? 1 : (int)max((int64_t)1, min((int64_t)p.most, (p.few ? kFewItems : kChunkItems) / p.items));
    p.batch = p.few && p.parts > 1 && dm.batch > 1 && (int64_t)dm.batch * dm.max_seqlen < (1ll << 31);
    if (p.batch) {                                       // (what the joining kernel takes by one, four or eight wavefronts: twice to eight times the mean)
        p.most = p.items >= 128 ? 16 : p.items >= 32 ? 64 : kMaxParts;
        p.parts = kFewItems / dm.Hkv + dm.batch;
    }
    if (!p.few && p.parts <= 16) p.most = min(p.most, 16);              // (of tiles with new tokens only: a wavefront joins up to 16)
    return p;
}
// (a bound that grows with each size: of the parts of few tiles)
size_t paged_attn_ws_bytes(const Dims &dm, int max_new) {
    if (dm.batch <= 0 || max_new <= 0) return 0;
    const bool few = (int64_t)max_new * dm.G <= 16;
    const int64_t items = min((int64_t)dm.batch * dm.Hkv * paged_tiles(dm, max_new), (int64_t)kFewItems);
    if (most_parts(dm, true) <= 1) return 0;
    const size_t rows = (size_t)((items + kFewItems + dm.Hkv) * (few ? 16 : kChunkRows));
    return align256(rows * kHeadDim * sizeof(float)) + align256(rows * sizeof(float2)) + align256(kFewItems * sizeof(int2));
}

int launch_paged_attn(const Dims &dm, Tensor q, const Pages &pg, NewTokens nt, const int32_t *seqlens, Tensor out, float *lse, void *ws, hipStream_t stream) {
    if (dm.batch <= 0 || nt.most <= 0) return 0;
    const int lg = __builtin_ctz(dm.G);
    const PagedPlan p = paged_plan(dm, nt.most);
    const int64_t rows = (int64_t)dm.batch * nt.most * dm.Hq;
    float *o_part = reinterpret_cast<float *>(ws);
    const size_t slots = !p.few ? (size_t)kChunkItems * kChunkRows : p.batch ? (size_t)p.parts * dm.Hkv * 16 : (size_t)rows * p.parts;
    float2 *ml_part = reinterpret_cast<float2 *>(reinterpret_cast<char *>(ws) + align256(slots * kHeadDim * sizeof(float)));
    int2 *plan = p.batch || (!p.few && p.parts > 1) ? reinterpret_cast<int2 *>(reinterpret_cast<char *>(ml_part) + align256(slots * sizeof(float2))) : nullptr;
    if (p.few) {
        timing_begin("paged_attn_few_kernel", stream);
        hipLaunchKernelGGL((p.batch ? paged_attn_few_kernel<true> : paged_attn_few_kernel<false>), dim3(p.batch ? kFewItems / dm.Hkv : p.parts, dm.Hkv, p.batch ? 1 : dm.batch), dim3(64 * kFewWaves), 0,
                           stream, dm, pg, nt, lg, q, seqlens, out, lse, o_part, ml_part, plan, kFewItems / dm.Hkv, p.most);
    } else {
        const int64_t items = p.parts > 1 ? kChunkItems : p.items;
        const int run = xcd_run_length(items);
        timing_begin("paged_attn_kernel", stream);
        hipLaunchKernelGGL((p.parts > 1 ? paged_attn_kernel<3, true> : p.groups ? paged_attn_kernel<3, false> : paged_attn_kernel<1, false>), dim3(xcd_grid(items, run)), dim3(p.groups ? 768 : 256), 0,
                           stream, dm, pg, nt, lg, p.parts > 1 ? p.most : p.tiles, run, q, seqlens, out, lse, o_part, ml_part, plan);
    }
    timing_end(stream);
    if (p.parts > 1) {
        timing_begin("paged_merge_kernel", stream);
        const int most = p.batch || !p.few ? p.most : p.parts, waves = most > 64 ? 8 : most > 16 ? 4 : 1;
        const auto join = !p.few ? (waves == 4 ? paged_merge_kernel<4, true> : paged_merge_kernel<1, true>)
                                 : waves == 8 ? paged_merge_kernel<8, false> : waves == 4 ? paged_merge_kernel<4, false> : paged_merge_kernel<1, false>;
        hipLaunchKernelGGL(join, dim3((unsigned)(waves > 1 ? rows : (rows + 3) / 4)), dim3(waves == 8 ? 512 : 256), 0, stream, dm, nt, p.parts, plan, rows, o_part,
                           ml_part, out, lse);
        timing_end(stream);
    }
    return (int)hipGetLastError();
}

}  // namespace infllmv2
