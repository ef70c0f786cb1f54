// What the cached rows of a sequence get of its new tokens' attention, summed over the tokens and the heads of a group.
//
// Keys are the rows of S = K . Q^T, so what a key gets is a sum over columns.  Each key belongs to one wavefront, and a sum's order is fixed.
#include "paged.h"

namespace infllmv2 {

// exp(score - lse) as a power of two: nothing for a head whose lse is -inf
__device__ __forceinline__ float lse_log2(float x) { return x == -INFINITY ? INFINITY : x * kLog2e; }

// Up to 16 query rows, all columns of one product; a wavefront takes units of 32 keys in turn.  grid (parts, Hkv, batch).  Bound by the keys' traffic
// (64 sequences of 4001 to 8191 rows: 43.7 us, 4.7 TB/s; one of 20000: 5.5, a chain of round trips).
__global__ __launch_bounds__(256) void paged_weights_few_kernel(Dims dm, Pages pg, NewTokens nt, int lg, Tensor q, const float *__restrict__ lse,
                                                                const int32_t *__restrict__ seqlens, const float *weights, int pitch, float *weights_out) {
    const int h = blockIdx.y, b = blockIdx.z, lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const Chunk ch(nt, seqlens, b, dm.max_seqlen);
    const int end = ch.L, units = (end + 31) >> 5, stride = 4 * gridDim.x, u0 = 4 * blockIdx.x + wave;
    const int count = u0 < units ? (units - u0 + stride - 1) / stride : 0;                    // units u0, u0 + stride, ..
    if (count == 0) return;
    const int token = n >> lg, hq = h * dm.G + (n & (dm.G - 1));
    const bool live = token < ch.n;
    bf16x8 bq[4];
    float z = INFINITY;
    if (ch.n > 0) {
        const __bf16 *qr = q.ptr + b * q.sb + (int64_t)min(token, ch.n - 1) * q.st + (int64_t)hq * q.sh + 8 * g;
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) bq[ks] = load8(qr + 32 * ks);
        if (live) z = lse_log2(lse[((int64_t)b * nt.most + token) * dm.Hq + hq]);
    } else {
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) bq[ks] = zero8();
    }
    const int last = live && z < INFINITY ? ch.before + token : -1;      // the last key that this column sees; a head without a sum adds nothing, whatever its scores are
    const char *k_head = reinterpret_cast<const char *>(pg.k.ptr + h * pg.k.sh);
    const uint32_t k_at = n * (2 * (uint32_t)pg.k.st) + 16 * g;
    const int32_t *table = pg.table + (int64_t)b * pg.ld;
    const int64_t row = ((int64_t)b * dm.Hkv + h) * pitch;
    struct Unit {
        bf16x8 k[2][4];
        float had;                                       // of key 16 (n / 4 % 2) + 4 g + n % 4, which this lane writes if n < 8
        uint32_t there;
        int k0;
    };
    UnitPages up;
    auto fetch = [&](Unit &u, int x) __attribute__((always_inline)) {
        if ((x & 63) == 0) up.load(pg, table, 32 * (u0 + stride * (x + lane)), x + lane < count ? end : 0);
        u.k0 = 32 * (u0 + stride * x);
        u.there = 0u;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const int page = __builtin_amdgcn_readlane(t ? up.hi : up.lo, x & 63), first = u.k0 + 16 * t;
            u.there |= page >= 0 ? 1u << t : 0u;
            const auto from = __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(k_head + page_bytes(pg.k, pg.lg, max(page, 0), first)), 0, 0xfffffffeu, 0x00027000);
            const uint32_t at = page >= 0 && first + n < end ? k_at : kNoRow;
#pragma unroll
            for (int ks = 0; ks < 4; ++ks)
                u.k[t][ks] = __builtin_bit_cast(bf16x8, (u32x4_t)__builtin_amdgcn_raw_buffer_load_b128(from, at, 64 * ks, 0));
        }
        const int key = u.k0 + 16 * (n >> 2) + 4 * g + (n & 3);
        u.had = weights && n < 8 && key < ch.before ? weights[row + key] : 0.f;
    };
    auto take = [&](const Unit &u) __attribute__((always_inline)) {
        float mine = 0.f;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int ks = 0; ks < 4; ++ks) s = mfma16(u.k[t][ks], bq[ks], s);
            const int at = (u.there >> t) & 1u ? last - u.k0 - 16 * t - 4 * g : -1;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float p = e <= at ? fast_exp2(__builtin_fmaf(s[e], dm.scale_log2, -z)) : 0.f;
                const float sum = row_reduce(p, [](float a, float d) { return a + d; });
                mine = n == 4 * t + e ? sum : mine;
            }
        }
        const int key = u.k0 + 16 * (n >> 2) + 4 * g + (n & 3);
        if (n < 8 && key < end) weights_out[row + key] = u.had + mine;
    };
    Unit a, c;
    fetch(a, 0);
    for (int x = 0; x < count; x += 2) {
        if (x + 1 < count) fetch(c, x + 1);
        take(a);
        if (x + 1 >= count) break;
        if (x + 2 < count) fetch(a, x + 2);
        take(c);
    }
}

// More rows: a workgroup takes 128 keys, 32 to a wavefront, which hold them in registers, and walks over the rows that see any of them, 32 at a time through LDS.
// What a lane adds up is one column's share of each of its keys.  Bound by the exponentials and the products, which are half of the attention's.
// 4096 new tokens over 32749 rows, 32 : 2 heads: 1.09 to 1.12 ms by card, 0.92 to 0.95 PFLOP/s, vector unit busy 71 %, matrix cores 53 %, at 1.84 GHz.
// Where tiles of keys are fewer than keep the chip evenly busy, a tile's rows are cut into parts, and a second kernel adds these up.
__global__ __launch_bounds__(256, 3) void paged_weights_kernel(Dims dm, Pages pg, NewTokens nt, int lg, int n_tiles, int n_part, int run, Tensor q, const float *__restrict__ lse,
                                                               const int32_t *__restrict__ seqlens, const float *weights, int pitch, float *weights_out,
                                                               float *__restrict__ partial) {
    __shared__ __align__(16) char slot0[kHalfTile], slot1[kHalfTile], slot2[kHalfTile];
    __shared__ int odd_s[4];
    const int item = xcd_item((blockIdx.y << kLgGroups) + blockIdx.x, run), bp = item / n_tiles, ti = item - bp * n_tiles, bh = bp / n_part, part = bp - bh * n_part, b = bh / dm.Hkv, h = bh - b * dm.Hkv;
    if (b >= dm.batch) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 31, hf = lane >> 5;
    const Chunk ch(nt, seqlens, b, dm.max_seqlen);
    const int first = 128 * ti, k0 = first + 32 * wave;
    if (first >= ch.L) return;
    const int32_t *table = pg.table + (int64_t)b * pg.ld;
    // ---- this wavefront's keys ----------------------------------------------------------------------------------------
    bf16x8 k[8];
    uint32_t there = 0u;
    {
        const int page = page_of(pg, table, k0 + (c & 16), ch.L), at = k0 + c;
        const bool some = page >= 0 && at < ch.L;
        const __bf16 *kr = pg.k.ptr + h * pg.k.sh + (some ? page_bytes(pg.k, pg.lg, page, at) / 2 : 0) + 8 * hf;
#pragma unroll
        for (int ks = 0; ks < 8; ++ks) k[ks] = some ? load8(kr + 16 * ks) : zero8();
        const uint32_t lanes = (uint32_t)__ballot(page >= 0);
        there = (lanes & 1u) | ((lanes >> 16) & 1u) << 1;
    }
    // ---- the rows: (token, head of the group), heads fastest, 32 to a unit -------------------------------------------------
    const int per = 32 >> lg, seen_from = max(0, first - ch.before) / per, all = (ch.n + per - 1) / per - seen_from;
    const int u0 = seen_from + (int)((int64_t)all * part / n_part), count = seen_from + (int)((int64_t)all * (part + 1) / n_part) - u0;
    const char *q_head = reinterpret_cast<const char *>(q.ptr + b * q.sb + (int64_t)h * dm.G * q.sh) + 64 * wave;
    uint32_t q_at[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const uint32_t row = 16 * j + (lane >> 2);
        q_at[j] = 2 * ((row >> lg) * (uint32_t)q.st + (row & (dm.G - 1)) * (uint32_t)q.sh) + 16 * copy_piece(lane);
    }
    auto stage = [&](char *dst, int x) __attribute__((always_inline)) {                        // two copies for every unit; rows behind the last are zeros
        const int t = per * (u0 + max(0, min(x, count - 1))), rows = x < count ? min(ch.n - t, per) << lg : 0;
        const char *from = q_head + 2 * (int64_t)t * q.st;
#pragma unroll
        for (int j = 0; j < 2; ++j) copy_rows(dst + wave * 2048 + j * 1024, from, 16 * j + (lane >> 2) < rows ? q_at[j] : kNoRow, 0);
    };
    const float *lse_at = lse + ((int64_t)b * nt.most + min(c >> lg, nt.most - 1)) * dm.Hq + h * dm.G + (c & (dm.G - 1));
    auto row_lse = [&](int x) __attribute__((always_inline)) {
        return lse_at[(int64_t)min(per * (u0 + x), max(0, ch.n - 1 - (c >> lg))) * dm.Hq];     // (of a row behind the last token: anything)
    };
    auto row_z = [&](float z, int x) __attribute__((always_inline)) {    // (made of it where it is used: it is two steps on its way)
        return x < count && per * (u0 + x) + (c >> lg) < ch.n ? lse_log2(z) : INFINITY;
    };
    const TileReader rd(lane);
    float sum[16];
    // 2^(score - inf) is 0 for a row behind the last token or without a sum, unless its score is NaN or infinite.  If a sum is no number, the walk is taken again with such rows left out by
    // comparison (in every unit at once, by a test of the row's z: 1071 -> 1112 us).
    bool careful = false;
    // Unit x lies in slot x % 3.  A step takes the exponentials of unit x and the products of unit x + 1, an instruction of one between those of the other: four wavefronts to a SIMD
    // that do one after the other overlap little (matrix cores 38 %, vector unit 60 % of the time, together all of it).
    auto arrived = [&]() __attribute__((always_inline)) {
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_waitcnt(0x0f72);              // all copies but the newest unit's two
        asm volatile("s_barrier" ::: "memory");          // everyone's, and everyone has read the unit before
        __builtin_amdgcn_sched_barrier(0);
    };
    float z0, z1, z2;
    f32x16 s;
    auto step = [&](const char *next, char *after, float &z, int x) __attribute__((always_inline)) {
        arrived();
        const float zx = row_z(z, x);
        z = row_lse(x + 3);
        stage(after, x + 3);
        bf16x8 qx[8];
#pragma unroll
        for (int ks = 0; ks < 8; ++ks) qx[ks] = rd.rows(next, ks);
        f32x16 s_next = zero16();
        const int t = ch.before + per * (u0 + x);        // position of the unit's first token
        if (k0 + 31 > t || careful) {
            const int at = zx < INFINITY ? t + (c >> lg) - k0 - 4 * hf : -1;          // keys up to this one are seen
#pragma unroll
            for (int e = 0; e < 16; ++e) sum[e] += 8 * (e >> 2) + (e & 3) <= at ? fast_exp2(__builtin_fmaf(s[e], dm.scale_log2, -zx)) : 0.f;
#pragma unroll
            for (int ks = 0; ks < 8; ++ks) s_next = mfma32(k[ks], qx[ks], s_next);
        } else {
#pragma unroll
            for (int ks = 0; ks < 8; ++ks) s_next = mfma32(k[ks], qx[ks], s_next);
#pragma unroll
            for (int e = 0; e < 16; ++e) sum[e] += fast_exp2(__builtin_fmaf(s[e], dm.scale_log2, -zx));
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);       // a product
                __builtin_amdgcn_sched_group_barrier(0x002, 2, 0);       // two to be scaled
                __builtin_amdgcn_sched_group_barrier(0x400, 2, 0);       // their exponentials
                __builtin_amdgcn_sched_group_barrier(0x002, 2, 0);       // added up
            }
        }
        settle<8>(s_next);
        s = s_next;
    };
#pragma unroll 1
    for (;;) {
#pragma unroll
        for (int e = 0; e < 16; ++e) sum[e] = 0.f;
        z0 = row_lse(0), z1 = row_lse(1), z2 = row_lse(2);
        stage(slot0, 0);
        stage(slot1, 1);
        arrived();
        s = zero16();
#pragma unroll
        for (int ks = 0; ks < 8; ++ks) s = mfma32(k[ks], rd.rows(slot0, ks), s);
        stage(slot2, 2);
        settle<8>(s);
        for (int x = 0; x < count; x += 3) {
            step(slot1, slot0, z0, x);
            if (x + 1 >= count) break;
            step(slot2, slot1, z1, x + 1);
            if (x + 2 >= count) break;
            step(slot0, slot2, z2, x + 2);
        }
        __builtin_amdgcn_s_waitcnt(0);                   // (the copies past the last unit have landed)
        if (careful) break;
        bool odd = false;
#pragma unroll
        for (int e = 0; e < 16; ++e) odd |= sum[e] != sum[e];
        if (lane == 0) odd_s[wave] = 0;
        if (odd) odd_s[wave] = 1;                        // (same wavefront: LDS keeps the order)
        __syncthreads();                                 // (the slots are free, too)
        if ((odd_s[0] | odd_s[1] | odd_s[2] | odd_s[3]) == 0) break;
        careful = true;
    }
    // ---- over the columns -------------------------------------------------------------------------------------------------
    float mine = 0.f;                                    // of key 8 (c / 4) + 4 hf + c % 4 in lanes c < 16
#pragma unroll
    for (int e = 0; e < 16; ++e) {
        const float half = row_reduce(sum[e], [](float a, float d) { return a + d; });
        const u32x2_t both = __builtin_amdgcn_permlane16_swap(__float_as_uint(half), __float_as_uint(half), false, false);
        const float all = __uint_as_float(both[0]) + __uint_as_float(both[1]);
        mine = c == e ? all : mine;
    }
    const int key = k0 + 8 * (c >> 2) + 4 * hf + (c & 3);
    if (c >= 16 || key >= ch.L) return;
    const int64_t at = (int64_t)bh * pitch + key;
    const bool seen = (there >> (c >> 3)) & 1u;          // (a row without a page gets nothing)
    if (n_part > 1) partial[(((int64_t)bh * n_tiles + ti) * n_part + part) * 128 + (key - first)] = seen ? mine : 0.f;
    else weights_out[at] = (weights && key < ch.before ? weights[at] : 0.f) + (seen ? mine : 0.f);
}

// grid (tiles, Hkv, batch), a thread to a key.
__global__ __launch_bounds__(128) void paged_weights_join_kernel(Dims dm, NewTokens nt, int n_part, const int32_t *__restrict__ seqlens,
                                                                 const float *__restrict__ partial, const float *weights, int pitch, float *weights_out) {
    const int h = blockIdx.y, b = blockIdx.z, key = 128 * blockIdx.x + threadIdx.x;
    const Chunk ch(nt, seqlens, b, dm.max_seqlen);
    if (key >= ch.L) return;
    const int64_t bh = (int64_t)b * dm.Hkv + h, at = bh * pitch + key;
    const float *from = partial + (bh * gridDim.x + blockIdx.x) * n_part * 128 + threadIdx.x;
    float sum = 0.f;
#pragma unroll 8
    for (int i = 0; i < n_part; ++i) sum += from[128 * i];
    weights_out[at] = (weights && key < ch.before ? weights[at] : 0.f) + sum;
}

// Workgroups run three to a compute unit.  Parts fill one such round, of at least four units of rows; four rounds, whose last is seldom empty for long, of at least 64 units
// (all of a tile / one round / four: 4096 tokens of 32749 rows, 32 : 2 heads, 1115 / 1114 / 1056 us; 1000 of 1000 201 / 18.7 / 27.9; 8 x 64 of 8192, 8 : 2, 19.5 / 18.6 / 27.6).
constexpr int kWeightRound = 3 * 256, kWeightItems = 4 * kWeightRound;
static int64_t weight_items(const Dims &dm) { return ((int64_t)dm.max_seqlen + 127) / 128 * dm.Hkv * dm.batch; }
int64_t paged_weights_groups(const Dims &dm) { return weight_items(dm); }
static int64_t most_weight_parts(const Dims &dm, int max_new) { return max((int64_t)1, (int64_t)max_new * dm.G / 128); }
static int weight_parts(const Dims &dm, int max_new) {
    const int64_t items = weight_items(dm), most = most_weight_parts(dm, max_new);
    return (int)max((int64_t)1, max(min(most, kWeightRound / items), min(most / 16, (kWeightItems + items - 1) / items)));
}
// (a bound that grows with each size)
size_t paged_weights_ws_bytes(const Dims &dm, int max_new) {
    const int64_t items = min(weight_items(dm), (int64_t)kWeightItems - 1), most = most_weight_parts(dm, max_new);
    if ((int64_t)max_new * dm.G <= 16 || most <= 1) return 0;
    return (size_t)min(items * most, items + kWeightItems) * 128 * sizeof(float);
}

int launch_paged_weights(const Dims &dm, Tensor q, const float *lse, const Pages &pg, NewTokens nt, const int32_t *seqlens, const float *weights, int pitch,
                         float *weights_out, void *ws, hipStream_t stream) {
    if (dm.batch <= 0 || nt.most <= 0 || dm.max_seqlen <= 0) return 0;
    const int lg = __builtin_ctz(dm.G);
    if ((int64_t)nt.most * dm.G <= 16) {
        const int64_t rows = (int64_t)dm.batch * dm.Hkv, units = ((int64_t)dm.max_seqlen + 31) / 32;
        const int parts = (int)max((int64_t)1, min((units + 3) / 4, (1024 + rows - 1) / rows));
        timing_begin("paged_weights_few_kernel", stream);
        hipLaunchKernelGGL(paged_weights_few_kernel, dim3(parts, dm.Hkv, dm.batch), dim3(256), 0, stream, dm, pg, nt, lg, q, lse, seqlens, weights, pitch,
                           weights_out);
        timing_end(stream);
        return (int)hipGetLastError();
    }
    const int tiles = (int)(((int64_t)dm.max_seqlen + 127) / 128);
    const int64_t items = weight_items(dm);
    const int parts = weight_parts(dm, nt.most);
    const int run = xcd_run_length(items * parts);
    float *partial = reinterpret_cast<float *>(ws);
    timing_begin("paged_weights_kernel", stream);
    const int64_t groups = xcd_grid(items * parts, run);
    hipLaunchKernelGGL(paged_weights_kernel, dim3(groups_x(groups), groups_beyond(groups)), dim3(256), 0, stream, dm, pg, nt, lg, tiles, parts, run, q, lse, seqlens,
                       weights, pitch, weights_out, partial);
    timing_end(stream);
    if (parts > 1) {
        timing_begin("paged_weights_join_kernel", stream);
        hipLaunchKernelGGL(paged_weights_join_kernel, dim3(tiles, dm.Hkv, dm.batch), dim3(128), 0, stream, dm, nt, parts, seqlens, partial, weights, pitch,
                           weights_out);
        timing_end(stream);
    }
    return (int)hipGetLastError();
}

}  // namespace infllmv2
