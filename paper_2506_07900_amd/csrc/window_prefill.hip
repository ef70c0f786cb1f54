// Attention over a sliding window and the first tokens, one query per cached token: one pass over the visible keys with a running
// maximum and sum.
//
// Query rows are (token, head of the group) with the heads fastest, so 128 of them see the same keys but for the few tokens they
// span, and a key tile is fetched once for them.  A wavefront takes 32 rows; key and value tiles of 64 tokens go from
// memory straight into LDS.  S^T = K . Q^T leaves a row's scores in a lane and its partner, so maxima and sums are
// per lane, and the probabilities are the second operand of O^T = V^T . P^T in the registers they come out in.
#include "window.h"

namespace infllmv2 {

constexpr int kFwdRows = 128;

// The running maximum follows a row's scores only where they exceed it by more than this (in powers of two): probabilities stay
// below 2^kSlack, and the outputs are rescaled once or twice per row instead of every tile.
constexpr float kSlack = 8.f;

// A wavefront's 32 rows: lane 32 hf + c holds row c.
struct QueryRows {
    WindowArgs win;
    float scale;                                         // to powers of two
    int lane, hf, i, hq, lo, hi;                         // the lane's token and head; first and last token of the wavefront
    TileReader rd;
    bf16x8 q[8];
    f32x16 o[4];                                         // channels 32 ct + 8 (e / 4) + 4 hf + e % 4
    float m, l;                                          // l: of this lane's keys
    __device__ __forceinline__ QueryRows(const Dims &dm, WindowArgs w, int lg, int t0, int first_row, int h, int lane)
        : win(w), scale(dm.scale_log2), lane(lane), hf(lane >> 5), rd(lane), m(-INFINITY), l(0.f) {
        const int row = first_row + (lane & 31);
        i = t0 + (row >> lg);
        hq = h * dm.G + (row & (dm.G - 1));
        lo = t0 + (first_row >> lg);
        hi = t0 + ((first_row + 31) >> lg);
    }
    __device__ __forceinline__ void load(const Tensor &t, int b, int L) {
        const __bf16 *qr = t.ptr + b * t.sb + (int64_t)min(i, L - 1) * t.st + (int64_t)hq * t.sh + 8 * hf;
#pragma unroll
        for (int ks = 0; ks < 8; ++ks) q[ks] = load8(qr + 16 * ks);
#pragma unroll
        for (int ct = 0; ct < 4; ++ct) o[ct] = zero16();
    }
    __device__ __forceinline__ void scores(const Tile64 &k, f32x16 (&s)[2]) const {
        s[0] = zero16();
        s[1] = zero16();
#pragma unroll
        for (int ks = 0; ks < 8; ++ks) {
            s[0] = mfma32(rd.rows(k.x, ks), q[ks], s[0]);
            s[1] = mfma32(rd.rows(k.x + kHalfTile, ks), q[ks], s[1]);
        }
    }
    __device__ __forceinline__ static float largest(const f32x16 (&s)[2]) {
        float a = max3(s[0][0], s[0][1], s[0][2]), d = max3(s[1][0], s[1][1], s[1][2]);
#pragma unroll
        for (int e = 3; e < 15; e += 2) {
            a = max3(a, s[0][e], s[0][e + 1]);
            d = max3(d, s[1][e], s[1][e + 1]);
        }
        return max3(max3(a, s[0][15], s[1][15]), d, d);
    }
    // the keys k0 .. k0 + 63 that a row does not see taken out, if there are any, and the largest of the others
    __device__ __forceinline__ void hide(f32x16 (&s)[2], int k0, float &mx) const {
        if (k0 + kWinKeys - 1 <= lo && (k0 + kWinKeys <= win.n_sink || hi - k0 < win.window)) return;
        int at = k0 + 4 * hf;
        asm volatile("" : "+v"(at));                     // (formed here: registers otherwise, held through the loop)
        const VisibleKeys visible(win, i);
#pragma unroll
        for (int kh = 0; kh < 2; ++kh)
#pragma unroll
            for (int e = 0; e < 16; ++e) s[kh][e] = visible(at + 32 * kh + 8 * (e >> 2) + (e & 3)) ? s[kh][e] : -INFINITY;
        mx = largest(s);
    }
    // mx: the largest of this lane's scores of a tile -> what its exponentials are referred to
    __device__ __forceinline__ float reference(float mx) {
        mx = half_reduce(mx, [](float a, float d) { return fmaxf(a, d); }) * scale;
        if (__any(mx > m + kSlack)) {
            const float m_new = fmaxf(m, mx), alpha = fast_exp2(m - (m_new == -INFINITY ? 0.f : m_new));
            m = m_new;
            l *= alpha;
#pragma unroll
            for (int ct = 0; ct < 4; ++ct) o[ct] *= alpha;
        }
        return m == -INFINITY ? 0.f : m;
    }
    __device__ __forceinline__ void add(f32x16 (&s)[2], float base, const Tile64 &v) {
        bf16x8 p[4];
        float sum[2] = {0.f, 0.f};
#pragma unroll
        for (int kh = 0; kh < 2; ++kh) {
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                s[kh][e] = fast_exp2(__builtin_fmaf(s[kh][e], scale, -base));
                sum[e & 1] += s[kh][e];
            }
            p[2 * kh] = pack8(s[kh], 0);                 // (bf16: what the matrix cores multiply; the sum is of what they were)
            p[2 * kh + 1] = pack8(s[kh], 1);
        }
        l += sum[0] + sum[1];
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int ct = 0; ct < 4; ++ct) o[ct] = mfma32(rd.columns(v.x + (j >> 1) * kHalfTile, j & 1, ct), p[j], o[ct]);
    }
};

// A unit of 32 keys, k0 ..: scores, and what they add.  kAhead: a wavefront that is alone on its SIMD asks for all operands before it uses them
// (4096 tokens, 4 : 1, whole window: 43.2 -> 41.5 us; dq 51.6 -> 50.0).
template <bool kAhead>
__device__ __forceinline__ void take_half(QueryRows &r, const KVHalf &cur, int k0) {
    f32x16 s = zero16();
    bf16x8 x[8];
    if constexpr (kAhead) {
#pragma unroll
        for (int ks = 0; ks < 8; ++ks) x[ks] = r.rd.rows(cur.k, ks);
        __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int ks = 0; ks < 8; ++ks) s = mfma32(kAhead ? x[ks] : r.rd.rows(cur.k, ks), r.q[ks], s);
    if constexpr (kAhead) {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = r.rd.columns(cur.v, i >> 2, i & 3);
        __builtin_amdgcn_sched_barrier(0);
    }
    settle<8>(s);
    if (!(k0 + 31 <= r.lo && (k0 + 32 <= r.win.n_sink || r.hi - k0 < r.win.window))) {
        int at = k0 + 4 * r.hf;
        asm volatile("" : "+v"(at));
        const VisibleKeys visible(r.win, r.i);
#pragma unroll
        for (int e = 0; e < 16; ++e) s[e] = visible(at + 8 * (e >> 2) + (e & 3)) ? s[e] : -INFINITY;
    }
    float mx = max3(s[0], s[1], s[2]);
#pragma unroll
    for (int e = 3; e < 15; e += 2) mx = max3(mx, s[e], s[e + 1]);
    const float base = r.reference(max3(mx, s[15], s[15]));
    float sum[2] = {0.f, 0.f};
#pragma unroll
    for (int e = 0; e < 16; ++e) {
        s[e] = fast_exp2(__builtin_fmaf(s[e], r.scale, -base));
        sum[e & 1] += s[e];
    }
    r.l += sum[0] + sum[1];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const bf16x8 p = pack8(s, j);
#pragma unroll
        for (int ct = 0; ct < 4; ++ct) r.o[ct] = mfma32(kAhead ? x[4 * j + ct] : r.rd.columns(cur.v, j, ct), p, r.o[ct]);
    }
}

// A product multiplies a key that a row does not see by a probability of 0, and 0 times an infinity or a NaN reaches the row's sum; and sums that are divided
// at the end only overflow where values are near the largest.  Rows that do not come out finite though the sum of their probabilities did are
// therefore taken again, all of the wavefront's at once: their maxima m and sums l stand (hidden scores are replaced, not multiplied), so probabilities are
// 2^(score - m - down) with a sum of 1/4 to 1/2.  In a unit of keys that not all rows see whole, values that are not finite are left out
// of the product and added to the rows that see them.  V goes through 8 KiB of LDS of the wavefront's own; nothing is asked for ahead.  With an
// infinity that all rows see: 777 tokens, 4 : 1, window 256 10.6 -> 82 us, 4096 tokens, 8 : 2, whole window 94 -> 365, 32K, 32 : 2, window 4096 2.09 -> 6.04 ms
// (key by key it was 430 us, 29 ms and 423 ms).
__device__ __forceinline__ int down_of(float l) { return __builtin_amdgcn_frexp_expf(l) + 1; }
__device__ __forceinline__ void take_again(QueryRows &r, const Tensor &k, const Tensor &v, int b, int h, int L, float m, float down, char *lds) {
    const KeyTiles<32> kt(r.win, r.lo, min(L, r.hi + 1));
    int lane = r.lane;
    asm volatile("" : "+v"(lane));                       // (nothing of this is worked out before it is needed)
    const int hf = lane >> 5;
    const TileReader rd(lane);
    const VisibleKeys visible(r.win, r.i);
    const int64_t k_head = b * k.sb + h * k.sh, v_head = b * v.sb + h * v.sh;
    const uint32_t v_at = (lane >> 2) * (2 * (uint32_t)v.st) + 16 * copy_piece(lane);
#pragma unroll
    for (int ct = 0; ct < 4; ++ct) r.o[ct] = zero16();
#pragma unroll 1
    for (int x = 0; x < kt.count; ++x) {
        const int k0 = kt.key0(x);
        const char *vb = reinterpret_cast<const char *>(v.ptr + v_head + (int64_t)k0 * v.st);
        const __bf16 *kr = k.ptr + k_head + (int64_t)min(k0 + (lane & 31), L - 1) * k.st + 8 * hf;
        reads_done();                                    // (the unit before)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int quarter = 0; quarter < 4; ++quarter)
                copy_rows(lds + quarter * 2048 + j * 1024, vb + 64 * quarter, k0 + 16 * j + (lane >> 2) < L ? v_at : kNoRow, 32 * j * (uint32_t)v.st);
        f32x16 s = zero16();
#pragma unroll
        for (int ks = 0; ks < 8; ++ks) {
            s = mfma32(load8(kr + 16 * ks), r.q[ks], s);
            if (ks == 3) __builtin_amdgcn_sched_barrier(0);          // (registers)
        }
#pragma unroll
        for (int e = 0; e < 16; ++e)
            s[e] = visible(k0 + 4 * hf + 8 * (e >> 2) + (e & 3)) ? fast_exp2(__builtin_fmaf(s[e], r.scale, -m) - down) : 0.f;
        const bool whole = k0 + 31 <= r.lo && (k0 + 32 <= r.win.n_sink || r.hi - k0 < r.win.window);
        bool odd = false;
        copies_landed(false);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const bf16x8 p = pack8(s, j);
#pragma unroll
            for (int ct = 0; ct < 4; ++ct) {
                u32x4_t y = __builtin_bit_cast(u32x4_t, rd.columns(lds, j, ct));
                if (!whole) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {        // the halves of a word whose exponents are all ones
                        const bool low = (y[i] & 0x7f80u) == 0x7f80u, high = (y[i] & 0x7f800000u) == 0x7f800000u;
                        y[i] = (low ? 0u : y[i] & 0xffffu) | (high ? 0u : y[i] & 0xffff0000u);
                        odd |= low | high;
                    }
                }
                r.o[ct] = mfma32(__builtin_bit_cast(bf16x8, y), p, r.o[ct]);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        if (!__any(odd)) continue;
#pragma unroll 1
        for (int t = 0; t < 32; ++t) {
            const bool sees = visible(k0 + t);
            const char *row = lds + 64 * t + 8 * hf;
#pragma unroll
            for (int ct = 0; ct < 4; ++ct)
#pragma unroll
                for (int e4 = 0; e4 < 4; ++e4) {
                    const uint2 y = *reinterpret_cast<const uint2 *>(row + ct * 2048 + ((e4 ^ ((t >> 2) & 3)) << 4));
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const uint32_t w = e < 2 ? y.x : y.y;
                        const float z = __uint_as_float(e & 1 ? w & 0xffff0000u : w << 16);
                        r.o[ct][4 * e4 + e] += sees && !(__builtin_fabsf(z) < INFINITY) ? z : 0.f;
                        __builtin_amdgcn_sched_barrier(0);               // (registers)
                    }
                }
        }
    }
}

// The end of a wavefront's 32 rows, with 8 KiB of LDS.
__device__ __forceinline__ void finish_rows(const Dims &dm, WindowArgs win, int lg, int t0, QueryRows &r, const Tensor &q, const Tensor &k, const Tensor &v,
                                            int b, int h, int L, int wave, int lane, char *lds, const Tensor &out, float *__restrict__ lse) {
    r.l = half_reduce(r.l, [](float a, float d) { return a + d; });
    const bool live = r.i < L;
    float check = 0.f;
#pragma unroll
    for (int ct = 0; ct < 4; ++ct)
#pragma unroll
        for (int e = 0; e < 16; ++e) check = __builtin_fmaf(r.o[ct][e], 0.f, check);
    const uint64_t bad_lanes = __ballot(live && check != 0.f && r.l == r.l), live_lanes = __ballot(live);
    const uint32_t bad = (uint32_t)bad_lanes | (uint32_t)(bad_lanes >> 32);
    const uint32_t alive = (uint32_t)live_lanes;
    if (alive != ~0u) {                                  // (rows behind the sequence: zeros, where they are written at all)
#pragma unroll
        for (int ct = 0; ct < 4; ++ct)
#pragma unroll
            for (int e = 0; e < 16; ++e) r.o[ct][e] = live ? r.o[ct][e] : 0.f;
    }
    auto to = [&](int row) __attribute__((always_inline)) {
        const int i = t0 + ((32 * wave + row) >> lg), hq = h * dm.G + ((32 * wave + row) & (dm.G - 1));
        return out.ptr + b * out.sb + (int64_t)i * out.st + (int64_t)hq * out.sh;
    };
    store_rows(lds, r.o, live ? 1.f / r.l : 0.f, lane, [&](int row) __attribute__((always_inline)) -> __bf16 * {
        const bool store = t0 + ((32 * wave + row) >> lg) < dm.max_seqlen && ((alive >> row) & 1u || dm.fill) && !((bad >> row) & 1u);
        return store ? to(row) : nullptr;
    });
    if (r.hf == 0 && r.i < dm.max_seqlen && (live || dm.fill)) lse[((int64_t)b * dm.max_seqlen + r.i) * dm.Hq + r.hq] = live ? lse_of(r.m, r.l) : 0.f;
    if (__builtin_expect(bad != 0u, 0)) {
        const int down = down_of(r.l);
        take_again(r, k, v, b, h, L, r.m, (float)down, lds);
        asm volatile("" : "+v"(lane));                   // (no addresses held meanwhile)
        store_rows(lds, r.o, 1.f / __builtin_ldexpf(r.l, -down), lane,
                   [&](int row) __attribute__((always_inline)) -> __bf16 * { return (bad >> row) & 1u ? to(row) : nullptr; });
    }
}
// A wavefront's rows that lie behind the sequence.
__device__ __forceinline__ void clear_rows(const Dims &dm, const QueryRows &r, int b, const Tensor &out, float *__restrict__ lse) {
    if (!dm.fill || r.i >= dm.max_seqlen) return;
    __bf16 *o_row = out.ptr + b * out.sb + (int64_t)r.i * out.st + (int64_t)r.hq * out.sh + 64 * r.hf;
    for (int c = 0; c < 8; ++c) reinterpret_cast<uint4 *>(o_row)[c] = uint4{0u, 0u, 0u, 0u};
    if (r.hf == 0) lse[((int64_t)b * dm.max_seqlen + r.i) * dm.Hq + r.hq] = 0.f;
}

// A workgroup's 128 rows by two halves, which take every other tile and are joined at the end; in each one tile's scores are ahead of another's
// exponentials.
__global__ __launch_bounds__(512, 2) void window_prefill_kernel(Dims dm, WindowArgs win, int lg, int n_tiles, int run, Tensor q, Tensor k, Tensor v,
                                                                const int32_t *__restrict__ seqlens, Tensor out, float *__restrict__ lse) {
    __shared__ Tile64 K0[2], K1[2], V0[2], V1[2];
    __shared__ float2 ml[4][64];
    const int item = xcd_item(blockIdx.x, run), bh = item / n_tiles, b = bh / dm.Hkv, h = bh - b * dm.Hkv;
    if (b >= dm.batch) return;
    const int ti = (bh + 1) * n_tiles - 1 - item;        // the last rows, which see most keys, first
    const int lane = threadIdx.x & 63, id = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = id >> 2, wave = id & 3;
    const int L = clamp_len(uniform_load(seqlens + b), dm.max_seqlen);
    const int t0 = ti * (kFwdRows >> lg), t1 = min(L, t0 + (kFwdRows >> lg));
    QueryRows r(dm, win, lg, t0, 32 * wave, h, lane);
    if (t0 >= L) {
        if (half == 0) clear_rows(dm, r, b, out, lse);
        return;
    }
    const KeyTiles<kWinKeys> kt(win, t0, t1);
    const int count = (kt.count + 1 - half) >> 1, steps = (kt.count + 1) >> 1;   // this half's tiles; the first one's
    auto key0 = [&](int x) __attribute__((always_inline)) { return kt.key0(2 * x + half); };
    const TileCopier keys(k, b, h, L, wave, lane), values(v, b, h, L, wave, lane);
    auto stage = [&](const TileCopier &from, Tile64 *to, int x) __attribute__((always_inline)) {
        if (x < count) from.copy(to[half], key0(x), wave, lane);
    };
    stage(keys, K0, 0);
    stage(values, V0, 0);
    stage(keys, K1, 1);
    stage(values, V1, 1);
    r.load(q, b, L);
    // Tile x: its probabilities and their product with the values, and between them the next tile's scores, so that the matrix cores have
    // work while the exponentials run.  (Behind the last tile: scores of what lies in LDS, not used.)
    auto step = [&](Tile64 *k_cur, const Tile64 *k_next, const Tile64 *v_cur, Tile64 *v_next, f32x16 (&s)[2], f32x16 (&s_next)[2], float &mx,
                    int x) __attribute__((always_inline)) {
        __builtin_amdgcn_s_waitcnt(0);                   // this wavefront's copies have landed
        __syncthreads();                                 // everyone's have, and everyone is past the tile before
        stage(keys, k_cur, x + 2);
        if (x > 0) stage(values, v_next, x + 1);         // (the first two at once: a short walk is a chain of round trips)
        if (x >= count) return;           // (the other half has one more)
        const float base = r.reference(mx);
        __builtin_amdgcn_sched_barrier(0);
        r.scores(k_next[half], s_next);
        r.add(s, base, v_cur[half]);
        mx = QueryRows::largest(s_next);
        __builtin_amdgcn_sched_barrier(0);
        if (x + 1 < count) r.hide(s_next, key0(x + 1), mx);
    };
    f32x16 sa[2], sb[2];
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
    r.scores(K0[half], sa);
    float mx = QueryRows::largest(sa);
    r.hide(sa, key0(0), mx);
    for (int x = 0; x < steps; x += 2) {
        step(K0, K1, V0, V1, sa, sb, mx, x);
        if (x + 1 < steps) step(K1, K0, V1, V0, sb, sa, mx, x + 1);
    }
    __syncthreads();                                     // the tiles are free
    // a row's state is in the same lanes of both halves: the second hands its own over
    char *at = (wave == 0 ? K0 : wave == 1 ? K1 : wave == 2 ? V0 : V1)[1].x + 16 * lane;
    if (half == 1) {
        ml[wave][lane] = float2{r.m, r.l};
#pragma unroll
        for (int ct = 0; ct < 4; ++ct)
#pragma unroll
            for (int e4 = 0; e4 < 4; ++e4)
                *reinterpret_cast<f32x4 *>(at + 1024 * (4 * ct + e4)) = f32x4{r.o[ct][4 * e4], r.o[ct][4 * e4 + 1], r.o[ct][4 * e4 + 2], r.o[ct][4 * e4 + 3]};
    }
    __syncthreads();
    if (half == 1) return;
    const float2 other = ml[wave][lane];
    const float M = fmaxf(r.m, other.x), base = M == -INFINITY ? 0.f : M, mine = fast_exp2(r.m - base), theirs = fast_exp2(other.x - base);
    r.m = M;
    r.l = r.l * mine + other.y * theirs;
#pragma unroll
    for (int ct = 0; ct < 4; ++ct)
#pragma unroll
        for (int e4 = 0; e4 < 4; ++e4) {
            const f32x4 x = *reinterpret_cast<const f32x4 *>(at + 1024 * (4 * ct + e4));
#pragma unroll
            for (int e = 0; e < 4; ++e) r.o[ct][4 * e4 + e] = r.o[ct][4 * e4 + e] * mine + x[e] * theirs;
        }
    finish_rows(dm, win, lg, t0, r, q, k, v, b, h, L, wave, lane, (wave < 2 ? K0 : K1)[0].x + (wave & 1) * kHalfTile, out, lse);
}

// The same for many rows: three workgroups of four wavefronts to a compute unit, so that one's exponentials run under another's products and round trips,
// with units of 32 keys, two ahead, in three slots, and a unit's scores at a time.  Its smaller units also leave less to hide.  32K tokens, 32 : 2
// heads, window 4096: 1.94 to 2.02 ms, 1.04 to 1.08 PFLOP/s; bound by the matrix cores' power (1.4 to 1.7 GHz under this load; a large library product
// reaches 1.36).  64 rows to a wavefront, which read each key and value from LDS half as often: 1.95 against 2.01 ms here, 607 against 591 us
// for 64K tokens x 4 heads and window 1024, so not taken.
__global__ __launch_bounds__(256, 3) void window_prefill_many_kernel(Dims dm, WindowArgs win, int lg, int n_tiles, int run, Tensor q, Tensor k,
                                                                     Tensor v, const int32_t *__restrict__ seqlens, Tensor out,
                                                                     float *__restrict__ lse) {
    __shared__ KVHalf slot0, slot1, slot2;
    const int item = xcd_item(blockIdx.x, run), bh = item / n_tiles, b = bh / dm.Hkv, h = bh - b * dm.Hkv;
    if (b >= dm.batch) return;
    const int ti = (bh + 1) * n_tiles - 1 - item;        // the last rows, which see most keys, first
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int L = clamp_len(uniform_load(seqlens + b), dm.max_seqlen);
    const int t0 = ti * (kFwdRows >> lg), t1 = min(L, t0 + (kFwdRows >> lg));
    QueryRows r(dm, win, lg, t0, 32 * wave, h, lane);
    if (t0 >= L) return clear_rows(dm, r, b, out, lse);
    const KeyTiles<32> kt(win, t0, t1);
    const char *k_head = reinterpret_cast<const char *>(k.ptr + b * k.sb + h * k.sh) + 64 * wave;
    const char *v_head = reinterpret_cast<const char *>(v.ptr + b * v.sb + h * v.sh) + 64 * wave;
    const uint32_t k_at = (lane >> 2) * (2 * (uint32_t)k.st) + 16 * copy_piece(lane), v_at = (lane >> 2) * (2 * (uint32_t)v.st) + 16 * copy_piece(lane);
    // four copies for every unit: those past the last bring zeros
    auto stage = [&](KVHalf &dst, int x) __attribute__((always_inline)) {
        const int k0 = kt.key0(min(x, kt.count - 1)), end = x < kt.count ? L : 0;
        const char *kb = k_head + (int64_t)k0 * (2 * k.st), *vb = v_head + (int64_t)k0 * (2 * v.st);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const bool row = k0 + 16 * j + (lane >> 2) < end;
            copy_rows(dst.k + wave * 2048 + j * 1024, kb, row ? k_at : kNoRow, 32 * j * (uint32_t)k.st);
            copy_rows(dst.v + wave * 2048 + j * 1024, vb, row ? v_at : kNoRow, 32 * j * (uint32_t)v.st);
        }
    };
    r.load(q, b, L);
    stage(slot0, 0);
    stage(slot1, 1);
    auto step = [&](const KVHalf &cur, KVHalf &next, int x) __attribute__((always_inline)) {
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_waitcnt(0x0f74);              // all copies but the next unit's four
        asm volatile("s_barrier" ::: "memory");          // everyone's, and everyone is past the unit before
        __builtin_amdgcn_sched_barrier(0);
        stage(next, x + 2);
        const int k0 = kt.key0(x);
        if (k0 <= r.hi && (k0 < win.n_sink || r.lo - (k0 + 31) < win.window)) take_half<false>(r, cur, k0);   // (some of the rows see some of the keys)
    };
    for (int x = 0; x < kt.count; x += 3) {
        step(slot0, slot2, x);
        if (x + 1 < kt.count) step(slot1, slot0, x + 1);
        if (x + 2 < kt.count) step(slot2, slot1, x + 2);
    }
    __builtin_amdgcn_s_waitcnt(0);                       // (the copies past the last unit have landed)
    __syncthreads();
    finish_rows(dm, win, lg, t0, r, q, k, v, b, h, L, wave, lane, (wave < 2 ? slot0.k : slot1.k) + (wave & 1) * kHalfTile, out, lse);
}

// The same for few rows: a workgroup takes 32 of them, its wavefronts every fourth unit of 32 keys each, fetched for itself and without a
// barrier; their four states are joined in LDS at the end.
__global__ __launch_bounds__(256, 1) void window_prefill_few_kernel(Dims dm, WindowArgs win, int lg, int n_tiles, Tensor q, Tensor k, Tensor v,
                                                                    const int32_t *__restrict__ seqlens, Tensor out, float *__restrict__ lse) {
    __shared__ KVHalf slot0[4], slot1[4];
    __shared__ float ml[2][4][32];
    const int bh = blockIdx.x / n_tiles, b = bh / dm.Hkv, h = bh - b * dm.Hkv;
    const int ti = (bh + 1) * n_tiles - 1 - (int)blockIdx.x;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int L = clamp_len(uniform_load(seqlens + b), dm.max_seqlen);
    const int t0 = ti * (32 >> lg), t1 = min(L, t0 + (32 >> lg));
    QueryRows r(dm, win, lg, t0, 0, h, lane);
    // the result's row and 16 channels of this thread
    const int row = tid >> 3, ch = 16 * (tid & 7), i = t0 + (row >> lg), hq = h * dm.G + (row & (dm.G - 1));
    __bf16 *o_row = out.ptr + b * out.sb + (int64_t)i * out.st + (int64_t)hq * out.sh + ch;
    float *lse_at = lse + ((int64_t)b * dm.max_seqlen + i) * dm.Hq + hq;
    const bool store = i < dm.max_seqlen && (i < L || dm.fill);
    if (t0 >= L) {
        if (store) {
            reinterpret_cast<uint4 *>(o_row)[0] = reinterpret_cast<uint4 *>(o_row)[1] = uint4{0u, 0u, 0u, 0u};
            if (ch == 0) *lse_at = 0.f;
        }
        return;
    }
    const KeyTiles<32> kt(win, t0, t1);
    r.load(q, b, L);
    walk_halves(slot0[wave], slot1[wave], k, v, b, h, kt, L, wave, lane,
                [&](const KVHalf &cur, int k0) __attribute__((always_inline)) { take_half<true>(r, cur, k0); });
    reads_done();
    r.l = half_reduce(r.l, [](float a, float d) { return a + d; });
    if (r.hf == 0) {
        ml[0][wave][lane] = r.m;
        ml[1][wave][lane] = r.l;
    }
    // [row][channel], 16-byte pieces XORed with the row
    float *mine = reinterpret_cast<float *>(&slot0[wave]);
#pragma unroll
    for (int ct = 0; ct < 4; ++ct)
#pragma unroll
        for (int e4 = 0; e4 < 4; ++e4)
            *reinterpret_cast<f32x4 *>(mine + (lane & 31) * kHeadDim + 4 * ((8 * ct + 2 * e4 + r.hf) ^ (lane & 7))) =
                f32x4{r.o[ct][4 * e4], r.o[ct][4 * e4 + 1], r.o[ct][4 * e4 + 2], r.o[ct][4 * e4 + 3]};
    __syncthreads();
    float M = -INFINITY, den = 0.f, y[16], check = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) M = fmaxf(M, ml[0][w][row]);
#pragma unroll
    for (int e = 0; e < 16; ++e) y[e] = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        const float f = fast_exp2(ml[0][w][row] - M);    // (a row sees its own key: M is a number)
        den += f * ml[1][w][row];
        const float *from = reinterpret_cast<const float *>(&slot0[w]) + row * kHeadDim;
#pragma unroll
        for (int e4 = 0; e4 < 4; ++e4) {
            const f32x4 a = *reinterpret_cast<const f32x4 *>(from + 4 * ((ch / 4 + e4) ^ (row & 7)));
#pragma unroll
            for (int e = 0; e < 4; ++e) y[4 * e4 + e] += f * a[e];
        }
    }
#pragma unroll
    for (int e = 0; e < 16; ++e) check = __builtin_fmaf(y[e], 0.f, check);
    const uint64_t bad = __ballot(i < L && check != 0.f && den == den);
    const bool whole = ((bad >> (lane & 56)) & 255u) == 0u;                    // this row's eight lanes
    if (store) {
        const float inv = 1.f / den;
        bf16x8 z[2];
#pragma unroll
        for (int e = 0; e < 16; ++e) z[e >> 3][e & 7] = (__bf16)(i < L ? y[e] * inv : 0.f);
        if (whole) {
            reinterpret_cast<uint4 *>(o_row)[0] = __builtin_bit_cast(uint4, z[0]);
            reinterpret_cast<uint4 *>(o_row)[1] = __builtin_bit_cast(uint4, z[1]);
        }
        if (ch == 0) *lse_at = i < L ? lse_of(M, den) : 0.f;
    }
    if (__builtin_expect(bad != 0ull, 0)) {              // of the 32 rows the eight of this wavefront's lanes
        uint32_t rows = 0u;
#pragma unroll
        for (int j = 0; j < 8; ++j) rows |= (uint32_t)((bad >> (8 * j)) & 255u ? 1u : 0u) << (8 * wave + j);
        const int n = lane & 31;
        float top = -INFINITY, sum = 0.f;
#pragma unroll
        for (int w = 0; w < 4; ++w) top = fmaxf(top, ml[0][w][n]);
#pragma unroll
        for (int w = 0; w < 4; ++w) sum += fast_exp2(ml[0][w][n] - top) * ml[1][w][n];
        const int down = down_of(sum);
        take_again(r, k, v, b, h, L, top, (float)down, slot1[wave].k);
        store_rows(slot1[wave].k, r.o, 1.f / __builtin_ldexpf(sum, -down), lane, [&](int at) __attribute__((always_inline)) -> __bf16 * {
            return (rows >> at) & 1u ? out.ptr + b * out.sb + (int64_t)(t0 + (at >> lg)) * out.st + (int64_t)(h * dm.G + (at & (dm.G - 1))) * out.sh : nullptr;
        });
    }
}

size_t window_prefill_ws_bytes(const Dims &, WindowArgs) { return 0; }

int launch_window_prefill(const Dims &dm, WindowArgs w, Tensor q, Tensor k, Tensor v, const int32_t *seqlens, Tensor out, float *lse,
                          void *, hipStream_t stream) {
    if (dm.batch <= 0 || dm.max_seqlen <= 0) return 0;
    const int lg = __builtin_ctz(dm.G);
    const int64_t heads = (int64_t)dm.Hkv * dm.batch;
    auto tiles = [&](int rows) { return (dm.max_seqlen + (rows >> lg) - 1) / (rows >> lg); };
    const int64_t items = tiles(kFwdRows) * heads;
    const int run = xcd_run_length(items);
    // few_rows: workgroups of 32 (2048 tokens, 4 heads : 1, whole window 42 -> 20 us; 4096 tokens, window 4096 / 1000 / 256: 79 / 28 / 13.8 -> 43 /
    // 27 / 15.6; twice as many rows, whole window: 84 -> 88).  by_halves (8192 tokens, 4 : 1, window 8192 / 3000 / 1000: 166 / 69 / 32 -> 123 / 55 / 30;
    // 8 : 2, window 8192: 245 -> 178, but 4096: 136 -> 147).  Beyond three workgroups per compute unit.
    const bool halves = by_halves(dm, w, items);
    if (few_rows(dm, w, items)) {
        timing_begin("window_prefill_few_kernel", stream);
        hipLaunchKernelGGL(window_prefill_few_kernel, dim3((unsigned)(tiles(32) * heads)), dim3(256), 0, stream, dm, w, lg, tiles(32), q, k, v,
                           seqlens, out, lse);
    } else {
        timing_begin(halves ? "window_prefill_kernel" : "window_prefill_many_kernel", stream);
        hipLaunchKernelGGL(halves ? window_prefill_kernel : window_prefill_many_kernel, dim3(xcd_grid(items, run)), dim3(halves ? 512 : 256), 0, stream,
                           dm, w, lg, tiles(kFwdRows), run, q, k, v, seqlens, out, lse);
    }
    timing_end(stream);
    return (int)hipGetLastError();
}

}  // namespace infllmv2
