// Gradients of the windowed attention.  With p = exp(scale <q_i, k_t> - lse_i) over the visible keys and D_i = <dout_i, out_i>:
//     dv_t = sum p dout_i      ds = p (<dout_i, v_t> - D_i)      dq_i = scale sum ds k_t      dk_t = scale sum ds q_i
// Two kernels, each of which sums what it owns in registers, so nothing is added atomically and results repeat: dq walks the
// keys of 128 query rows as the forward does and leaves every row's log-sum-exp and D for the other; dk/dv walks the rows that see 128
// keys.  The scores are computed in both (7 products instead of 5: the other way is 4 bytes of atomics per row, channel and key
// tile).
#include "window.h"

namespace infllmv2 {

constexpr int kDqRows = 128;
struct KVTile {
    Tile64 k, v;
};

// What the forward leaves of a row (token, head of the group): its log-sum-exp in powers of two and -D, 32 and 32 floats for 32 rows.
__host__ __device__ static inline int64_t row_blocks(const Dims &dm) { return ((int64_t)dm.max_seqlen * dm.G + 31) / 32; }   // per (sequence, head)

// dq of 128 rows, and what the rows leave for the other kernel.  A wavefront's 32 rows of q and dout stay in registers, keys and values come in tiles of 64,
// one ahead; two workgroups to a compute unit, so that one's exponentials run under the other's products.  32K tokens, 32 : 2 heads, window
// 4096: 2.65 ms, 1.18 PFLOP/s of its three products, bound by the matrix cores' power as dk/dv is.  kHalves 2, as in the forward: 4096 tokens, 8 : 2,
// whole window, 106 -> 88 us; 8192, 8 : 2, whole window 316 -> 224, but window 4096 183 -> 191.  Half a tile's exponentials stand between the other half's
// products, and a product's operands are read one ahead (2 x 4096, 16 : 2, window 1000: 110.4 -> 104; two ahead the same).
template <int kHalves>
__global__ __launch_bounds__(256 * kHalves, 2) void window_dq_kernel(Dims dm, WindowArgs win, float scale, int lg, int n_tiles, int run, Tensor q,
                                                                     Tensor k, Tensor v, Tensor out, Tensor dout, const float *__restrict__ lse,
                                                                     const int32_t *__restrict__ seqlens, Tensor dq, float *__restrict__ rows) {
    __shared__ KVTile tile0[kHalves], tile1[kHalves];
    const int item = xcd_item(blockIdx.x, run), bh = item / n_tiles, b = bh / dm.Hkv, h = bh - b * dm.Hkv;
    if (b >= dm.batch) return;
    const int ti = (bh + 1) * n_tiles - 1 - item;        // the last rows, which see most keys, first
    const int tid = threadIdx.x, lane = tid & 63, id = __builtin_amdgcn_readfirstlane(tid >> 6), half = kHalves == 1 ? 0 : id >> 2, wave = id & 3;
    const int c32 = lane & 31, hf = lane >> 5;
    const int L = clamp_len(uniform_load(seqlens + b), dm.max_seqlen);
    const int t0 = ti * (kDqRows >> lg), t1 = min(L, t0 + (kDqRows >> lg));
    const int row = 32 * wave + c32, i = t0 + (row >> lg), hq = h * dm.G + (row & (dm.G - 1));
    __bf16 *dq_row = dq.ptr + b * dq.sb + (int64_t)i * dq.st + (int64_t)hq * dq.sh + 4 * hf;
    if (t0 >= L) {
        if (dm.fill && half == 0 && i < dm.max_seqlen)
            for (int c = 0; c < 16; ++c) *reinterpret_cast<uint2 *>(dq_row + 8 * c) = uint2{0u, 0u};
        return;
    }
    const KeyTiles<kWinKeys> kt(win, t0, t1);
    const TileCopier keys(k, b, h, L, wave, lane), values(v, b, h, L, wave, lane);
    const int count = (kt.count + kHalves - 1 - half) / kHalves, steps = (kt.count + kHalves - 1) / kHalves;   // this half's tiles; the first one's
    auto key0 = [&](int x) __attribute__((always_inline)) { return kt.key0(kHalves * x + half); };
    auto stage = [&](KVTile *dst, int x) __attribute__((always_inline)) {
        if (x >= count) return;
        keys.copy(dst[half].k, key0(x), wave, lane);
        values.copy(dst[half].v, key0(x), wave, lane);
    };
    stage(tile0, 0);
    bf16x8 qf[8], gf[8];
    float D = 0.f, ref;
    {
        const int64_t t = min(i, L - 1);
        const __bf16 *qr = q.ptr + b * q.sb + t * q.st + (int64_t)hq * q.sh + 8 * hf;
        const __bf16 *gr = dout.ptr + b * dout.sb + t * dout.st + (int64_t)hq * dout.sh + 8 * hf;
        const __bf16 *orow = out.ptr + b * out.sb + t * out.st + (int64_t)hq * out.sh + 8 * hf;
#pragma unroll
        for (int ks = 0; ks < 8; ++ks) {
            qf[ks] = load8(qr + 16 * ks);
            gf[ks] = load8(gr + 16 * ks);
            const bf16x8 x = load8(orow + 16 * ks);
#pragma unroll
            for (int e = 0; e < 8; ++e) D = __builtin_fmaf((float)gf[ks][e], (float)x[e], D);
        }
        D = half_reduce(D, [](float a, float d) { return a + d; });
        ref = lse[((int64_t)b * dm.max_seqlen + t) * dm.Hq + hq] * kLog2e;
        const int64_t r = (int64_t)ti * kDqRows + row;
        if (i < L && half == 0) rows[((int64_t)bh * row_blocks(dm) + (r >> 5)) * 64 + 32 * hf + (r & 31)] = hf ? -D : ref;
    }
    const TileReader rd(lane);
    const float c = dm.scale_log2;
    f32x16 acc[4];
#pragma unroll
    for (int ct = 0; ct < 4; ++ct) acc[ct] = zero16();
    const int w_lo = t0 + ((32 * wave) >> lg), w_hi = t0 + ((32 * wave + 31) >> lg);
    auto step = [&](const KVTile *cur, KVTile *next, int x) __attribute__((always_inline)) {
        __builtin_amdgcn_s_waitcnt(0);
        __syncthreads();
        stage(next, x + 1);
        if (kHalves > 1 && x >= count) return;           // (the other half has one more)
        const int k0 = key0(x);
        const bool some = k0 <= w_hi && (k0 < win.n_sink || w_lo - (k0 + kWinKeys - 1) < win.window);
        if (!some) return;
        const bool all = k0 + kWinKeys - 1 <= w_lo && (k0 + kWinKeys <= win.n_sink || w_hi - k0 < win.window);
        f32x16 s[2], dp[2];                              // (dp - D straight from the product)
        // (the next operands are under way while the matrix cores work; `more`: vector work to put between)
        auto products = [&](int kh, auto more) __attribute__((always_inline)) {
            const char *kr = cur[half].k.x + kh * kHalfTile, *vr = cur[half].v.x + kh * kHalfTile;
            bf16x8 xk[2] = {rd.rows(kr, 0)}, xv[2] = {rd.rows(vr, 0)};
            s[kh] = zero16();
#pragma unroll
            for (int e = 0; e < 16; ++e) dp[kh][e] = -D;
#pragma unroll
            for (int ks = 0; ks < 8; ++ks) {
                if (ks < 7) {
                    xk[(ks + 1) & 1] = rd.rows(kr, ks + 1);
                    xv[(ks + 1) & 1] = rd.rows(vr, ks + 1);
                }
                __builtin_amdgcn_sched_barrier(0);
                s[kh] = mfma32(xk[ks & 1], qf[ks], s[kh]);
                dp[kh] = mfma32(xv[ks & 1], gf[ks], dp[kh]);
                more(ks);
            }
        };
        auto exponentials = [&](int kh, int i) __attribute__((always_inline)) {
#pragma unroll
            for (int e = 2 * i; e < 2 * i + 2; ++e) s[kh][e] = fast_exp2(__builtin_fmaf(s[kh][e], c, -ref)) * dp[kh][e];
        };
        auto hide = [&](int kh) __attribute__((always_inline)) {
            if (all) return;                             // (what is not visible may be anything: replaced, not multiplied)
            int at = k0 + 32 * kh + 4 * hf;
            asm volatile("" : "+v"(at));
            const VisibleKeys visible(win, i);
#pragma unroll
            for (int e = 0; e < 16; ++e) s[kh][e] = visible(at + 8 * (e >> 2) + (e & 3)) ? s[kh][e] : 0.f;
        };
        auto sums = [&](int kh, auto more) __attribute__((always_inline)) {
            const char *kr = cur[half].k.x + kh * kHalfTile;
            bf16x8 xk[2] = {rd.columns(kr, 0, 0)};
            const bf16x8 ds[2] = {pack8(s[kh], 0), pack8(s[kh], 1)};
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if (j < 7) xk[(j + 1) & 1] = rd.columns(kr, (j + 1) >> 2, (j + 1) & 3);
                __builtin_amdgcn_sched_barrier(0);
                acc[j & 3] = mfma32(xk[j & 1], ds[j >> 2], acc[j & 3]);
                more(j);
            }
        };
        // one half's exponentials under the other's products
        products(0, [](int) {});
        products(1, [&](int j) __attribute__((always_inline)) { exponentials(0, j); });
        __builtin_amdgcn_sched_barrier(0);
        hide(0);
        sums(0, [&](int j) __attribute__((always_inline)) { exponentials(1, j); });
        __builtin_amdgcn_sched_barrier(0);
        hide(1);
        sums(1, [](int) {});
    };
    for (int x = 0; x < steps; x += 2) {
        step(tile0, tile1, x);
        if (x + 1 < steps) step(tile1, tile0, x + 1);
    }
    __syncthreads();                                     // the tiles are free
    if constexpr (kHalves == 2) {                        // (as in the forward)
        KVTile &theirs = (wave & 1 ? tile1 : tile0)[1];
        char *at = (wave < 2 ? theirs.k : theirs.v).x + 16 * lane;
#pragma unroll
        for (int ct = 0; ct < 4; ++ct)
#pragma unroll
            for (int e4 = 0; e4 < 4; ++e4)
                if (half == 1)
                    *reinterpret_cast<f32x4 *>(at + 1024 * (4 * ct + e4)) = f32x4{acc[ct][4 * e4], acc[ct][4 * e4 + 1], acc[ct][4 * e4 + 2], acc[ct][4 * e4 + 3]};
        __syncthreads();
        if (half == 1) return;
#pragma unroll
        for (int ct = 0; ct < 4; ++ct)
#pragma unroll
            for (int e4 = 0; e4 < 4; ++e4) {
                const f32x4 x = *reinterpret_cast<const f32x4 *>(at + 1024 * (4 * ct + e4));
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[ct][4 * e4 + e] += x[e];
            }
    }
    const bool live = i < L;
    const uint32_t alive = (uint32_t)__ballot(live);
    if (alive != ~0u) {                                  // (rows behind the sequence: zeros, where they are written at all)
#pragma unroll
        for (int ct = 0; ct < 4; ++ct)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[ct][e] = live ? acc[ct][e] : 0.f;
    }
    store_rows((wave < 2 ? tile0[0].k.x : tile0[0].v.x) + (wave & 1) * kHalfTile, acc, scale, lane, [&](int r) __attribute__((always_inline)) -> __bf16 * {
        const int t = t0 + ((32 * wave + r) >> lg), head = h * dm.G + ((32 * wave + r) & (dm.G - 1));
        return t < dm.max_seqlen && ((alive >> r) & 1u || dm.fill) ? dq.ptr + b * dq.sb + (int64_t)t * dq.st + (int64_t)head * dq.sh : nullptr;
    });
}

// The same for few rows, as in the forward: 32 rows to a workgroup, every fourth unit of 32 keys to a wavefront, four sums joined in LDS.
__global__ __launch_bounds__(256, 1) void window_dq_few_kernel(Dims dm, WindowArgs win, float scale, int lg, int n_tiles, Tensor q, Tensor k,
                                                               Tensor v, Tensor out, Tensor dout, const float *__restrict__ lse,
                                                               const int32_t *__restrict__ seqlens, Tensor dq, float *__restrict__ rows) {
    __shared__ KVHalf slot0[4], slot1[4];
    const int bh = blockIdx.x / n_tiles, b = bh / dm.Hkv, h = bh - b * dm.Hkv;
    const int ti = (bh + 1) * n_tiles - 1 - (int)blockIdx.x;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), hf = lane >> 5;
    const int L = clamp_len(uniform_load(seqlens + b), dm.max_seqlen);
    const int t0 = ti * (32 >> lg), t1 = min(L, t0 + (32 >> lg));
    // the result's row and 16 channels of this thread
    const int o_row = tid >> 3, ch = 16 * (tid & 7), o_i = t0 + (o_row >> lg), o_hq = h * dm.G + (o_row & (dm.G - 1));
    __bf16 *dq_row = dq.ptr + b * dq.sb + (int64_t)o_i * dq.st + (int64_t)o_hq * dq.sh + ch;
    const bool store = o_i < dm.max_seqlen && (o_i < L || dm.fill);
    if (t0 >= L) {
        if (store) reinterpret_cast<uint4 *>(dq_row)[0] = reinterpret_cast<uint4 *>(dq_row)[1] = uint4{0u, 0u, 0u, 0u};
        return;
    }
    const KeyTiles<32> kt(win, t0, t1);
    const int row = lane & 31, i = t0 + (row >> lg), hq = h * dm.G + (row & (dm.G - 1));
    bf16x8 qf[8], gf[8];
    float D = 0.f;
    const int64_t t = min(i, L - 1);
    const __bf16 *qr = q.ptr + b * q.sb + t * q.st + (int64_t)hq * q.sh + 8 * hf;
    const __bf16 *gr = dout.ptr + b * dout.sb + t * dout.st + (int64_t)hq * dout.sh + 8 * hf;
    const __bf16 *orow = out.ptr + b * out.sb + t * out.st + (int64_t)hq * out.sh + 8 * hf;
#pragma unroll
    for (int ks = 0; ks < 8; ++ks) {
        qf[ks] = load8(qr + 16 * ks);
        gf[ks] = load8(gr + 16 * ks);
        const bf16x8 x = load8(orow + 16 * ks);
#pragma unroll
        for (int e = 0; e < 8; ++e) D = __builtin_fmaf((float)gf[ks][e], (float)x[e], D);
    }
    D = half_reduce(D, [](float a, float d) { return a + d; });
    const float ref = lse[((int64_t)b * dm.max_seqlen + t) * dm.Hq + hq] * kLog2e, c = dm.scale_log2;
    if (wave == 0 && i < L) {
        const int64_t r = (int64_t)ti * 32 + row;
        rows[((int64_t)bh * row_blocks(dm) + (r >> 5)) * 64 + 32 * hf + (r & 31)] = hf ? -D : ref;
    }
    const TileReader rd(lane);
    f32x16 acc[4];
#pragma unroll
    for (int ct = 0; ct < 4; ++ct) acc[ct] = zero16();
    const int hi = t0 + (31 >> lg);
    walk_halves(slot0[wave], slot1[wave], k, v, b, h, kt, L, wave, lane, [&](const KVHalf &cur, int k0) __attribute__((always_inline)) {
        f32x16 s = zero16(), dp;
#pragma unroll
        for (int e = 0; e < 16; ++e) dp[e] = -D;
        bf16x8 x[8], y[8];                               // (alone on its SIMD: all operands asked for before any is used)
#pragma unroll
        for (int ks = 0; ks < 8; ++ks) {
            x[ks] = rd.rows(cur.k, ks);
            y[ks] = rd.rows(cur.v, ks);
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int ks = 0; ks < 8; ++ks) {
            s = mfma32(x[ks], qf[ks], s);
            dp = mfma32(y[ks], gf[ks], dp);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = rd.columns(cur.k, j >> 2, j & 3);
        __builtin_amdgcn_sched_barrier(0);
        settle<8>(s, dp);
#pragma unroll
        for (int e = 0; e < 16; ++e) s[e] = fast_exp2(__builtin_fmaf(s[e], c, -ref)) * dp[e];
        if (!(k0 + 31 <= t0 && (k0 + 32 <= win.n_sink || hi - k0 < win.window))) {
            const VisibleKeys visible(win, i);
#pragma unroll
            for (int e = 0; e < 16; ++e) s[e] = visible(k0 + 4 * hf + 8 * (e >> 2) + (e & 3)) ? s[e] : 0.f;
        }
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const bf16x8 ds = pack8(s, j);
#pragma unroll
            for (int ct = 0; ct < 4; ++ct) acc[ct] = mfma32(x[4 * j + ct], ds, acc[ct]);
        }
    });
    reads_done();
    // [row][channel], 16-byte pieces XORed with the row
    float *mine = reinterpret_cast<float *>(&slot0[wave]);
#pragma unroll
    for (int ct = 0; ct < 4; ++ct)
#pragma unroll
        for (int e4 = 0; e4 < 4; ++e4)
            *reinterpret_cast<f32x4 *>(mine + row * kHeadDim + 4 * ((8 * ct + 2 * e4 + hf) ^ (lane & 7))) =
                f32x4{acc[ct][4 * e4], acc[ct][4 * e4 + 1], acc[ct][4 * e4 + 2], acc[ct][4 * e4 + 3]};
    __syncthreads();
    if (!store) return;
    bf16x8 z[2];
#pragma unroll
    for (int e4 = 0; e4 < 4; ++e4) {
        f32x4 y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < 4; ++w)
            y += *reinterpret_cast<const f32x4 *>(reinterpret_cast<const float *>(&slot0[w]) + o_row * kHeadDim + 4 * ((ch / 4 + e4) ^ (o_row & 7)));
#pragma unroll
        for (int e = 0; e < 4; ++e) z[e4 >> 1][4 * (e4 & 1) + e] = (__bf16)(o_i < L ? y[e] * scale : 0.f);
    }
    reinterpret_cast<uint4 *>(dq_row)[0] = __builtin_bit_cast(uint4, z[0]);
    reinterpret_cast<uint4 *>(dq_row)[1] = __builtin_bit_cast(uint4, z[1]);
}

// ---- dk, dv ------------------------------------------------------------------------------------------------------------------
// A workgroup takes 128 keys, 32 to a wavefront (as columns: their K stays in registers, their V in LDS: both would not fit 256 registers),
// and the rows of a span of tokens that see any of them, in steps of 32; rows and their scalars go straight into LDS one step ahead.
// S = Q . K^T and dP = dout . V^T leave a key in a lane, so P and dS are the second operands of dV^T = dout^T . P and dK^T = Q^T . dS as they
// come out.
// The spans are the same for all keys, and the workgroups of a span are neighbours: they walk the same rows at the same time, which then
// come out of their XCD's L2 (cut from each key tile's own first row on instead, 94 % of 17 GB came from beyond it: 32K tokens, window 4096).
// Sums of a tile whose rows lie in several spans go to scratch and are added up in order.
constexpr int kKvKeys = 128, kKvRows = 32;
struct BwdPlan {
    int tiles, sink_tiles;                               // key tiles of a sequence; those with any of the first n_sink tokens
    int span, spans;                                     // tokens of a span (a multiple of a step's), spans
    int per_span;                                        // key tiles a span may have
    int parts;                                           // spans a tile may have, sinks' tiles apart
    __host__ __device__ int64_t slot(int tile) const {
        return tile < sink_tiles ? (int64_t)tile * spans : (int64_t)sink_tiles * spans + (int64_t)(tile - sink_tiles) * parts;
    }
    // the first key tile behind the sinks' that a query of span s sees
    __host__ __device__ int first_tile(WindowArgs w, int s) const {
        const int64_t key = (int64_t)s * span + 1 - w.window;
        const int t = key > 0 ? (int)(key / kKvKeys) : 0;
        return t > sink_tiles ? t : sink_tiles;
    }
};
struct KvSpans {                                         // the tokens that see key tile `tile`, the first and the last of their spans
    int from, to, first, last;
    __device__ __forceinline__ KvSpans(const BwdPlan &plan, WindowArgs w, int tile, int L) {
        from = tile * kKvKeys;
        to = tile < plan.sink_tiles ? L : (int)min((int64_t)L, (int64_t)from + kKvKeys - 1 + w.window);
        first = from / plan.span;
        last = max(to - 1, from) / plan.span;
    }
};
struct __align__(16) KvRows {
    char q[kHalfTile], g[kHalfTile];
    float ref[32], minus_D[32];
};

// dk, dv of 128 keys from one span's rows: a step is 32 rows, brought into LDS one step ahead (three steps ahead, one workgroup to a compute unit: nothing
// where there are fewer workgroups than that, 20 % more time where there are more).  32K tokens, 32 : 2 heads, window 4096: 3.9 to 4.2 ms, 1.0
// PFLOP/s of its four products; matrix cores busy 69 % of the time in which a SIMD has its two wavefronts, at the 1.7 GHz that the power limit
// leaves (a large library product: 1.36 PFLOP/s).
__global__ __launch_bounds__(256, 2) void window_dkdv_kernel(Dims dm, WindowArgs win, float scale, int lg, BwdPlan plan, Tensor q, Tensor k,
                                                             Tensor v, Tensor dout, const float *__restrict__ rows,
                                                             const int32_t *__restrict__ seqlens, Tensor dk, Tensor dv,
                                                             float *__restrict__ part) {
    __shared__ KvRows slot0, slot1;
    __shared__ __align__(16) char vt[kKvKeys * 256];
    const int item = xcd_item(blockIdx.x, plan.per_span), group = item / plan.per_span, bh = group / plan.spans;     // a span is a run
    const int b = bh / dm.Hkv, h = bh - b * dm.Hkv, span = (bh + 1) * plan.spans - 1 - group, at = item - group * plan.per_span;
    if (b >= dm.batch) return;
    // the sinks' tiles; from the span's first tile back, which all of its queries see, down to the window's edge; the span's other tiles
    const int begin = max(plan.sink_tiles, (int)((int64_t)span * plan.span / kKvKeys)), back = begin - plan.first_tile(win, span), y = at - plan.sink_tiles;
    const int tile = y < 0 ? at : y <= back ? begin - y : begin + y - back;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int c32 = lane & 31, hf = lane >> 5;
    const int L = clamp_len(uniform_load(seqlens + b), dm.max_seqlen);
    if (tile >= plan.tiles) return;
    const KvSpans rows_of(plan, win, tile, L);
    if (span < rows_of.first || span > rows_of.last) return;
    const int from = max(rows_of.from, span * plan.span), to = (int)min((int64_t)rows_of.to, (int64_t)(span + 1) * plan.span);
    if (from >= to && !dm.fill) return;
    const int per = kKvRows >> lg, x1 = from < to ? (to - from + per - 1) / per : 0;
    const int t = tile * kKvKeys + 32 * wave + c32;      // this lane's key
    bf16x8 kf[8];
    if (x1 > 0) {
        const __bf16 *kr = k.ptr + b * k.sb + h * k.sh + (int64_t)min(t, L - 1) * k.st + 8 * hf;
#pragma unroll
        for (int ks = 0; ks < 8; ++ks) kf[ks] = load8(kr + 16 * ks);
        const int k0 = tile * kKvKeys;
        const char *vb = reinterpret_cast<const char *>(v.ptr + b * v.sb + h * v.sh + (int64_t)k0 * v.st) + 64 * wave;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const bool row = k0 + 16 * j + (lane >> 2) < L;
            copy_rows(vt + (j >> 1) * kHalfTile + wave * 2048 + (j & 1) * 1024, vb,
                      row ? (uint32_t)(lane >> 2) * 2u * (uint32_t)v.st + 16 * copy_piece(lane) : kNoRow, 32 * j * (uint32_t)v.st);
        }
    }
    const char *q_head = reinterpret_cast<const char *>(q.ptr + b * q.sb + (int64_t)h * dm.G * q.sh) + 64 * wave;
    const char *g_head = reinterpret_cast<const char *>(dout.ptr + b * dout.sb + (int64_t)h * dm.G * dout.sh) + 64 * wave;
    const float *row_head = rows + (int64_t)bh * row_blocks(dm) * 64;
    uint32_t q_at[2], g_at[2];                           // this lane's row of either half of a step, and its piece
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const uint32_t r = 16 * j + (lane >> 2), tok = r >> lg, g = r & (dm.G - 1), piece = 16 * copy_piece(lane);
        q_at[j] = 2u * (tok * (uint32_t)q.st + g * (uint32_t)q.sh) + piece;
        g_at[j] = 2u * (tok * (uint32_t)dout.st + g * (uint32_t)dout.sh) + piece;
    }
    auto stage = [&](KvRows &dst, int x) __attribute__((always_inline)) {
        if (x >= x1) return;
        const int i0 = from + x * per;
        const char *qb = q_head + (int64_t)i0 * (2 * q.st), *gb = g_head + (int64_t)i0 * (2 * dout.st);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const bool row = i0 + ((16 * j + (lane >> 2)) >> lg) < L;
            copy_rows(dst.q + wave * 2048 + j * 1024, qb, row ? q_at[j] : kNoRow, 0);
            copy_rows(dst.g + wave * 2048 + j * 1024, gb, row ? g_at[j] : kNoRow, 0);
        }
        if (lane >> 4 == wave)
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)(row_head + ((int64_t)i0 >> (5 - lg)) * 64 + lane),
                                             (__attribute__((address_space(3))) void *)dst.ref, 4, 0, 0);
    };
    stage(slot0, 0);
    const TileReader rd(lane);
    const float c = dm.scale_log2;
    f32x16 dka[4], dva[4];
#pragma unroll
    for (int ct = 0; ct < 4; ++ct) dka[ct] = dva[ct] = zero16();
    const int k_lo = tile * kKvKeys + 32 * wave, k_hi = k_lo + 31;
    auto step = [&](const KvRows &cur, KvRows &next, int x) __attribute__((always_inline)) {
        __builtin_amdgcn_s_waitcnt(0);
        __syncthreads();
        stage(next, x + 1);
        const int i0 = from + x * per, i1 = i0 + per - 1;
        const bool some = k_lo <= i1 && (k_lo < win.n_sink || i0 - k_hi < win.window);
        if (!some) return;
        const bool all = k_hi <= i0 && (k_hi < win.n_sink || i1 - k_lo < win.window) && i1 < L;
        const char *qr = cur.q, *gr = cur.g, *vr = vt + wave * kHalfTile;
        // entry e: row 8 (e / 4) + 4 hf + e % 4; dp - D straight from the product
        f32x16 s = zero16(), dp;
#pragma unroll
        for (int e4 = 0; e4 < 4; ++e4) {
            const f32x4 d = *reinterpret_cast<const f32x4 *>(&cur.minus_D[8 * e4 + 4 * hf]);
#pragma unroll
            for (int e = 0; e < 4; ++e) dp[4 * e4 + e] = d[e];
        }
        // the next operands are under way while the matrix cores work, and no more: there are no registers (two to seven ahead: slower also where
        // a wavefront is alone on its SIMD)
        constexpr int kAhead = 1, kRing = kAhead + 1;
        bf16x8 xq[kRing], xg[kRing], xv[kRing];
#pragma unroll
        for (int ks = 0; ks < kAhead; ++ks) {
            xq[ks] = rd.rows(qr, ks);
            xg[ks] = rd.rows(gr, ks);
            xv[ks] = rd.rows(vr, ks);
        }
#pragma unroll
        for (int ks = 0; ks < 8; ++ks) {
            if (ks + kAhead < 8) {
                xq[(ks + kAhead) % kRing] = rd.rows(qr, ks + kAhead);
                xg[(ks + kAhead) % kRing] = rd.rows(gr, ks + kAhead);
                xv[(ks + kAhead) % kRing] = rd.rows(vr, ks + kAhead);
            }
            __builtin_amdgcn_sched_barrier(0);
            s = mfma32(xq[ks % kRing], kf[ks], s);
            dp = mfma32(xg[ks % kRing], xv[ks % kRing], dp);
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int e4 = 0; e4 < 4; ++e4) {
            const f32x4 ref = *reinterpret_cast<const f32x4 *>(&cur.ref[8 * e4 + 4 * hf]);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                s[4 * e4 + e] = fast_exp2(__builtin_fmaf(s[4 * e4 + e], c, -ref[e]));
                dp[4 * e4 + e] *= s[4 * e4 + e];
            }
        }
        if (!all) {                                      // the key is visible to tokens t .. t + reach - 1
            const int reach = max(0, min(t < win.n_sink ? 0x7fffffff : win.window, L - t));
            int at = 4 * hf;
            asm volatile("" : "+v"(at));                 // (formed here: sixteen registers otherwise, held through the loop)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const bool seen = (uint32_t)(i0 + ((8 * (e >> 2) + (e & 3) + at) >> lg) - t) < (uint32_t)reach;
                s[e] = seen ? s[e] : 0.f;
                dp[e] = seen ? dp[e] : 0.f;
            }
        }
        __builtin_amdgcn_sched_barrier(0);
        const bf16x8 p[2] = {pack8(s, 0), pack8(s, 1)}, ds[2] = {pack8(dp, 0), pack8(dp, 1)};
        bf16x8 cg[kRing], cq[kRing];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            cg[i] = rd.columns(gr, i >> 2, i & 3);
            cq[i] = rd.columns(qr, i >> 2, i & 3);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {                    // (half s of the rows, channel tile ct) = (i / 4, i % 4)
            const int j = i + kAhead;
            if (j < 8) {
                cg[j % kRing] = rd.columns(gr, j >> 2, j & 3);
                cq[j % kRing] = rd.columns(qr, j >> 2, j & 3);
            }
            __builtin_amdgcn_sched_barrier(0);
            dva[i & 3] = mfma32(cg[i % kRing], p[i >> 2], dva[i & 3]);
            dka[i & 3] = mfma32(cq[i % kRing], ds[i >> 2], dka[i & 3]);
        }
    };
    for (int x = 0; x < x1; x += 2) {
        step(slot0, slot1, x);
        if (x + 1 < x1) step(slot1, slot0, x + 1);
    }
    if (rows_of.first != rows_of.last) {                 // [key][channel], dk then dv
        const int64_t slot = (int64_t)bh * plan.slot(plan.tiles) + plan.slot(tile) + span - rows_of.first;
        float *p = part + slot * (2 * kKvKeys * kHeadDim) + (32 * wave + c32) * kHeadDim + 4 * hf;
#pragma unroll
        for (int ct = 0; ct < 4; ++ct)
#pragma unroll
            for (int e4 = 0; e4 < 4; ++e4) {
                *reinterpret_cast<float4 *>(p + 32 * ct + 8 * e4) =
                    float4{dka[ct][4 * e4] * scale, dka[ct][4 * e4 + 1] * scale, dka[ct][4 * e4 + 2] * scale, dka[ct][4 * e4 + 3] * scale};
                *reinterpret_cast<float4 *>(p + kKvKeys * kHeadDim + 32 * ct + 8 * e4) =
                    float4{dva[ct][4 * e4], dva[ct][4 * e4 + 1], dva[ct][4 * e4 + 2], dva[ct][4 * e4 + 3]};
            }
        return;
    }
    if (t >= dm.max_seqlen || (t >= L && !dm.fill)) return;
    __bf16 *dkr = dk.ptr + b * dk.sb + h * dk.sh + (int64_t)t * dk.st + 4 * hf, *dvr = dv.ptr + b * dv.sb + h * dv.sh + (int64_t)t * dv.st + 4 * hf;
#pragma unroll
    for (int ct = 0; ct < 4; ++ct)
#pragma unroll
        for (int e4 = 0; e4 < 4; ++e4) {
            bf16x4 x, y;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                x[e] = (__bf16)(t < L ? dka[ct][4 * e4 + e] * scale : 0.f);
                y[e] = (__bf16)(t < L ? dva[ct][4 * e4 + e] : 0.f);
            }
            *reinterpret_cast<uint2 *>(dkr + 32 * ct + 8 * e4) = __builtin_bit_cast(uint2, x);
            *reinterpret_cast<uint2 *>(dvr + 32 * ct + 8 * e4) = __builtin_bit_cast(uint2, y);
        }
}

// The spans' sums of a key tile, added in order.  grid (keys / 8, Hkv, batch): 8 keys a workgroup, a thread 4 channels of dk and dv, four sums
// of each asked for at once.  Traffic alone: 32K tokens x 2 heads, three to five spans a tile, 57 to 70 us.
__global__ __launch_bounds__(256) void window_join_kernel(Dims dm, WindowArgs win, BwdPlan plan, const int32_t *__restrict__ seqlens,
                                                          const float *__restrict__ part, Tensor dk, Tensor dv) {
    const int h = blockIdx.y, b = blockIdx.z, bh = b * dm.Hkv + h;
    const int t = 8 * (int)blockIdx.x + (threadIdx.x >> 5), c4 = 4 * (threadIdx.x & 31), tile = t / kKvKeys;
    if (t >= dm.max_seqlen) return;
    const int L = clamp_len(uniform_load(seqlens + b), dm.max_seqlen);
    const KvSpans rows_of(plan, win, tile, L);
    if (rows_of.first == rows_of.last || (t >= L && !dm.fill)) return;
    const int n = t < L ? rows_of.last - rows_of.first + 1 : 0;
    constexpr int64_t kPart = 2 * kKvKeys * kHeadDim;
    const float *p = part + ((int64_t)bh * plan.slot(plan.tiles) + plan.slot(tile)) * kPart + (t % kKvKeys) * kHeadDim + c4;
    f32x4 x = {0.f, 0.f, 0.f, 0.f}, y = x;
    int i = 0;
    for (; i + 4 <= n; i += 4, p += 4 * kPart) {
        f32x4 a[4], d[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            a[j] = *reinterpret_cast<const f32x4 *>(p + j * kPart);
            d[j] = *reinterpret_cast<const f32x4 *>(p + j * kPart + kKvKeys * kHeadDim);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            x += a[j];
            y += d[j];
        }
    }
    for (; i < n; ++i, p += kPart) {
        x += *reinterpret_cast<const f32x4 *>(p);
        y += *reinterpret_cast<const f32x4 *>(p + kKvKeys * kHeadDim);
    }
    bf16x4 r, s;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        r[e] = (__bf16)x[e];
        s[e] = (__bf16)y[e];
    }
    *reinterpret_cast<uint2 *>(dk.ptr + b * dk.sb + h * dk.sh + (int64_t)t * dk.st + c4) = __builtin_bit_cast(uint2, r);
    *reinterpret_cast<uint2 *>(dv.ptr + b * dv.sb + h * dv.sh + (int64_t)t * dv.st + c4) = __builtin_bit_cast(uint2, s);
}

// ---- host side -------------------------------------------------------------------------------------------------------------
// Scratch tiles a call may use in all: a number that grows with the batch and with max_seqlen, so that a buffer for a call is large
// enough for every smaller one.
static int64_t most_slots(int64_t tiles) { return min(32 * tiles, 4096 + 2 * tiles); }

// The span: of some lengths the one whose workgroups the chip, which holds 512, is through with first: all steps, about 50 more per
// workgroup for its start and its sums but for the first 256, which have a compute unit each (not less than the longest workgroup), and half a
// longest workgroup's steps in which not all have work.  (4096 tokens, 4 heads : 1, window 256, spans of 32 / 64 / 128 tokens: dk/dv and join 31 /
// 26 / 32 us; 2 x 4096, 16 : 2, window 1000, of 128 / 256 / 384 / 512: 183 / 208 / 180 / 218.)
static BwdPlan bwd_plan(const Dims &dm, WindowArgs w) {
    BwdPlan best{};
    const int per = kKvRows / dm.G;
    const int64_t heads = (int64_t)dm.batch * dm.Hkv;
    const int64_t all_steps = (dm.max_seqlen + per - 1) / per, window_steps = min(all_steps, ((int64_t)w.window + kKvKeys - 1 + per - 1) / per);
    BwdPlan p;
    p.tiles = (dm.max_seqlen + kKvKeys - 1) / kKvKeys;
    p.sink_tiles = (w.n_sink + kKvKeys - 1) / kKvKeys;
    const int64_t steps = heads * (p.sink_tiles * all_steps + (p.tiles - p.sink_tiles) * window_steps), whole = (int64_t)p.tiles * kKvKeys;
    int64_t least = INT64_MAX;
    for (int64_t span = max(16, per);; span = span < kKvKeys ? 2 * span : span + (span / kKvKeys + 3) / 4 * kKvKeys) {
        span = min(span, whole);
        p.span = (int)span;
        p.spans = (int)((dm.max_seqlen + span - 1) / span);
        p.per_span = (int)min((int64_t)p.tiles, p.sink_tiles + (span + w.window - 2) / kKvKeys + 2);
        p.parts = (int)min((int64_t)p.spans, ((int64_t)w.window + 126) / span + 2);
        const int64_t items = heads * p.spans * p.per_span / (p.per_span == p.tiles ? 2 : 1);   // (of whole pasts half exist)
        const int64_t longest = (min(span, (int64_t)dm.max_seqlen) + per - 1) / per;
        const int64_t cost = max((steps + 50 * max((int64_t)0, items - 256)) / 512, longest) + longest / 2;
        if (heads * p.slot(p.tiles) <= most_slots(heads * p.tiles) && cost < least) {
            least = cost;
            best = p;
        }
        if (span == whole) return best;                  // (one span: a slot per tile at most)
    }
}

static size_t row_bytes(const Dims &dm) { return (size_t)dm.batch * dm.Hkv * row_blocks(dm) * 64 * sizeof(float); }
constexpr size_t kSlotBytes = 2 * kKvKeys * kHeadDim * sizeof(float);

size_t window_bwd_ws_bytes(const Dims &dm, WindowArgs) {
    const int64_t tiles = (int64_t)dm.batch * dm.Hkv * ((dm.max_seqlen + kKvKeys - 1) / kKvKeys);
    return row_bytes(dm) + (size_t)most_slots(tiles) * kSlotBytes;
}

// What a call of these arguments uses of it: the slots of its plan (2 x 4096 tokens, 16 : 2, window 1000: 72 MB of 538; 32K, 32 : 2, window 4096:
// 419 of 679).
size_t window_bwd_scratch_bytes(const Dims &dm, WindowArgs w) {
    if (dm.batch <= 0 || dm.max_seqlen <= 0) return 0;
    const BwdPlan plan = bwd_plan(dm, w);
    return row_bytes(dm) + (plan.spans == 1 ? 0 : (size_t)((int64_t)dm.batch * dm.Hkv * plan.slot(plan.tiles)) * kSlotBytes);
}

int launch_window_bwd(const Dims &dm, WindowArgs w, Tensor q, Tensor k, Tensor v, Tensor out, Tensor dout, const float *lse,
                      const int32_t *seqlens, Tensor dq, Tensor dk, Tensor dv, void *ws, hipStream_t stream) {
    if (dm.batch <= 0 || dm.max_seqlen <= 0) return 0;
    const int lg = __builtin_ctz(dm.G), per = kDqRows >> lg, n_tiles = (dm.max_seqlen + per - 1) / per;
    const float scale = dm.scale_log2 * kLn2;
    float *rows = reinterpret_cast<float *>(ws), *part = rows + row_bytes(dm) / sizeof(float);
    const BwdPlan plan = bwd_plan(dm, w);
    const int64_t heads = (int64_t)dm.batch * dm.Hkv;
    const int few_tiles = (dm.max_seqlen + (32 >> lg) - 1) / (32 >> lg), run = xcd_run_length(n_tiles * heads);
    const bool halves = by_halves(dm, w, n_tiles * heads);
    timing_begin("window_dq_kernel", stream);
    if (few_rows(dm, w, n_tiles * heads))
        hipLaunchKernelGGL(window_dq_few_kernel, dim3((unsigned)(few_tiles * heads)), dim3(256), 0, stream, dm, w, scale, lg, few_tiles, q, k, v, out,
                           dout, lse, seqlens, dq, rows);
    else
        hipLaunchKernelGGL(halves ? window_dq_kernel<2> : window_dq_kernel<1>, dim3(xcd_grid(n_tiles * heads, run)), dim3(halves ? 512 : 256), 0,
                           stream, dm, w, scale, lg, n_tiles, run, q, k, v, out, dout, lse, seqlens, dq, rows);
    timing_end(stream);
    timing_begin("window_dkdv_kernel", stream);
    hipLaunchKernelGGL(window_dkdv_kernel, dim3(xcd_grid(heads * plan.spans * plan.per_span, plan.per_span)), dim3(256), 0, stream, dm, w, scale, lg, plan,
                       q, k, v, dout, rows, seqlens, dk, dv, part);
    timing_end(stream);
    if (plan.spans == 1) return (int)hipGetLastError();
    timing_begin("window_join_kernel", stream);
    hipLaunchKernelGGL(window_join_kernel, dim3((dm.max_seqlen + 7) / 8, dm.Hkv, dm.batch), dim3(256), 0, stream, dm, w, plan, seqlens, part,
                       dk, dv);
    timing_end(stream);
    return (int)hipGetLastError();
}

}  // namespace infllmv2
