// Gradients of the windowed attention.  With p = exp(scale <q_i, k_t> - lse_i) over the visible keys and D_i = <dout_i, out_i>:
//     dv_t = sum p dout_i      ds = p (<dout_i, v_t> - D_i)      dq_i = scale sum ds k_t      dk_t = scale sum ds q_i
// Two kernels, each of which sums what it owns in registers, so nothing is added atomically and results repeat: dq walks the
// keys of 128 query rows as the forward does and leaves every row's log-sum-exp and D for the other; dk/dv walks the rows that see 128
// keys.  The scores are computed in both (7 products instead of 5: the other way is 4 bytes of atomics per row, channel and key
// tile).
#include "window.h"

namespace infllmv2 {

constexpr int kDqRows = 128;
struct __align__(16) DqTile {
    char k[kWinKeys * 256], v[kWinKeys * 256];
};

// rows: (lse in powers of two, D) of row (token, head of the group), [batch, Hkv, max_seqlen * G]
__global__ __launch_bounds__(256, 2) void window_dq_kernel(Dims dm, WindowArgs win, float scale, int lg, int n_tiles, Tensor q, Tensor k,
                                                           Tensor v, Tensor out, Tensor dout, const float *__restrict__ lse,
                                                           const int32_t *__restrict__ seqlens, Tensor dq, float2 *__restrict__ rows) {
    __shared__ DqTile tile0, tile1;
    const int id = xcd_run(blockIdx.x, gridDim.x);
    const int ti = id % n_tiles, bh = id / n_tiles, b = bh / dm.Hkv, h = bh - b * dm.Hkv;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int c32 = lane & 31, hf = lane >> 5;
    const int L = clamp_len(uniform_load(seqlens + b), dm.max_seqlen);
    const int t0 = ti * (kDqRows >> lg), t1 = min(L, t0 + (kDqRows >> lg));
    const int row = 32 * wave + c32, i = t0 + (row >> lg), hq = h * dm.G + (row & (dm.G - 1));
    __bf16 *dq_row = dq.ptr + b * dq.sb + (int64_t)i * dq.st + (int64_t)hq * dq.sh + 4 * hf;
    if (t0 >= L) {
        if (dm.fill && i < dm.max_seqlen)
            for (int c = 0; c < 16; ++c) *reinterpret_cast<uint2 *>(dq_row + 8 * c) = uint2{0u, 0u};
        return;
    }
    const KeyTiles kt(win, t0, t1);
    const char *k_head = reinterpret_cast<const char *>(k.ptr + b * k.sb + h * k.sh), *v_head = reinterpret_cast<const char *>(v.ptr + b * v.sb + h * v.sh);
    auto stage = [&](DqTile &dst, int x) __attribute__((always_inline)) {
        if (x >= kt.count) return;
        const int k0 = kt.key0(x);
#pragma unroll
        for (int j = 0; j < 4; ++j) {                    // (as in the forward)
            const int r = 16 * wave + 4 * j + (lane >> 4);
            const int64_t t = min(k0 + r, L - 1);
            const int piece = 16 * ((lane & 15) ^ row_swizzle(r));
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)(k_head + t * (2 * k.st) + piece),
                                             (__attribute__((address_space(3))) void *)(dst.k + (16 * wave + 4 * j) * 256), 16, 0, 0);
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)(v_head + t * (2 * v.st) + piece),
                                             (__attribute__((address_space(3))) void *)(dst.v + (16 * wave + 4 * j) * 256), 16, 0, 0);
        }
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
        if (hf == 0 && i < L) rows[((int64_t)bh * dm.max_seqlen + i) * dm.G + (row & (dm.G - 1))] = float2{ref, D};
    }
    const TileReader rd(lane);
    const float c = dm.scale_log2;
    f32x16 acc[4];
#pragma unroll
    for (int ct = 0; ct < 4; ++ct) acc[ct] = zero16();
    const int w_lo = t0 + ((32 * wave) >> lg), w_hi = t0 + ((32 * wave + 31) >> lg);
    auto step = [&](const DqTile &cur, DqTile &next, int x) __attribute__((always_inline)) {
        __builtin_amdgcn_s_waitcnt(0);
        __syncthreads();
        stage(next, x + 1);
        const int k0 = kt.key0(x);
        const bool some = k0 <= w_hi && (k0 < win.n_sink || w_lo - (k0 + kWinKeys - 1) < win.window);
        if (!some) return;
        const bool all = k0 + kWinKeys - 1 <= w_lo && (k0 + kWinKeys <= win.n_sink || w_hi - k0 < win.window);
#pragma unroll
        for (int kh = 0; kh < 2; ++kh) {
            const char *kr = cur.k + kh * 32 * 256, *vr = cur.v + kh * 32 * 256;
            f32x16 s = zero16(), dp = zero16();
#pragma unroll
            for (int ks = 0; ks < 8; ++ks) {
                s = mfma32(rd.rows(kr, ks), qf[ks], s);
                dp = mfma32(rd.rows(vr, ks), gf[ks], dp);
            }
#pragma unroll
            for (int e = 0; e < 16; ++e) s[e] = fast_exp2(__builtin_fmaf(s[e], c, -ref)) * (dp[e] - D);
            if (!all) {                                  // (what is not visible may be anything: replaced, not multiplied)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int t = k0 + 32 * kh + 8 * (e >> 2) + 4 * hf + (e & 3);
                    if (!(t <= i && (t < win.n_sink || i - t < win.window))) s[e] = 0.f;
                }
            }
#pragma unroll
            for (int s2 = 0; s2 < 2; ++s2) {
                const bf16x8 ds = pack8(s, s2);
#pragma unroll
                for (int ct = 0; ct < 4; ++ct) acc[ct] = mfma32(rd.columns(kr, s2, ct), ds, acc[ct]);
            }
        }
    };
    for (int x = 0; x < kt.count; x += 2) {
        step(tile0, tile1, x);
        if (x + 1 < kt.count) step(tile1, tile0, x + 1);
    }
    if (i >= dm.max_seqlen || (i >= L && !dm.fill)) return;
    const float f = i < L ? scale : 0.f;
#pragma unroll
    for (int ct = 0; ct < 4; ++ct)
#pragma unroll
        for (int e4 = 0; e4 < 4; ++e4) {
            bf16x4 r;
#pragma unroll
            for (int e = 0; e < 4; ++e) r[e] = (__bf16)(i < L ? acc[ct][4 * e4 + e] * f : 0.f);
            *reinterpret_cast<uint2 *>(dq_row + 32 * ct + 8 * e4) = __builtin_bit_cast(uint2, r);
        }
}

// ---- dk, dv ------------------------------------------------------------------------------------------------------------------
// A workgroup takes 128 keys, 32 to a wavefront (as columns: their K stays in registers, their V in LDS: both would not fit 256 registers), and a chunk of the steps of 32
// query rows that see any of them; rows and their scalars go straight into LDS one step ahead.  S = Q . K^T and dP = dout . V^T leave a key
// in a lane, so P and dS are the second operands of dV^T = dout^T . P and dK^T = Q^T . dS as they come out.  A tile's
// steps are cut into chunks where there are fewer tiles than the chip holds, and those of the first tokens, which all later rows see;
// the chunks' sums go to scratch and are added up in order.
constexpr int kKvKeys = 128, kKvRows = 32;
struct BwdPlan {
    int tiles, sink_tiles;                               // key tiles of a sequence; those with any of the first n_sink tokens
    int chunk;                                           // steps per chunk
    int sink_chunks, chunks;                             // chunks a tile may have
    int slots;                                           // scratch tiles per (sequence, key-value head)
    __host__ __device__ int first_slot(int tile) const { return tile < sink_tiles ? tile * sink_chunks : sink_tiles * sink_chunks + (tile - sink_tiles) * chunks; }
    __host__ __device__ int of(int tile) const { return tile < sink_tiles ? sink_chunks : chunks; }
};
struct KvSteps {                                         // the rows that see key tile `tile`: tokens from .. to - 1
    int from, to, count;
    __device__ __forceinline__ KvSteps(WindowArgs w, int tile, bool sink, int L, int lg) {
        from = tile * kKvKeys;
        to = sink ? L : (int)min((int64_t)L, (int64_t)from + kKvKeys - 1 + w.window);
        const int per = kKvRows >> lg;
        count = to > from ? (to - from + per - 1) / per : 0;
    }
};
struct __align__(16) KvRows {
    char q[kKvRows * 256], g[kKvRows * 256];
    float2 ld[kKvRows];
};

__global__ __launch_bounds__(256, 2) void window_dkdv_kernel(Dims dm, WindowArgs win, float scale, int lg, BwdPlan plan, Tensor q, Tensor k,
                                                             Tensor v, Tensor dout, const float2 *__restrict__ rows,
                                                             const int32_t *__restrict__ seqlens, Tensor dk, Tensor dv,
                                                             float *__restrict__ part) {
    __shared__ KvRows slot0, slot1;
    __shared__ __align__(16) char vt[kKvKeys * 256];
    const int per_head = plan.sink_tiles * plan.sink_chunks + (plan.tiles - plan.sink_tiles) * plan.chunks;
    const int id = xcd_run(blockIdx.x, gridDim.x), bh = id / per_head, b = bh / dm.Hkv, h = bh - b * dm.Hkv;
    int at = id - bh * per_head;
    const bool sink = at < plan.sink_tiles * plan.sink_chunks;
    if (!sink) at -= plan.sink_tiles * plan.sink_chunks;
    const int n_ch = sink ? plan.sink_chunks : plan.chunks, tile = at / n_ch + (sink ? 0 : plan.sink_tiles), chunk = at % n_ch;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int c32 = lane & 31, hf = lane >> 5;
    const int L = clamp_len(uniform_load(seqlens + b), dm.max_seqlen);
    const KvSteps steps(win, tile, sink, L, lg);
    const int x0 = chunk * plan.chunk, x1 = min(steps.count, x0 + plan.chunk);
    if (n_ch > 1 ? x0 >= x1 : !dm.fill && x0 >= x1) return;
    const int t = tile * kKvKeys + 32 * wave + c32;      // this lane's key
    bf16x8 kf[8];
    if (x0 < x1) {
        const __bf16 *kr = k.ptr + b * k.sb + h * k.sh + (int64_t)min(t, L - 1) * k.st + 8 * hf;
#pragma unroll
        for (int ks = 0; ks < 8; ++ks) kf[ks] = load8(kr + 16 * ks);
        const char *v_head = reinterpret_cast<const char *>(v.ptr + b * v.sb + h * v.sh);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int r = 32 * wave + 4 * j + (lane >> 4);
            const int64_t row = min(tile * kKvKeys + r, L - 1);
            const int piece = 16 * ((lane & 15) ^ row_swizzle(r));
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)(v_head + row * (2 * v.st) + piece),
                                             (__attribute__((address_space(3))) void *)(vt + (32 * wave + 4 * j) * 256), 16, 0, 0);
        }
    }
    const int per = kKvRows >> lg;
    const char *q_head = reinterpret_cast<const char *>(q.ptr + b * q.sb + (int64_t)h * dm.G * q.sh);
    const char *g_head = reinterpret_cast<const char *>(dout.ptr + b * dout.sb + (int64_t)h * dm.G * dout.sh);
    const char *ld_head = reinterpret_cast<const char *>(rows + (int64_t)bh * dm.max_seqlen * dm.G);
    auto stage = [&](KvRows &dst, int x) __attribute__((always_inline)) {
        if (x >= x1) return;
        const int i0 = steps.from + x * per;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int r = 8 * wave + 4 * j + (lane >> 4);
            const int64_t i = min(i0 + (r >> lg), L - 1), g = r & (dm.G - 1);
            const int piece = 16 * ((lane & 15) ^ row_swizzle(r));
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)(q_head + 2 * (i * q.st + g * q.sh) + piece),
                                             (__attribute__((address_space(3))) void *)(dst.q + (8 * wave + 4 * j) * 256), 16, 0, 0);
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)(g_head + 2 * (i * dout.st + g * dout.sh) + piece),
                                             (__attribute__((address_space(3))) void *)(dst.g + (8 * wave + 4 * j) * 256), 16, 0, 0);
        }
        if (wave == 0) {                                 // 32 (lse, D): 256 bytes
            const int r = lane >> 1;
            const int64_t i = min(i0 + (r >> lg), L - 1);
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)(ld_head + 8 * (i * dm.G + (r & (dm.G - 1))) + 4 * (lane & 1)),
                                             (__attribute__((address_space(3))) void *)dst.ld, 4, 0, 0);
        }
    };
    stage(slot0, x0);
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
        const int i0 = steps.from + x * per, i1 = i0 + per - 1;
        const bool some = k_lo <= i1 && (k_lo < win.n_sink || i0 - k_hi < win.window);
        if (!some) return;
        const bool all = k_hi <= i0 && (k_hi < win.n_sink || i1 - k_lo < win.window) && i1 < L;
        const char *qr = cur.q, *gr = cur.g, *vr = vt + wave * 32 * 256;
        f32x16 s = zero16(), dp = zero16();
#pragma unroll
        for (int ks = 0; ks < 8; ++ks) {
            s = mfma32(rd.rows(qr, ks), kf[ks], s);
            dp = mfma32(rd.rows(gr, ks), rd.rows(vr, ks), dp);
        }
        // entry e: row 8 (e / 4) + 4 hf + e % 4
#pragma unroll
        for (int e4 = 0; e4 < 4; ++e4) {
            const float4 *ld = reinterpret_cast<const float4 *>(&cur.ld[8 * e4 + 4 * hf]);
            const float4 a = ld[0], d = ld[1];
            const float ref[4] = {a.x, a.z, d.x, d.z}, D[4] = {a.y, a.w, d.y, d.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float p = fast_exp2(__builtin_fmaf(s[4 * e4 + e], c, -ref[e]));
                s[4 * e4 + e] = p;
                dp[4 * e4 + e] = p * (dp[4 * e4 + e] - D[e]);
            }
        }
        if (!all) {
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const int i = i0 + ((8 * (e >> 2) + 4 * hf + (e & 3)) >> lg);
                if (!(t <= i && i < L && (t < win.n_sink || i - t < win.window))) s[e] = dp[e] = 0.f;
            }
        }
#pragma unroll
        for (int s2 = 0; s2 < 2; ++s2) {
            const bf16x8 p = pack8(s, s2), ds = pack8(dp, s2);
#pragma unroll
            for (int ct = 0; ct < 4; ++ct) {
                dva[ct] = mfma32(rd.columns(gr, s2, ct), p, dva[ct]);
                dka[ct] = mfma32(rd.columns(qr, s2, ct), ds, dka[ct]);
            }
        }
    };
    for (int x = x0; x < x1; x += 2) {
        step(slot0, slot1, x);
        if (x + 1 < x1) step(slot1, slot0, x + 1);
    }
    if (n_ch > 1) {                                      // [key][channel], dk then dv
        float *p = part + ((int64_t)bh * plan.slots + plan.first_slot(tile) + chunk) * (2 * kKvKeys * kHeadDim) + (32 * wave + c32) * kHeadDim + 4 * hf;
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

// The chunks' sums of a key tile, added in order.  grid (keys / 16, Hkv, batch) over the tiles that may have several: 16 keys a workgroup, a thread
// 8 channels of dk and dv.
__global__ __launch_bounds__(256) void window_join_kernel(Dims dm, WindowArgs win, int lg, BwdPlan plan, const int32_t *__restrict__ seqlens,
                                                          const float *__restrict__ part, Tensor dk, Tensor dv) {
    const int h = blockIdx.y, b = blockIdx.z, bh = b * dm.Hkv + h;
    const int t = 16 * (int)blockIdx.x + (threadIdx.x >> 4), c8 = 8 * (threadIdx.x & 15), tile = t / kKvKeys;
    if (plan.of(tile) == 1 || t >= dm.max_seqlen) return;
    const int L = clamp_len(uniform_load(seqlens + b), dm.max_seqlen);
    if (t >= L && !dm.fill) return;
    const KvSteps steps(win, tile, tile < plan.sink_tiles, L, lg);
    const int n = t < L ? (steps.count + plan.chunk - 1) / plan.chunk : 0;
    const float *p = part + ((int64_t)bh * plan.slots + plan.first_slot(tile)) * (2 * kKvKeys * kHeadDim) + (t % kKvKeys) * kHeadDim + c8;
    float x[8], y[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = y[e] = 0.f;
    for (int i = 0; i < n; ++i, p += 2 * kKvKeys * kHeadDim) {
        const f32x4 a = *reinterpret_cast<const f32x4 *>(p), d = *reinterpret_cast<const f32x4 *>(p + 4);
        const f32x4 e0 = *reinterpret_cast<const f32x4 *>(p + kKvKeys * kHeadDim), e1 = *reinterpret_cast<const f32x4 *>(p + kKvKeys * kHeadDim + 4);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            x[e] += a[e];
            x[4 + e] += d[e];
            y[e] += e0[e];
            y[4 + e] += e1[e];
        }
    }
    bf16x8 r, s;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        r[e] = (__bf16)x[e];
        s[e] = (__bf16)y[e];
    }
    *reinterpret_cast<uint4 *>(dk.ptr + b * dk.sb + h * dk.sh + (int64_t)t * dk.st + c8) = __builtin_bit_cast(uint4, r);
    *reinterpret_cast<uint4 *>(dv.ptr + b * dv.sb + h * dv.sh + (int64_t)t * dv.st + c8) = __builtin_bit_cast(uint4, s);
}

// ---- host side -------------------------------------------------------------------------------------------------------------
static inline size_t align256(size_t x) { return (x + 255) / 256 * 256; }

// Scratch tiles a call may use in all: a number that grows with the batch and with max_seqlen, so that a buffer for a call is large
// enough for every smaller one.
static int64_t most_slots(int64_t tiles) { return min(8 * tiles, 2048 + tiles); }

static BwdPlan bwd_plan(const Dims &dm, WindowArgs w) {
    BwdPlan p;
    const int per = kKvRows / dm.G;
    const int64_t heads = (int64_t)dm.batch * dm.Hkv;
    p.tiles = (dm.max_seqlen + kKvKeys - 1) / kKvKeys;
    p.sink_tiles = (w.n_sink + kKvKeys - 1) / kKvKeys;
    const int64_t sink_steps = (dm.max_seqlen + per - 1) / per;
    const int64_t steps = min(sink_steps, ((int64_t)w.window + kKvKeys - 1 + per - 1) / per);
    const int64_t total = heads * (p.sink_tiles * sink_steps + (p.tiles - p.sink_tiles) * steps);
    for (int64_t chunk = max((int64_t)8, total / 1024);; chunk += (chunk + 3) / 4) {
        p.chunk = (int)min(chunk, (int64_t)1 << 30);
        p.sink_chunks = (int)((sink_steps + chunk - 1) / chunk);
        p.chunks = (int)((steps + chunk - 1) / chunk);
        const int64_t slots = (int64_t)p.sink_tiles * p.sink_chunks + (int64_t)(p.tiles - p.sink_tiles) * (p.chunks > 1 ? p.chunks : 0);
        p.slots = (int)slots;
        if (heads * slots <= most_slots(heads * p.tiles)) return p;
    }
}

size_t window_bwd_ws_bytes(const Dims &dm, WindowArgs) {
    const size_t rows = align256((size_t)dm.batch * dm.Hq * dm.max_seqlen * sizeof(float2));
    const int64_t tiles = (int64_t)dm.batch * dm.Hkv * ((dm.max_seqlen + kKvKeys - 1) / kKvKeys);
    return rows + (size_t)most_slots(tiles) * (2 * kKvKeys * kHeadDim * sizeof(float));
}

int launch_window_bwd(const Dims &dm, WindowArgs w, Tensor q, Tensor k, Tensor v, Tensor out, Tensor dout, const float *lse,
                      const int32_t *seqlens, Tensor dq, Tensor dk, Tensor dv, void *ws, hipStream_t stream) {
    if (dm.batch <= 0 || dm.max_seqlen <= 0) return 0;
    const int lg = __builtin_ctz(dm.G), per = kDqRows >> lg, n_tiles = (dm.max_seqlen + per - 1) / per;
    const float scale = dm.scale_log2 * kLn2;
    float2 *rows = reinterpret_cast<float2 *>(ws);
    float *part = reinterpret_cast<float *>(reinterpret_cast<char *>(ws) + align256((size_t)dm.batch * dm.Hq * dm.max_seqlen * sizeof(float2)));
    const BwdPlan plan = bwd_plan(dm, w);
    const int64_t heads = (int64_t)dm.batch * dm.Hkv;
    timing_begin("window_dq_kernel", stream);
    hipLaunchKernelGGL(window_dq_kernel, dim3((unsigned)(n_tiles * heads)), dim3(256), 0, stream, dm, w, scale, lg, n_tiles, q, k, v, out,
                       dout, lse, seqlens, dq, rows);
    timing_end(stream);
    timing_begin("window_dkdv_kernel", stream);
    const int64_t items = (int64_t)plan.sink_tiles * plan.sink_chunks + (int64_t)(plan.tiles - plan.sink_tiles) * plan.chunks;
    hipLaunchKernelGGL(window_dkdv_kernel, dim3((unsigned)(items * heads)), dim3(256), 0, stream, dm, w, scale, lg, plan, q, k, v, dout,
                       rows, seqlens, dk, dv, part);
    timing_end(stream);
    if (plan.chunks == 1 && (plan.sink_tiles == 0 || plan.sink_chunks == 1)) return (int)hipGetLastError();
    const int keys = plan.chunks > 1 ? dm.max_seqlen : min(dm.max_seqlen, plan.sink_tiles * kKvKeys);
    timing_begin("window_join_kernel", stream);
    hipLaunchKernelGGL(window_join_kernel, dim3((keys + 15) / 16, dm.Hkv, dm.batch), dim3(256), 0, stream, dm, w, lg, plan, seqlens, part,
                       dk, dv);
    timing_end(stream);
    return (int)hipGetLastError();
}

}  // namespace infllmv2
