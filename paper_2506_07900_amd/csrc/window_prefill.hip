// Attention over a sliding window and the first tokens, one query per cached token: one pass over the visible keys with a running
// maximum and sum.
//
// A workgroup takes 128 query rows, (token, head of the group) with the heads fastest, so its rows see the same keys but for
// the few tokens they span, and every key tile is fetched once for them.  Four wavefronts of 32 rows; key and value tiles of 64 tokens go from
// memory straight into LDS, one tile ahead.  S^T = K . Q^T leaves a row's scores in a lane and its partner, so maxima and sums are
// per lane, and the probabilities are the second operand of O^T = V^T . P^T in the registers they come out in.
#include "window.h"

namespace infllmv2 {

constexpr int kFwdRows = 128;
struct __align__(16) KVTile {
    char k[kWinKeys * 256], v[kWinKeys * 256];
};

// The running maximum follows a row's scores only where they exceed it by more than this (in powers of two): probabilities stay
// below 2^kSlack, and the outputs are rescaled once or twice per row instead of every tile.
constexpr float kSlack = 8.f;

__global__ __launch_bounds__(256, 2) void window_prefill_kernel(Dims dm, WindowArgs win, int lg, int n_tiles, Tensor q, Tensor k, Tensor v,
                                                                const int32_t *__restrict__ seqlens, Tensor out, float *__restrict__ lse) {
    __shared__ KVTile tile0, tile1;
    const int id = xcd_run(blockIdx.x, gridDim.x);
    const int ti = id % n_tiles, bh = id / n_tiles, b = bh / dm.Hkv, h = bh - b * dm.Hkv;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int c32 = lane & 31, hf = lane >> 5;
    const int L = clamp_len(uniform_load(seqlens + b), dm.max_seqlen);
    const int t0 = ti * (kFwdRows >> lg), t1 = min(L, t0 + (kFwdRows >> lg));
    const int row = 32 * wave + c32, i = t0 + (row >> lg), hq = h * dm.G + (row & (dm.G - 1));
    __bf16 *o_row = out.ptr + b * out.sb + (int64_t)i * out.st + (int64_t)hq * out.sh + 4 * hf;
    float *lse_at = lse + ((int64_t)b * dm.max_seqlen + i) * dm.Hq + hq;
    if (t0 >= L) {
        if (dm.fill && i < dm.max_seqlen) {
            for (int c = 0; c < 16; ++c) *reinterpret_cast<uint2 *>(o_row + 8 * c) = uint2{0u, 0u};
            if (hf == 0) *lse_at = 0.f;
        }
        return;
    }
    const KeyTiles kt(win, t0, t1);
    const char *k_head = reinterpret_cast<const char *>(k.ptr + b * k.sb + h * k.sh), *v_head = reinterpret_cast<const char *>(v.ptr + b * v.sb + h * v.sh);
    auto stage = [&](KVTile &dst, int x) __attribute__((always_inline)) {
        if (x >= kt.count) return;
        const int k0 = kt.key0(x);
#pragma unroll
        for (int j = 0; j < 4; ++j) {                    // 1 KiB: rows 16 wave + 4 j + lane / 16 (past the sequence: its last again)
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
    bf16x8 qf[8];
    {
        const __bf16 *qr = q.ptr + b * q.sb + (int64_t)min(i, L - 1) * q.st + (int64_t)hq * q.sh + 8 * hf;
#pragma unroll
        for (int ks = 0; ks < 8; ++ks) qf[ks] = load8(qr + 16 * ks);
    }
    const TileReader rd(lane);
    const float c = dm.scale_log2;
    f32x16 o[4];
#pragma unroll
    for (int ct = 0; ct < 4; ++ct) o[ct] = zero16();
    float m = -INFINITY, l = 0.f;
    // tokens of this wavefront's rows
    const int w_lo = t0 + ((32 * wave) >> lg), w_hi = t0 + ((32 * wave + 31) >> lg);
    auto step = [&](const KVTile &cur, KVTile &next, int x) __attribute__((always_inline)) {
        __builtin_amdgcn_s_waitcnt(0);                   // this wavefront's copies have landed
        __syncthreads();                                 // everyone's have, and everyone is past the tile before
        stage(next, x + 1);
        const int k0 = kt.key0(x);
        // any of this wavefront's rows sees any of the keys?
        const bool some = k0 <= w_hi && (k0 < win.n_sink || w_lo - (k0 + kWinKeys - 1) < win.window);
        if (!some) return;
        f32x16 s[2];
        s[0] = zero16();
        s[1] = zero16();
#pragma unroll
        for (int ks = 0; ks < 8; ++ks) {
            s[0] = mfma32(rd.rows(cur.k, ks), qf[ks], s[0]);
            s[1] = mfma32(rd.rows(cur.k + 32 * 256, ks), qf[ks], s[1]);
        }
        // all of them all of the keys?
        const bool all = k0 + kWinKeys - 1 <= w_lo && (k0 + kWinKeys <= win.n_sink || w_hi - k0 < win.window);
        if (!all) {
#pragma unroll
            for (int kh = 0; kh < 2; ++kh)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int t = k0 + 32 * kh + 8 * (e >> 2) + 4 * hf + (e & 3);
                    if (!(t <= i && (t < win.n_sink || i - t < win.window))) s[kh][e] = -INFINITY;
                }
        }
        float mx = fmaxf(s[0][0], s[1][0]);
#pragma unroll
        for (int e = 1; e < 16; ++e) mx = fmaxf(mx, fmaxf(s[0][e], s[1][e]));
        mx = half_reduce(mx, [](float a, float d) { return fmaxf(a, d); }) * c;
        if (__any(mx > m + kSlack)) {
            const float m_new = fmaxf(m, mx), alpha = fast_exp2(m - (m_new == -INFINITY ? 0.f : m_new));
            m = m_new;
            l *= alpha;
#pragma unroll
            for (int ct = 0; ct < 4; ++ct) o[ct] *= alpha;
        }
        const float base = m == -INFINITY ? 0.f : m;
#pragma unroll
        for (int kh = 0; kh < 2; ++kh)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                s[kh][e] = fast_exp2(__builtin_fmaf(s[kh][e], c, -base));
                l += s[kh][e];
            }
#pragma unroll
        for (int kh = 0; kh < 2; ++kh)
#pragma unroll
            for (int s2 = 0; s2 < 2; ++s2) {
                const bf16x8 p = pack8(s[kh], s2);
#pragma unroll
                for (int ct = 0; ct < 4; ++ct) o[ct] = mfma32(rd.columns(cur.v, 2 * kh + s2, ct), p, o[ct]);
            }
    };
    for (int x = 0; x < kt.count; x += 2) {
        step(tile0, tile1, x);
        if (x + 1 < kt.count) step(tile1, tile0, x + 1);
    }
    l = half_reduce(l, [](float a, float d) { return a + d; });
    if (i >= dm.max_seqlen || (i >= L && !dm.fill)) return;
    const bool live = i < L;
#pragma unroll
    for (int ct = 0; ct < 4; ++ct)
#pragma unroll
        for (int e4 = 0; e4 < 4; ++e4) {
            bf16x4 r;
#pragma unroll
            for (int e = 0; e < 4; ++e) r[e] = (__bf16)(live ? o[ct][4 * e4 + e] / l : 0.f);
            *reinterpret_cast<uint2 *>(o_row + 32 * ct + 8 * e4) = __builtin_bit_cast(uint2, r);
        }
    if (hf == 0) *lse_at = live ? lse_of(m, l) : 0.f;
}

size_t window_prefill_ws_bytes(const Dims &, WindowArgs) { return 0; }

int launch_window_prefill(const Dims &dm, WindowArgs w, Tensor q, Tensor k, Tensor v, const int32_t *seqlens, Tensor out, float *lse,
                          void *, hipStream_t stream) {
    if (dm.batch <= 0 || dm.max_seqlen <= 0) return 0;
    const int lg = __builtin_ctz(dm.G), per = kFwdRows >> lg, n_tiles = (dm.max_seqlen + per - 1) / per;
    timing_begin("window_prefill_kernel", stream);
    hipLaunchKernelGGL(window_prefill_kernel, dim3((unsigned)((int64_t)n_tiles * dm.Hkv * dm.batch)), dim3(256), 0, stream, dm, w, lg,
                       n_tiles, q, k, v, seqlens, out, lse);
    timing_end(stream);
    return (int)hipGetLastError();
}

}  // namespace infllmv2
