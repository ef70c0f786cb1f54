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

// The running maximum follows a row's scores only where they exceed it by more than this (in powers of two): probabilities stay
// below 2^kSlack, and the outputs are rescaled once or twice per row instead of every tile.
constexpr float kSlack = 8.f;

__global__ __launch_bounds__(256, 2) void window_prefill_kernel(Dims dm, WindowArgs win, int lg, int n_tiles, Tensor q, Tensor k, Tensor v,
                                                                const int32_t *__restrict__ seqlens, Tensor out, float *__restrict__ lse) {
    __shared__ Tile64 K0, K1, V0, V1;
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
    const TileCopier keys(k, b, h, L, wave, lane), values(v, b, h, L, wave, lane);
    auto stage = [&](const TileCopier &from, Tile64 &to, int x) __attribute__((always_inline)) {
        if (x < kt.count) from.copy(to, kt.key0(x), wave, lane);
    };
    stage(keys, K0, 0);
    stage(values, V0, 0);
    stage(keys, K1, 1);
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
    const auto larger = [](float a, float d) { return fmaxf(a, d); };
    auto scores = [&](const Tile64 &kt_, f32x16 (&s)[2]) __attribute__((always_inline)) {
        s[0] = zero16();
        s[1] = zero16();
#pragma unroll
        for (int ks = 0; ks < 8; ++ks) {
            s[0] = mfma32(rd.rows(kt_.x, ks), qf[ks], s[0]);
            s[1] = mfma32(rd.rows(kt_.x + kHalfTile, ks), qf[ks], s[1]);
        }
    };
    auto largest = [&](const f32x16 (&s)[2]) __attribute__((always_inline)) {
        float a = max3(s[0][0], s[0][1], s[0][2]), d = max3(s[1][0], s[1][1], s[1][2]);
#pragma unroll
        for (int e = 3; e < 15; e += 2) {
            a = max3(a, s[0][e], s[0][e + 1]);
            d = max3(d, s[1][e], s[1][e + 1]);
        }
        return max3(max3(a, s[0][15], s[1][15]), d, d);
    };
    // the keys a row does not see out of tile x, if there are any, and the largest of the others
    auto hide = [&](f32x16 (&s)[2], int x, float &mx) __attribute__((always_inline)) {
        const int k0 = kt.key0(x);
        if (k0 + kWinKeys - 1 <= w_lo && (k0 + kWinKeys <= win.n_sink || w_hi - k0 < win.window)) return;
        int at = k0 + 4 * hf;
        asm volatile("" : "+v"(at));
        const VisibleKeys visible(win, i);
#pragma unroll
        for (int kh = 0; kh < 2; ++kh)
#pragma unroll
            for (int e = 0; e < 16; ++e) s[kh][e] = visible(at + 32 * kh + 8 * (e >> 2) + (e & 3)) ? s[kh][e] : -INFINITY;
        mx = largest(s);
    };
    // Tile x: its probabilities and their product with the values, and between them the next tile's scores, so that the matrix cores have
    // work while the exponentials run.  (Behind the last tile: scores of what lies in LDS, not used.)
    auto step = [&](Tile64 &k_cur, const Tile64 &k_next, const Tile64 &v_cur, Tile64 &v_next, f32x16 (&s)[2], f32x16 (&s_next)[2], float &mx,
                    int x) __attribute__((always_inline)) {
        __builtin_amdgcn_s_waitcnt(0);                   // this wavefront's copies have landed
        __syncthreads();                                 // everyone's have, and everyone is past the tile before
        stage(keys, k_cur, x + 2);
        stage(values, v_next, x + 1);
        mx = half_reduce(mx, larger) * c;
        if (__any(mx > m + kSlack)) {
            const float m_new = fmaxf(m, mx), alpha = fast_exp2(m - (m_new == -INFINITY ? 0.f : m_new));
            m = m_new;
            l *= alpha;
#pragma unroll
            for (int ct = 0; ct < 4; ++ct) o[ct] *= alpha;
        }
        const float base = m == -INFINITY ? 0.f : m;
        __builtin_amdgcn_sched_barrier(0);
        scores(k_next, s_next);
        bf16x8 p[4];
        float sum[2] = {0.f, 0.f};
#pragma unroll
        for (int kh = 0; kh < 2; ++kh) {
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                s[kh][e] = fast_exp2(__builtin_fmaf(s[kh][e], c, -base));
                sum[e & 1] += s[kh][e];
            }
            p[2 * kh] = pack8(s[kh], 0);
            p[2 * kh + 1] = pack8(s[kh], 1);
        }
        l += sum[0] + sum[1];
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int ct = 0; ct < 4; ++ct) o[ct] = mfma32(rd.columns(v_cur.x + (j >> 1) * kHalfTile, j & 1, ct), p[j], o[ct]);
        mx = largest(s_next);
        __builtin_amdgcn_sched_barrier(0);
        if (x + 1 < kt.count) hide(s_next, x + 1, mx);
    };
    f32x16 sa[2], sb[2];
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
    scores(K0, sa);
    float mx = largest(sa);
    hide(sa, 0, mx);
    for (int x = 0; x < kt.count; x += 2) {
        step(K0, K1, V0, V1, sa, sb, mx, x);
        if (x + 1 < kt.count) step(K1, K0, V1, V0, sb, sa, mx, x + 1);
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
