// Attention of single queries over a cache in 4 bits (the selected blocks, or a window) and over the window of a bf16 cache.
//
// The keys of a query row are walked in units of 32 tokens: halves of the selected blocks, or the units that hold the first
// n_sink tokens and the window.  A workgroup takes a run of a row's units, its four wavefronts every fourth of them, each by
// itself: keys as rows of the first product (S^T = K . Q^T, 16 heads as columns), a running maximum and sum per head, the values through
// 8 KiB of LDS of the wavefront's own (stored as rows, read transposed) into the second (O^T = V^T . P^T).  The order of keys within a product is free,
// so the probabilities are the second product's operand in the registers they come out in.  At the end the four
// states are joined in LDS; where a row is split over workgroups, decode_merge_kernel joins those.
#include "quant.h"
#include "token_union.h"

namespace infllmv2 {

constexpr int kUnit = 32;                                // tokens

struct RowSource {                                       // a cache of either kind
    Tensor k, v;
    QuantTensor kq, vq;
};


// One unit of K and V on its way.  Lane (n, g): key rows n and 16 + n.
template <bool kQuant>
struct UnitRows;
template <>
struct UnitRows<false> {
    bf16x8 k[2][4];                                      // channels 32 ks + 8 g ..
    uint4 v[8];                                          // row lane / 16 + 4 i, channels 8 (lane % 16) ..
    __device__ __forceinline__ void load(const RowSource &s, int64_t k_head, int64_t v_head, int key0, int last, int lane) {
        const int n = lane & 15, g = lane >> 4;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const __bf16 *kr = s.k.ptr + k_head + (int64_t)min(key0 + 16 * t + n, last) * s.k.st + 8 * g;
#pragma unroll
            for (int ks = 0; ks < 4; ++ks) k[t][ks] = load8(kr + 32 * ks);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i)
            v[i] = *reinterpret_cast<const uint4 *>(s.v.ptr + v_head + (int64_t)min(key0 + g + 4 * i, last) * s.v.st + 8 * n);
    }
    __device__ __forceinline__ bf16x8 key(int t, int ks) const { return k[t][ks]; }
    __device__ __forceinline__ void values(char *vs, uint32_t allow, int lane) const {
        const int n = lane & 15, g = lane >> 4;
#pragma unroll
        for (int i = 0; i < 8; ++i) {                    // (rows the query does not see as zeros: 0 * garbage must stay 0)
            const int r = g + 4 * i;
            const uint4 y = (allow >> r) & 1u ? v[i] : uint4{0u, 0u, 0u, 0u};
            *reinterpret_cast<uint4 *>(vs + r * 256 + ((n ^ row_swizzle(r)) << 4)) = y;
        }
    }
};
template <>
struct UnitRows<true> {
    uint4 k[2], v[2];                                    // K: channels 32 g .. of its row; V: row lane / 4 + 16 i, channels 32 (lane % 4) ..
    uint8_t ke[2], ve[2];
    __device__ __forceinline__ void load(const RowSource &s, int64_t, int64_t, int key0, int last, int lane, int b, int h) {
        const int n = lane & 15, g = lane >> 4;
        const int64_t kc = b * s.kq.sb + h * s.kq.sh, kx = b * s.kq.eb + h * s.kq.eh;
        const int64_t vc = b * s.vq.sb + h * s.vq.sh, vx = b * s.vq.eb + h * s.vq.eh;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const int64_t r = min(key0 + 16 * t + n, last), rv = min(key0 + 16 * t + (lane >> 2), last);
            k[t] = *reinterpret_cast<const uint4 *>(s.kq.codes + kc + r * s.kq.st + 16 * g);
            ke[t] = s.kq.scales[kx + r * s.kq.et + g];
            v[t] = *reinterpret_cast<const uint4 *>(s.vq.codes + vc + rv * s.vq.st + 16 * (lane & 3));
            ve[t] = s.vq.scales[vx + rv * s.vq.et + (lane & 3)];
        }
    }
    __device__ __forceinline__ bf16x8 key(int t, int ks) const {
        const uint32_t w = ks == 0 ? k[t].x : ks == 1 ? k[t].y : ks == 2 ? k[t].z : k[t].w;
        return __builtin_bit_cast(bf16x8, dequant8(w, ke[t]));
    }
    __device__ __forceinline__ void values(char *vs, uint32_t allow, int lane) const {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const int r = 16 * t + (lane >> 2);
            const bool seen = (allow >> r) & 1u;
            const uint32_t w[4] = {v[t].x, v[t].y, v[t].z, v[t].w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint4 y = seen ? dequant8(w[i], ve[t]) : uint4{0u, 0u, 0u, 0u};
                *reinterpret_cast<uint4 *>(vs + r * 256 + (((4 * (lane & 3) + i) ^ row_swizzle(r)) << 4)) = y;
            }
        }
    }
};

// grid (splits, Hkv, rows).  kList: a row's units are the halves of its list's entries, `per` entries to a split; otherwise its share
// of the units of its window.  With one split the result is written as it is, else as a partial (o, maximum, sum).
template <bool kQuant, bool kList>
__global__ __launch_bounds__(256) void stream_attn_kernel(Dims dm, WindowArgs win, Tensor q, RowSource src, const int32_t *__restrict__ seqlens,
                                                          const int32_t *__restrict__ block_idx, const uint64_t *__restrict__ tree_mask,
                                                          int per, Tensor out, float *__restrict__ lse, float *__restrict__ o_part,
                                                          float2 *__restrict__ ml_part) {
    __shared__ __align__(16) char Vs[4][kUnit * 256];
    __shared__ float2 ml_s[4][16];
    const int split = blockIdx.x, n_split = gridDim.x, h = blockIdx.y, bv = blockIdx.z;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n = lane & 15, g = lane >> 4, G = dm.G;
    int b, qi;
    const int L = query_row(dm, seqlens, bv, b, qi);
    // ---- the query: lane (n, g) holds head n, channels 32 ks + 8 g .. (4-bit keys: 32 g + 8 ks ..) --------------------
    bf16x8 bq[4];
    {
        const __bf16 *qr = q.ptr + b * q.sb + qi * q.st + (int64_t)(h * G + min(n, G - 1)) * q.sh;
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) bq[ks] = load8(qr + (kQuant ? 32 * g + 8 * ks : 32 * ks + 8 * g));
    }
    // ---- the row's units ---------------------------------------------------------------------------------------------
    const int L_all = L + (dm.n_q - 1 - qi);             // cache rows of the sequence (when L >= 1)
    uint64_t mask_word = 0ull;
    int entry = -1, u = 0, u_end = 0, sinks = 0, skip = 0, lo = 0;
    if constexpr (kList) {
        const int e0 = split * per, e1 = min(e0 + per, dm.topk);
        if (tree_mask) {
            mask_word = tree_mask[bv];
            if (dm.n_q < 64) mask_word &= (1ull << dm.n_q) - 1ull;
        }
        if (e0 + lane < e1) entry = block_idx[(((int64_t)b * dm.Hkv + h) * dm.n_q + qi) * dm.topk + e0 + lane];
        u = wave;
        u_end = L >= 1 ? 2 * (e1 - e0) : 0;
    } else if (L >= 1) {
        lo = max(0, L - win.window);
        sinks = (min(win.n_sink, lo) + kUnit - 1) / kUnit;
        const int w0 = max(lo / kUnit, sinks);
        skip = w0 - sinks;
        const int all = sinks + (L - 1) / kUnit - w0 + 1;
        u = (int)((int64_t)all * split / n_split) + wave;
        u_end = (int)((int64_t)all * (split + 1) / n_split);
    }
    // the first key of unit x, and which of its keys the row sees (bit r: key0 + r); uniform over the wavefront
    auto place = [&](int x, int &key0) __attribute__((always_inline)) -> uint32_t {
        if (x >= u_end) return 0u;
        if constexpr (kList) {
            const int blk = __builtin_amdgcn_readlane(entry, x >> 1);
            const int64_t at = (int64_t)blk * kBlock + kUnit * (x & 1);
            if (blk < 0 || at >= (tree_mask ? L_all : L)) return 0u;
            key0 = (int)at;
            const int valid = tree_mask ? L_all - dm.n_q - key0 : L - key0;   // keys before the drafted tokens; up to the query's own
            uint32_t allow = valid >= kUnit ? ~0u : valid <= 0 ? 0u : (1u << valid) - 1u;
            if (tree_mask && valid < kUnit) allow |= valid >= 0 ? (uint32_t)(mask_word << valid) : -valid < 64 ? (uint32_t)(mask_word >> -valid) : 0u;
            return allow;
        } else {
            key0 = kUnit * (x < sinks ? x : x + skip);
            uint32_t allow = L - key0 >= kUnit ? ~0u : (1u << (L - key0)) - 1u;
            if (key0 < lo) {                             // of the keys before the window the first n_sink
                const uint32_t old = lo - key0 >= kUnit ? ~0u : (1u << (lo - key0)) - 1u;
                const int s = win.n_sink - key0;
                allow &= ~old | (s >= kUnit ? ~0u : s <= 0 ? 0u : (1u << s) - 1u);
            }
            return allow;
        }
    };
    const int64_t k_head = kQuant ? 0 : b * src.k.sb + h * src.k.sh, v_head = kQuant ? 0 : b * src.v.sb + h * src.v.sh;
    const int last = dm.max_seqlen - 1;
    auto fetch = [&](UnitRows<kQuant> &x, int key0) __attribute__((always_inline)) {
        if constexpr (kQuant) x.load(src, 0, 0, key0, last, lane, b, h);
        else x.load(src, k_head, v_head, key0, last, lane);
    };
    // ---- the walk ------------------------------------------------------------------------------------------------------
    f32x4 o[8];
#pragma unroll
    for (int c = 0; c < 8; ++c) o[c] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m = -INFINITY, l = 0.f;
    char *vs = Vs[wave];
    auto attend = [&](const UnitRows<kQuant> &x, uint32_t allow) __attribute__((always_inline)) {
        f32x4 s[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            s[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int ks = 0; ks < 4; ++ks) s[t] = mfma16(x.key(t, ks), bq[ks], s[t]);
        }
        x.values(vs, allow, lane);
        float y[8], mx = -INFINITY;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int j = 0; j < 4; ++j) {                // key 16 t + 4 g + j
                y[4 * t + j] = (allow >> (16 * t + 4 * g + j)) & 1u ? s[t][j] * dm.scale_log2 : -INFINITY;
                mx = fmaxf(mx, y[4 * t + j]);
            }
        const float m_new = fmaxf(m, xgroup_max(mx)), base = m_new == -INFINITY ? 0.f : m_new;
        const float alpha = fast_exp2(m - base);
        m = m_new;
        float ps = 0.f;
        bf16x8 p;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float e = fast_exp2(y[j] - base);
            ps += e;
            p[j] = (__bf16)e;
        }
        l = l * alpha + ps;                              // (this lane's keys only: joined over g at the end)
        __builtin_amdgcn_wave_barrier();                 // same wavefront: LDS keeps the order
#pragma unroll
        for (int c = 0; c < 8; ++c) {                    // A: channel 16 c + n, keys 4 g .. and 16 + 4 g ..
            const int r = 4 * g + (n >> 2);
            const char *at = vs + 8 * (n & 1);
            const int piece = 2 * c + ((n & 3) >> 1);
            const s16x4 x0 = lds_read_tr16(at + r * 256 + ((piece ^ row_swizzle(r)) << 4));
            const s16x4 x1 = lds_read_tr16(at + (r + 16) * 256 + ((piece ^ row_swizzle(r + 16)) << 4));
            o[c] = mfma16(__builtin_bit_cast(bf16x8, __builtin_shufflevector(x0, x1, 0, 1, 2, 3, 4, 5, 6, 7)), p, o[c] * alpha);
        }
        __builtin_amdgcn_wave_barrier();
    };
    // the next unit of the wavefront that has a visible key
    auto advance = [&](int x, int &key0, uint32_t &allow) __attribute__((always_inline)) {
        while (x < u_end && (allow = place(x, key0)) == 0u) x += 4;
        return x;
    };
    UnitRows<kQuant> a, c;
    int ka = 0, kc = 0;
    uint32_t aa = 0u, ac = 0u;
    u = advance(u, ka, aa);
    if (u < u_end) fetch(a, ka);
    while (u < u_end) {
        int next = advance(u + 4, kc, ac);
        if (next < u_end) fetch(c, kc);
        attend(a, aa);
        u = next;
        if (u >= u_end) break;
        next = advance(u + 4, ka, aa);
        if (next < u_end) fetch(a, ka);
        attend(c, ac);
        u = next;
    }
    l = xgroup_sum(l);
    // ---- the four wavefronts' states into one --------------------------------------------------------------------------
    if (g == 0) ml_s[wave][n] = float2{m, l};
    __syncthreads();
    const float M = fmaxf(fmaxf(ml_s[0][n].x, ml_s[1][n].x), fmaxf(ml_s[2][n].x, ml_s[3][n].x)), base = M == -INFINITY ? 0.f : M;
    const float w = fast_exp2(m - base);
    float *mine = reinterpret_cast<float *>(vs);         // [head][channel]: its 8 KiB
#pragma unroll
    for (int ch = 0; ch < 8; ++ch)
        *reinterpret_cast<f32x4 *>(mine + n * kHeadDim + 16 * (ch ^ (n & 7)) + 4 * g) = o[ch] * w;
    __syncthreads();
    const int head = tid >> 4, c8 = 8 * (tid & 15);      // eight channels of a head
    if (head < G) {
        float den = 0.f, Mh = -INFINITY;
#pragma unroll
        for (int i = 0; i < 4; ++i) Mh = fmaxf(Mh, ml_s[i][head].x);
        const float bh = Mh == -INFINITY ? 0.f : Mh;
        float y[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            den += ml_s[i][head].y * fast_exp2(ml_s[i][head].x - bh);
            const float *from = reinterpret_cast<const float *>(Vs[i]) + head * kHeadDim + 16 * ((c8 >> 4) ^ (head & 7)) + (c8 & 15);
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] += from[e];
        }
        const int hq = h * G + head;
        if (n_split == 1) {
            bf16x8 r;
#pragma unroll
            for (int e = 0; e < 8; ++e) r[e] = (__bf16)(den > 0.f ? y[e] / den : 0.f);
            *reinterpret_cast<uint4 *>(out.ptr + b * out.sb + qi * out.st + (int64_t)hq * out.sh + c8) = __builtin_bit_cast(uint4, r);
            if (c8 == 0) lse[(int64_t)bv * dm.Hq + hq] = den > 0.f ? lse_of(bh, den) : -INFINITY;
        } else {
            const int64_t at = ((int64_t)bv * dm.Hq + hq) * n_split + split;
            float4 *op = reinterpret_cast<float4 *>(o_part + at * kHeadDim + c8);
            op[0] = float4{y[0], y[1], y[2], y[3]};
            op[1] = float4{y[4], y[5], y[6], y[7]};
            if (c8 == 0) ml_part[at] = float2{Mh, den};
        }
    }
}

// ---- host side -------------------------------------------------------------------------------------------------------------
static inline size_t align256(size_t x) { return (x + 255) / 256 * 256; }

// How many workgroups a row's `units` are split over: enough to fill the chip, at least four units (one per wavefront) each.
constexpr int kMaxSplits = 64;                           // what decode_merge_kernel joins
static int stream_splits(const Dims &dm, int64_t units) {
    const int64_t rows = max((int64_t)1, (int64_t)dm.batch * dm.n_q * dm.Hkv);
    const int64_t want = (1024 + rows - 1) / rows, most = (units + 3) / 4;
    return (int)max((int64_t)1, min(min(want, most), (int64_t)kMaxSplits));
}
// The most units a window may touch: the sinks', and one more than fill the window.
static int64_t window_units(const Dims &dm, WindowArgs w) {
    const int64_t whole = ((int64_t)dm.max_seqlen + kUnit - 1) / kUnit;
    return min(whole, ((int64_t)w.n_sink + kUnit - 1) / kUnit + ((int64_t)w.window + kUnit - 1) / kUnit + 1);
}

template <bool kQuant, bool kList>
static int launch_stream(const char *name, const Dims &dm, WindowArgs win, int splits, int per, Tensor q, const RowSource &src,
                         const int32_t *seqlens, const int32_t *block_idx, const uint64_t *tree_mask, Tensor out, float *lse, void *ws,
                         hipStream_t stream) {
    float *o_part = reinterpret_cast<float *>(ws);
    float2 *ml_part = reinterpret_cast<float2 *>(reinterpret_cast<char *>(ws) +
                                                 align256((size_t)dm.batch * dm.n_q * dm.Hq * splits * kHeadDim * sizeof(float)));
    timing_begin(name, stream);
    hipLaunchKernelGGL((stream_attn_kernel<kQuant, kList>), dim3(splits, dm.Hkv, dm.batch * dm.n_q), dim3(256), 0, stream, dm, win, q, src,
                       seqlens, block_idx, tree_mask, per, out, lse, o_part, ml_part);
    timing_end(stream);
    if (splits == 1) return (int)hipGetLastError();
    Dims parts = dm;
    parts.topk = splits;
    return launch_decode_merge(parts, o_part, ml_part, out, lse, stream);
}

int launch_attn_decode_quant(const Dims &dm, Tensor q, QuantTensor kq, QuantTensor vq, const int32_t *seqlens,
                             const int32_t *block_idx, const uint64_t *tree_mask, Tensor out, float *lse, void *ws,
                             hipStream_t stream) {
    if (dm.batch <= 0) return 0;
    const int want = stream_splits(dm, 2 * dm.topk), per = (dm.topk + want - 1) / want;
    return launch_stream<true, true>("sparse_attn_quant_kernel", dm, WindowArgs{0, 0}, (dm.topk + per - 1) / per, per, q,
                                     RowSource{Tensor{}, Tensor{}, kq, vq}, seqlens, block_idx, tree_mask, out, lse, ws, stream);
}

size_t window_decode_ws_bytes(const Dims &dm, WindowArgs w) {
    const size_t rows = (size_t)dm.batch * dm.Hq * stream_splits(dm, window_units(dm, w));
    return align256(rows * kHeadDim * sizeof(float)) + align256(rows * sizeof(float2));
}

int launch_window_decode(const Dims &dm, WindowArgs w, Tensor q, Tensor k, Tensor v, const int32_t *seqlens, Tensor out, float *lse,
                         void *ws, hipStream_t stream) {
    if (dm.batch <= 0) return 0;
    return launch_stream<false, false>("window_decode_kernel", dm, w, stream_splits(dm, window_units(dm, w)), 0, q,
                                       RowSource{k, v, QuantTensor{}, QuantTensor{}}, seqlens, nullptr, nullptr, out, lse, ws, stream);
}

int launch_window_decode_quant(const Dims &dm, WindowArgs w, Tensor q, QuantTensor kq, QuantTensor vq, const int32_t *seqlens,
                               Tensor out, float *lse, void *ws, hipStream_t stream) {
    if (dm.batch <= 0) return 0;
    return launch_stream<true, false>("window_decode_quant_kernel", dm, w, stream_splits(dm, window_units(dm, w)), 0, q,
                                      RowSource{Tensor{}, Tensor{}, kq, vq}, seqlens, nullptr, nullptr, out, lse, ws, stream);
}

}  // namespace infllmv2
