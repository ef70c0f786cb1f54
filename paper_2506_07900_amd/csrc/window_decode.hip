// Attention of single queries over a cache in 4 bits (the selected blocks, or a window) and over the window of a bf16 cache.
//
// The keys of a query row are walked in units of 32 tokens: halves of the selected blocks, or the units that hold the first
// n_sink tokens and the window.  A workgroup takes a run of a row's units, its wavefronts (four, or eight) take them in turn, each by
// itself: keys as rows of the first product (S^T = K . Q^T, 16 heads as columns), a running maximum and sum per head, the values through
// 8 KiB of LDS of the wavefront's own (stored as rows, read transposed) into the second (O^T = V^T . P^T).  The order of keys within a product is free,
// so the probabilities are the second product's operand in the registers they come out in.  At the end their
// states are joined in LDS; where a row is split over workgroups, decode_merge_kernel joins those.
#include <type_traits>

#include "quant.h"
#include "window.h"

namespace infllmv2 {

constexpr int kUnit = 32;                                // tokens

struct RowSource {                                       // a cache of either kind
    Tensor k, v;
    QuantTensor kq, vq;
};


// An address that is the same for all lanes, in scalar registers.
__device__ __forceinline__ const uint8_t *uniform(const uint8_t *p) {
    const uint64_t x = (uint64_t)(uintptr_t)p;
    return (const uint8_t *)(uintptr_t)((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(x >> 32)) << 32 |
                                        (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)x));
}

// One unit of K and V on its way.  Lane (n, g): key rows n and 16 + n.
template <bool kQuant>
struct UnitRows;
template <>
struct UnitRows<false> {
    struct Head {
        __device__ __forceinline__ Head(const RowSource &, int, int, int) {}
    };
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
    uint4 k[2], v[2];                                    // row n + 16 t, channels 32 g ..
    uint32_t ke[2], ve[2];
    // The head's first row, and bytes from a unit's first row to this lane's codes and exponents, of K and of V.
    struct Head {
        const uint8_t *kc, *ke, *vc, *ve;
        uint32_t at[4];
        __device__ __forceinline__ Head(const RowSource &s, int b, int h, int lane)
            : kc(uniform(s.kq.codes + b * s.kq.sb + h * s.kq.sh)), ke(uniform(s.kq.scales + b * s.kq.eb + h * s.kq.eh)),
              vc(uniform(s.vq.codes + b * s.vq.sb + h * s.vq.sh)), ve(uniform(s.vq.scales + b * s.vq.eb + h * s.vq.eh)) {
            const uint32_t n = lane & 15, g = lane >> 4;
            at[0] = n * (uint32_t)s.kq.st + 16 * g;
            at[1] = n * (uint32_t)s.kq.et + g;
            at[2] = n * (uint32_t)s.vq.st + 16 * g;
            at[3] = n * (uint32_t)s.vq.et + g;
        }
    };
    __device__ __forceinline__ void load(const RowSource &s, const Head &head, int key0, int rows, int lane) {    // the cache has `rows` from key0 on
        typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
        key0 = __builtin_amdgcn_readfirstlane(key0);
        auto from = [&](const uint8_t *p, int64_t st) __attribute__((always_inline)) {
            return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(p + key0 * st), 0, 0xfffffffeu, 0x00027000);
        };
        const auto kc = from(head.kc, s.kq.st), ke_ = from(head.ke, s.kq.et), vc = from(head.vc, s.vq.st), ve_ = from(head.ve, s.vq.et);
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const bool row = (lane & 15) + 16 * t < rows;
            k[t] = __builtin_bit_cast(uint4, (u32x4)__builtin_amdgcn_raw_buffer_load_b128(kc, row ? head.at[0] + 16 * t * (uint32_t)s.kq.st : kNoRow, 0, 0));
            v[t] = __builtin_bit_cast(uint4, (u32x4)__builtin_amdgcn_raw_buffer_load_b128(vc, row ? head.at[2] + 16 * t * (uint32_t)s.vq.st : kNoRow, 0, 0));
            ke[t] = __builtin_amdgcn_raw_buffer_load_b8(ke_, row ? head.at[1] + 16 * t * (uint32_t)s.kq.et : kNoRow, 0, 0);
            ve[t] = __builtin_amdgcn_raw_buffer_load_b8(ve_, row ? head.at[3] + 16 * t * (uint32_t)s.vq.et : kNoRow, 0, 0);
        }
    }
    __device__ __forceinline__ bf16x8 key(int t, int ks) const {
        const uint32_t w = ks == 0 ? k[t].x : ks == 1 ? k[t].y : ks == 2 ? k[t].z : k[t].w;
        return __builtin_bit_cast(bf16x8, dequant8(w, ke[t]));
    }
    // Values into LDS: four quarters of 32 channels, in each 32 rows of 64 bytes, whose four pieces are XORed with row / 4 % 4, its bits
    // exchanged: a store takes a piece of each of 16 rows, two groups of lanes of a transposing load 32 bytes of each of 8; sixteen lanes of either touch every
    // bank once, eight of a store's half of them twice.  By the counters 0.45 to 0.5 of this kernel's LDS time are bank conflicts all the same, the join's
    // stores at the end among them (16 heads at a pitch of 512 bytes, exchanged in pieces of 64: 16 lanes on four places of 16 bytes).
    __device__ __forceinline__ static uint32_t swizzle(uint32_t i) { return ((i & 1) << 1) | (i >> 1); }
    __device__ __forceinline__ void values(char *vs, uint32_t allow, int lane) const {
        const uint32_t n = lane & 15, g = lane >> 4;
        char *at = vs + g * 2048 + n * 64;
        const uint32_t x = swizzle(n >> 2) << 4;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            uint32_t w[4] = {v[t].x, v[t].y, v[t].z, v[t].w}, e = ve[t];
            if (allow != ~0u) {                          // what is not seen: zeros
                const uint32_t seen = 0u - ((allow >> (16 * t + n)) & 1u);
                e = seen ? e : 127u;
#pragma unroll
                for (int i = 0; i < 4; ++i) w[i] &= seen;
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) *reinterpret_cast<uint4 *>(at + 1024 * t + ((16 * i) ^ x)) = dequant8(w[i], e);
        }
    }
};

// grid (splits, Hkv, rows).  kList: a row's units are the halves of its list's entries, `per` entries to a split; otherwise its share
// of the units of its window.  With one split the result is written as it is, else as a partial (o, maximum, sum).
// A unit is 4.25 KiB of a 4-bit cache or 16 KiB of a bf16 one; a wavefront asks for its next one before it works on its present one.  Many rows are bound by
// traffic (64 sequences of up to 32K, window 8192, 4 bits: 26.4 us, 5.0 TB/s), few by round trips: a launch, a list or a length, a unit, about 5 us
// (one sequence, 16 blocks or 4096 tokens), and the joining launch 2 to 4 us.
template <bool kQuant, bool kList, int kWaves>
__global__ __launch_bounds__(64 * kWaves, kWaves == 4 && kQuant ? 3 : 2) void stream_attn_kernel(
    Dims dm, WindowArgs win, Tensor q, RowSource src, const int32_t *__restrict__ seqlens, const int32_t *__restrict__ block_idx,
    const uint64_t *__restrict__ tree_mask, int per, Tensor out, float *__restrict__ lse, float *__restrict__ o_part,
    float2 *__restrict__ ml_part) {
    __shared__ __align__(16) char Vs[kWaves][kUnit * 256];
    __shared__ float2 ml_s[kWaves][16];
    __shared__ bool again_s[kWaves];
    const int split = blockIdx.x, n_split = gridDim.x, h = blockIdx.y, bv = blockIdx.z;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    int lane = tid & 63, n = lane & 15, g = lane >> 4;
    const int G = dm.G;
    int b, qi;
    const int L = __builtin_amdgcn_readfirstlane(query_row(dm, seqlens, bv, b, qi));
    b = __builtin_amdgcn_readfirstlane(b);               // (uniform: the compiler divides in vector registers)
    qi = __builtin_amdgcn_readfirstlane(qi);
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
    const typename UnitRows<kQuant>::Head rows_of(src, b, h, lane);
    auto fetch = [&](UnitRows<kQuant> &x, int key0) __attribute__((always_inline)) {
        if constexpr (kQuant) x.load(src, rows_of, key0, dm.max_seqlen - key0, lane);
        else x.load(src, k_head, v_head, key0, last, lane);
    };
    // ---- the walk ------------------------------------------------------------------------------------------------------
    f32x4 o[8];
    float m, l, shift = 0.f;                             // probabilities are 2^(score - m - shift)
    char *vs = Vs[wave];
    auto attend = [&](const UnitRows<kQuant> &x, uint32_t allow) __attribute__((always_inline)) {
        f32x4 s[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            s[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int ks = 0; ks < 4; ++ks) s[t] = mfma16(x.key(t, ks), bq[ks], s[t]);
            if constexpr (kQuant) __builtin_amdgcn_sched_barrier(0);   // (one tile's keys in bf16 at a time: registers)
        }
        x.values(vs, allow, lane);
        if constexpr (kQuant) __builtin_amdgcn_sched_barrier(0);
        float y[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = s[e >> 2][e & 3];         // key 16 (e / 4) + 4 g + e % 4
        if (allow != ~0u) {
            const uint32_t mine = allow >> (4 * g);
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = (mine >> (16 * (e >> 2) + (e & 3))) & 1u ? y[e] : -INFINITY;
        }
        const float mx = xgroup_max(max3(max3(max3(y[0], y[1], y[2]), y[3], y[4]), max3(y[5], y[6], y[7]), y[7])) * dm.scale_log2;
        // the maximum follows only where scores exceed it by a factor of 2^8: outputs are rescaled once or twice, not every unit
        if (__any(mx > m + 8.f)) {
            const float m_new = fmaxf(m, mx), alpha = fast_exp2(m - (m_new == -INFINITY ? 0.f : m_new));
            m = m_new;
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
        __builtin_amdgcn_wave_barrier();                 // same wavefront: LDS keeps the order
#pragma unroll
        for (int c = 0; c < 8; ++c) {                    // A: channel 16 c + n, keys 4 g .. and 16 + 4 g ..
            const int r = 4 * g + (n >> 2);
            s16x4 x0, x1;
            if constexpr (kQuant) {
                const char *at = vs + (r * 64 + (((2 * (c & 1) + ((n & 3) >> 1)) ^ UnitRows<true>::swizzle(g)) << 4) + 8 * (n & 1)) + (c >> 1) * 2048;
                x0 = lds_read_tr16(at);
                x1 = lds_read_tr16(at + 1024);
            } else {
                const char *at = vs + 8 * (n & 1);
                const int piece = 2 * c + ((n & 3) >> 1);
                x0 = lds_read_tr16(at + r * 256 + ((piece ^ row_swizzle(r)) << 4));
                x1 = lds_read_tr16(at + (r + 16) * 256 + ((piece ^ row_swizzle(r + 16)) << 4));
            }
            o[c] = mfma16(__builtin_bit_cast(bf16x8, __builtin_shufflevector(x0, x1, 0, 1, 2, 3, 4, 5, 6, 7)), p, o[c]);
        }
        __builtin_amdgcn_wave_barrier();
    };
    // the next unit of the wavefront that has a visible key
    auto advance = [&](int x, int &key0, uint32_t &allow) __attribute__((always_inline)) {
        while (x < u_end && (allow = place(x, key0)) == 0u) x += kWaves;
        return x;
    };
    // A pass: the walk, the wavefronts' states into one, the result.  -> whether a sum of a row that has one came out as no number
    const int first = u, head = tid >> 4, c8 = 8 * (tid & 15);       // (a thread joins eight channels of a head)
    auto pass = [&](auto ahead) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
        m = -INFINITY;
        l = 0.f;
        UnitRows<kQuant> a, c;
        int ka = 0, kc = 0;
        uint32_t aa = 0u, ac = 0u;
        u = first;
        if constexpr (!ahead) {
            asm volatile("" : "+s"(u), "+v"(lane), "+v"(n), "+v"(g));   // (nothing of this pass is worked out before the other)
            u = advance(u, ka, aa);
            for (; u < u_end; u = advance(u + kWaves, ka, aa)) {
                fetch(a, ka);
                attend(a, aa);
            }
        } else if ((u = advance(u, ka, aa)) < u_end) {
            fetch(a, ka);
            for (;;) {
                int next = advance(u + kWaves, kc, ac);
                if (next < u_end) fetch(c, kc);
                attend(a, aa);
                u = next;
                if (u >= u_end) break;
                next = advance(u + kWaves, ka, aa);
                if (next < u_end) fetch(a, ka);
                attend(c, ac);
                u = next;
                if (u >= u_end) break;
            }
        }
        l = xgroup_sum(l);
        // ---- the wavefronts' states into one ----------------------------------------------------------------------
        if (g == 0) ml_s[wave][n] = float2{m, l};
        __syncthreads();
        float M = -INFINITY;
#pragma unroll
        for (int i = 0; i < kWaves; ++i) M = fmaxf(M, ml_s[i][n].x);
        const float base = M == -INFINITY ? 0.f : M;
        const float w = fast_exp2(m - base);
        float *mine = reinterpret_cast<float *>(vs);     // [head][channel]: its 8 KiB
#pragma unroll
        for (int ch = 0; ch < 8; ++ch)
            *reinterpret_cast<f32x4 *>(mine + n * kHeadDim + 16 * (ch ^ (n & 7)) + 4 * g) = o[ch] * w;
        __syncthreads();
        if (head >= G) return false;                     // (of eight wavefronts the first four have heads)
        float den = 0.f, Mh = -INFINITY;
#pragma unroll
        for (int i = 0; i < kWaves; ++i) Mh = fmaxf(Mh, ml_s[i][head].x);
        const float bh = Mh == -INFINITY ? 0.f : Mh;
        float y[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = 0.f;
#pragma unroll
        for (int i = 0; i < kWaves; ++i) {
            den += ml_s[i][head].y * fast_exp2(ml_s[i][head].x - bh);
            const float *from = reinterpret_cast<const float *>(Vs[i]) + head * kHeadDim + 16 * ((c8 >> 4) ^ (head & 7)) + (c8 & 15);
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] += from[e];
        }
        const int hq = h * G + head;
        if (n_split == 1) {
            bf16x8 r;
#pragma unroll
            for (int e = 0; e < 8; ++e) r[e] = (__bf16)(den == 0.f ? 0.f : y[e] / den);   // (0: no key is seen; a NaN among the scores stays one)
            *reinterpret_cast<uint4 *>(out.ptr + b * out.sb + qi * out.st + (int64_t)hq * out.sh + c8) = __builtin_bit_cast(uint4, r);
            if (c8 == 0) lse[(int64_t)bv * dm.Hq + hq] = den == 0.f ? -INFINITY : lse_of(bh + shift, den);
        } else {
            const int64_t at = ((int64_t)bv * dm.Hq + hq) * n_split + split;
            float4 *op = reinterpret_cast<float4 *>(o_part + at * kHeadDim + c8);
            op[0] = float4{y[0], y[1], y[2], y[3]};
            op[1] = float4{y[4], y[5], y[6], y[7]};
            if (c8 == 0) ml_part[at] = float2{Mh + shift, den};
        }
        float odd = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) odd = __builtin_fmaf(y[e], 0.f, odd);
        return odd != 0.f && den == den;
    };
    // The sums are divided at the end only, so values near the largest, which have a mean, may overflow in them.  Then the workgroup takes its units
    // again with all probabilities 2^-40 of what they were (2^30 keys at 2^8 weigh 1/4 together), and writes over what it wrote.  The question comes
    // behind the result's stores, which the workgroup waits for anyway.
    const bool again = __any(pass(std::true_type()));
    if (lane == 0) again_s[wave] = again;
    reads_done();                                        // (LDS is all that the barrier needs: it does not wait for the stores)
    asm volatile("s_barrier" ::: "memory");
    bool any = false;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) any |= again_s[i];
    if (__builtin_expect(any, 0)) {
        shift = 40.f;
        pass(std::false_type());
    }
}

// ---- host side -------------------------------------------------------------------------------------------------------------
static inline size_t align256(size_t x) { return (x + 255) / 256 * 256; }

// Whether each row is one workgroup of eight wavefronts, and the call one launch.  Where rows fill the chip once (64 to 512 of them)
// and a wavefront has at most five units, that beats a split over workgroups of four with a second launch to join them (4 bits, 1024
// tokens: 128 rows 11.6 / 13.3 us, 512 rows 24.5 / 27; bf16: 64 rows of 450 tokens 8.6 / 10, 256 rows of 1000 tokens 24 / 27).  With more
// rows three workgroups of four per compute unit hide more than the one of eight that fits (1024 rows 44 / 36).  With fewer the units
// that a wavefront takes one after the other are what is waited for (2 rows of 1024 tokens 10.4 / 8.7), but for up to two of them at
// 4 bits (7.0 / 8.1).
static bool stream_alone(const Dims &dm, int64_t units, bool quant) {
    const int64_t rows = (int64_t)dm.batch * dm.n_q * dm.Hkv;
    return units <= 40 && rows <= 512 && (rows >= 64 || (quant && units <= 16));
}
// The rest is split over workgroups of four wavefronts, as many as the chip holds (three per compute unit; two with a bf16 cache, whose
// rows take more registers), and a number of units to each that its wavefronts share evenly.  With more workgroups the last of them wait
// for the first ones' places (64 sequences, window 8192, 4 bits: 1024 / 768 / 512 workgroups 35 / 30 / 33 us), uneven ones do as if they
// had more (16 drafted tokens x 32 blocks, 6 / 8 units each: 11.8 / 10.1 us).
constexpr int kMaxSplits = 64;                           // what decode_merge_kernel joins
static int stream_units(const Dims &dm, int64_t units, bool quant) {
    if (stream_alone(dm, units, quant)) return (int)max((int64_t)1, units);
    const int64_t rows = max((int64_t)1, (int64_t)dm.batch * dm.n_q * dm.Hkv), chip = quant ? 768 : 512;
    const int64_t want = min((chip + rows - 1) / rows, (int64_t)kMaxSplits);
    return (int)max((int64_t)4, (units + 4 * want - 1) / (4 * want) * 4);   // (no units: a cache of no rows)
}
static int stream_splits(const Dims &dm, int64_t units, bool quant) {
    const int each = stream_units(dm, units, quant);
    return (int)max((int64_t)1, (units + each - 1) / each);
}
// The most units a window may touch: the sinks', and one more than fill the window.
static int64_t window_units(const Dims &dm, WindowArgs w) {
    const int64_t whole = ((int64_t)dm.max_seqlen + kUnit - 1) / kUnit;
    return min(whole, ((int64_t)w.n_sink + kUnit - 1) / kUnit + ((int64_t)w.window + kUnit - 1) / kUnit + 1);
}

template <bool kQuant, bool kList>
static int launch_stream(const char *name, const Dims &dm, WindowArgs win, int64_t units, int splits, int per, Tensor q, const RowSource &src,
                         const int32_t *seqlens, const int32_t *block_idx, const uint64_t *tree_mask, Tensor out, float *lse, void *ws,
                         hipStream_t stream) {
    float *o_part = reinterpret_cast<float *>(ws);
    float2 *ml_part = reinterpret_cast<float2 *>(reinterpret_cast<char *>(ws) +
                                                 align256((size_t)dm.batch * dm.n_q * dm.Hq * splits * kHeadDim * sizeof(float)));
    timing_begin(name, stream);
    const bool alone = stream_alone(dm, units, kQuant);
    hipLaunchKernelGGL((alone ? stream_attn_kernel<kQuant, kList, 8> : stream_attn_kernel<kQuant, kList, 4>), dim3(splits, dm.Hkv, dm.batch * dm.n_q),
                       dim3(alone ? 512 : 256), 0, stream, dm, win, q, src, seqlens, block_idx, tree_mask, per, out, lse, o_part, ml_part);
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
    const int per = min(stream_units(dm, 2 * dm.topk, true) / 2, dm.topk);
    return launch_stream<true, true>("sparse_attn_quant_kernel", dm, WindowArgs{0, 0}, 2 * dm.topk, (dm.topk + per - 1) / per, per, q,
                                     RowSource{Tensor{}, Tensor{}, kq, vq}, seqlens, block_idx, tree_mask, out, lse, ws, stream);
}

// (An upper bound that grows with the batch and with max_seqlen: a buffer for a call is large enough for every smaller one.)
size_t window_decode_ws_bytes(const Dims &dm, WindowArgs w) {
    const int64_t rows = (int64_t)dm.batch * dm.Hkv, most = min((int64_t)kMaxSplits, (window_units(dm, w) + 3) / 4);
    const size_t parts = (size_t)(min(rows * most, rows + 768) * dm.G);
    return align256(parts * kHeadDim * sizeof(float)) + align256(parts * sizeof(float2));
}

int launch_window_decode(const Dims &dm, WindowArgs w, Tensor q, Tensor k, Tensor v, const int32_t *seqlens, Tensor out, float *lse,
                         void *ws, hipStream_t stream) {
    if (dm.batch <= 0) return 0;
    return launch_stream<false, false>("window_decode_kernel", dm, w, window_units(dm, w), stream_splits(dm, window_units(dm, w), false), 0, q,
                                       RowSource{k, v, QuantTensor{}, QuantTensor{}}, seqlens, nullptr, nullptr, out, lse, ws, stream);
}

int launch_window_decode_quant(const Dims &dm, WindowArgs w, Tensor q, QuantTensor kq, QuantTensor vq, const int32_t *seqlens,
                               Tensor out, float *lse, void *ws, hipStream_t stream) {
    if (dm.batch <= 0) return 0;
    return launch_stream<true, false>("window_decode_quant_kernel", dm, w, window_units(dm, w), stream_splits(dm, window_units(dm, w), true), 0, q,
                                      RowSource{Tensor{}, Tensor{}, kq, vq}, seqlens, nullptr, nullptr, out, lse, ws, stream);
}

}  // namespace infllmv2
