// Rotary positions of queries and keys, and the append of new tokens to the pages with the rotation on the way.
//
// Eight lanes take a row of a head, eight pairs of channels each (32 bytes), or 16 channels that do not rotate; a wavefront takes one token and eight heads at
// a time.  A token's cosines and sines are worked out once to a wavefront, a pair to a lane (eight to each lane that uses them: the vector unit busy 87 % of the time).
#include "paged.h"

namespace infllmv2 {

struct RotateArgs {
    Tensor q, k, v, q_out, k_out;
    Pages pg;                                            // kPaged: where keys and values go
    NewTokens nt;
    const int32_t *positions;
    Rotation rot;
    int rows, heads, q_heads, per;                       // rows of a sequence; heads of a token (queries', keys', values'); steps of eight of them a wavefront takes
    int chunks;                                          // wavefronts to a token
};

// cos and sin of x / 2^32 turns.  The angle is brought to an eighth of a turn on either side of a multiple of a quarter as a whole number, exactly;
// from there Taylor's polynomials, whose next terms (x^11 / 11!, x^12 / 12!) are below 2e-9 and 2e-10 there.
__device__ __forceinline__ void turn(uint32_t x, float &c, float &s) {
    const uint32_t quarter = (x + 0x20000000u) >> 30;
    const float r = (float)(int32_t)(x - (quarter << 30)) * 1.4629180792671596e-9f;            // 2 pi / 2^32
    const float z = r * r;
    float sn = __builtin_fmaf(z, 2.7557319e-6f, -1.9841270e-4f);
    sn = __builtin_fmaf(z, sn, 8.3333333e-3f);
    sn = __builtin_fmaf(z, sn, -1.6666667e-1f);
    sn = __builtin_fmaf(z * r, sn, r);
    float cs = __builtin_fmaf(z, -2.7557319e-7f, 2.4801587e-5f);
    cs = __builtin_fmaf(z, cs, -1.3888889e-3f);
    cs = __builtin_fmaf(z, cs, 4.1666667e-2f);
    cs = __builtin_fmaf(z, cs, -0.5f);
    cs = __builtin_fmaf(z, cs, 1.f);
    const float a = quarter & 1u ? sn : cs, b = quarter & 1u ? cs : sn;
    c = (quarter + 1u) & 2u ? -a : a;
    s = quarter & 2u ? -b : b;
}

// Bound by traffic where rows are many (32768 tokens of 34 heads: 95 us, 6.0 TB/s), by the launch and round trips where they are few (777 tokens of 5: 4.1 us).
template <bool kPaged, bool kStream>
__global__ __launch_bounds__(256) void rotate_kernel(Dims dm, RotateArgs a, const int32_t *__restrict__ seqlens) {
    const int lane = threadIdx.x & 63, id = __builtin_amdgcn_readfirstlane(((blockIdx.z << kLgGroups) + blockIdx.x) * 4 + (threadIdx.x >> 6)), b = blockIdx.y;
    const int t = id / a.chunks, chunk = id - t * a.chunks;
    if (t >= a.rows) return;
    int n, before = 0;
    bool keep = true;                                    // kPaged: keys and values have a page
    int64_t k_at = 0, v_at = 0;
    if constexpr (kPaged) {
        const Chunk ch(a.nt, seqlens, b, dm.max_seqlen);
        n = ch.L == 0 || uniform_load(seqlens + b) > dm.max_seqlen ? 0 : ch.n;
        if (t >= n) return;
        before = ch.before;
        const int row = before + t, page = uniform_load(a.pg.table + (int64_t)b * a.pg.ld + (row >> a.pg.lg));
        keep = (uint32_t)page < (uint32_t)a.pg.count;
        k_at = page_bytes(a.pg.k, a.pg.lg, page, row);
        v_at = page_bytes(a.pg.v, a.pg.lg, page, row);
    } else {
        n = clamp_len(uniform_load(seqlens + b), dm.max_seqlen);
        if (t >= n && !dm.fill) return;
    }
    const int r = lane & 7, rot = a.rot.dim;
    const bool turns = 16 * r < rot;
    // bytes of this lane's two pieces of 16 from the row's start
    const int at0 = !turns || a.rot.interleaved ? 32 * r : 16 * r, at1 = !turns || a.rot.interleaved ? 32 * r + 16 : 16 * r + rot;
    // a lane a pair; then eight pairs to a lane, through LDS of the wavefront's own
    __shared__ __align__(16) float2 turned[4][64];
    float2 *const mine = turned[threadIdx.x >> 6];
    float c[8], s[8];
    if (rot > 0) {
        if (lane < rot / 2) {
            const uint32_t p = (uint32_t)(a.positions ? uniform_load(a.positions + (int64_t)b * a.rows + t) : before + t);
            const uint64_t step = a.rot.steps[lane];
            const uint32_t lo = (uint32_t)step, hi = (uint32_t)(step >> 32);
            float x, y;
            turn(p * hi + __umulhi(p, lo) - ((int32_t)p < 0 ? lo : 0u), x, y);             // the high word of p step, p signed
            mine[lane] = float2{x * a.rot.amplitude, y * (a.rot.amplitude * a.rot.sign)};
        }
        __builtin_amdgcn_wave_barrier();                 // same wavefront: LDS keeps the order
        if (turns) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float4 x = *reinterpret_cast<const float4 *>(mine + 8 * r + 2 * i);
                c[2 * i] = x.x;
                s[2 * i] = x.y;
                c[2 * i + 1] = x.z;
                s[2 * i + 1] = x.w;
            }
        }
    }
    auto place = [&](int head, const char *&from, char *&to) __attribute__((always_inline)) {  // false: this lane has none
        if (head >= a.heads) return false;
        if (head < a.q_heads) {
            from = reinterpret_cast<const char *>(a.q.ptr + b * a.q.sb + (int64_t)t * a.q.st + (int64_t)head * a.q.sh);
            to = reinterpret_cast<char *>(a.q_out.ptr + b * a.q_out.sb + (int64_t)t * a.q_out.st + (int64_t)head * a.q_out.sh);
            return true;
        }
        head -= a.q_heads;
        if (head < dm.Hkv) {
            from = reinterpret_cast<const char *>(a.k.ptr + b * a.k.sb + (int64_t)t * a.k.st + (int64_t)head * a.k.sh);
            to = kPaged ? reinterpret_cast<char *>(a.pg.k.ptr + (int64_t)head * a.pg.k.sh) + k_at
                        : reinterpret_cast<char *>(a.k_out.ptr + b * a.k_out.sb + (int64_t)t * a.k_out.st + (int64_t)head * a.k_out.sh);
            return keep;
        }
        head -= dm.Hkv;
        from = reinterpret_cast<const char *>(a.v.ptr + b * a.v.sb + (int64_t)t * a.v.st + (int64_t)head * a.v.sh);
        to = reinterpret_cast<char *>(a.pg.v.ptr + (int64_t)head * a.pg.v.sh) + v_at;
        return keep;
    };
    const int first = 8 * chunk * a.per + (lane >> 3);
    for (int i = 0; i < a.per; ++i) {
        const int head = first + 8 * i;
        const char *from;
        char *to;
        if (!place(head, from, to)) continue;
        if (!kPaged && t >= n) {
            store16<kStream>(to + at0, u32x4_t{0u, 0u, 0u, 0u});
            store16<kStream>(to + at1, u32x4_t{0u, 0u, 0u, 0u});
            continue;
        }
        const uint4 u = *reinterpret_cast<const uint4 *>(from + at0), v = *reinterpret_cast<const uint4 *>(from + at1);
        uint32_t w[8] = {u.x, u.y, u.z, u.w, v.x, v.y, v.z, v.w};
        if (turns && (!kPaged || head < a.q_heads + dm.Hkv)) {
            auto low = [](uint32_t x) { return __uint_as_float(x << 16); };
            auto high = [](uint32_t x) { return __uint_as_float(x & 0xffff0000u); };
            auto pack = [](float x, float y) {
                bf16x2_t z;
                z[0] = (__bf16)x;
                z[1] = (__bf16)y;
                return __builtin_bit_cast(uint32_t, z);
            };
            if (a.rot.interleaved) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float x = low(w[j]), y = high(w[j]);
                    w[j] = pack(__builtin_fmaf(x, c[j], -(y * s[j])), __builtin_fmaf(y, c[j], x * s[j]));
                }
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float x0 = low(w[j]), x1 = high(w[j]), y0 = low(w[4 + j]), y1 = high(w[4 + j]);
                    w[j] = pack(__builtin_fmaf(x0, c[2 * j], -(y0 * s[2 * j])), __builtin_fmaf(x1, c[2 * j + 1], -(y1 * s[2 * j + 1])));
                    w[4 + j] = pack(__builtin_fmaf(y0, c[2 * j], x0 * s[2 * j]), __builtin_fmaf(y1, c[2 * j + 1], x1 * s[2 * j + 1]));
                }
            }
        }
        store16<kStream>(to + at0, u32x4_t{w[0], w[1], w[2], w[3]});
        store16<kStream>(to + at1, u32x4_t{w[4], w[5], w[6], w[7]});
    }
}

int64_t rotate_wavefronts(int64_t rows, int64_t heads) { return rows * ((heads + 7) / 8); }

template <bool kPaged>
static int launch_rotate(const char *name, const Dims &dm, RotateArgs a, const int32_t *seqlens, hipStream_t stream) {
    if (dm.batch <= 0 || a.rows <= 0 || a.heads <= 0) return 0;
    const int steps = (a.heads + 7) / 8;
    a.per = (int64_t)a.rows * dm.batch >= 4096 ? min(steps, 2) : 1;      // (32768 tokens, 34 heads: 1 / 2 / 3 / 5 of 5: 111 / 98 / 100 / 105 us)
    a.chunks = (steps + a.per - 1) / a.per;
    const bool past = (int64_t)a.rows * dm.batch * a.heads * (2 * kHeadDim) > kAllL2;
    const int64_t groups = ((int64_t)a.rows * a.chunks + 3) / 4;
    timing_begin(name, stream);
    hipLaunchKernelGGL((past ? rotate_kernel<kPaged, true> : rotate_kernel<kPaged, false>), dim3(groups_x(groups), dm.batch, groups_beyond(groups)), dim3(256), 0, stream, dm, a, seqlens);
    timing_end(stream);
    return (int)hipGetLastError();
}

int launch_rope(const Dims &dm, const Rotation &rot, const Tensor *q, const Tensor *k, const int32_t *positions, const int32_t *seqlens, const Tensor *q_out,
                const Tensor *k_out, hipStream_t stream) {
    RotateArgs a{};
    if (q) a.q = *q, a.q_out = *q_out;
    if (k) a.k = *k, a.k_out = *k_out;
    a.positions = positions;
    a.rot = rot;
    a.rows = dm.max_seqlen;
    a.q_heads = q ? dm.Hq : 0;
    a.heads = a.q_heads + (k ? dm.Hkv : 0);
    return launch_rotate<false>("rope_kernel", dm, a, seqlens, stream);
}

int launch_paged_append(const Dims &dm, const Rotation &rot, Tensor k_new, Tensor v_new, const Tensor *q, const Pages &pg, const int32_t *positions,
                        NewTokens nt, const int32_t *seqlens, const Tensor *q_out, hipStream_t stream) {
    RotateArgs a{};
    if (q) a.q = *q, a.q_out = *q_out;
    a.k = k_new;
    a.v = v_new;
    a.pg = pg;
    a.nt = nt;
    a.positions = positions;
    a.rot = rot;
    a.rows = nt.most;
    a.q_heads = q ? dm.Hq : 0;
    a.heads = a.q_heads + 2 * dm.Hkv;
    return launch_rotate<true>("paged_append_kernel", dm, a, seqlens, stream);
}

}  // namespace infllmv2
