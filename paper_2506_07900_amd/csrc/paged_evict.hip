// Eviction by weight: which rows of a sequence and head stay, and these rows, in order, into other pages.
#include "paged.h"

namespace infllmv2 {

constexpr int kPickThreads = 1024, kPickWaves = kPickThreads / 64;

// Numbers in the order of the floats they are made of: -0 as 0, a NaN above all.
__device__ __forceinline__ uint32_t order_of(float x) {
    if (x != x) return 0xffffffffu;
    const uint32_t u = __float_as_uint(x + 0.f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// A workgroup to a sequence and head: the smallest weight that stays, by digits of 11, 11 and 10 bits from the highest on (11: exponents and two bits of mantissa spread a
// wavefront's counts over many words; all lanes' in one word cost an addition); then the rows above it and the first of those equal to it, in order.  A wavefront holds a run of
// rows, of up to 64 kPer in registers, of more it reads them again for each pass.
// 32749 rows to 4096: 18 us, of which the weights' way 2.5, the first digits 4, the list 3, a count, a sum and three barriers for each digit; 64 of 5001 to 9001 rows at a time 13.
constexpr int kDigits = 2048, kListed = 512;
template <int kPer>
__global__ __launch_bounds__(kPickThreads) void evict_pick_kernel(Dims dm, const float *__restrict__ weights, int pitch, const int32_t *__restrict__ seqlens,
                                                                  int budget, int first, int recent, int32_t *__restrict__ kept) {
    __shared__ uint32_t hist[kDigits];
    __shared__ uint32_t wave_sums[kPickWaves];
    __shared__ uint32_t found[2];                        // the digit, and how many are above it
    __shared__ int2 counts[kPickWaves];
    __shared__ uint32_t list[kPickWaves][kListed];
    __shared__ int over;
    const int h = blockIdx.x, b = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int L = clamp_len(uniform_load(seqlens + b), dm.max_seqlen);
    const int64_t bh = (int64_t)b * dm.Hkv + h;
    int32_t *out = kept + bh * budget;
    if (L <= budget) {
        for (int j = tid; j < budget; j += kPickThreads) out[j] = j < L ? j : -1;
        return;
    }
    for (int j = tid; j < first; j += kPickThreads) out[j] = j;
    for (int j = tid; j < recent; j += kPickThreads) out[budget - recent + j] = L - recent + j;
    const int lo = first, hi = L - recent, want = budget - first - recent;                     // want < hi - lo
    if (want == 0) return;
    const float *w = weights + bh * pitch;
    const int each = ((hi - lo + kPickWaves - 1) / kPickWaves + 63) / 64, from = min(hi, lo + wave * 64 * each), to = min(hi, from + 64 * each);
    const bool held = each <= kPer;
    uint32_t x[kPer];                                    // row from + 64 i + lane
    auto load = [&](int base) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int j = base + 64 * i + lane;
            x[i] = j < to ? __float_as_uint(w[j]) : 0u;
        }
#pragma unroll
        for (int i = 0; i < kPer; ++i) x[i] = base + 64 * i + lane < to ? order_of(__uint_as_float(x[i])) : 0u;    // (0: of no number)
    };
    // f(i, base) over a run's rows, kPer steps at a time
    auto rows = [&](auto f) __attribute__((always_inline)) {
        for (int base = from; base < to; base += 64 * kPer) {
            if (!held) load(base);
#pragma unroll
            for (int i = 0; i < kPer; ++i)
                if (base + 64 * i < to) f(x[i], base + 64 * i);
        }
    };
    if (held) load(from);
    uint32_t prefix = 0u, mask = 0u;
    int left = want, above = 0, equal = 0;               // how many of those with this prefix; this run's rows above the last one that stays, and equal to it
    int listed = 0;                                      // this run's numbers with the first digit, in LDS unless some run has more than fit
    bool fits = false;
    auto count = [&](uint32_t y, uint32_t digits, int shift) __attribute__((always_inline)) {
        const uint64_t who = __ballot((y & mask) == prefix);             // (numbers that are none count as the lowest, which are never reached)
        if (!who) return;
        const uint32_t digit = (y >> shift) & digits, some = (uint32_t)__builtin_amdgcn_readlane((int)digit, __builtin_ctzll(who));
        const uint64_t same = __ballot(digit == some);
        if ((who & ~same) == 0ull) {
            if (lane == 0) atomicAdd(&hist[some], (uint32_t)__popcll(who));
        } else if ((who >> lane) & 1ull) {
            atomicAdd(&hist[digit], 1u);
        }
    };
#pragma unroll 1
    for (int shift = 21; shift >= 0; shift = shift == 21 ? 10 : shift - 10) {
        const uint32_t digits = shift == 0 ? 1023u : kDigits - 1u;
        hist[tid] = hist[tid + kPickThreads] = 0u;
        if (shift == 21 && tid == 0) over = 0;           // (once: a later pass would clear it before all have read it)
        __syncthreads();
        if (shift == 21) {
            rows([&](uint32_t y, int) __attribute__((always_inline)) {
                const uint32_t digit = y >> 21, some = (uint32_t)__builtin_amdgcn_readfirstlane((int)digit);
                if (__ballot(digit != some) != 0ull) atomicAdd(&hist[digit], 1u);
                else if (lane == 0) atomicAdd(&hist[digit], 64u);
            });
        } else if (fits) {
            for (int j = lane; j - lane < listed; j += 64) count(j < listed ? list[wave][j] : 0u, digits, shift);
        } else {
            rows([&](uint32_t y, int) __attribute__((always_inline)) { count(y, digits, shift); });
        }
        __syncthreads();
        // thread i: digits 2047 - 2 i and the one below, so that sums run from the highest on
        const uint32_t c0 = hist[kDigits - 1 - 2 * tid], c1 = hist[kDigits - 2 - 2 * tid];
        const uint32_t upto = wave_scan(c0 + c1, lane);
        if (lane == 63) wave_sums[wave] = upto;
        __syncthreads();
        const uint32_t before = wave_scan(lane < kPickWaves ? wave_sums[lane] : 0u, lane);
        const uint32_t more = upto - c0 - c1 + (wave ? (uint32_t)__builtin_amdgcn_readlane((int)before, wave - 1) : 0u);
        if (more < (uint32_t)left && (uint32_t)left <= more + c0 + c1) {
            const bool second = (uint32_t)left > more + c0;
            found[0] = kDigits - 1 - 2 * tid - (second ? 1 : 0);
            found[1] = more + (second ? c0 : 0u);
        }
        __syncthreads();
        const uint32_t digit = found[0];
        prefix |= digit << shift;
        mask |= digits << shift;
        left -= (int)found[1];
        if (shift < 21) continue;
        rows([&](uint32_t y, int) __attribute__((always_inline)) {       // (the other digits are looked for among few)
            above += __popcll(__ballot((y >> 21) > digit));
            const uint64_t who = __ballot((y >> 21) == digit);
            if (!who) return;
            const int at = listed + __builtin_amdgcn_mbcnt_hi((uint32_t)(who >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)who, 0u));
            if (((who >> lane) & 1ull) && at < kListed) list[wave][at] = y;
            listed += __popcll(who);
        });
        if (listed > kListed) over = 1;
        __syncthreads();
        fits = over == 0;
    }
    // rows above `prefix`, and the first `left` of those equal to it
    if (fits) {
        for (int j = lane; j - lane < listed; j += 64) {
            const uint32_t y = j < listed ? list[wave][j] : 0u;
            above += __popcll(__ballot(y > prefix));
            equal += __popcll(__ballot(y == prefix));
        }
    } else {
        above = 0;
        rows([&](uint32_t y, int) __attribute__((always_inline)) {
            above += __popcll(__ballot(y > prefix));
            equal += __popcll(__ballot(y == prefix));
        });
    }
    if (lane == 0) counts[wave] = int2{above, equal};
    __syncthreads();
    const int2 mine = lane < kPickWaves ? counts[lane] : int2{0, 0};
    const int above_upto = (int)wave_scan((uint32_t)mine.x, lane), equal_upto = (int)wave_scan((uint32_t)mine.y, lane);
    int ties = wave ? __builtin_amdgcn_readlane(equal_upto, wave - 1) : 0;                     // equal rows before this run, and rows kept
    int at = first + (wave ? __builtin_amdgcn_readlane(above_upto, wave - 1) : 0) + min(ties, left);
    if (__builtin_amdgcn_readlane(equal_upto, 63) == left) {             // all that are equal stay
        rows([&](uint32_t y, int base) __attribute__((always_inline)) {
            const uint64_t who = __ballot(y >= prefix);
            if (y >= prefix) out[at + __builtin_amdgcn_mbcnt_hi((uint32_t)(who >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)who, 0u))] = base + lane;
            at += __popcll(who);
        });
        return;
    }
    const uint64_t below = (1ull << lane) - 1ull;
    rows([&](uint32_t y, int base) __attribute__((always_inline)) {
        const uint64_t eq = __ballot(y == prefix);
        const bool keep = y > prefix || (y == prefix && ties + __popcll(eq & below) < left);
        const uint64_t who = __ballot(keep);
        if (keep) out[at + __popcll(who & below)] = base + lane;
        at += __popcll(who);
        ties += __popcll(eq);
    });
}

// 16 lanes to a row, 64 rows to a workgroup; grid (rows / 64, Hkv, batch).  Bound by traffic (144000 rows, 295 MB: 57 us, 5.2 TB/s).
template <bool kStream>
__global__ __launch_bounds__(256) void evict_move_kernel(Dims dm, const float *__restrict__ weights, int pitch, Pages from, const int32_t *__restrict__ seqlens,
                                                         int budget, Pages to, const int32_t *__restrict__ kept, float *__restrict__ weights_out,
                                                         int32_t *__restrict__ seqlens_out) {
    const int h = blockIdx.y, b = blockIdx.z, piece = threadIdx.x & 15;
    const int64_t bh = (int64_t)b * dm.Hkv + h;
    if (blockIdx.x == 0 && h == 0 && threadIdx.x == 0) seqlens_out[b] = min(clamp_len(seqlens[b], dm.max_seqlen), budget);
    const char *kf = reinterpret_cast<const char *>(from.k.ptr + h * from.k.sh) + 16 * piece, *vf = reinterpret_cast<const char *>(from.v.ptr + h * from.v.sh) + 16 * piece;
    char *kt = reinterpret_cast<char *>(to.k.ptr + h * to.k.sh) + 16 * piece, *vt = reinterpret_cast<char *>(to.v.ptr + h * to.v.sh) + 16 * piece;
    u32x4_t x[4], y[4];
    int row[4], src[4], dst[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int j = 64 * blockIdx.x + 16 * i + (threadIdx.x >> 4);
        row[i] = j < budget ? kept[bh * budget + j] : -1;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int j = 64 * blockIdx.x + 16 * i + (threadIdx.x >> 4);
        src[i] = row[i] >= 0 ? from.table[(int64_t)b * from.ld + (row[i] >> from.lg)] : -1;
        dst[i] = row[i] >= 0 ? to.table[(int64_t)b * to.ld + (j >> to.lg)] : -1;               // (its table may end with the rows that there can be)
        if (weights_out && piece == 0 && j < budget) weights_out[bh * budget + j] = row[i] >= 0 ? weights[bh * pitch + row[i]] : 0.f;
    }
    bool moves[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        moves[i] = (uint32_t)src[i] < (uint32_t)from.count && (uint32_t)dst[i] < (uint32_t)to.count;
        x[i] = y[i] = u32x4_t{0u, 0u, 0u, 0u};
        if (moves[i]) {
            x[i] = *reinterpret_cast<const u32x4_t *>(kf + page_bytes(from.k, from.lg, src[i], row[i]));
            y[i] = *reinterpret_cast<const u32x4_t *>(vf + page_bytes(from.v, from.lg, src[i], row[i]));
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int j = 64 * blockIdx.x + 16 * i + (threadIdx.x >> 4);
        if (!moves[i]) continue;
        store16<kStream>(kt + page_bytes(to.k, to.lg, dst[i], j), x[i]);
        store16<kStream>(vt + page_bytes(to.v, to.lg, dst[i], j), y[i]);
    }
}

size_t paged_evict_ws_bytes(const Dims &) { return 0; }

int launch_paged_evict(const Dims &dm, const float *weights, int pitch, const Pages &from, const int32_t *seqlens, int budget, int first, int recent,
                       const Pages &to, int32_t *kept, float *weights_out, int32_t *seqlens_out, void *, hipStream_t stream) {
    if (dm.batch <= 0) return 0;
    timing_begin("evict_pick_kernel", stream);
    const int64_t rows = (dm.max_seqlen + kPickThreads - 1) / kPickThreads;
    hipLaunchKernelGGL((rows <= 8 ? evict_pick_kernel<8> : evict_pick_kernel<32>), dim3(dm.Hkv, dm.batch), dim3(kPickThreads), 0, stream, dm, weights, pitch, seqlens, budget, first, recent, kept);
    timing_end(stream);
    timing_begin("evict_move_kernel", stream);
    const bool past = (int64_t)budget * dm.Hkv * dm.batch * (4 * kHeadDim) > kAllL2;
    hipLaunchKernelGGL((past ? evict_move_kernel<true> : evict_move_kernel<false>), dim3((budget + 63) / 64, dm.Hkv, dm.batch), dim3(256), 0, stream, dm, weights, pitch, from, seqlens, budget, to, kept,
                       weights_out, seqlens_out);
    timing_end(stream);
    return (int)hipGetLastError();
}

}  // namespace infllmv2
