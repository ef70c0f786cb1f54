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
// up to 64 kPer rows in registers.
// 64 of 5001 to 9001 rows at a time: 9.6 us, of which the weights' way 2.5; counts, sums and three barriers for each digit, and the list of those that have the first.
constexpr int kDigits = 2048, kListed = 512, kMostPer = 16;
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
    uint32_t x[kPer];                                    // row from + 64 i + lane, 0 (of no number): none
#pragma unroll
    for (int i = 0; i < kPer; ++i) x[i] = from + 64 * i + lane < to ? __float_as_uint(w[from + 64 * i + lane]) : 0u;
#pragma unroll
    for (int i = 0; i < kPer; ++i) x[i] = from + 64 * i + lane < to ? order_of(__uint_as_float(x[i])) : 0u;
    // f(number, row - lane) over the run
    auto rows = [&](auto f) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < kPer; ++i)
            if (from + 64 * i < to) f(x[i], from + 64 * i);
    };
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
                if (__ballot(digit != some) != 0ull) atomicAdd(&hist[digit], 1u);             // (those of no number are digit 0, which is never reached)
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

// ---- more rows -----------------------------------------------------------------------------------------------------------------

// Parts of `rows` rows, a workgroup to a part, three launches: the first digits' counts of each part; from all parts' the first digit, and each part's numbers that have it into a list;
// from all lists the other digits, and each part's rows that stay.  Every workgroup of a sequence and head works the digits out for itself.  Bound by launches and, in each, round trips:
// 32749 rows of two heads 3.6 + 5.6 + 7.2 us (a workgroup to a head, its rows in registers: 18.2), 131072 25 (73).
constexpr int kPartRows = 4096, kMostParts = 64, kGathered = 16384;
struct EvictParts {
    int rows, most;                                      // parts that there can be
    uint32_t *hist, *list;                               // [batch, Hkv, most, kDigits]; [batch, Hkv, most rows]
    int2 *of;                                            // [batch, Hkv, most]: a part's numbers above the first digit, and those that have it
    int2 *state;                                         // [batch, Hkv]: the first digit, and how many of those that have it stay
};
struct EvictRange {
    int L, lo, hi, want, parts, from, to;                // rows to choose from, and of this part
    int64_t bh;
    __device__ __forceinline__ EvictRange(const Dims &dm, const int32_t *__restrict__ seqlens, int budget, int first, int recent, const EvictParts &ep) {
        const int b = blockIdx.z;
        bh = (int64_t)b * dm.Hkv + blockIdx.y;
        L = clamp_len(uniform_load(seqlens + b), dm.max_seqlen);
        lo = first;
        hi = L - recent;
        want = L > budget ? budget - first - recent : 0;                 // want < hi - lo
        parts = want > 0 ? (int)(((int64_t)hi - lo + ep.rows - 1) / ep.rows) : 0;
        from = (int)min((int64_t)hi, lo + (int64_t)blockIdx.x * ep.rows);
        to = (int)min((int64_t)hi, (int64_t)from + ep.rows);
    }
};
// Rows at + 64 i + lane of a wavefront's run, in the order of their numbers; 0 behind `to`.
__device__ __forceinline__ void load_orders(uint32_t (&x)[4], const float *__restrict__ w, int at, int to, int lane) {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = at + 64 * i + lane < to ? __float_as_uint(w[at + 64 * i + lane]) : 0u;
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = at + 64 * i + lane < to ? order_of(__uint_as_float(x[i])) : 0u;
}

__global__ __launch_bounds__(kPickThreads) void evict_count_kernel(Dims dm, const float *__restrict__ weights, int pitch, const int32_t *__restrict__ seqlens, int budget, int first,
                                                                   int recent, EvictParts ep) {
    __shared__ __align__(16) uint32_t hist[kDigits];
    const EvictRange r(dm, seqlens, budget, first, recent, ep);
    if ((int)blockIdx.x >= r.parts) return;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const float *w = weights + r.bh * pitch;
    uint32_t x[4];
    load_orders(x, w, r.from + 256 * wave, r.to, lane);
    hist[tid] = hist[tid + kPickThreads] = 0u;
    __syncthreads();
    for (int base = r.from;;) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t digit = x[i] >> 21, some = (uint32_t)__builtin_amdgcn_readfirstlane((int)digit);
            if (__ballot(digit != some) != 0ull) {
                if (x[i]) atomicAdd(&hist[digit], 1u);
            } else if (lane == 0 && x[i]) {
                atomicAdd(&hist[digit], 64u);
            }
        }
        base += kPartRows;
        if (base >= r.to) break;
        load_orders(x, w, base + 256 * wave, r.to, lane);
    }
    __syncthreads();
    reinterpret_cast<uint2 *>(ep.hist + (r.bh * ep.most + blockIdx.x) * kDigits)[tid] = reinterpret_cast<const uint2 *>(hist)[tid];
}

// The digit, from the highest on, at which `left` is reached by counts c0 of digit 2047 - 2 tid and c1 of the one below; -> it and how many are above it.
__device__ __forceinline__ uint2 find_digit(uint32_t c0, uint32_t c1, int left, uint32_t *wave_sums, uint32_t *found) {
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
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
    return uint2{found[0], found[1]};
}

__global__ __launch_bounds__(kPickThreads) void evict_list_kernel(Dims dm, const float *__restrict__ weights, int pitch, const int32_t *__restrict__ seqlens, int budget, int first,
                                                                  int recent, EvictParts ep) {
    __shared__ uint32_t wave_sums[kPickWaves], found[2];
    __shared__ int above_s, listed_s;
    const EvictRange r(dm, seqlens, budget, first, recent, ep);
    if ((int)blockIdx.x >= r.parts) return;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const float *w = weights + r.bh * pitch;
    uint32_t x[4];
    load_orders(x, w, r.from + 256 * wave, r.to, lane);
    if (tid == 0) above_s = listed_s = 0;
    uint32_t c0 = 0u, c1 = 0u;
    const uint2 *hist = reinterpret_cast<const uint2 *>(ep.hist + r.bh * ep.most * kDigits) + (kPickThreads - 1 - tid);
#pragma unroll 8
    for (int p = 0; p < r.parts; ++p) {
        const uint2 c = hist[(int64_t)p * (kDigits / 2)];
        c0 += c.y;
        c1 += c.x;
    }
    const uint2 digit = find_digit(c0, c1, r.want, wave_sums, found);
    uint32_t *list = ep.list + (r.bh * ep.most + blockIdx.x) * ep.rows;
    int above = 0;
    for (int base = r.from;;) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            above += __popcll(__ballot((x[i] >> 21) > digit.x));
            const uint64_t who = __ballot((x[i] >> 21) == digit.x && x[i] != 0u);
            if (!who) continue;
            int at = lane == 0 ? atomicAdd(&listed_s, (int)__popcll(who)) : 0;                  // (their order does not matter)
            at = __builtin_amdgcn_readfirstlane(at) + __builtin_amdgcn_mbcnt_hi((uint32_t)(who >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)who, 0u));
            if ((who >> lane) & 1ull) list[at] = x[i];
        }
        base += kPartRows;
        if (base >= r.to) break;
        load_orders(x, w, base + 256 * wave, r.to, lane);
    }
    if (lane == 0 && above) atomicAdd(&above_s, above);
    __syncthreads();
    if (tid == 0) {
        ep.of[r.bh * ep.most + blockIdx.x] = int2{above_s, listed_s};
        if (blockIdx.x == 0) ep.state[r.bh] = int2{(int)digit.x, r.want - (int)digit.y};
    }
}

__global__ __launch_bounds__(kPickThreads) void evict_choose_kernel(Dims dm, const float *__restrict__ weights, int pitch, const int32_t *__restrict__ seqlens, int budget, int first,
                                                                    int recent, EvictParts ep, int32_t *__restrict__ kept) {
    __shared__ uint32_t hist[kDigits], gathered[kGathered];
    __shared__ uint32_t wave_sums[kPickWaves], found[2];
    __shared__ int2 counts[kPickWaves];
    __shared__ int above_s, equal_s;
    const EvictRange r(dm, seqlens, budget, first, recent, ep);
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), part = blockIdx.x;
    int32_t *out = kept + r.bh * budget;
    if (part == 0) {
        if (r.L <= budget) {
            for (int j = tid; j < budget; j += kPickThreads) out[j] = j < r.L ? j : -1;
        } else {
            for (int j = tid; j < first; j += kPickThreads) out[j] = j;
            for (int j = tid; j < recent; j += kPickThreads) out[budget - recent + j] = r.L - recent + j;
        }
    }
    if (part >= r.parts) return;
    const float *w = weights + r.bh * pitch;
    // this wavefront's run of rows: kPartRows / kPickWaves, or as many times that as a part is longer
    const int each = ep.rows / kPickWaves, from = min(r.to, r.from + wave * each), to = min(r.to, from + each);
    const bool held = each <= 256;
    uint32_t x[4];
    load_orders(x, w, from, to, lane);
    const int2 of = lane < r.parts ? ep.of[r.bh * ep.most + lane] : int2{0, 0};
    const int2 state = ep.state[r.bh];
    const int above_upto = (int)wave_scan((uint32_t)of.x, lane), listed_upto = (int)wave_scan((uint32_t)of.y, lane);
    const int listed = __builtin_amdgcn_readlane(listed_upto, 63), earlier = __builtin_amdgcn_readlane(listed_upto - of.y, part);   // in all lists, in those of earlier parts
    const uint32_t *lists = ep.list + r.bh * ep.most * ep.rows;
    const bool fits = listed <= kGathered;
    if (tid == 0) above_s = equal_s = 0;
    if (fits) {                                          // the lists, one behind the other
        for (int p = wave; p < r.parts; p += kPickWaves) {
            const int n = __builtin_amdgcn_readlane(of.y, p), start = __builtin_amdgcn_readlane(listed_upto, p) - n;
            const uint32_t *l = lists + (int64_t)p * ep.rows;
#pragma unroll 4
            for (int j = lane; j < n; j += 64) gathered[start + j] = l[j];
        }
    }
    // f(number, whether it is of an earlier part) over all listed numbers, 0 for lanes without one
    auto all = [&](auto f) __attribute__((always_inline)) {
        if (fits) {
            for (int j = 64 * wave + lane; j - lane < listed; j += kPickThreads) f(j < listed ? gathered[j] : 0u, j < earlier);
        } else {
            for (int p = 0; p < r.parts; ++p) {
                const int n = __builtin_amdgcn_readlane(of.y, p);
                for (int j = 64 * wave + lane; j - lane < n; j += kPickThreads) f(j < n ? lists[(int64_t)p * ep.rows + j] : 0u, p < part);
            }
        }
    };
    uint32_t prefix = (uint32_t)state.x << 21, mask = 0xffe00000u;
    int left = state.y;
#pragma unroll 1
    for (int shift = 10; shift >= 0; shift -= 10) {
        const uint32_t digits = shift == 0 ? 1023u : kDigits - 1u;
        hist[tid] = hist[tid + kPickThreads] = 0u;
        __syncthreads();
        all([&](uint32_t y, bool) __attribute__((always_inline)) {
            const uint64_t who = __ballot(y != 0u && (y & mask) == prefix);
            if (!who) return;
            const uint32_t digit = (y >> shift) & digits, some = (uint32_t)__builtin_amdgcn_readlane((int)digit, __builtin_ctzll(who));
            if ((who & ~__ballot(digit == some)) == 0ull) {
                if (lane == 0) atomicAdd(&hist[some], (uint32_t)__popcll(who));
            } else if ((who >> lane) & 1ull) {
                atomicAdd(&hist[digit], 1u);
            }
        });
        __syncthreads();
        const uint2 digit = find_digit(hist[kDigits - 1 - 2 * tid], hist[kDigits - 2 - 2 * tid], left, wave_sums, found);
        prefix |= digit.x << shift;
        mask |= digits << shift;
        left -= (int)digit.y;
    }
    // ---- `prefix` is the smallest number that stays, `left` of those equal to it do -------------------------------------------
    int above = 0, equal = 0;
    all([&](uint32_t y, bool before) __attribute__((always_inline)) {
        above += __popcll(__ballot(before && y > prefix));
        equal += __popcll(__ballot(before && y == prefix));
    });
    if (lane == 0 && above) atomicAdd(&above_s, above);
    if (lane == 0 && equal) atomicAdd(&equal_s, equal);
    // f(number, row - lane) over this wavefront's rows
    auto rows = [&](auto f) __attribute__((always_inline)) {
        for (int base = from; base < to; base += 256) {
            if (!held) load_orders(x, w, base, to, lane);
#pragma unroll
            for (int i = 0; i < 4; ++i) f(x[i], base + 64 * i);
        }
    };
    above = equal = 0;
    rows([&](uint32_t y, int) __attribute__((always_inline)) {
        above += __popcll(__ballot(y > prefix));
        equal += __popcll(__ballot(y == prefix));
    });
    if (lane == 0) counts[wave] = int2{above, equal};
    __syncthreads();
    const int2 mine = lane < kPickWaves ? counts[lane] : int2{0, 0};
    const int a = (int)wave_scan((uint32_t)mine.x, lane), e = (int)wave_scan((uint32_t)mine.y, lane);
    int ties = equal_s + (wave ? __builtin_amdgcn_readlane(e, wave - 1) : 0);                  // equal rows before this run, and rows kept
    int at = first + __builtin_amdgcn_readlane(above_upto - of.x, part) + above_s + (wave ? __builtin_amdgcn_readlane(a, wave - 1) : 0) + min(ties, left);
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
    // (a kept row without a page goes as zeros: its place counts as a row of the sequence, and what lay there is another's)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[i] = y[i] = u32x4_t{0u, 0u, 0u, 0u};
        if ((uint32_t)src[i] < (uint32_t)from.count && (uint32_t)dst[i] < (uint32_t)to.count) {
            x[i] = *reinterpret_cast<const u32x4_t *>(kf + page_bytes(from.k, from.lg, src[i], row[i]));
            y[i] = *reinterpret_cast<const u32x4_t *>(vf + page_bytes(from.v, from.lg, src[i], row[i]));
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int j = 64 * blockIdx.x + 16 * i + (threadIdx.x >> 4);
        if ((uint32_t)dst[i] >= (uint32_t)to.count) continue;
        store16<kStream>(kt + page_bytes(to.k, to.lg, dst[i], j), x[i]);
        store16<kStream>(vt + page_bytes(to.v, to.lg, dst[i], j), y[i]);
    }
}

// (one sequence of 9000 / 16000 / 32749 rows, the move too, in one workgroup a head: 16.8 / 20.5 / 23.3 us, in parts 19.5 / 20.2 / 20.8; 64 of 16000 58 / 66)
constexpr int64_t kPickRows = (int64_t)kMostPer * kPickThreads;
static inline size_t align256(size_t x) { return (x + 255) / 256 * 256; }
// (a bound that grows with each size: of parts of kPartRows up to kMostParts of them, and of lists of all rows and a part more)
static EvictParts evict_parts(const Dims &dm, char *ws, size_t *bytes) {
    EvictParts ep;
    const int64_t times = ((int64_t)dm.max_seqlen + (int64_t)kPartRows * kMostParts - 1) / ((int64_t)kPartRows * kMostParts), bh = (int64_t)dm.batch * dm.Hkv;
    ep.rows = (int)(kPartRows * times);
    ep.most = (int)(((int64_t)dm.max_seqlen + ep.rows - 1) / ep.rows);
    const int64_t parts = min((int64_t)kMostParts, ((int64_t)dm.max_seqlen + kPartRows - 1) / kPartRows);
    const size_t hist = align256(bh * parts * kDigits * sizeof(uint32_t)), list = align256(bh * ((int64_t)dm.max_seqlen + ep.rows) * sizeof(uint32_t)), of = align256(bh * parts * sizeof(int2));
    ep.hist = reinterpret_cast<uint32_t *>(ws);
    ep.list = reinterpret_cast<uint32_t *>(ws + hist);
    ep.of = reinterpret_cast<int2 *>(ws + hist + list);
    ep.state = reinterpret_cast<int2 *>(ws + hist + list + of);
    *bytes = hist + list + of + align256(bh * sizeof(int2));
    return ep;
}
size_t paged_evict_ws_bytes(const Dims &dm) {
    if (dm.batch <= 0 || dm.max_seqlen <= kPickRows) return 0;
    size_t bytes;
    evict_parts(dm, nullptr, &bytes);
    return bytes;
}

int launch_paged_evict(const Dims &dm, const float *weights, int pitch, const Pages &from, const int32_t *seqlens, int budget, int first, int recent,
                       const Pages &to, int32_t *kept, float *weights_out, int32_t *seqlens_out, void *ws, hipStream_t stream) {
    if (dm.batch <= 0) return 0;
    if (dm.max_seqlen > kPickRows) {
        size_t bytes;
        const EvictParts ep = evict_parts(dm, static_cast<char *>(ws), &bytes);
        const dim3 grid(ep.most, dm.Hkv, dm.batch);
        timing_begin("evict_count_kernel", stream);
        hipLaunchKernelGGL(evict_count_kernel, grid, dim3(kPickThreads), 0, stream, dm, weights, pitch, seqlens, budget, first, recent, ep);
        timing_end(stream);
        timing_begin("evict_list_kernel", stream);
        hipLaunchKernelGGL(evict_list_kernel, grid, dim3(kPickThreads), 0, stream, dm, weights, pitch, seqlens, budget, first, recent, ep);
        timing_end(stream);
        timing_begin("evict_choose_kernel", stream);
        hipLaunchKernelGGL(evict_choose_kernel, grid, dim3(kPickThreads), 0, stream, dm, weights, pitch, seqlens, budget, first, recent, ep, kept);
        timing_end(stream);
    } else {
        timing_begin("evict_pick_kernel", stream);
        hipLaunchKernelGGL((dm.max_seqlen <= 8 * kPickThreads ? evict_pick_kernel<8> : evict_pick_kernel<kMostPer>), dim3(dm.Hkv, dm.batch), dim3(kPickThreads), 0, stream, dm, weights, pitch, seqlens,
                           budget, first, recent, kept);
        timing_end(stream);
    }
    timing_begin("evict_move_kernel", stream);
    const bool past = (int64_t)budget * dm.Hkv * dm.batch * (4 * kHeadDim) > kAllL2;
    hipLaunchKernelGGL((past ? evict_move_kernel<true> : evict_move_kernel<false>), dim3((budget + 63) / 64, dm.Hkv, dm.batch), dim3(256), 0, stream, dm, weights, pitch, from, seqlens, budget, to, kept,
                       weights_out, seqlens_out);
    timing_end(stream);
    return (int)hipGetLastError();
}

}  // namespace infllmv2
