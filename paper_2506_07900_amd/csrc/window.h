// What the prefill and backward kernels of the windowed attention share: rows of 128 channels copied from memory into LDS
// tiles, matrix operands read from them, and which keys a tile of queries sees.
#pragma once
#include "quant.h"
#include "token_union.h"

namespace infllmv2 {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
__device__ __forceinline__ f32x16 mfma32(bf16x8 a, bf16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x16 zero16() {
    f32x16 x;
#pragma unroll
    for (int v = 0; v < 16; ++v) x[v] = 0.f;
    return x;
}
// A value of this lane and of its partner in the other half of the wavefront, joined.
template <typename F>
__device__ __forceinline__ float half_reduce(float v, F f) {
    const u32x2_t a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return f(__uint_as_float(a[0]), __uint_as_float(a[1]));
}

// 32 rows of 128 channels in LDS, as operands of 32x32x16 products: four quarters of 32 channels, in each 32 rows of 64 bytes, whose four 16-byte
// pieces are XORed with the row's second bit pair.  A row operand takes one piece of 32 rows, a transposing load 32 bytes of each of 4
// consecutive rows; both touch every bank once, and what changes from one operand to the next is a constant (with whole rows of 256
// bytes it is an exclusive or, a register and an instruction each).
constexpr int kHalfTile = 32 * 256;
struct TileReader {
    uint32_t row_at[2], col_at[2];
    __device__ __forceinline__ explicit TileReader(int lane) {           // lane = 32 hf + c
        const uint32_t ln = lane, hf = ln >> 5, r = ln & 31, t_r = 4u * hf + ((ln & 15) >> 2), t_c = 2u * ((ln >> 4) & 1) + ((ln & 3) >> 1);
#pragma unroll
        for (uint32_t i = 0; i < 2; ++i) {
            row_at[i] = r * 64u + (((2u * i + hf) ^ ((r >> 2) & 3u)) << 4);
            col_at[i] = (8u * i + t_r) * 64u + ((t_c ^ (2u * i + (t_r >> 2))) << 4) + 8u * (ln & 1);
        }
    }
    // row c, channels 16 ks + 8 hf .. +7
    __device__ __forceinline__ bf16x8 rows(const char *tile, int ks) const {
        return __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4_t *>(tile + (row_at[ks & 1] + (ks >> 1) * 2048)));
    }
    // channel 32 ct + c of rows 16 s + 4 hf .. +3 and 16 s + 8 + 4 hf .. +3: the rows a lane holds of a product's result
    __device__ __forceinline__ bf16x8 columns(const char *tile, int s, int ct) const {
        const s16x4 x0 = lds_read_tr16(tile + (col_at[0] + ct * 2048 + s * 1024));
        const s16x4 x1 = lds_read_tr16(tile + (col_at[1] + ct * 2048 + s * 1024));
        return __builtin_bit_cast(bf16x8, __builtin_shufflevector(x0, x1, 0, 1, 2, 3, 4, 5, 6, 7));
    }
};
// Filling it: a copy is 1 KiB, 16 rows of a quarter; lane l brings row l / 4, and of the quarter's four pieces this one.
__device__ __forceinline__ int copy_piece(int lane) { return (lane & 3) ^ ((lane >> 4) & 3); }
constexpr uint32_t kNoRow = 0xffffffffu;                 // an offset that lies outside: reads 0
__device__ __forceinline__ void copy_rows(char *to, const char *base, uint32_t offset, uint32_t more) {
    const auto src = __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(base), 0, 0xfffffffeu, 0x00027000);
    __builtin_amdgcn_raw_ptr_buffer_load_lds(src, (__attribute__((address_space(3))) void *)to, 16, (int)offset, (int)more, 0, 0);
}

// Entries 8 s .. 8 s + 7 of a product's result as the second operand of the next product: rows 16 s + 4 hf .. and 16 s + 8 + 4 hf ..
__device__ __forceinline__ bf16x8 pack8(const f32x16 &x, int s) {
    bf16x8 r;
#pragma unroll
    for (int j = 0; j < 8; ++j) r[j] = (__bf16)x[8 * s + j];
    return r;
}

// A wavefront's result, channel 32 ct + 8 (e / 4) + 4 hf + e % 4 of row c in lane 32 hf + c, times the lane's factor, to rows of memory: through 8 KiB
// of LDS of its own, so that 16 lanes write a row's 256 bytes together (as the lanes hold it, an instruction would write 16 bytes of each of 32
// rows).  to(row): where row `row` goes, null: nowhere.
template <typename F>
__device__ __forceinline__ void store_rows(char *lds, const f32x16 (&o)[4], float factor, int lane, F to) {
    const uint32_t c = lane & 31, hf = lane >> 5;
#pragma unroll
    for (int ct = 0; ct < 4; ++ct)
#pragma unroll
        for (int e4 = 0; e4 < 4; ++e4) {
            bf16x4 y;
#pragma unroll
            for (int e = 0; e < 4; ++e) y[e] = (__bf16)(o[ct][4 * e4 + e] * factor);
            *reinterpret_cast<uint2 *>(lds + c * 256 + (((4 * ct + e4) ^ (c & 15)) << 4) + 8 * hf) = __builtin_bit_cast(uint2, y);
        }
    __builtin_amdgcn_wave_barrier();                     // same wavefront: LDS keeps the order
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const uint32_t row = 4 * j + (lane >> 4), piece = lane & 15;
        const uint4 y = *reinterpret_cast<const uint4 *>(lds + row * 256 + ((piece ^ (row & 15)) << 4));
        __bf16 *p = to((int)row);
        if (p) *reinterpret_cast<uint4 *>(p + 8 * piece) = y;
    }
}

// Tiles of kKeys keys that any of the queries t0 .. t1 - 1 sees: `sinks` tiles from the first on, then those from `first` to the last.
constexpr int kWinKeys = 64;
template <int kKeys>
struct KeyTiles {
    int sinks, first, count;
    __device__ __forceinline__ KeyTiles(WindowArgs w, int t0, int t1) {
        const int lo = max(0, t0 - w.window + 1);
        sinks = (min(w.n_sink, lo) + kKeys - 1) / kKeys;
        first = max(lo / kKeys, sinks);
        count = sinks + (t1 - 1) / kKeys - first + 1;
    }
    __device__ __forceinline__ int key0(int i) const { return kKeys * (i < sinks ? i : first + i - sinks); }
};

// Whether the query at position i sees a key.  No branches: a wavefront tests sixteen keys at a time.
struct VisibleKeys {
    int i;
    uint32_t window, sinks;
    __device__ __forceinline__ VisibleKeys(WindowArgs w, int i) : i(i), window(w.window), sinks(min(w.n_sink, i + 1)) {}
    __device__ __forceinline__ bool operator()(int t) const { return ((uint32_t)(i - t) < window) | ((uint32_t)t < sinks); }
};

// Tiles of 64 keys or values, and their copies by a workgroup of four wavefronts, wavefront w the quarter w of the channels.
struct __align__(16) Tile64 {
    char x[2 * kHalfTile];
};
struct TileCopier {
    const char *head;                                    // the head's first row, at this wavefront's channels
    uint32_t step, at;                                   // bytes from row to row; of this lane's row and piece
    int L;
    __device__ __forceinline__ TileCopier(const Tensor &t, int b, int h, int L, int wave, int lane) : L(L) {
        head = reinterpret_cast<const char *>(t.ptr + b * t.sb + h * t.sh) + 64 * wave;
        step = 2 * (uint32_t)t.st;
        at = (lane >> 2) * step + 16 * copy_piece(lane);
    }
    // rows r0 .. r0 + 63; those past the sequence as zeros
    __device__ __forceinline__ void copy(Tile64 &dst, int r0, int wave, int lane) const {
        const char *base = head + (int64_t)r0 * step;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            copy_rows(dst.x + ((j >> 1) * kHalfTile + wave * 2048 + (j & 1) * 1024), base, r0 + 16 * j + (lane >> 2) < L ? at : kNoRow, 16 * j * step);
    }
};
// The same for few rows, a wavefront by itself: 32 keys and their values, all four quarters, into tiles of its own.
struct __align__(16) KVHalf {
    char k[kHalfTile], v[kHalfTile];
};
__device__ __forceinline__ void copy_half(KVHalf &dst, const Tensor &k, const Tensor &v, int64_t k_head, int64_t v_head, int k0, int L, int lane) {
    const char *kb = reinterpret_cast<const char *>(k.ptr + k_head + (int64_t)k0 * k.st), *vb = reinterpret_cast<const char *>(v.ptr + v_head + (int64_t)k0 * v.st);
    const uint32_t piece = 16 * copy_piece(lane), k_at = (lane >> 2) * (2 * (uint32_t)k.st) + piece, v_at = (lane >> 2) * (2 * (uint32_t)v.st) + piece;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const bool row = k0 + 16 * j + (lane >> 2) < L;
#pragma unroll
        for (int quarter = 0; quarter < 4; ++quarter) {
            copy_rows(dst.k + quarter * 2048 + j * 1024, kb + 64 * quarter, row ? k_at : kNoRow, 32 * j * (uint32_t)k.st);
            copy_rows(dst.v + quarter * 2048 + j * 1024, vb + 64 * quarter, row ? v_at : kNoRow, 32 * j * (uint32_t)v.st);
        }
    }
}
// All copies have landed, or all but the newest half's sixteen.
__device__ __forceinline__ void copies_landed(bool but_the_newest) {
    __builtin_amdgcn_sched_barrier(0);
    if (but_the_newest) __builtin_amdgcn_s_waitcnt(0x4f70);              // vmcnt 16
    else __builtin_amdgcn_s_waitcnt(0x0f70);                             // vmcnt 0
    __builtin_amdgcn_sched_barrier(0);
}
// This wavefront's LDS reads have ended: what they read may be overwritten.
__device__ __forceinline__ void reads_done() {
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_waitcnt(0xc07f);                  // lgkmcnt 0
    __builtin_amdgcn_sched_barrier(0);
}
// A wavefront's walk over units wave, wave + 4, ..: one ahead under way.
template <typename F>
__device__ __forceinline__ void walk_halves(KVHalf &slot0, KVHalf &slot1, const Tensor &k, const Tensor &v, int b, int h, const KeyTiles<32> &kt, int L,
                                            int wave, int lane, F unit) {
    const int64_t k_head = b * k.sb + h * k.sh, v_head = b * v.sb + h * v.sh;
    auto step = [&](const KVHalf &cur, KVHalf &next, int x) __attribute__((always_inline)) {
        reads_done();
        if (x + 4 < kt.count) copy_half(next, k, v, k_head, v_head, kt.key0(x + 4), L, lane);
        copies_landed(x + 4 < kt.count);
        unit(cur, kt.key0(x));
    };
    if (wave < kt.count) copy_half(slot0, k, v, k_head, v_head, kt.key0(wave), L, lane);
    for (int x = wave; x < kt.count; x += 8) {
        step(slot0, slot1, x);
        if (x + 4 < kt.count) step(slot1, slot0, x + 4);
    }
}

// The largest of three numbers, one instruction (fmaxf first makes the results of a product canonical, an instruction each).  NaN if any is.
__device__ __forceinline__ float max3(float a, float b, float c) { return __builtin_elementwise_maximum(__builtin_elementwise_maximum(a, b), c); }

// Workgroup -> item: runs of `run` neighbouring items, which read the same rows and should find them in one L2, go to the eight XCDs in turn (to which
// the hardware deals workgroups one by one), every eight runs from the next XCD on: rows are dealt last to first, those of a sequence's start see
// fewer keys, and with a multiple of eight runs to a head one XCD would get all of them (8 x 4096 tokens, 16 : 2 heads, whole window: forward
// 885 -> 546 us; 32 : 2, backward 4.58 -> 3.57 ms).  The grid is a whole number of runs per XCD; items past the last one do not exist.
__device__ __forceinline__ int xcd_item(int id, int run) {
    const int slot = id >> 3, r = slot / run;
    return (r * 8 + ((id + r) & 7)) * run + slot - r * run;
}
inline unsigned xcd_grid(int64_t items, int run) { return (unsigned)((items + 8 * run - 1) / (8 * run) * (8 * run)); }
// What an XCD holds at a time, or less so that each gets sixteen runs: with few it has more or less work than the others (ragged sequences, a
// sequence's start; dq of 2 x 4096 tokens, runs of 8 / 32 / 128 of its 1024 workgroups: 113 / 123 / 119 us).
inline int xcd_run_length(int64_t items) { return (int)max((int64_t)1, min((int64_t)64, items / 128)); }

// Whether rows see 512 keys or more, at which walks shared by wavefronts and joined are shorter by more than the joining costs.
inline bool long_walks(const Dims &dm, WindowArgs w) { return min((int64_t)dm.max_seqlen, (int64_t)w.window + w.n_sink) >= 512; }
// Whether workgroups of 128 rows are so few that a wavefront's walk over its keys is what is waited for: then a workgroup takes 32 rows and its
// wavefronts share the keys.
inline bool few_rows(const Dims &dm, WindowArgs w, int64_t items) { return items <= (long_walks(dm, w) ? 128 : 64); }

// Whether a workgroup of 128 rows is two halves that share its walk: walks are long, and there are fewer workgroups than compute units, or up to twice as many
// where windows are whole, so that walks are of all lengths and a compute unit's second place would stand empty behind a short one.
inline bool by_halves(const Dims &dm, WindowArgs w, int64_t items) {
    return long_walks(dm, w) && items <= ((int64_t)w.window + w.n_sink >= dm.max_seqlen ? 512 : 256);
}

}  // namespace infllmv2
