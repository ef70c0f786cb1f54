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

// Operand reads of 32x32x16 products from a tile of 256-byte rows (swizzled, see row_swizzle).  Lane = 32 hf + c.
struct TileReader {
    uint32_t row_at, col_at;
    __device__ __forceinline__ explicit TileReader(int lane) {
        const uint32_t ln = lane, hf = ln >> 5;
        row_at = (ln & 31) * 256u + ((hf ^ (uint32_t)row_swizzle((int)(ln & 15))) << 4);
        const uint32_t t_r = 4u * hf + ((ln & 15) >> 2), t_c = 2u * ((ln >> 4) & 1) + ((ln & 3) >> 1);
        col_at = t_r * 256u + ((t_c ^ (uint32_t)row_swizzle((int)t_r)) << 4) + 8u * (ln & 1);
    }
    // row c of the 32 from `tile` on, channels 16 ks + 8 hf .. +7
    __device__ __forceinline__ bf16x8 rows(const char *tile, int ks) const {
        return __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4_t *>(tile + (row_at ^ (uint32_t)(ks << 5))));
    }
    // channel 32 ct + c of rows 16 s + 4 hf .. +3 and 16 s + 8 + 4 hf .. +3: the rows a lane holds of a product's result
    __device__ __forceinline__ bf16x8 columns(const char *tile, int s, int ct) const {
        const s16x4 x0 = lds_read_tr16(tile + ((col_at ^ (uint32_t)(ct << 6)) + 16 * s * 256u));
        const s16x4 x1 = lds_read_tr16(tile + ((col_at ^ (uint32_t)((ct << 6) | (2 << 4))) + (16 * s + 8) * 256u));
        return __builtin_bit_cast(bf16x8, __builtin_shufflevector(x0, x1, 0, 1, 2, 3, 4, 5, 6, 7));
    }
};

// Entries 8 s .. 8 s + 7 of a product's result as the second operand of the next product: rows 16 s + 4 hf .. and 16 s + 8 + 4 hf ..
__device__ __forceinline__ bf16x8 pack8(const f32x16 &x, int s) {
    bf16x8 r;
#pragma unroll
    for (int j = 0; j < 8; ++j) r[j] = (__bf16)x[8 * s + j];
    return r;
}

// Tiles of kKeys keys that any of the queries t0 .. t1 - 1 sees: `sinks` tiles from the first on, then those from `first` to `last`.
constexpr int kWinKeys = 64;
struct KeyTiles {
    int sinks, first, count;
    __device__ __forceinline__ KeyTiles(WindowArgs w, int t0, int t1) {
        const int lo = max(0, t0 - w.window + 1);
        sinks = (min(w.n_sink, lo) + kWinKeys - 1) / kWinKeys;
        first = max(lo / kWinKeys, sinks);
        count = sinks + (t1 - 1) / kWinKeys - first + 1;
    }
    __device__ __forceinline__ int key0(int i) const { return kWinKeys * (i < sinks ? i : first + i - sinks); }
};

// Workgroups in runs of neighbours per XCD (the hardware deals them to the eight XCDs in turn): neighbours read the same keys, which then
// lie in one L2.
__device__ __forceinline__ int xcd_run(int id, int total) {
    const int xcd = id & 7, slot = id >> 3, each = total >> 3, rest = total & 7;
    return xcd * each + min(xcd, rest) + slot;
}

}  // namespace infllmv2
