// The 4-bit cache: a row of 128 channels is 64 bytes of codes and 4 exponent bytes, one for each 32 channels.
// A code is a sign and the index of 0, 0.5, 1, 1.5, 2, 3, 4, 6 (two bits of exponent, one of mantissa), channel 2c in the low half
// of byte c; its value is that number times 2^(byte - 127).  Every value is a bf16 number, so reading back rounds nothing, and
// the hardware converts two codes and applies the exponent in one instruction.
// The exponent is that of the group's largest magnitude rounded to two significant bits, less 2: the largest magnitude lies in
// [3.5, 7) of its units, so no element is clipped by more than the half step it would be rounded by anyway (taking the
// exponent as it is clips magnitudes of 7 to 8 units to 6).  The byte is at least 2, which keeps all values normal numbers, and at most 252, which keeps
// them finite (magnitudes from 1.75 x 2^127 on are clipped to 1.5 x 2^127).  A group with an infinity or a NaN gets byte 255 and reads back as NaN.
#pragma once
#include "common.h"

namespace infllmv2 {

struct QuantTensor {                                     // strides in bytes
    uint8_t *codes, *scales;
    int64_t sb, sh, st;
    int64_t eb, eh, et;
};

typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));

// The exponent byte of a group whose largest |x| has these bits (bf16, no sign).
__device__ __forceinline__ uint32_t quant_exponent(uint32_t amax) {
    const uint32_t e = (amax + 0x20u) >> 7;              // a mantissa of 1.75 and more carries into the exponent
    return amax >= 0x7f80u ? 255u : min(max(e, 4u), 254u) - 2u;
}

// Two channels (a bf16 pair) -> one byte of codes; ties go to the even code, a group with byte 255 gets codes 0.
__device__ __forceinline__ uint32_t quant_pair(uint32_t pair, uint32_t exponent) {
    const uint32_t c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(0u, __builtin_bit_cast(bf16x2_t, pair), __uint_as_float(exponent << 23), 0);
    return exponent == 255u ? 0u : c & 0xffu;
}

// Byte kSel of a word of codes -> a bf16 pair.
template <int kSel>
__device__ __forceinline__ uint32_t dequant_pair(uint32_t word, uint32_t exponent) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, __uint_as_float(exponent << 23), kSel));
}
// Eight channels.
__device__ __forceinline__ uint4 dequant8(uint32_t word, uint32_t exponent) {
    return uint4{dequant_pair<0>(word, exponent), dequant_pair<1>(word, exponent), dequant_pair<2>(word, exponent), dequant_pair<3>(word, exponent)};
}

// Launchers (quant_kv.hip, window_decode.hip); each returns a hipError_t as int.
int launch_quantize_kv(const Dims &dm, Tensor k, Tensor v, const int32_t *seqlens, int32_t n_new_tokens, QuantTensor kq,
                       QuantTensor vq, hipStream_t stream);
int launch_dequantize_kv(const Dims &dm, QuantTensor kq, QuantTensor vq, const int32_t *seqlens, int32_t n_new_tokens, Tensor k,
                         Tensor v, hipStream_t stream);
int launch_append_kv_quant(const Dims &dm, Tensor k_new, Tensor v_new, QuantTensor kq, QuantTensor vq, const Tensor *ck,
                           const int32_t *seqlens, hipStream_t stream);   // dm.n_q rows per sequence
int launch_attn_decode_quant(const Dims &dm, Tensor q, QuantTensor kq, QuantTensor vq, const int32_t *seqlens,
                             const int32_t *block_idx, const uint64_t *tree_mask, Tensor out, float *lse, void *ws,
                             hipStream_t stream);

// Attention over a window: key t is visible to the query at position i when t <= i and (t < n_sink or i - t < window).
struct WindowArgs {
    int32_t n_sink, window;                              // both at most max_seqlen
};
size_t window_decode_ws_bytes(const Dims &dm, WindowArgs w);
int launch_window_decode(const Dims &dm, WindowArgs w, Tensor q, Tensor k, Tensor v, const int32_t *seqlens, Tensor out, float *lse,
                         void *ws, hipStream_t stream);
int launch_window_decode_quant(const Dims &dm, WindowArgs w, Tensor q, QuantTensor kq, QuantTensor vq, const int32_t *seqlens,
                               Tensor out, float *lse, void *ws, hipStream_t stream);
// The prefill and backward kernels address rows with 32-bit offsets from a tile's first: what the strides of a call may be.
constexpr int64_t kMaxTokenStride = 1ll << 23, kMaxHeadSpan = 1ll << 29;   // elements; of a token, and of the heads of a group
constexpr int64_t kMaxQuantStride = 1ll << 26;               // bytes; of a row of a cache in 4 bits that the attention reads
size_t window_prefill_ws_bytes(const Dims &dm, WindowArgs w);
int launch_window_prefill(const Dims &dm, WindowArgs w, Tensor q, Tensor k, Tensor v, const int32_t *seqlens, Tensor out, float *lse,
                          void *ws, hipStream_t stream);
size_t window_bwd_ws_bytes(const Dims &dm, WindowArgs w);        // enough for all calls with fewer sequences or tokens, whatever their window
size_t window_bwd_scratch_bytes(const Dims &dm, WindowArgs w);   // what a call uses
int launch_window_bwd(const Dims &dm, WindowArgs w, Tensor q, Tensor k, Tensor v, Tensor out, Tensor dout, const float *lse,
                      const int32_t *seqlens, Tensor dq, Tensor dk, Tensor dv, void *ws, hipStream_t stream);

}  // namespace infllmv2
