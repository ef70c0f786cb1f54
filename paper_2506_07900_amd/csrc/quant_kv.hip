// The 4-bit cache as it is written and read back (format: quant.h): a prompt's rows, the rows of a decode or verification
// step with the semantic kernels they complete, and the way back to bf16.
#include "quant.h"

namespace infllmv2 {

constexpr int kQuantRows = 64;                           // cache rows per workgroup: 16 at a time, of K and V

// The largest of a value's bits over a quad of lanes.
__device__ __forceinline__ uint32_t quad_max(uint32_t x) {
    x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, kSwap1, 0xf, 0xf, false));
    return max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, kSwap2, 0xf, 0xf, false));
}
// The larger magnitude of a bf16 pair, as bits.
__device__ __forceinline__ uint32_t pair_max(uint32_t pair) { return max(pair & 0x7fffu, (pair >> 16) & 0x7fffu); }

// Rows [max(0, l - n_new), l) of every sequence, l = its length; with dm.fill also rows [l, max_seqlen), as zeros.
// A thread takes 8 channels of a row, a quad a group of 32.  Pure traffic: 256 bytes in and 68 out per row of K and of V.  128K tokens x 2 heads 27 to
// 33 us, 5.1 to 6.3 TB/s (some of it from the last-level cache; a large copy: 5.25).
__global__ __launch_bounds__(256) void quantize_kv_kernel(Dims dm, Tensor k, Tensor v, const int32_t *__restrict__ seqlens,
                                                          int32_t n_new, QuantTensor kq, QuantTensor vq) {
    const int h = blockIdx.y, b = blockIdx.z;
    const int L = clamp_len(uniform_load(seqlens + b), dm.max_seqlen);
    const int first = (n_new > 0 ? max(0, L - n_new) : 0) + (int)blockIdx.x * kQuantRows;
    const int end = dm.fill ? dm.max_seqlen : L;
    if (first >= end) return;
    const int c16 = threadIdx.x & 15, r0 = threadIdx.x >> 4;
    const __bf16 *src[2] = {k.ptr + b * k.sb + h * k.sh + 8 * c16, v.ptr + b * v.sb + h * v.sh + 8 * c16};
    uint8_t *codes[2] = {kq.codes + b * kq.sb + h * kq.sh + 4 * c16, vq.codes + b * vq.sb + h * vq.sh + 4 * c16};
    uint8_t *scales[2] = {kq.scales + b * kq.eb + h * kq.eh, vq.scales + b * vq.eb + h * vq.eh};
    const int64_t st[2] = {k.st, v.st}, ct[2] = {kq.st, vq.st}, et[2] = {kq.et, vq.et};
    uint4 x[2][4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const int t = first + r0 + 16 * i;
            x[s][i] = uint4{0u, 0u, 0u, 0u};
            if (t < L) x[s][i] = *reinterpret_cast<const uint4 *>(src[s] + (int64_t)t * st[s]);
        }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const int t = first + r0 + 16 * i;
            const uint4 y = x[s][i];
            const uint32_t amax = quad_max(max(max(pair_max(y.x), pair_max(y.y)), max(pair_max(y.z), pair_max(y.w))));
            const uint32_t e = t < L ? quant_exponent(amax) : 0u;
            const uint32_t w = quant_pair(y.x, e) | quant_pair(y.y, e) << 8 | quant_pair(y.z, e) << 16 | quant_pair(y.w, e) << 24;
            // the row's four exponents in its first lane: lanes 4, 8 and 12 further on
            const uint32_t e4 = e | (uint32_t)__builtin_amdgcn_update_dpp(0, (int)e, 0x104, 0xf, 0xf, true) << 8 |
                                (uint32_t)__builtin_amdgcn_update_dpp(0, (int)e, 0x108, 0xf, 0xf, true) << 16 |
                                (uint32_t)__builtin_amdgcn_update_dpp(0, (int)e, 0x10c, 0xf, 0xf, true) << 24;
            if (t < end) {
                *reinterpret_cast<uint32_t *>(codes[s] + (int64_t)t * ct[s]) = w;
                if (c16 == 0) *reinterpret_cast<uint32_t *>(scales[s] + (int64_t)t * et[s]) = e4;
            }
        }
}

// The way back, the same split; 26 us for 128K tokens x 2 heads.
__global__ __launch_bounds__(256) void dequantize_kv_kernel(Dims dm, QuantTensor kq, QuantTensor vq, const int32_t *__restrict__ seqlens,
                                                            int32_t n_new, Tensor k, Tensor v) {
    const int h = blockIdx.y, b = blockIdx.z;
    const int L = clamp_len(uniform_load(seqlens + b), dm.max_seqlen);
    const int first = (n_new > 0 ? max(0, L - n_new) : 0) + (int)blockIdx.x * kQuantRows;
    const int end = dm.fill ? dm.max_seqlen : L;
    if (first >= end) return;
    const int c16 = threadIdx.x & 15, r0 = threadIdx.x >> 4;
    __bf16 *dst[2] = {k.ptr + b * k.sb + h * k.sh + 8 * c16, v.ptr + b * v.sb + h * v.sh + 8 * c16};
    const uint8_t *codes[2] = {kq.codes + b * kq.sb + h * kq.sh + 4 * c16, vq.codes + b * vq.sb + h * vq.sh + 4 * c16};
    const uint8_t *scales[2] = {kq.scales + b * kq.eb + h * kq.eh, vq.scales + b * vq.eb + h * vq.eh};
    const int64_t st[2] = {k.st, v.st}, ct[2] = {kq.st, vq.st}, et[2] = {kq.et, vq.et};
    uint32_t w[2][4], e4[2][4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const int t = first + r0 + 16 * i;
            w[s][i] = e4[s][i] = 0u;
            if (t < L) {
                w[s][i] = *reinterpret_cast<const uint32_t *>(codes[s] + (int64_t)t * ct[s]);
                e4[s][i] = *reinterpret_cast<const uint32_t *>(scales[s] + (int64_t)t * et[s]);
            }
        }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const int t = first + r0 + 16 * i;
            const uint4 y = dequant8(w[s][i], (e4[s][i] >> (8 * (c16 >> 2))) & 255u);
            if (t < end) *reinterpret_cast<uint4 *>(dst[s] + (int64_t)t * st[s]) = t < L ? y : uint4{0u, 0u, 0u, 0u};
        }
}

// New rows into the cache and the semantic kernels they complete, in one launch: a wavefront per task, lane = two channels (16
// lanes are a group of the format, so its largest magnitude is a row reduction).  Tasks 0 .. 2 n_q - 1 of a (sequence,
// key-value head) quantise a row of K (even) or V; the others build a kernel each from its 32 rows' values as the cache holds them: older
// rows from the cache, new ones from k_new through the same quantisation.  So the kernel's bits are those that
// compress_keys gives for the cache as read back.  A sequence shorter than n_q is skipped as a whole.  One launch of latency: 4.3 us for a token, 5.7 for
// 8 sequences x 16 tokens.
__device__ __forceinline__ uint32_t group_exponent(uint32_t pair) {
    return quant_exponent(row_reduce_u32(pair_max(pair), [](uint32_t a, uint32_t b) { return max(a, b); }));
}
template <bool kWithCk>
__global__ __launch_bounds__(256) void append_kv_quant_kernel(Dims dm, Tensor k_new, Tensor v_new, QuantTensor kq, QuantTensor vq,
                                                              Tensor ck, const int32_t *__restrict__ seqlens) {
    const int h = blockIdx.y, b = blockIdx.z, lane = threadIdx.x & 63;
    const int task = (int)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int L = uniform_load(seqlens + b);
    if (L < dm.n_q || L > dm.max_seqlen) return;
    const int first_new = L - dm.n_q;
    if (task < 2 * dm.n_q) {
        const int qi = task >> 1;
        const bool is_v = task & 1;
        const Tensor &src = is_v ? v_new : k_new;
        const QuantTensor &dst = is_v ? vq : kq;
        const uint32_t pair = reinterpret_cast<const uint32_t *>(src.ptr + b * src.sb + h * src.sh + qi * src.st)[lane];
        const uint32_t e = group_exponent(pair);
        const int64_t t = first_new + qi;
        dst.codes[b * dst.sb + h * dst.sh + t * dst.st + lane] = (uint8_t)quant_pair(pair, e);
        if ((lane & 15) == 0) dst.scales[b * dst.eb + h * dst.eh + t * dst.et + (lane >> 4)] = (uint8_t)e;
        return;
    }
    if constexpr (kWithCk) {
        const int jh = num_kernels(first_new) + task - 2 * dm.n_q;
        if (jh >= num_kernels(L)) return;
        const uint8_t *codes = kq.codes + b * kq.sb + h * kq.sh + lane, *scales = kq.scales + b * kq.eb + h * kq.eh + (lane >> 4);
        const __bf16 *fresh = k_new.ptr + b * k_new.sb + h * k_new.sh;
        uint32_t x[kKernel], e[kKernel];
#pragma unroll
        for (int t = 0; t < kKernel; ++t) {              // (uniform over the wavefront; all asked for before any is used)
            const int r = jh * kStride + t;
            if (r >= first_new) {
                x[t] = reinterpret_cast<const uint32_t *>(fresh + (int64_t)(r - first_new) * k_new.st)[lane];
            } else {
                x[t] = codes[(int64_t)r * kq.st];
                e[t] = scales[(int64_t)r * kq.et];
            }
        }
#pragma unroll
        for (int t = 0; t < kKernel; ++t) {
            if (jh * kStride + t >= first_new) {
                e[t] = group_exponent(x[t]);
                x[t] = quant_pair(x[t], e[t]);
            }
            x[t] = dequant_pair<0>(x[t], e[t]);
        }
        reinterpret_cast<uint32_t *>(ck.ptr + b * ck.sb + h * ck.sh + (int64_t)jh * ck.st)[lane] = kernel_mean(x);
    }
}

static int kv_groups(const Dims &dm, int32_t n_new) {
    const int rows = n_new > 0 && !dm.fill ? min(n_new, dm.max_seqlen) : dm.max_seqlen;
    return (rows + kQuantRows - 1) / kQuantRows;
}

int launch_quantize_kv(const Dims &dm, Tensor k, Tensor v, const int32_t *seqlens, int32_t n_new, QuantTensor kq, QuantTensor vq,
                       hipStream_t stream) {
    if (dm.batch <= 0 || dm.max_seqlen <= 0) return 0;
    timing_begin("quantize_kv_kernel", stream);
    hipLaunchKernelGGL(quantize_kv_kernel, dim3(kv_groups(dm, n_new), dm.Hkv, dm.batch), dim3(256), 0, stream, dm, k, v, seqlens, n_new,
                       kq, vq);
    timing_end(stream);
    return (int)hipGetLastError();
}

int launch_dequantize_kv(const Dims &dm, QuantTensor kq, QuantTensor vq, const int32_t *seqlens, int32_t n_new, Tensor k, Tensor v,
                         hipStream_t stream) {
    if (dm.batch <= 0 || dm.max_seqlen <= 0) return 0;
    timing_begin("dequantize_kv_kernel", stream);
    hipLaunchKernelGGL(dequantize_kv_kernel, dim3(kv_groups(dm, n_new), dm.Hkv, dm.batch), dim3(256), 0, stream, dm, kq, vq, seqlens,
                       n_new, k, v);
    timing_end(stream);
    return (int)hipGetLastError();
}

int launch_append_kv_quant(const Dims &dm, Tensor k_new, Tensor v_new, QuantTensor kq, QuantTensor vq, const Tensor *ck,
                           const int32_t *seqlens, hipStream_t stream) {
    if (dm.batch <= 0) return 0;
    const int tasks = 2 * dm.n_q + (ck ? (dm.n_q + kStride - 1) / kStride : 0);   // n rows complete at most ceil(n / s) kernels
    const dim3 grid((tasks + 3) / 4, dm.Hkv, dm.batch), block(256);
    timing_begin("append_kv_quant_kernel", stream);
    if (ck) hipLaunchKernelGGL(append_kv_quant_kernel<true>, grid, block, 0, stream, dm, k_new, v_new, kq, vq, *ck, seqlens);
    else hipLaunchKernelGGL(append_kv_quant_kernel<false>, grid, block, 0, stream, dm, k_new, v_new, kq, vq, Tensor{}, seqlens);
    timing_end(stream);
    return (int)hipGetLastError();
}

}  // namespace infllmv2
