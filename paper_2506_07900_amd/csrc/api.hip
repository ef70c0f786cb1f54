// C ABI of the library: argument validation (host only, before any HIP call) and dispatch to
// the kernel launchers.  See include/infllmv2.h for the contract of every entry point.
#include <math.h>

#include "common.h"
#include "internal.h"
#include "paged.h"
#include "quant.h"

using namespace infllmv2;

namespace {

#define RETURN_IF_ERR(x)                   \
    do {                                   \
        int32_t _s = (x);                  \
        if (_s != INFLLMV2_OK) return _s;  \
    } while (0)

constexpr int32_t kMaxDecodeSeqlen = 262144;   // decode selection: at most 256 log-sum-exp partials per head
constexpr int32_t kMaxDraft = 64;              // one uint64 mask word per drafted token

int32_t check_params(const infllmv2_params *p) {
    if (!p) return INFLLMV2_ERR_INVALID_ARGUMENT;
    if (p->n_q_heads <= 0 || p->n_kv_heads <= 0 || p->topk <= 0 || p->n_init_blocks < 0 ||
        p->n_local_blocks < 0 || p->head_dim <= 0 || p->block_size <= 0 || p->kernel_size <= 0 ||
        p->kernel_stride <= 0)
        return INFLLMV2_ERR_INVALID_ARGUMENT;
    if (!(p->softmax_scale > 0.f) || !(p->softmax_scale < 1e30f)) return INFLLMV2_ERR_INVALID_ARGUMENT;
    if (p->n_q_heads % p->n_kv_heads != 0) return INFLLMV2_ERR_INVALID_ARGUMENT;
    if (p->topk < p->n_init_blocks + p->n_local_blocks) return INFLLMV2_ERR_INVALID_ARGUMENT;
    if (p->head_dim != kHeadDim || p->block_size != kBlock || p->kernel_size != kKernel ||
        p->kernel_stride != kStride)
        return INFLLMV2_ERR_UNSUPPORTED;
    const int g = p->n_q_heads / p->n_kv_heads;
    if (!(g == 1 || g == 2 || g == 4 || g == 8 || g == 16)) return INFLLMV2_ERR_UNSUPPORTED;
    if (p->topk > kMaxTopk) return INFLLMV2_ERR_UNSUPPORTED;
    if (p->lse_coarse_ratio < 0) return INFLLMV2_ERR_INVALID_ARGUMENT;
    if (p->lse_coarse_ratio > 1) {                       // approximate log-sum-exp
        const int rho = p->lse_coarse_ratio;
        if (!(rho == 2 || rho == 4) || g != 16) return INFLLMV2_ERR_UNSUPPORTED;
        // a query that has candidate blocks must see at least one coarse kernel
        if ((p->n_init_blocks + p->n_local_blocks) * p->block_size < 2 * rho * p->kernel_stride)
            return INFLLMV2_ERR_UNSUPPORTED;
    }
    return INFLLMV2_OK;
}

int32_t check_sizes(int32_t batch, int32_t max_seqlen) {
    if (batch < 0 || max_seqlen < 0) return INFLLMV2_ERR_INVALID_ARGUMENT;
    if (batch > 65535) return INFLLMV2_ERR_UNSUPPORTED;
    return INFLLMV2_OK;
}

// query rows of a verification step: one grid-z slot each
int32_t check_draft(int32_t batch, int32_t n_draft) {
    if (n_draft < 1) return INFLLMV2_ERR_INVALID_ARGUMENT;
    if (n_draft > kMaxDraft || (int64_t)batch * n_draft > 65535) return INFLLMV2_ERR_UNSUPPORTED;
    return INFLLMV2_OK;
}

int32_t check_tensor(const infllmv2_tensor *t) {
    if (!t || !t->ptr) return INFLLMV2_ERR_INVALID_ARGUMENT;
    if ((reinterpret_cast<uintptr_t>(t->ptr) & 15u) != 0) return INFLLMV2_ERR_INVALID_ARGUMENT;
    if (t->stride_b < 0 || t->stride_h < 0 || t->stride_t < 0) return INFLLMV2_ERR_INVALID_ARGUMENT;
    if ((t->stride_b % 8) || (t->stride_h % 8) || (t->stride_t % 8)) return INFLLMV2_ERR_INVALID_ARGUMENT;
    return INFLLMV2_OK;
}

Dims make_dims(const infllmv2_params *p, int32_t batch, int32_t max_seqlen, int32_t n_q = 1, int32_t fill = 0) {
    Dims d;
    d.Hq = p->n_q_heads;
    d.Hkv = p->n_kv_heads;
    d.G = p->n_q_heads / p->n_kv_heads;
    d.topk = p->topk;
    d.n_init = p->n_init_blocks;
    d.n_local = p->n_local_blocks;
    d.batch = batch;
    d.max_seqlen = max_seqlen;
    d.scale_log2 = p->softmax_scale * kLog2e;
    d.rho = p->lse_coarse_ratio > 1 ? p->lse_coarse_ratio : 1;
    d.n_q = n_q;
    d.n_q_inv = n_q > 1 ? (uint32_t)((1ull << 32) / (uint32_t)n_q) + 1u : 0u;
    d.shared_q = 0;
    d.fill = fill;
    return d;
}

Tensor make_tensor(const infllmv2_tensor *t) {
    Tensor r;
    r.ptr = reinterpret_cast<__bf16 *>(t->ptr);
    r.sb = t->stride_b;
    r.sh = t->stride_h;
    r.st = t->stride_t;
    return r;
}

// a cache in 4 bits; strides in bytes
int32_t check_quant(const infllmv2_quant_tensor *t) {
    if (!t || !t->codes || !t->scales) return INFLLMV2_ERR_INVALID_ARGUMENT;
    if ((reinterpret_cast<uintptr_t>(t->codes) & 15u) || (reinterpret_cast<uintptr_t>(t->scales) & 3u)) return INFLLMV2_ERR_INVALID_ARGUMENT;
    const int64_t codes[3] = {t->stride_b, t->stride_h, t->stride_t}, scales[3] = {t->scale_stride_b, t->scale_stride_h, t->scale_stride_t};
    for (int i = 0; i < 3; ++i)
        if (codes[i] < 0 || scales[i] < 0 || codes[i] % 16 || scales[i] % 4) return INFLLMV2_ERR_INVALID_ARGUMENT;
    return INFLLMV2_OK;
}

QuantTensor make_quant(const infllmv2_quant_tensor *t) {
    return QuantTensor{reinterpret_cast<uint8_t *>(t->codes), reinterpret_cast<uint8_t *>(t->scales), t->stride_b, t->stride_h, t->stride_t,
                       t->scale_stride_b, t->scale_stride_h, t->scale_stride_t};
}

// (the kernels number a cache's rows, rounded up to tiles, in 32 bits)
int32_t check_capacity(int32_t max_seqlen) { return max_seqlen > (1 << 30) ? INFLLMV2_ERR_UNSUPPORTED : INFLLMV2_OK; }

int32_t check_window(int32_t n_sink, int32_t window) { return n_sink < 0 || window < 1 ? INFLLMV2_ERR_INVALID_ARGUMENT : INFLLMV2_OK; }

WindowArgs make_window(int32_t n_sink, int32_t window, int32_t max_seqlen) {   // (none of a sequence lies behind max_seqlen)
    const int32_t most = max_seqlen > 1 ? max_seqlen : 1;
    return WindowArgs{n_sink < most ? n_sink : most, window < most ? window : most};
}

// the prefill and backward kernels address a tile's rows with 32-bit offsets: tokens of k, v, and in the backward of q and dout and
// their heads of a group
int32_t check_spans(const infllmv2_params *p, const infllmv2_tensor *k, const infllmv2_tensor *v, const infllmv2_tensor *q, const infllmv2_tensor *dout) {
    const infllmv2_tensor *ts[4] = {k, v, q, dout};
    for (int i = 0; i < 4; ++i) {
        if (!ts[i]) continue;
        if (ts[i]->stride_t > kMaxTokenStride) return INFLLMV2_ERR_UNSUPPORTED;
        if (i >= 2 && (p->n_q_heads / p->n_kv_heads) * ts[i]->stride_h > kMaxHeadSpan) return INFLLMV2_ERR_UNSUPPORTED;
    }
    return INFLLMV2_OK;
}

// and so do the attention calls in the rows of a cache in 4 bits
int32_t check_rows(const infllmv2_quant_tensor *kq, const infllmv2_quant_tensor *vq) {
    const int64_t st[4] = {kq->stride_t, kq->scale_stride_t, vq->stride_t, vq->scale_stride_t};
    for (int i = 0; i < 4; ++i)
        if (st[i] > kMaxQuantStride) return INFLLMV2_ERR_UNSUPPORTED;
    return INFLLMV2_OK;
}

int32_t check_workspace(const void *workspace, size_t bytes, size_t need) {
    return need > 0 && (!workspace || bytes < need || (reinterpret_cast<uintptr_t>(workspace) & 255u) != 0) ? INFLLMV2_ERR_WORKSPACE : INFLLMV2_OK;
}

// a cache in pages, with tables of `rows` rows per sequence
int32_t check_pages(const infllmv2_pages *p, int64_t rows) {
    if (!p || !p->table || p->n_pages < 0 || p->page_size <= 0 || p->table_stride < 0) return INFLLMV2_ERR_INVALID_ARGUMENT;
    RETURN_IF_ERR(check_tensor(&p->k));
    RETURN_IF_ERR(check_tensor(&p->v));
    if ((p->page_size & (p->page_size - 1)) != 0 || p->page_size < 16 || p->page_size > 1024) return INFLLMV2_ERR_UNSUPPORTED;
    if ((int64_t)p->table_stride * p->page_size < rows) return INFLLMV2_ERR_INVALID_ARGUMENT;
    if (p->k.stride_t > kMaxTokenStride || p->v.stride_t > kMaxTokenStride) return INFLLMV2_ERR_UNSUPPORTED;
    return INFLLMV2_OK;
}

Pages make_pages(const infllmv2_pages *p) {
    return Pages{make_tensor(&p->k), make_tensor(&p->v), p->table, p->table_stride, __builtin_ctz((unsigned)p->page_size), p->n_pages};
}

int32_t check_rotation(const infllmv2_rotation *r) {
    if (!r || !r->steps || (reinterpret_cast<uintptr_t>(r->steps) & 15u) || r->rot_dim <= 0 || !isfinite(r->amplitude)) return INFLLMV2_ERR_INVALID_ARGUMENT;
    return r->rot_dim % 16 || r->rot_dim > kHeadDim ? INFLLMV2_ERR_UNSUPPORTED : INFLLMV2_OK;
}

Rotation make_rotation(const infllmv2_rotation *r, bool back) {
    return r ? Rotation{r->steps, r->rot_dim, r->interleaved, r->amplitude, back ? -1.f : 1.f} : Rotation{nullptr, 0, 0, 1.f, 1.f};
}

int32_t check_new(const infllmv2_params *prm, int32_t max_new) {
    if (max_new < 1) return INFLLMV2_ERR_INVALID_ARGUMENT;
    return max_new > (1 << 24) || (int64_t)max_new * prm->n_q_heads > (1ll << 30) ? INFLLMV2_ERR_UNSUPPORTED : INFLLMV2_OK;
}

int32_t hip_status(int e) { return e == 0 ? INFLLMV2_OK : INFLLMV2_ERR_HIP; }

}  // namespace

namespace infllmv2 {
// Host-side validation of the stage-3 decode arguments, shared by the entry points that differ only in
// where their scratch memory comes from.
int32_t validate_attn_decode(const infllmv2_params *prm, const infllmv2_tensor *q, const infllmv2_tensor *k,
                             const infllmv2_tensor *v, const int32_t *seqlens, int32_t batch, int32_t max_seqlen,
                             const int32_t *block_idx, const infllmv2_tensor *out, const float *lse, Dims *dm,
                             Tensor *tq, Tensor *tk, Tensor *tv, Tensor *tout) {
    RETURN_IF_ERR(check_params(prm));
    RETURN_IF_ERR(check_sizes(batch, max_seqlen));
    RETURN_IF_ERR(check_tensor(q));
    RETURN_IF_ERR(check_tensor(k));
    RETURN_IF_ERR(check_tensor(v));
    RETURN_IF_ERR(check_tensor(out));
    if (!seqlens || !block_idx || !lse) return INFLLMV2_ERR_INVALID_ARGUMENT;
    *dm = make_dims(prm, batch, max_seqlen);
    *tq = make_tensor(q);
    *tk = make_tensor(k);
    *tv = make_tensor(v);
    *tout = make_tensor(out);
    return INFLLMV2_OK;
}
}  // namespace infllmv2

extern "C" {

const char *infllmv2_status_string(int32_t status) {
    switch (status) {
        case INFLLMV2_OK: return "ok";
        case INFLLMV2_ERR_INVALID_ARGUMENT: return "invalid argument";
        case INFLLMV2_ERR_UNSUPPORTED: return "unsupported shape";
        case INFLLMV2_ERR_WORKSPACE: return "workspace missing or too small";
        case INFLLMV2_ERR_HIP: return "HIP error";
    }
    return "unknown status";
}

size_t infllmv2_workspace_bytes(int32_t op, const infllmv2_params *prm, int32_t batch,
                                int32_t max_seqlen) {
    if (check_params(prm) != INFLLMV2_OK || check_sizes(batch, max_seqlen) != INFLLMV2_OK) return 0;
    const Dims dm = make_dims(prm, batch, max_seqlen);
    switch (op) {
        case INFLLMV2_OP_SELECT_PREFILL: return select_prefill_ws_bytes(dm);
        case INFLLMV2_OP_SELECT_DECODE: return max_seqlen > kMaxDecodeSeqlen ? 0 : select_decode_ws_bytes(dm);
        case INFLLMV2_OP_ATTN_PREFILL: return attn_prefill_ws_bytes(dm);
        case INFLLMV2_OP_ATTN_DECODE: return attn_decode_ws_bytes(dm);
        case INFLLMV2_OP_ATTN_BWD: return attn_bwd_ws_bytes(dm);
        case INFLLMV2_OP_SELECT_SHARED: {
            Dims ds = dm;
            ds.shared_q = 1;
            return select_prefill_ws_bytes(ds);
        }
        case INFLLMV2_OP_DECODE_STEP:
            return max_seqlen > kMaxDecodeSeqlen ? 0 : select_decode_ws_bytes(dm) + attn_decode_ws_bytes(dm);
    }
    return 0;
}

size_t infllmv2_verify_workspace_bytes(int32_t op, const infllmv2_params *prm, int32_t batch,
                                       int32_t max_seqlen, int32_t n_draft) {
    if (check_params(prm) != INFLLMV2_OK || check_sizes(batch, max_seqlen) != INFLLMV2_OK ||
        check_draft(batch, n_draft) != INFLLMV2_OK)
        return 0;
    const Dims dm = make_dims(prm, batch, max_seqlen, n_draft);
    switch (op) {
        case INFLLMV2_OP_SELECT_VERIFY: return max_seqlen > kMaxDecodeSeqlen ? 0 : select_decode_ws_bytes(dm);
        case INFLLMV2_OP_ATTN_VERIFY: return attn_decode_ws_bytes(dm);
        case INFLLMV2_OP_VERIFY_STEP:
            return max_seqlen > kMaxDecodeSeqlen ? 0 : select_decode_ws_bytes(dm) + attn_decode_ws_bytes(dm);
    }
    return 0;
}

int32_t infllmv2i_compress_keys(const infllmv2_params *prm, const infllmv2_tensor *k,
                                const int32_t *seqlens, int32_t batch, int32_t max_seqlen,
                                int32_t n_new_tokens, const infllmv2_tensor *ck, void *stream, int32_t fill) {
    RETURN_IF_ERR(check_params(prm));
    RETURN_IF_ERR(check_sizes(batch, max_seqlen));
    RETURN_IF_ERR(check_tensor(k));
    RETURN_IF_ERR(check_tensor(ck));
    if (!seqlens) return INFLLMV2_ERR_INVALID_ARGUMENT;
    const Dims dm = make_dims(prm, batch, max_seqlen, 1, fill);
    return hip_status(launch_compress_keys(dm, make_tensor(k), make_tensor(ck), seqlens, n_new_tokens,
                                           reinterpret_cast<hipStream_t>(stream)));
}

int32_t infllmv2_compress_keys(const infllmv2_params *prm, const infllmv2_tensor *k,
                               const int32_t *seqlens, int32_t batch, int32_t max_seqlen,
                               int32_t n_new_tokens, const infllmv2_tensor *ck, void *stream) {
    return infllmv2i_compress_keys(prm, k, seqlens, batch, max_seqlen, n_new_tokens, ck, stream, 0);
}

int32_t infllmv2_append_kv(const infllmv2_params *prm, const infllmv2_tensor *k_new,
                           const infllmv2_tensor *v_new, const infllmv2_tensor *k,
                           const infllmv2_tensor *v, const infllmv2_tensor *ck, const int32_t *seqlens,
                           int32_t batch, int32_t max_seqlen, void *stream) {
    RETURN_IF_ERR(check_params(prm));
    RETURN_IF_ERR(check_sizes(batch, max_seqlen));
    RETURN_IF_ERR(check_tensor(k_new));
    RETURN_IF_ERR(check_tensor(v_new));
    RETURN_IF_ERR(check_tensor(k));
    RETURN_IF_ERR(check_tensor(v));
    if (ck) RETURN_IF_ERR(check_tensor(ck));
    if (!seqlens) return INFLLMV2_ERR_INVALID_ARGUMENT;
    const Dims dm = make_dims(prm, batch, max_seqlen);
    Tensor ckt;
    if (ck) ckt = make_tensor(ck);
    return hip_status(launch_append_kv(dm, make_tensor(k_new), make_tensor(v_new), make_tensor(k),
                                       make_tensor(v), ck ? &ckt : nullptr, seqlens,
                                       reinterpret_cast<hipStream_t>(stream)));
}

int32_t infllmv2_append_kv_verify(const infllmv2_params *prm, const infllmv2_tensor *k_new,
                                  const infllmv2_tensor *v_new, const infllmv2_tensor *k,
                                  const infllmv2_tensor *v, const infllmv2_tensor *ck, const int32_t *seqlens,
                                  int32_t batch, int32_t max_seqlen, int32_t n_draft, void *stream) {
    RETURN_IF_ERR(check_params(prm));
    RETURN_IF_ERR(check_sizes(batch, max_seqlen));
    RETURN_IF_ERR(check_draft(batch, n_draft));
    RETURN_IF_ERR(check_tensor(k_new));
    RETURN_IF_ERR(check_tensor(v_new));
    RETURN_IF_ERR(check_tensor(k));
    RETURN_IF_ERR(check_tensor(v));
    if (ck) RETURN_IF_ERR(check_tensor(ck));
    if (!seqlens) return INFLLMV2_ERR_INVALID_ARGUMENT;
    const Dims dm = make_dims(prm, batch, max_seqlen, n_draft);
    Tensor ckt;
    if (ck) ckt = make_tensor(ck);
    return hip_status(launch_append_kv(dm, make_tensor(k_new), make_tensor(v_new), make_tensor(k),
                                       make_tensor(v), ck ? &ckt : nullptr, seqlens,
                                       reinterpret_cast<hipStream_t>(stream)));
}

int32_t infllmv2_select_blocks_verify(const infllmv2_params *prm, const infllmv2_tensor *q,
                                      const infllmv2_tensor *ck, const int32_t *seqlens, int32_t batch,
                                      int32_t max_seqlen, int32_t n_draft, int32_t *block_idx,
                                      void *workspace, size_t workspace_bytes, void *stream) {
    RETURN_IF_ERR(check_params(prm));
    RETURN_IF_ERR(check_sizes(batch, max_seqlen));
    RETURN_IF_ERR(check_draft(batch, n_draft));
    RETURN_IF_ERR(check_tensor(q));
    RETURN_IF_ERR(check_tensor(ck));
    if (!seqlens || !block_idx) return INFLLMV2_ERR_INVALID_ARGUMENT;
    if (max_seqlen > kMaxDecodeSeqlen) return INFLLMV2_ERR_UNSUPPORTED;
    const Dims dm = make_dims(prm, batch, max_seqlen, n_draft);
    const size_t need = select_decode_ws_bytes(dm);
    if (need > 0 && (!workspace || workspace_bytes < need ||
                     (reinterpret_cast<uintptr_t>(workspace) & 255u) != 0))
        return INFLLMV2_ERR_WORKSPACE;
    return hip_status(launch_select_decode(dm, make_tensor(q), make_tensor(ck), seqlens, block_idx,
                                           workspace, reinterpret_cast<hipStream_t>(stream)));
}

int32_t infllmv2_sparse_attn_verify(const infllmv2_params *prm, const infllmv2_tensor *q,
                                    const infllmv2_tensor *k, const infllmv2_tensor *v,
                                    const int32_t *seqlens, int32_t batch, int32_t max_seqlen,
                                    int32_t n_draft, const uint64_t *tree_mask, const int32_t *block_idx,
                                    const infllmv2_tensor *out, float *lse, void *workspace,
                                    size_t workspace_bytes, void *stream) {
    RETURN_IF_ERR(check_params(prm));
    RETURN_IF_ERR(check_sizes(batch, max_seqlen));
    RETURN_IF_ERR(check_draft(batch, n_draft));
    RETURN_IF_ERR(check_tensor(q));
    RETURN_IF_ERR(check_tensor(k));
    RETURN_IF_ERR(check_tensor(v));
    RETURN_IF_ERR(check_tensor(out));
    if (!seqlens || !block_idx || !lse) return INFLLMV2_ERR_INVALID_ARGUMENT;
    if (tree_mask && (reinterpret_cast<uintptr_t>(tree_mask) & 7u) != 0) return INFLLMV2_ERR_INVALID_ARGUMENT;
    const Dims dm = make_dims(prm, batch, max_seqlen, n_draft);
    const size_t need = attn_decode_ws_bytes(dm);
    if (need > 0 && (!workspace || workspace_bytes < need ||
                     (reinterpret_cast<uintptr_t>(workspace) & 255u) != 0))
        return INFLLMV2_ERR_WORKSPACE;
    return hip_status(launch_attn_decode(dm, make_tensor(q), make_tensor(k), make_tensor(v), seqlens,
                                         block_idx, tree_mask, make_tensor(out), lse, workspace,
                                         reinterpret_cast<hipStream_t>(stream)));
}

int32_t infllmv2_verify_step(const infllmv2_params *prm, const infllmv2_tensor *q,
                             const infllmv2_tensor *k_new, const infllmv2_tensor *v_new,
                             const infllmv2_tensor *k, const infllmv2_tensor *v, const infllmv2_tensor *ck,
                             const int32_t *seqlens, int32_t batch, int32_t max_seqlen, int32_t n_draft,
                             const uint64_t *tree_mask, int32_t *block_idx, const infllmv2_tensor *out,
                             float *lse, void *workspace, size_t workspace_bytes, void *stream) {
    RETURN_IF_ERR(check_params(prm));
    RETURN_IF_ERR(check_sizes(batch, max_seqlen));
    RETURN_IF_ERR(check_draft(batch, n_draft));
    const infllmv2_tensor *ts[7] = {q, k_new, v_new, k, v, ck, out};
    for (int i = 0; i < 7; ++i) RETURN_IF_ERR(check_tensor(ts[i]));
    if (!seqlens || !block_idx || !lse) return INFLLMV2_ERR_INVALID_ARGUMENT;
    if (tree_mask && (reinterpret_cast<uintptr_t>(tree_mask) & 7u) != 0) return INFLLMV2_ERR_INVALID_ARGUMENT;
    if (max_seqlen > kMaxDecodeSeqlen) return INFLLMV2_ERR_UNSUPPORTED;
    const Dims dm = make_dims(prm, batch, max_seqlen, n_draft);
    const size_t sel = select_decode_ws_bytes(dm), need = sel + attn_decode_ws_bytes(dm);
    if (need > 0 && (!workspace || workspace_bytes < need ||
                     (reinterpret_cast<uintptr_t>(workspace) & 255u) != 0))
        return INFLLMV2_ERR_WORKSPACE;
    const AppendArgs ap = {make_tensor(k_new), make_tensor(v_new), make_tensor(k), make_tensor(v)};
    return hip_status(launch_verify_step(dm, make_tensor(q), make_tensor(ck), ap, seqlens, tree_mask, block_idx,
                                         make_tensor(out), lse, workspace, reinterpret_cast<char *>(workspace) + sel,
                                         reinterpret_cast<hipStream_t>(stream)));
}

int32_t infllmv2_decode_step(const infllmv2_params *prm, const infllmv2_tensor *q,
                             const infllmv2_tensor *k_new, const infllmv2_tensor *v_new,
                             const infllmv2_tensor *k, const infllmv2_tensor *v, const infllmv2_tensor *ck,
                             const int32_t *seqlens, int32_t batch, int32_t max_seqlen, int32_t *block_idx,
                             const infllmv2_tensor *out, float *lse, void *workspace, size_t workspace_bytes,
                             void *stream) {
    RETURN_IF_ERR(check_params(prm));
    RETURN_IF_ERR(check_sizes(batch, max_seqlen));
    const infllmv2_tensor *ts[7] = {q, k_new, v_new, k, v, ck, out};
    for (int i = 0; i < 7; ++i) RETURN_IF_ERR(check_tensor(ts[i]));
    if (!seqlens || !block_idx || !lse) return INFLLMV2_ERR_INVALID_ARGUMENT;
    if (max_seqlen > kMaxDecodeSeqlen) return INFLLMV2_ERR_UNSUPPORTED;
    const Dims dm = make_dims(prm, batch, max_seqlen);
    const size_t sel = select_decode_ws_bytes(dm), need = sel + attn_decode_ws_bytes(dm);
    if (need > 0 && (!workspace || workspace_bytes < need ||
                     (reinterpret_cast<uintptr_t>(workspace) & 255u) != 0))
        return INFLLMV2_ERR_WORKSPACE;
    hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    const AppendArgs ap = {make_tensor(k_new), make_tensor(v_new), make_tensor(k), make_tensor(v)};
    return hip_status(launch_decode_step(dm, make_tensor(q), make_tensor(ck), ap, seqlens, block_idx, make_tensor(out),
                                         lse, workspace, reinterpret_cast<char *>(workspace) + sel, st));
}

int32_t infllmv2i_select_blocks(const infllmv2_params *prm, int32_t mode, const infllmv2_tensor *q,
                               const infllmv2_tensor *ck, const int32_t *seqlens, int32_t batch,
                               int32_t max_seqlen, int32_t *block_idx, void *workspace,
                               size_t workspace_bytes, void *stream, int32_t fill) {
    RETURN_IF_ERR(check_params(prm));
    RETURN_IF_ERR(check_sizes(batch, max_seqlen));
    if (mode != INFLLMV2_MODE_PREFILL && mode != INFLLMV2_MODE_DECODE) return INFLLMV2_ERR_INVALID_ARGUMENT;
    RETURN_IF_ERR(check_tensor(q));
    RETURN_IF_ERR(check_tensor(ck));
    if (!seqlens || !block_idx) return INFLLMV2_ERR_INVALID_ARGUMENT;
    if (mode == INFLLMV2_MODE_DECODE && max_seqlen > kMaxDecodeSeqlen) return INFLLMV2_ERR_UNSUPPORTED;
    const Dims dm = make_dims(prm, batch, max_seqlen, 1, fill);
    const size_t need = mode == INFLLMV2_MODE_PREFILL ? select_prefill_ws_bytes(dm) : select_decode_ws_bytes(dm);
    if (need > 0 && (!workspace || workspace_bytes < need ||
                     (reinterpret_cast<uintptr_t>(workspace) & 255u) != 0))
        return INFLLMV2_ERR_WORKSPACE;
    hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    if (mode == INFLLMV2_MODE_PREFILL)
        return hip_status(launch_select_prefill(dm, make_tensor(q), make_tensor(ck), seqlens, block_idx,
                                                workspace, st));
    return hip_status(launch_select_decode(dm, make_tensor(q), make_tensor(ck), seqlens, block_idx,
                                           workspace, st));
}

int32_t infllmv2_select_blocks(const infllmv2_params *prm, int32_t mode, const infllmv2_tensor *q,
                               const infllmv2_tensor *ck, const int32_t *seqlens, int32_t batch,
                               int32_t max_seqlen, int32_t *block_idx, void *workspace,
                               size_t workspace_bytes, void *stream) {
    return infllmv2i_select_blocks(prm, mode, q, ck, seqlens, batch, max_seqlen, block_idx, workspace, workspace_bytes, stream, 0);
}

int32_t infllmv2_block_scores(const infllmv2_params *prm, const infllmv2_tensor *q, const infllmv2_tensor *ck,
                              const int32_t *seqlens, int32_t batch, int32_t max_seqlen, float *block_scores,
                              int32_t scores_pitch, void *workspace, size_t workspace_bytes, void *stream) {
    RETURN_IF_ERR(check_params(prm));
    RETURN_IF_ERR(check_sizes(batch, max_seqlen));
    RETURN_IF_ERR(check_tensor(q));
    RETURN_IF_ERR(check_tensor(ck));
    if (!seqlens || !block_scores || scores_pitch < (max_seqlen + prm->block_size - 1) / prm->block_size)
        return INFLLMV2_ERR_INVALID_ARGUMENT;
    const Dims dm = make_dims(prm, batch, max_seqlen);
    const size_t need = select_prefill_ws_bytes(dm);
    if (need > 0 && (!workspace || workspace_bytes < need ||
                     (reinterpret_cast<uintptr_t>(workspace) & 255u) != 0))
        return INFLLMV2_ERR_WORKSPACE;
    return hip_status(launch_select_prefill(dm, make_tensor(q), make_tensor(ck), seqlens, nullptr, workspace,
                                            reinterpret_cast<hipStream_t>(stream), block_scores, scores_pitch));
}

int32_t infllmv2_select_blocks_shared(const infllmv2_params *prm, const infllmv2_tensor *q,
                                      const infllmv2_tensor *ck, const int32_t *seqlens, int32_t batch,
                                      int32_t max_seqlen, int32_t *block_idx, void *workspace,
                                      size_t workspace_bytes, void *stream) {
    RETURN_IF_ERR(check_params(prm));
    RETURN_IF_ERR(check_sizes(batch, max_seqlen));
    RETURN_IF_ERR(check_tensor(q));
    RETURN_IF_ERR(check_tensor(ck));
    if (!seqlens || !block_idx) return INFLLMV2_ERR_INVALID_ARGUMENT;
    Dims dm = make_dims(prm, batch, max_seqlen);
    dm.shared_q = 1;
    const size_t need = select_prefill_ws_bytes(dm);
    if (need > 0 && (!workspace || workspace_bytes < need ||
                     (reinterpret_cast<uintptr_t>(workspace) & 255u) != 0))
        return INFLLMV2_ERR_WORKSPACE;
    return hip_status(launch_select_prefill(dm, make_tensor(q), make_tensor(ck), seqlens, block_idx, workspace,
                                            reinterpret_cast<hipStream_t>(stream)));
}

int32_t infllmv2i_sparse_attn_prefill(const infllmv2_params *prm, const infllmv2_tensor *q,
                                     const infllmv2_tensor *k, const infllmv2_tensor *v,
                                     const int32_t *seqlens, int32_t batch, int32_t max_seqlen,
                                     const int32_t *block_idx, const infllmv2_tensor *out, float *lse,
                                     void *workspace, size_t workspace_bytes, void *stream, int32_t fill) {
    RETURN_IF_ERR(check_params(prm));
    RETURN_IF_ERR(check_sizes(batch, max_seqlen));
    RETURN_IF_ERR(check_tensor(q));
    RETURN_IF_ERR(check_tensor(k));
    RETURN_IF_ERR(check_tensor(v));
    RETURN_IF_ERR(check_tensor(out));
    if (!seqlens || !block_idx || !lse) return INFLLMV2_ERR_INVALID_ARGUMENT;
    const Dims dm = make_dims(prm, batch, max_seqlen, 1, fill);
    const size_t need = attn_prefill_ws_bytes(dm);
    if (need > 0 && (!workspace || workspace_bytes < need ||
                     (reinterpret_cast<uintptr_t>(workspace) & 255u) != 0))
        return INFLLMV2_ERR_WORKSPACE;
    return hip_status(launch_attn_prefill(dm, make_tensor(q), make_tensor(k), make_tensor(v), seqlens,
                                          block_idx, make_tensor(out), lse, workspace,
                                          reinterpret_cast<hipStream_t>(stream)));
}

int32_t infllmv2_sparse_attn_prefill(const infllmv2_params *prm, const infllmv2_tensor *q,
                                     const infllmv2_tensor *k, const infllmv2_tensor *v,
                                     const int32_t *seqlens, int32_t batch, int32_t max_seqlen,
                                     const int32_t *block_idx, const infllmv2_tensor *out, float *lse,
                                     void *workspace, size_t workspace_bytes, void *stream) {
    return infllmv2i_sparse_attn_prefill(prm, q, k, v, seqlens, batch, max_seqlen, block_idx, out, lse, workspace,
                                         workspace_bytes, stream, 0);
}

int32_t infllmv2_sparse_attn_prefill_shared(const infllmv2_params *prm, const infllmv2_tensor *q,
                                            const infllmv2_tensor *k, const infllmv2_tensor *v,
                                            const int32_t *seqlens, int32_t batch, int32_t max_seqlen,
                                            const int32_t *block_idx, const infllmv2_tensor *out, float *lse,
                                            void *workspace, size_t workspace_bytes, void *stream) {
    RETURN_IF_ERR(check_params(prm));
    RETURN_IF_ERR(check_sizes(batch, max_seqlen));
    RETURN_IF_ERR(check_tensor(q));
    RETURN_IF_ERR(check_tensor(k));
    RETURN_IF_ERR(check_tensor(v));
    RETURN_IF_ERR(check_tensor(out));
    if (!seqlens || !block_idx || !lse) return INFLLMV2_ERR_INVALID_ARGUMENT;
    Dims dm = make_dims(prm, batch, max_seqlen);
    dm.shared_q = 1;
    const size_t need = attn_prefill_ws_bytes(dm);
    if (need > 0 && (!workspace || workspace_bytes < need ||
                     (reinterpret_cast<uintptr_t>(workspace) & 255u) != 0))
        return INFLLMV2_ERR_WORKSPACE;
    return hip_status(launch_attn_prefill(dm, make_tensor(q), make_tensor(k), make_tensor(v), seqlens,
                                          block_idx, make_tensor(out), lse, workspace,
                                          reinterpret_cast<hipStream_t>(stream)));
}

int32_t infllmv2i_sparse_attn_bwd(const infllmv2_params *prm, const infllmv2_tensor *q,
                                 const infllmv2_tensor *k, const infllmv2_tensor *v,
                                 const infllmv2_tensor *out, const infllmv2_tensor *dout, const float *lse,
                                 const int32_t *seqlens, int32_t batch, int32_t max_seqlen,
                                 const int32_t *block_idx, const infllmv2_tensor *dq,
                                 const infllmv2_tensor *dk, const infllmv2_tensor *dv, void *workspace,
                                 size_t workspace_bytes, void *stream, int32_t fill) {
    RETURN_IF_ERR(check_params(prm));
    RETURN_IF_ERR(check_sizes(batch, max_seqlen));
    const infllmv2_tensor *ts[8] = {q, k, v, out, dout, dq, dk, dv};
    for (int i = 0; i < 8; ++i) RETURN_IF_ERR(check_tensor(ts[i]));
    if (!seqlens || !block_idx || !lse) return INFLLMV2_ERR_INVALID_ARGUMENT;
    // the dk/dv kernel addresses the heads of a group with 32-bit element offsets from the group's first head
    const int64_t head_span = (int64_t)(prm->n_q_heads / prm->n_kv_heads) * (q->stride_h > dout->stride_h ? q->stride_h : dout->stride_h);
    if (head_span > (int64_t)1 << 30) return INFLLMV2_ERR_UNSUPPORTED;
    const Dims dm = make_dims(prm, batch, max_seqlen, 1, fill);
    const size_t need = attn_bwd_ws_bytes(dm);
    if (need > 0 && (!workspace || workspace_bytes < need ||
                     (reinterpret_cast<uintptr_t>(workspace) & 255u) != 0))
        return INFLLMV2_ERR_WORKSPACE;
    return hip_status(launch_attn_bwd(dm, make_tensor(q), make_tensor(k), make_tensor(v), make_tensor(out),
                                      make_tensor(dout), lse, seqlens, block_idx, make_tensor(dq), make_tensor(dk),
                                      make_tensor(dv), workspace, reinterpret_cast<hipStream_t>(stream)));
}

int32_t infllmv2_sparse_attn_bwd(const infllmv2_params *prm, const infllmv2_tensor *q,
                                 const infllmv2_tensor *k, const infllmv2_tensor *v,
                                 const infllmv2_tensor *out, const infllmv2_tensor *dout, const float *lse,
                                 const int32_t *seqlens, int32_t batch, int32_t max_seqlen,
                                 const int32_t *block_idx, const infllmv2_tensor *dq,
                                 const infllmv2_tensor *dk, const infllmv2_tensor *dv, void *workspace,
                                 size_t workspace_bytes, void *stream) {
    return infllmv2i_sparse_attn_bwd(prm, q, k, v, out, dout, lse, seqlens, batch, max_seqlen, block_idx, dq, dk, dv,
                                     workspace, workspace_bytes, stream, 0);
}

int32_t infllmv2_sparse_attn_decode(const infllmv2_params *prm, const infllmv2_tensor *q,
                                    const infllmv2_tensor *k, const infllmv2_tensor *v,
                                    const int32_t *seqlens, int32_t batch, int32_t max_seqlen,
                                    const int32_t *block_idx, const infllmv2_tensor *out, float *lse,
                                    void *workspace, size_t workspace_bytes, void *stream) {
    Dims dm;
    Tensor tq, tk, tv, tout;
    RETURN_IF_ERR(validate_attn_decode(prm, q, k, v, seqlens, batch, max_seqlen, block_idx, out, lse, &dm, &tq, &tk,
                                       &tv, &tout));
    const size_t need = attn_decode_ws_bytes(dm);
    if (need > 0 && (!workspace || workspace_bytes < need ||
                     (reinterpret_cast<uintptr_t>(workspace) & 255u) != 0))
        return INFLLMV2_ERR_WORKSPACE;
    return hip_status(launch_attn_decode(dm, tq, tk, tv, seqlens, block_idx, nullptr, tout, lse, workspace,
                                         reinterpret_cast<hipStream_t>(stream)));
}

int32_t infllmv2i_quantize_kv(const infllmv2_params *prm, const infllmv2_tensor *k, const infllmv2_tensor *v,
                              const int32_t *seqlens, int32_t batch, int32_t max_seqlen, int32_t n_new_tokens,
                              const infllmv2_quant_tensor *kq, const infllmv2_quant_tensor *vq, void *stream, int32_t fill) {
    RETURN_IF_ERR(check_params(prm));
    RETURN_IF_ERR(check_sizes(batch, max_seqlen));
    RETURN_IF_ERR(check_capacity(max_seqlen));
    RETURN_IF_ERR(check_tensor(k));
    RETURN_IF_ERR(check_tensor(v));
    RETURN_IF_ERR(check_quant(kq));
    RETURN_IF_ERR(check_quant(vq));
    if (!seqlens) return INFLLMV2_ERR_INVALID_ARGUMENT;
    return hip_status(launch_quantize_kv(make_dims(prm, batch, max_seqlen, 1, fill), make_tensor(k), make_tensor(v), seqlens, n_new_tokens,
                                         make_quant(kq), make_quant(vq), reinterpret_cast<hipStream_t>(stream)));
}

int32_t infllmv2_quantize_kv(const infllmv2_params *prm, const infllmv2_tensor *k, const infllmv2_tensor *v,
                             const int32_t *seqlens, int32_t batch, int32_t max_seqlen, int32_t n_new_tokens,
                             const infllmv2_quant_tensor *kq, const infllmv2_quant_tensor *vq, void *stream) {
    return infllmv2i_quantize_kv(prm, k, v, seqlens, batch, max_seqlen, n_new_tokens, kq, vq, stream, 0);
}

int32_t infllmv2i_dequantize_kv(const infllmv2_params *prm, const infllmv2_quant_tensor *kq, const infllmv2_quant_tensor *vq,
                                const int32_t *seqlens, int32_t batch, int32_t max_seqlen, int32_t n_new_tokens,
                                const infllmv2_tensor *k, const infllmv2_tensor *v, void *stream, int32_t fill) {
    RETURN_IF_ERR(check_params(prm));
    RETURN_IF_ERR(check_sizes(batch, max_seqlen));
    RETURN_IF_ERR(check_capacity(max_seqlen));
    RETURN_IF_ERR(check_quant(kq));
    RETURN_IF_ERR(check_quant(vq));
    RETURN_IF_ERR(check_tensor(k));
    RETURN_IF_ERR(check_tensor(v));
    if (!seqlens) return INFLLMV2_ERR_INVALID_ARGUMENT;
    return hip_status(launch_dequantize_kv(make_dims(prm, batch, max_seqlen, 1, fill), make_quant(kq), make_quant(vq), seqlens, n_new_tokens,
                                           make_tensor(k), make_tensor(v), reinterpret_cast<hipStream_t>(stream)));
}

int32_t infllmv2_dequantize_kv(const infllmv2_params *prm, const infllmv2_quant_tensor *kq, const infllmv2_quant_tensor *vq,
                               const int32_t *seqlens, int32_t batch, int32_t max_seqlen, int32_t n_new_tokens,
                               const infllmv2_tensor *k, const infllmv2_tensor *v, void *stream) {
    return infllmv2i_dequantize_kv(prm, kq, vq, seqlens, batch, max_seqlen, n_new_tokens, k, v, stream, 0);
}

int32_t infllmv2_append_kv_quant(const infllmv2_params *prm, const infllmv2_tensor *k_new, const infllmv2_tensor *v_new,
                                 const infllmv2_quant_tensor *kq, const infllmv2_quant_tensor *vq, const infllmv2_tensor *ck,
                                 const int32_t *seqlens, int32_t batch, int32_t max_seqlen, int32_t n_draft, void *stream) {
    RETURN_IF_ERR(check_params(prm));
    RETURN_IF_ERR(check_sizes(batch, max_seqlen));
    RETURN_IF_ERR(check_capacity(max_seqlen));
    RETURN_IF_ERR(check_draft(batch, n_draft));
    RETURN_IF_ERR(check_tensor(k_new));
    RETURN_IF_ERR(check_tensor(v_new));
    RETURN_IF_ERR(check_quant(kq));
    RETURN_IF_ERR(check_quant(vq));
    if (ck) RETURN_IF_ERR(check_tensor(ck));
    if (!seqlens) return INFLLMV2_ERR_INVALID_ARGUMENT;
    Tensor ckt;
    if (ck) ckt = make_tensor(ck);
    return hip_status(launch_append_kv_quant(make_dims(prm, batch, max_seqlen, n_draft), make_tensor(k_new), make_tensor(v_new), make_quant(kq),
                                             make_quant(vq), ck ? &ckt : nullptr, seqlens, reinterpret_cast<hipStream_t>(stream)));
}

int32_t infllmv2_sparse_attn_verify_quant(const infllmv2_params *prm, const infllmv2_tensor *q, const infllmv2_quant_tensor *kq,
                                          const infllmv2_quant_tensor *vq, const int32_t *seqlens, int32_t batch, int32_t max_seqlen,
                                          int32_t n_draft, const uint64_t *tree_mask, const int32_t *block_idx,
                                          const infllmv2_tensor *out, float *lse, void *workspace, size_t workspace_bytes,
                                          void *stream) {
    RETURN_IF_ERR(check_params(prm));
    RETURN_IF_ERR(check_sizes(batch, max_seqlen));
    RETURN_IF_ERR(check_capacity(max_seqlen));
    RETURN_IF_ERR(check_draft(batch, n_draft));
    RETURN_IF_ERR(check_tensor(q));
    RETURN_IF_ERR(check_quant(kq));
    RETURN_IF_ERR(check_quant(vq));
    RETURN_IF_ERR(check_tensor(out));
    if (!seqlens || !block_idx || !lse) return INFLLMV2_ERR_INVALID_ARGUMENT;
    if (tree_mask && (reinterpret_cast<uintptr_t>(tree_mask) & 7u) != 0) return INFLLMV2_ERR_INVALID_ARGUMENT;
    RETURN_IF_ERR(check_rows(kq, vq));
    const Dims dm = make_dims(prm, batch, max_seqlen, n_draft);
    RETURN_IF_ERR(check_workspace(workspace, workspace_bytes, attn_decode_ws_bytes(dm)));
    return hip_status(launch_attn_decode_quant(dm, make_tensor(q), make_quant(kq), make_quant(vq), seqlens, block_idx, tree_mask,
                                               make_tensor(out), lse, workspace, reinterpret_cast<hipStream_t>(stream)));
}

int32_t infllmv2_sparse_attn_decode_quant(const infllmv2_params *prm, const infllmv2_tensor *q, const infllmv2_quant_tensor *kq,
                                          const infllmv2_quant_tensor *vq, const int32_t *seqlens, int32_t batch, int32_t max_seqlen,
                                          const int32_t *block_idx, const infllmv2_tensor *out, float *lse, void *workspace,
                                          size_t workspace_bytes, void *stream) {
    return infllmv2_sparse_attn_verify_quant(prm, q, kq, vq, seqlens, batch, max_seqlen, 1, nullptr, block_idx, out, lse, workspace,
                                             workspace_bytes, stream);
}

size_t infllmv2_window_workspace_bytes(int32_t op, const infllmv2_params *prm, int32_t n_sink, int32_t window, int32_t batch,
                                       int32_t max_seqlen) {
    if (check_params(prm) != INFLLMV2_OK || check_window(n_sink, window) != INFLLMV2_OK || check_sizes(batch, max_seqlen) != INFLLMV2_OK ||
        check_capacity(max_seqlen) != INFLLMV2_OK)
        return 0;
    const Dims dm = make_dims(prm, batch, max_seqlen);
    const WindowArgs w = make_window(n_sink, window, max_seqlen);
    switch (op) {
        case INFLLMV2_OP_WINDOW_PREFILL: return window_prefill_ws_bytes(dm, w);
        case INFLLMV2_OP_WINDOW_BWD: return window_bwd_ws_bytes(dm, w);
        case INFLLMV2_OP_WINDOW_DECODE: return window_decode_ws_bytes(dm, w);
    }
    return 0;
}

size_t infllmv2i_window_bwd_scratch_bytes(const infllmv2_params *prm, int32_t n_sink, int32_t window, int32_t batch, int32_t max_seqlen) {
    if (check_params(prm) != INFLLMV2_OK || check_window(n_sink, window) != INFLLMV2_OK || check_sizes(batch, max_seqlen) != INFLLMV2_OK ||
        check_capacity(max_seqlen) != INFLLMV2_OK)
        return 0;
    return window_bwd_scratch_bytes(make_dims(prm, batch, max_seqlen), make_window(n_sink, window, max_seqlen));
}

int32_t infllmv2i_window_attn_prefill(const infllmv2_params *prm, int32_t n_sink, int32_t window, const infllmv2_tensor *q,
                                      const infllmv2_tensor *k, const infllmv2_tensor *v, const int32_t *seqlens, int32_t batch,
                                      int32_t max_seqlen, const infllmv2_tensor *out, float *lse, void *workspace,
                                      size_t workspace_bytes, void *stream, int32_t fill) {
    RETURN_IF_ERR(check_params(prm));
    RETURN_IF_ERR(check_window(n_sink, window));
    RETURN_IF_ERR(check_sizes(batch, max_seqlen));
    RETURN_IF_ERR(check_capacity(max_seqlen));
    RETURN_IF_ERR(check_tensor(q));
    RETURN_IF_ERR(check_tensor(k));
    RETURN_IF_ERR(check_tensor(v));
    RETURN_IF_ERR(check_tensor(out));
    if (!seqlens || !lse) return INFLLMV2_ERR_INVALID_ARGUMENT;
    RETURN_IF_ERR(check_spans(prm, k, v, nullptr, nullptr));
    const Dims dm = make_dims(prm, batch, max_seqlen, 1, fill);
    const WindowArgs w = make_window(n_sink, window, max_seqlen);
    RETURN_IF_ERR(check_workspace(workspace, workspace_bytes, window_prefill_ws_bytes(dm, w)));
    return hip_status(launch_window_prefill(dm, w, make_tensor(q), make_tensor(k), make_tensor(v), seqlens, make_tensor(out), lse, workspace,
                                            reinterpret_cast<hipStream_t>(stream)));
}

int32_t infllmv2_window_attn_prefill(const infllmv2_params *prm, int32_t n_sink, int32_t window, const infllmv2_tensor *q,
                                     const infllmv2_tensor *k, const infllmv2_tensor *v, const int32_t *seqlens, int32_t batch,
                                     int32_t max_seqlen, const infllmv2_tensor *out, float *lse, void *workspace,
                                     size_t workspace_bytes, void *stream) {
    return infllmv2i_window_attn_prefill(prm, n_sink, window, q, k, v, seqlens, batch, max_seqlen, out, lse, workspace, workspace_bytes, stream, 0);
}

int32_t infllmv2i_window_attn_bwd(const infllmv2_params *prm, int32_t n_sink, int32_t window, const infllmv2_tensor *q,
                                  const infllmv2_tensor *k, const infllmv2_tensor *v, const infllmv2_tensor *out,
                                  const infllmv2_tensor *dout, const float *lse, const int32_t *seqlens, int32_t batch,
                                  int32_t max_seqlen, const infllmv2_tensor *dq, const infllmv2_tensor *dk,
                                  const infllmv2_tensor *dv, void *workspace, size_t workspace_bytes, void *stream, int32_t fill) {
    RETURN_IF_ERR(check_params(prm));
    RETURN_IF_ERR(check_window(n_sink, window));
    RETURN_IF_ERR(check_sizes(batch, max_seqlen));
    RETURN_IF_ERR(check_capacity(max_seqlen));
    const infllmv2_tensor *ts[8] = {q, k, v, out, dout, dq, dk, dv};
    for (int i = 0; i < 8; ++i) RETURN_IF_ERR(check_tensor(ts[i]));
    if (!seqlens || !lse) return INFLLMV2_ERR_INVALID_ARGUMENT;
    RETURN_IF_ERR(check_spans(prm, k, v, q, dout));
    const Dims dm = make_dims(prm, batch, max_seqlen, 1, fill);
    const WindowArgs w = make_window(n_sink, window, max_seqlen);
    RETURN_IF_ERR(check_workspace(workspace, workspace_bytes, window_bwd_scratch_bytes(dm, w)));
    return hip_status(launch_window_bwd(dm, w, make_tensor(q), make_tensor(k), make_tensor(v), make_tensor(out), make_tensor(dout), lse,
                                        seqlens, make_tensor(dq), make_tensor(dk), make_tensor(dv), workspace,
                                        reinterpret_cast<hipStream_t>(stream)));
}

int32_t infllmv2_window_attn_bwd(const infllmv2_params *prm, int32_t n_sink, int32_t window, const infllmv2_tensor *q,
                                 const infllmv2_tensor *k, const infllmv2_tensor *v, const infllmv2_tensor *out,
                                 const infllmv2_tensor *dout, const float *lse, const int32_t *seqlens, int32_t batch,
                                 int32_t max_seqlen, const infllmv2_tensor *dq, const infllmv2_tensor *dk,
                                 const infllmv2_tensor *dv, void *workspace, size_t workspace_bytes, void *stream) {
    // (its workspace is infllmv2_window_workspace_bytes; where that is 0 the call below has nothing to do or refuses the arguments)
    if (workspace_bytes < infllmv2_window_workspace_bytes(INFLLMV2_OP_WINDOW_BWD, prm, n_sink, window, batch, max_seqlen)) workspace = nullptr;
    return infllmv2i_window_attn_bwd(prm, n_sink, window, q, k, v, out, dout, lse, seqlens, batch, max_seqlen, dq, dk, dv, workspace,
                                     workspace_bytes, stream, 0);
}

int32_t infllmv2_window_attn_decode(const infllmv2_params *prm, int32_t n_sink, int32_t window, const infllmv2_tensor *q,
                                    const infllmv2_tensor *k, const infllmv2_tensor *v, const int32_t *seqlens, int32_t batch,
                                    int32_t max_seqlen, const infllmv2_tensor *out, float *lse, void *workspace,
                                    size_t workspace_bytes, void *stream) {
    RETURN_IF_ERR(check_params(prm));
    RETURN_IF_ERR(check_window(n_sink, window));
    RETURN_IF_ERR(check_sizes(batch, max_seqlen));
    RETURN_IF_ERR(check_capacity(max_seqlen));
    RETURN_IF_ERR(check_tensor(q));
    RETURN_IF_ERR(check_tensor(k));
    RETURN_IF_ERR(check_tensor(v));
    RETURN_IF_ERR(check_tensor(out));
    if (!seqlens || !lse) return INFLLMV2_ERR_INVALID_ARGUMENT;
    const Dims dm = make_dims(prm, batch, max_seqlen);
    const WindowArgs w = make_window(n_sink, window, max_seqlen);
    RETURN_IF_ERR(check_workspace(workspace, workspace_bytes, window_decode_ws_bytes(dm, w)));
    return hip_status(launch_window_decode(dm, w, make_tensor(q), make_tensor(k), make_tensor(v), seqlens, make_tensor(out), lse, workspace,
                                           reinterpret_cast<hipStream_t>(stream)));
}

int32_t infllmv2_window_attn_decode_quant(const infllmv2_params *prm, int32_t n_sink, int32_t window, const infllmv2_tensor *q,
                                          const infllmv2_quant_tensor *kq, const infllmv2_quant_tensor *vq, const int32_t *seqlens,
                                          int32_t batch, int32_t max_seqlen, const infllmv2_tensor *out, float *lse, void *workspace,
                                          size_t workspace_bytes, void *stream) {
    RETURN_IF_ERR(check_params(prm));
    RETURN_IF_ERR(check_window(n_sink, window));
    RETURN_IF_ERR(check_sizes(batch, max_seqlen));
    RETURN_IF_ERR(check_capacity(max_seqlen));
    RETURN_IF_ERR(check_tensor(q));
    RETURN_IF_ERR(check_quant(kq));
    RETURN_IF_ERR(check_quant(vq));
    RETURN_IF_ERR(check_tensor(out));
    if (!seqlens || !lse) return INFLLMV2_ERR_INVALID_ARGUMENT;
    RETURN_IF_ERR(check_rows(kq, vq));
    const Dims dm = make_dims(prm, batch, max_seqlen);
    const WindowArgs w = make_window(n_sink, window, max_seqlen);
    RETURN_IF_ERR(check_workspace(workspace, workspace_bytes, window_decode_ws_bytes(dm, w)));
    return hip_status(launch_window_decode_quant(dm, w, make_tensor(q), make_quant(kq), make_quant(vq), seqlens, make_tensor(out), lse,
                                                 workspace, reinterpret_cast<hipStream_t>(stream)));
}

int32_t infllmv2_rope_table(const infllmv2_rope_config *cfg, uint64_t *steps, float *amplitude) {
    if (!cfg || !steps || !amplitude || cfg->rot_dim <= 0) return INFLLMV2_ERR_INVALID_ARGUMENT;
    if (cfg->rot_dim % 16 || cfg->rot_dim > kHeadDim) return INFLLMV2_ERR_UNSUPPORTED;
    const int kind = cfg->scaling, half = cfg->rot_dim / 2;
    if (kind < INFLLMV2_ROPE_NONE || kind > INFLLMV2_ROPE_FACTORS) return INFLLMV2_ERR_INVALID_ARGUMENT;
    if (!(cfg->base > 1.0) || !isfinite(cfg->base) || !(cfg->amplitude >= 0.0) || !(cfg->amplitude < 1e30)) return INFLLMV2_ERR_INVALID_ARGUMENT;
    if (kind != INFLLMV2_ROPE_NONE && (!(cfg->factor >= 1.0) || !isfinite(cfg->factor))) return INFLLMV2_ERR_INVALID_ARGUMENT;
    const bool trained = kind == INFLLMV2_ROPE_YARN || (kind == INFLLMV2_ROPE_FACTORS && cfg->amplitude == 0.0);
    if (trained && cfg->original_len < 2) return INFLLMV2_ERR_INVALID_ARGUMENT;
    if (kind == INFLLMV2_ROPE_YARN && (!(cfg->beta_fast > cfg->beta_slow) || !(cfg->beta_slow >= 0.0) || !isfinite(cfg->beta_fast)))
        return INFLLMV2_ERR_INVALID_ARGUMENT;
    if (kind == INFLLMV2_ROPE_FACTORS) {
        if (!cfg->pair_factors) return INFLLMV2_ERR_INVALID_ARGUMENT;
        for (int j = 0; j < half; ++j)
            if (!(cfg->pair_factors[j] >= 1e-3) || !isfinite(cfg->pair_factors[j])) return INFLLMV2_ERR_INVALID_ARGUMENT;
    }
    // (in 64-bit mantissas: an angle after 2^31 positions is then exact to 2^-33 turns)
    const long double factor = cfg->factor, two_pi = 6.283185307179586476925286766559L;
    long double base = cfg->base;
    if (kind == INFLLMV2_ROPE_NTK) base *= powl(factor, (long double)cfg->rot_dim / (cfg->rot_dim - 2));
    for (int j = 0; j < half; ++j) {
        long double turns = powl(base, -2.0L * j / cfg->rot_dim) / two_pi;                     // per position
        if (kind == INFLLMV2_ROPE_LINEAR) turns /= factor;
        if (kind == INFLLMV2_ROPE_YARN) {
            long double keep = (cfg->original_len * turns - cfg->beta_slow) / ((long double)cfg->beta_fast - cfg->beta_slow);
            keep = keep < 0.0L ? 0.0L : keep > 1.0L ? 1.0L : keep;
            turns *= keep + (1.0L - keep) / factor;
        }
        if (kind == INFLLMV2_ROPE_FACTORS) turns /= cfg->pair_factors[j];
        turns -= floorl(turns);                          // (a pair factor below 1 / (2 pi) makes it more than one)
        const long double scaled = roundl(ldexpl(turns, 64));
        steps[j] = scaled >= 18446744073709551616.0L ? 0u : (uint64_t)scaled;
    }
    double a = cfg->amplitude;
    if (a == 0.0) {
        a = 1.0;
        if (kind == INFLLMV2_ROPE_YARN) a = 0.1 * log(cfg->factor) + 1.0;
        if (kind == INFLLMV2_ROPE_FACTORS) a = sqrt(1.0 + log(cfg->factor) / log((double)cfg->original_len));
    }
    *amplitude = (float)a;
    return INFLLMV2_OK;
}

int32_t infllmv2i_rope(const infllmv2_params *prm, const infllmv2_rotation *rot, const infllmv2_tensor *q, const infllmv2_tensor *k,
                       const int32_t *positions, const int32_t *seqlens, int32_t batch, int32_t max_seqlen, const infllmv2_tensor *q_out,
                       const infllmv2_tensor *k_out, void *stream, int32_t back, int32_t fill) {
    RETURN_IF_ERR(check_params(prm));
    RETURN_IF_ERR(check_sizes(batch, max_seqlen));
    RETURN_IF_ERR(check_capacity(max_seqlen));
    RETURN_IF_ERR(check_rotation(rot));
    if (!q != !q_out || !k != !k_out || !seqlens) return INFLLMV2_ERR_INVALID_ARGUMENT;
    if (rotate_wavefronts(max_seqlen, (int64_t)prm->n_q_heads + prm->n_kv_heads) > (1ll << 30)) return INFLLMV2_ERR_UNSUPPORTED;
    const infllmv2_tensor *ts[4] = {q, q_out, k, k_out};
    Tensor made[4];
    for (int i = 0; i < 4; ++i) {
        if (!ts[i]) continue;
        RETURN_IF_ERR(check_tensor(ts[i]));
        made[i] = make_tensor(ts[i]);
    }
    return hip_status(launch_rope(make_dims(prm, batch, max_seqlen, 1, fill), make_rotation(rot, back != 0), q ? &made[0] : nullptr, k ? &made[2] : nullptr,
                                  positions, seqlens, q ? &made[1] : nullptr, k ? &made[3] : nullptr, reinterpret_cast<hipStream_t>(stream)));
}

int32_t infllmv2_rope(const infllmv2_params *prm, const infllmv2_rotation *rot, const infllmv2_tensor *q, const infllmv2_tensor *k,
                      const int32_t *positions, const int32_t *seqlens, int32_t batch, int32_t max_seqlen, const infllmv2_tensor *q_out,
                      const infllmv2_tensor *k_out, void *stream) {
    return infllmv2i_rope(prm, rot, q, k, positions, seqlens, batch, max_seqlen, q_out, k_out, stream, 0, 0);
}

int32_t infllmv2_rope_bwd(const infllmv2_params *prm, const infllmv2_rotation *rot, const infllmv2_tensor *dq_out, const infllmv2_tensor *dk_out,
                          const int32_t *positions, const int32_t *seqlens, int32_t batch, int32_t max_seqlen, const infllmv2_tensor *dq,
                          const infllmv2_tensor *dk, void *stream) {
    return infllmv2i_rope(prm, rot, dq_out, dk_out, positions, seqlens, batch, max_seqlen, dq, dk, stream, 1, 0);
}

size_t infllmv2_paged_workspace_bytes(int32_t op, const infllmv2_params *prm, int32_t batch, int32_t max_seqlen, int32_t max_new) {
    if (check_params(prm) != INFLLMV2_OK || check_sizes(batch, max_seqlen) != INFLLMV2_OK || check_capacity(max_seqlen) != INFLLMV2_OK) return 0;
    const Dims dm = make_dims(prm, batch, max_seqlen);
    if (op == INFLLMV2_OP_PAGED_EVICT) return paged_evict_ws_bytes(dm);
    if (check_new(prm, max_new) != INFLLMV2_OK) return 0;
    switch (op) {
        case INFLLMV2_OP_PAGED_ATTN: return paged_attn_ws_bytes(dm, max_new);
        case INFLLMV2_OP_PAGED_WEIGHTS: return paged_weights_ws_bytes(dm, max_new);
    }
    return 0;
}

int32_t infllmv2_paged_append(const infllmv2_params *prm, const infllmv2_rotation *rot, const infllmv2_tensor *k_new, const infllmv2_tensor *v_new,
                              const infllmv2_tensor *q, const infllmv2_pages *pages, const int32_t *positions, const int32_t *n_new,
                              const int32_t *seqlens, int32_t batch, int32_t max_seqlen, int32_t max_new, const infllmv2_tensor *q_out,
                              void *stream) {
    RETURN_IF_ERR(check_params(prm));
    RETURN_IF_ERR(check_sizes(batch, max_seqlen));
    RETURN_IF_ERR(check_capacity(max_seqlen));
    RETURN_IF_ERR(check_new(prm, max_new));
    if (rot) RETURN_IF_ERR(check_rotation(rot));
    RETURN_IF_ERR(check_tensor(k_new));
    RETURN_IF_ERR(check_tensor(v_new));
    RETURN_IF_ERR(check_pages(pages, max_seqlen));
    if (!q != !q_out || (q && !rot) || !seqlens) return INFLLMV2_ERR_INVALID_ARGUMENT;
    Tensor qt, ot;
    if (q) {
        RETURN_IF_ERR(check_tensor(q));
        RETURN_IF_ERR(check_tensor(q_out));
        qt = make_tensor(q);
        ot = make_tensor(q_out);
    }
    return hip_status(launch_paged_append(make_dims(prm, batch, max_seqlen), make_rotation(rot, false), make_tensor(k_new), make_tensor(v_new),
                                          q ? &qt : nullptr, make_pages(pages), positions, NewTokens{n_new, max_new}, seqlens, q ? &ot : nullptr,
                                          reinterpret_cast<hipStream_t>(stream)));
}

int32_t infllmv2i_paged_attn(const infllmv2_params *prm, const infllmv2_tensor *q, const infllmv2_pages *pages, const int32_t *n_new,
                             const int32_t *seqlens, int32_t batch, int32_t max_seqlen, int32_t max_new, const infllmv2_tensor *out, float *lse,
                             void *workspace, size_t workspace_bytes, void *stream, int32_t fill) {
    RETURN_IF_ERR(check_params(prm));
    RETURN_IF_ERR(check_sizes(batch, max_seqlen));
    RETURN_IF_ERR(check_capacity(max_seqlen));
    RETURN_IF_ERR(check_new(prm, max_new));
    RETURN_IF_ERR(check_tensor(q));
    RETURN_IF_ERR(check_pages(pages, max_seqlen));
    RETURN_IF_ERR(check_tensor(out));
    if (!seqlens || !lse) return INFLLMV2_ERR_INVALID_ARGUMENT;
    RETURN_IF_ERR(check_spans(prm, nullptr, nullptr, q, nullptr));
    const Dims dm = make_dims(prm, batch, max_seqlen, 1, fill);
    if (paged_attn_groups(dm, max_new) > (1ll << kLgGroups)) return INFLLMV2_ERR_UNSUPPORTED;
    RETURN_IF_ERR(check_workspace(workspace, workspace_bytes, paged_attn_ws_bytes(dm, max_new)));
    return hip_status(launch_paged_attn(dm, make_tensor(q), make_pages(pages), NewTokens{n_new, max_new}, seqlens, make_tensor(out), lse, workspace,
                                        reinterpret_cast<hipStream_t>(stream)));
}

int32_t infllmv2_paged_attn(const infllmv2_params *prm, const infllmv2_tensor *q, const infllmv2_pages *pages, const int32_t *n_new,
                            const int32_t *seqlens, int32_t batch, int32_t max_seqlen, int32_t max_new, const infllmv2_tensor *out, float *lse,
                            void *workspace, size_t workspace_bytes, void *stream) {
    return infllmv2i_paged_attn(prm, q, pages, n_new, seqlens, batch, max_seqlen, max_new, out, lse, workspace, workspace_bytes, stream, 0);
}

int32_t infllmv2_paged_attn_weights(const infllmv2_params *prm, const infllmv2_tensor *q, const float *lse, const infllmv2_pages *pages,
                                    const int32_t *n_new, const int32_t *seqlens, int32_t batch, int32_t max_seqlen, int32_t max_new,
                                    const float *weights, int32_t weights_pitch, float *weights_out, void *workspace, size_t workspace_bytes,
                                    void *stream) {
    RETURN_IF_ERR(check_params(prm));
    RETURN_IF_ERR(check_sizes(batch, max_seqlen));
    RETURN_IF_ERR(check_capacity(max_seqlen));
    RETURN_IF_ERR(check_new(prm, max_new));
    RETURN_IF_ERR(check_tensor(q));
    RETURN_IF_ERR(check_pages(pages, max_seqlen));
    if (!seqlens || !lse || !weights_out || weights_pitch < max_seqlen) return INFLLMV2_ERR_INVALID_ARGUMENT;
    RETURN_IF_ERR(check_spans(prm, nullptr, nullptr, q, nullptr));
    const Dims dm = make_dims(prm, batch, max_seqlen);
    if (paged_weights_groups(dm) > (1ll << 30)) return INFLLMV2_ERR_UNSUPPORTED;
    RETURN_IF_ERR(check_workspace(workspace, workspace_bytes, paged_weights_ws_bytes(dm, max_new)));
    return hip_status(launch_paged_weights(dm, make_tensor(q), lse, make_pages(pages), NewTokens{n_new, max_new}, seqlens, weights, weights_pitch, weights_out,
                                           workspace, reinterpret_cast<hipStream_t>(stream)));
}

int32_t infllmv2_paged_evict(const infllmv2_params *prm, const float *weights, int32_t weights_pitch, const infllmv2_pages *from,
                             const int32_t *seqlens, int32_t batch, int32_t max_seqlen, int32_t budget, int32_t n_first, int32_t n_recent,
                             const infllmv2_pages *to, int32_t *kept, float *weights_out, int32_t *seqlens_out, void *workspace,
                             size_t workspace_bytes, void *stream) {
    RETURN_IF_ERR(check_params(prm));
    RETURN_IF_ERR(check_sizes(batch, max_seqlen));
    RETURN_IF_ERR(check_capacity(max_seqlen));
    if (budget < 1 || n_first < 0 || n_recent < 0 || (int64_t)n_first + n_recent > budget) return INFLLMV2_ERR_INVALID_ARGUMENT;
    if (budget > (1 << 30) - 64) return INFLLMV2_ERR_UNSUPPORTED;          // (64 of them to a workgroup of 256 threads: the last are kept below 2^32)
    RETURN_IF_ERR(check_pages(from, max_seqlen));
    RETURN_IF_ERR(check_pages(to, budget < max_seqlen ? budget : max_seqlen));
    if (!weights || !seqlens || !kept || !seqlens_out || weights_pitch < max_seqlen) return INFLLMV2_ERR_INVALID_ARGUMENT;
    const Dims dm = make_dims(prm, batch, max_seqlen);
    RETURN_IF_ERR(check_workspace(workspace, workspace_bytes, paged_evict_ws_bytes(dm)));
    return hip_status(launch_paged_evict(dm, weights, weights_pitch, make_pages(from), seqlens, budget, n_first, n_recent, make_pages(to), kept, weights_out,
                                         seqlens_out, workspace, reinterpret_cast<hipStream_t>(stream)));
}

}  // extern "C"
