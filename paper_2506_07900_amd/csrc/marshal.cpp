// Python extension behind binding.py: tensors -> pointers and strides -> one call of the library.
//
// A decode step is 20 us on the GPU; marshalling its arguments in Python (seven descriptors, the stream, the parameter
// block, the size query) took 13 us of host time on top of the launches and bounded an eager step.  Here it is under
// 1 us.  Results the caller did not provide are allocated uninitialised; the library clears the rows its kernels leave
// alone in kernels it launches anyway (internal.h), where torch's fills cost a launch and a pass over memory each.
#include <dlfcn.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <ATen/ATen.h>
#include <c10/hip/HIPStream.h>

#include <algorithm>
#include <stdexcept>
#include <string>

#include "internal.h"

namespace {

struct MarshalError : std::runtime_error {
    using std::runtime_error::runtime_error;
};

PyObject *g_error = nullptr;                              // binding.InfLLMv2Error

// The library binding.py loaded (libinfllmv2.so, its bench build, or another build named by the caller).
struct Library {
#define INFLLMV2_FN(name) decltype(&infllmv2_##name) name = nullptr
#define INFLLMV2_FNI(name) decltype(&infllmv2i_##name) name = nullptr
    INFLLMV2_FN(status_string);
    INFLLMV2_FN(workspace_bytes);
    INFLLMV2_FN(verify_workspace_bytes);
    INFLLMV2_FN(append_kv);
    INFLLMV2_FN(sparse_attn_decode);
    INFLLMV2_FN(decode_step);
    INFLLMV2_FN(append_kv_verify);
    INFLLMV2_FN(select_blocks_verify);
    INFLLMV2_FN(sparse_attn_verify);
    INFLLMV2_FN(verify_step);
    INFLLMV2_FNI(compress_keys);
    INFLLMV2_FNI(select_blocks);
    INFLLMV2_FNI(sparse_attn_prefill);
    INFLLMV2_FNI(sparse_attn_bwd);
    INFLLMV2_FN(append_kv_quant);
    INFLLMV2_FN(sparse_attn_decode_quant);
    INFLLMV2_FN(sparse_attn_verify_quant);
    INFLLMV2_FN(window_workspace_bytes);
    INFLLMV2_FN(window_attn_decode);
    INFLLMV2_FN(window_attn_decode_quant);
    INFLLMV2_FNI(quantize_kv);
    INFLLMV2_FNI(dequantize_kv);
    INFLLMV2_FNI(window_attn_prefill);
    INFLLMV2_FNI(window_attn_bwd);
    INFLLMV2_FNI(window_bwd_scratch_bytes);
#undef INFLLMV2_FN
#undef INFLLMV2_FNI
} lib;

template <typename F>
void symbol(void *handle, const char *name, F &f) {
    f = reinterpret_cast<F>(dlsym(handle, name));
    if (!f) throw MarshalError(std::string("the library does not export ") + name);
}

const at::Tensor &tensor(PyObject *o, const char *name) {
    if (!THPVariable_Check(o)) throw MarshalError(std::string(name) + " must be a tensor");
    return THPVariable_Unpack(o);
}

const at::Tensor &bf16_4d(PyObject *o, const char *name) {
    if (!THPVariable_Check(o)) throw MarshalError(std::string(name) + " must be a 4-d bf16 device tensor");
    const at::Tensor &t = THPVariable_Unpack(o);
    if (!t.is_cuda() || t.scalar_type() != at::kBFloat16 || t.dim() != 4)
        throw MarshalError(std::string(name) + " must be a 4-d bf16 device tensor");
    if (t.stride(3) != 1) throw MarshalError(std::string(name) + ": head_dim axis must be contiguous");
    return t;
}

// caches, compressed keys, new rows: [B, Hkv, T, d]
infllmv2_tensor cache(const at::Tensor &t) { return {t.data_ptr(), t.stride(0), t.stride(1), t.stride(2)}; }
infllmv2_tensor cache(PyObject *o, const char *name) { return cache(bf16_4d(o, name)); }
// queries, outputs: [B, T, Hq, d]
infllmv2_tensor rows(const at::Tensor &t) { return {t.data_ptr(), t.stride(0), t.stride(2), t.stride(1)}; }
infllmv2_tensor rows(PyObject *o, const char *name) { return rows(bf16_4d(o, name)); }

int32_t *i32(PyObject *o, const char *name) {
    if (THPVariable_Check(o)) {
        const at::Tensor &t = THPVariable_Unpack(o);
        if (t.is_cuda() && t.scalar_type() == at::kInt && t.is_contiguous()) return static_cast<int32_t *>(t.data_ptr());
    }
    throw MarshalError(std::string(name) + " must be a contiguous int32 device tensor");
}

int32_t integer(PyObject *o) {
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw python_error();
    if (v != static_cast<int32_t>(v)) throw MarshalError("an integer argument does not fit 32 bits");
    return static_cast<int32_t>(v);
}

const infllmv2_params *params(PyObject *o) {
    if (!PyBytes_Check(o) || PyBytes_GET_SIZE(o) != static_cast<Py_ssize_t>(sizeof(infllmv2_params)))
        throw MarshalError("prm must be the packed parameter block");
    return reinterpret_cast<const infllmv2_params *>(PyBytes_AS_STRING(o));
}

void *current_stream() { return c10::hip::getCurrentHIPStream().stream(); }

// A result: the caller's tensor, or one made here.
struct Result {
    PyObject *given;
    at::Tensor own;
    explicit Result(PyObject *o) : given(o == Py_None ? nullptr : o) {}
    bool make() const { return given == nullptr; }
    PyObject *release() {
        if (!given) return THPVariable_Wrap(std::move(own));
        Py_INCREF(given);
        return given;
    }
};

// The kernels write every row of a tensor shaped like q (like k): it has no heads or channels beyond the parameters'.
bool q_shaped(const at::Tensor &q, const infllmv2_params *prm) { return q.size(2) == prm->n_q_heads && q.size(3) == prm->head_dim; }
bool k_shaped(const at::Tensor &k, const infllmv2_params *prm) { return k.size(1) == prm->n_kv_heads && k.size(3) == prm->head_dim; }

at::TensorOptions like(const at::Tensor &t, at::ScalarType type) { return at::TensorOptions().dtype(type).device(t.device()); }

// The caller's workspace, or scratch that lives until the call has been enqueued (the allocator reuses it in stream order).
struct Workspace {
    at::Tensor t;
    void *ptr;
    size_t bytes;
    Workspace(PyObject *o, size_t need, const at::Tensor &device_of) {
        t = o == Py_None ? at::empty({static_cast<int64_t>(std::max<size_t>(need, 256))}, like(device_of, at::kByte))
                         : tensor(o, "workspace");
        ptr = t.data_ptr();
        bytes = static_cast<size_t>(t.numel()) * t.element_size();
    }
};

template <typename F>
void run(const char *what, F f) {                         // without the interpreter lock, as any foreign call
    int32_t status;
    Py_BEGIN_ALLOW_THREADS
    status = f();
    Py_END_ALLOW_THREADS
    if (status != INFLLMV2_OK)
        throw MarshalError(std::string(what) + " failed: " + lib.status_string(status) + " (" + std::to_string(status) + ")");
}

PyObject *tuple2(Result &a, Result &b) {
    PyObject *r = PyTuple_New(2);
    PyTuple_SET_ITEM(r, 0, a.release());
    PyTuple_SET_ITEM(r, 1, b.release());
    return r;
}
PyObject *tuple3(Result &a, Result &b, Result &c) {
    PyObject *r = PyTuple_New(3);
    PyTuple_SET_ITEM(r, 0, a.release());
    PyTuple_SET_ITEM(r, 1, b.release());
    PyTuple_SET_ITEM(r, 2, c.release());
    return r;
}

using Args = PyObject *const *;

// (prm, k, seqlens, max_seqlen, ck | None, n_new_tokens)
PyObject *compress_keys(Args a) {
    const infllmv2_params *prm = params(a[0]);
    const at::Tensor &k = bf16_4d(a[1], "k");
    const int32_t T = integer(a[3]), n_new = integer(a[5]);
    Result ck(a[4]);
    int32_t fill = 0;
    if (ck.make()) {
        const bool kernels = prm->kernel_size > 0 && prm->kernel_stride > 0 && T >= prm->kernel_size;   // (the library refuses the rest)
        const int64_t n = kernels ? (T - prm->kernel_size) / prm->kernel_stride + 1 : 0;
        const at::IntArrayRef::value_type shape[4] = {k.size(0), k.size(1), std::max<int64_t>(n, 1), k.size(3)};
        fill = n > 0 && n_new <= 0 && k_shaped(k, prm);   // otherwise the kernel does not visit every row
        ck.own = fill ? at::empty(shape, like(k, at::kBFloat16)) : at::zeros(shape, like(k, at::kBFloat16));
    }
    const infllmv2_tensor kd = cache(k), cd = ck.make() ? cache(ck.own) : cache(ck.given, "ck");
    const int32_t *sl = i32(a[2], "seqlens");
    const int32_t B = static_cast<int32_t>(k.size(0));
    run("infllmv2_compress_keys", [&] { return lib.compress_keys(prm, &kd, sl, B, T, n_new, &cd, current_stream(), fill); });
    return ck.release();
}

// (prm, k_new, v_new, k, v, seqlens, max_seqlen, ck | None)
PyObject *append_kv(Args a) {
    const infllmv2_params *prm = params(a[0]);
    const infllmv2_tensor kn = cache(a[1], "k_new"), vn = cache(a[2], "v_new"), k = cache(a[3], "k"), v = cache(a[4], "v");
    infllmv2_tensor ck{};
    if (a[7] != Py_None) ck = cache(a[7], "ck");
    const int32_t *sl = i32(a[5], "seqlens");
    const int32_t T = integer(a[6]), B = static_cast<int32_t>(tensor(a[3], "k").size(0));
    run("infllmv2_append_kv", [&] {
        return lib.append_kv(prm, &kn, &vn, &k, &v, a[7] != Py_None ? &ck : nullptr, sl, B, T, current_stream());
    });
    Py_RETURN_NONE;
}

// (prm, k_new, v_new, k, v, seqlens, max_seqlen, ck | None)
PyObject *append_kv_verify(Args a) {
    const infllmv2_params *prm = params(a[0]);
    const infllmv2_tensor kn = cache(a[1], "k_new"), vn = cache(a[2], "v_new"), k = cache(a[3], "k"), v = cache(a[4], "v");
    infllmv2_tensor ck{};
    if (a[7] != Py_None) ck = cache(a[7], "ck");
    const int32_t *sl = i32(a[5], "seqlens");
    const int32_t T = integer(a[6]), B = static_cast<int32_t>(tensor(a[3], "k").size(0));
    const int32_t n = static_cast<int32_t>(tensor(a[1], "k_new").size(2));
    run("infllmv2_append_kv_verify", [&] {
        return lib.append_kv_verify(prm, &kn, &vn, &k, &v, a[7] != Py_None ? &ck : nullptr, sl, B, T, n, current_stream());
    });
    Py_RETURN_NONE;
}

// (prm, mode, q, ck, seqlens, max_seqlen, block_idx | None, workspace | None)
PyObject *select_blocks(Args a) {
    const infllmv2_params *prm = params(a[0]);
    const int32_t mode = integer(a[1]), T = integer(a[5]);
    const at::Tensor &q = bf16_4d(a[2], "q");
    const int32_t B = static_cast<int32_t>(q.size(0));
    const bool prefill = mode == INFLLMV2_MODE_PREFILL;
    Result idx(a[6]);
    if (idx.make())                                       // (a decode row is written whole)
        idx.own = at::empty({B, prm->n_kv_heads, prefill ? T : 1, prm->topk}, like(q, at::kInt));
    const int32_t op = prefill ? INFLLMV2_OP_SELECT_PREFILL : INFLLMV2_OP_SELECT_DECODE;
    const Workspace ws(a[7], a[7] == Py_None ? lib.workspace_bytes(op, prm, B, T) : 0, q);
    const infllmv2_tensor qd = rows(q), cd = cache(a[3], "ck");
    const int32_t *sl = i32(a[4], "seqlens");
    int32_t *ip = idx.make() ? static_cast<int32_t *>(idx.own.data_ptr()) : i32(idx.given, "block_idx");
    const int32_t fill = idx.make();
    run("infllmv2_select_blocks",
        [&] { return lib.select_blocks(prm, mode, &qd, &cd, sl, B, T, ip, ws.ptr, ws.bytes, current_stream(), fill); });
    return idx.release();
}

// (prm, q, ck, seqlens, max_seqlen, block_idx | None, workspace | None)
PyObject *select_blocks_verify(Args a) {
    const infllmv2_params *prm = params(a[0]);
    const at::Tensor &q = bf16_4d(a[1], "q");
    const int32_t T = integer(a[4]), B = static_cast<int32_t>(q.size(0)), n = static_cast<int32_t>(q.size(1));
    Result idx(a[5]);
    if (idx.make()) idx.own = at::empty({B, prm->n_kv_heads, n, prm->topk}, like(q, at::kInt));   // every row is written whole
    const Workspace ws(a[6], a[6] == Py_None ? lib.verify_workspace_bytes(INFLLMV2_OP_SELECT_VERIFY, prm, B, T, n) : 0, q);
    const infllmv2_tensor qd = rows(q), cd = cache(a[2], "ck");
    const int32_t *sl = i32(a[3], "seqlens");
    int32_t *ip = idx.make() ? static_cast<int32_t *>(idx.own.data_ptr()) : i32(idx.given, "block_idx");
    run("infllmv2_select_blocks_verify",
        [&] { return lib.select_blocks_verify(prm, &qd, &cd, sl, B, T, n, ip, ws.ptr, ws.bytes, current_stream()); });
    return idx.release();
}

// (prm, q, k, v, seqlens, max_seqlen, block_idx, out | None, lse | None, workspace | None)
PyObject *sparse_attn_prefill(Args a) {
    const infllmv2_params *prm = params(a[0]);
    const at::Tensor &q = bf16_4d(a[1], "q");
    const int32_t T = integer(a[5]), B = static_cast<int32_t>(q.size(0));
    Result out(a[7]), lse(a[8]);
    // the call clears rows up to max_seqlen: only where `out`, shaped like q, has just those.  Rows past max_seqlen of a longer
    // tensor, a tensor shorter than max_seqlen, and a tensor next to one of the caller's (whose other rows stay as they
    // are), are cleared by torch
    const bool fill = out.make() && lse.make() && q.size(1) == T && q_shaped(q, prm);
    if (out.make()) out.own = fill ? at::empty_like(q) : at::zeros_like(q);
    if (lse.make())
        lse.own = fill ? at::empty({B, T, prm->n_q_heads}, like(q, at::kFloat)) : at::zeros({B, T, prm->n_q_heads}, like(q, at::kFloat));
    const Workspace ws(a[9], a[9] == Py_None ? lib.workspace_bytes(INFLLMV2_OP_ATTN_PREFILL, prm, B, T) : 0, q);
    const infllmv2_tensor qd = rows(q), kd = cache(a[2], "k"), vd = cache(a[3], "v"),
                          od = out.make() ? rows(out.own) : rows(out.given, "out");
    const int32_t *sl = i32(a[4], "seqlens"), *ip = i32(a[6], "block_idx");
    float *lp = static_cast<float *>((lse.make() ? lse.own : tensor(lse.given, "lse")).data_ptr());
    run("infllmv2_sparse_attn_prefill", [&] {
        return lib.sparse_attn_prefill(prm, &qd, &kd, &vd, sl, B, T, ip, &od, lp, ws.ptr, ws.bytes, current_stream(), fill);
    });
    return tuple2(out, lse);
}

// (prm, q, k, v, seqlens, max_seqlen, block_idx, out | None, lse | None, workspace | None)
PyObject *sparse_attn_decode(Args a) {
    const infllmv2_params *prm = params(a[0]);
    const at::Tensor &q = bf16_4d(a[1], "q");
    const int32_t T = integer(a[5]), B = static_cast<int32_t>(q.size(0));
    Result out(a[7]), lse(a[8]);
    if (out.make()) out.own = q.size(1) == 1 && q_shaped(q, prm) ? at::empty_like(q) : at::zeros_like(q);           // (every row is written)
    if (lse.make()) lse.own = at::empty({B, prm->n_q_heads}, like(q, at::kFloat));
    const Workspace ws(a[9], a[9] == Py_None ? lib.workspace_bytes(INFLLMV2_OP_ATTN_DECODE, prm, B, T) : 0, q);
    const infllmv2_tensor qd = rows(q), kd = cache(a[2], "k"), vd = cache(a[3], "v"),
                          od = out.make() ? rows(out.own) : rows(out.given, "out");
    const int32_t *sl = i32(a[4], "seqlens"), *ip = i32(a[6], "block_idx");
    float *lp = static_cast<float *>((lse.make() ? lse.own : tensor(lse.given, "lse")).data_ptr());
    run("infllmv2_sparse_attn_decode",
        [&] { return lib.sparse_attn_decode(prm, &qd, &kd, &vd, sl, B, T, ip, &od, lp, ws.ptr, ws.bytes, current_stream()); });
    return tuple2(out, lse);
}

const uint64_t *tree_mask(PyObject *o, int64_t B, int64_t n) {
    if (o == Py_None) return nullptr;
    if (THPVariable_Check(o)) {
        const at::Tensor &t = THPVariable_Unpack(o);
        if (t.is_cuda() && t.scalar_type() == at::kLong && t.is_contiguous() && t.dim() == 2 && t.size(0) == B && t.size(1) == n)
            return static_cast<const uint64_t *>(t.data_ptr());
    }
    throw MarshalError("tree_mask must be a contiguous int64 device tensor [B, n_draft]");
}

// (prm, q, k, v, seqlens, max_seqlen, block_idx, tree_mask | None, out | None, lse | None, workspace | None)
PyObject *sparse_attn_verify(Args a) {
    const infllmv2_params *prm = params(a[0]);
    const at::Tensor &q = bf16_4d(a[1], "q");
    const int32_t T = integer(a[5]), B = static_cast<int32_t>(q.size(0)), n = static_cast<int32_t>(q.size(1));
    Result out(a[8]), lse(a[9]);
    if (out.make()) out.own = q_shaped(q, prm) ? at::empty_like(q) : at::zeros_like(q);
    if (lse.make()) lse.own = at::empty({B, n, prm->n_q_heads}, like(q, at::kFloat));
    const uint64_t *mask = tree_mask(a[7], B, n);
    const Workspace ws(a[10], a[10] == Py_None ? lib.verify_workspace_bytes(INFLLMV2_OP_ATTN_VERIFY, prm, B, T, n) : 0, q);
    const infllmv2_tensor qd = rows(q), kd = cache(a[2], "k"), vd = cache(a[3], "v"),
                          od = out.make() ? rows(out.own) : rows(out.given, "out");
    const int32_t *sl = i32(a[4], "seqlens"), *ip = i32(a[6], "block_idx");
    float *lp = static_cast<float *>((lse.make() ? lse.own : tensor(lse.given, "lse")).data_ptr());
    run("infllmv2_sparse_attn_verify", [&] {
        return lib.sparse_attn_verify(prm, &qd, &kd, &vd, sl, B, T, n, mask, ip, &od, lp, ws.ptr, ws.bytes, current_stream());
    });
    return tuple2(out, lse);
}

// (prm, q, k_new, v_new, k, v, ck, seqlens, max_seqlen, block_idx | None, out | None, lse | None, workspace | None)
PyObject *decode_step(Args a) {
    const infllmv2_params *prm = params(a[0]);
    const at::Tensor &q = bf16_4d(a[1], "q");
    const int32_t T = integer(a[8]), B = static_cast<int32_t>(q.size(0));
    Result idx(a[9]), out(a[10]), lse(a[11]);             // every row of every result is written
    if (idx.make()) idx.own = at::empty({B, prm->n_kv_heads, 1, prm->topk}, like(q, at::kInt));
    if (out.make()) out.own = q.size(1) == 1 && q_shaped(q, prm) ? at::empty_like(q) : at::zeros_like(q);
    if (lse.make()) lse.own = at::empty({B, prm->n_q_heads}, like(q, at::kFloat));
    const Workspace ws(a[12], a[12] == Py_None ? lib.workspace_bytes(INFLLMV2_OP_DECODE_STEP, prm, B, T) : 0, q);
    const infllmv2_tensor qd = rows(q), kn = cache(a[2], "k_new"), vn = cache(a[3], "v_new"), k = cache(a[4], "k"),
                          v = cache(a[5], "v"), ck = cache(a[6], "ck"), od = out.make() ? rows(out.own) : rows(out.given, "out");
    const int32_t *sl = i32(a[7], "seqlens");
    int32_t *ip = idx.make() ? static_cast<int32_t *>(idx.own.data_ptr()) : i32(idx.given, "block_idx");
    float *lp = static_cast<float *>((lse.make() ? lse.own : tensor(lse.given, "lse")).data_ptr());
    run("infllmv2_decode_step", [&] {
        return lib.decode_step(prm, &qd, &kn, &vn, &k, &v, &ck, sl, B, T, ip, &od, lp, ws.ptr, ws.bytes, current_stream());
    });
    return tuple3(idx, out, lse);
}

// (prm, q, k_new, v_new, k, v, ck, seqlens, max_seqlen, tree_mask | None, block_idx | None, out | None, lse | None,
//  workspace | None)
PyObject *verify_step(Args a) {
    const infllmv2_params *prm = params(a[0]);
    const at::Tensor &q = bf16_4d(a[1], "q");
    const int32_t T = integer(a[8]), B = static_cast<int32_t>(q.size(0)), n = static_cast<int32_t>(q.size(1));
    Result idx(a[10]), out(a[11]), lse(a[12]);            // every row of every result is written
    if (idx.make()) idx.own = at::empty({B, prm->n_kv_heads, n, prm->topk}, like(q, at::kInt));
    if (out.make()) out.own = q_shaped(q, prm) ? at::empty_like(q) : at::zeros_like(q);
    if (lse.make()) lse.own = at::empty({B, n, prm->n_q_heads}, like(q, at::kFloat));
    const uint64_t *mask = tree_mask(a[9], B, n);
    const Workspace ws(a[13], a[13] == Py_None ? lib.verify_workspace_bytes(INFLLMV2_OP_VERIFY_STEP, prm, B, T, n) : 0, q);
    const infllmv2_tensor qd = rows(q), kn = cache(a[2], "k_new"), vn = cache(a[3], "v_new"), k = cache(a[4], "k"),
                          v = cache(a[5], "v"), ck = cache(a[6], "ck"), od = out.make() ? rows(out.own) : rows(out.given, "out");
    const int32_t *sl = i32(a[7], "seqlens");
    int32_t *ip = idx.make() ? static_cast<int32_t *>(idx.own.data_ptr()) : i32(idx.given, "block_idx");
    float *lp = static_cast<float *>((lse.make() ? lse.own : tensor(lse.given, "lse")).data_ptr());
    run("infllmv2_verify_step", [&] {
        return lib.verify_step(prm, &qd, &kn, &vn, &k, &v, &ck, sl, B, T, n, mask, ip, &od, lp, ws.ptr, ws.bytes, current_stream());
    });
    return tuple3(idx, out, lse);
}

// (prm, q, k, v, out, dout, lse, seqlens, max_seqlen, block_idx, dq | None, dk | None, dv | None, workspace | None)
PyObject *sparse_attn_bwd(Args a) {
    const infllmv2_params *prm = params(a[0]);
    const at::Tensor &q = bf16_4d(a[1], "q"), &k = bf16_4d(a[2], "k"), &v = bf16_4d(a[3], "v");
    const int32_t T = integer(a[8]), B = static_cast<int32_t>(q.size(0));
    Result dq(a[10]), dk(a[11]), dv(a[12]);
    const bool fill = dq.make() && dk.make() && dv.make() && q.size(1) == T && k.size(2) == T && v.size(2) == T && q_shaped(q, prm) &&
                      k_shaped(k, prm) && k_shaped(v, prm) && k.size(0) == B && v.size(0) == B;   // (as for sparse_attn_prefill)
    if (dq.make()) dq.own = fill ? at::empty_like(q) : at::zeros_like(q);
    if (dk.make()) dk.own = fill ? at::empty_like(k) : at::zeros_like(k);
    if (dv.make()) dv.own = fill ? at::empty_like(v) : at::zeros_like(v);
    const Workspace ws(a[13], a[13] == Py_None ? lib.workspace_bytes(INFLLMV2_OP_ATTN_BWD, prm, B, T) : 0, q);
    const infllmv2_tensor qd = rows(q), kd = cache(k), vd = cache(v), od = rows(a[4], "out"), gd = rows(a[5], "dout"),
                          dqd = dq.make() ? rows(dq.own) : rows(dq.given, "dq"),
                          dkd = dk.make() ? cache(dk.own) : cache(dk.given, "dk"),
                          dvd = dv.make() ? cache(dv.own) : cache(dv.given, "dv");
    const at::Tensor &lse = tensor(a[6], "lse");
    if (!lse.is_cuda() || lse.scalar_type() != at::kFloat || !lse.is_contiguous())
        throw MarshalError("lse must be a contiguous fp32 device tensor");
    const float *lp = static_cast<const float *>(lse.data_ptr());
    const int32_t *sl = i32(a[7], "seqlens"), *ip = i32(a[9], "block_idx");
    run("infllmv2_sparse_attn_bwd", [&] {
        return lib.sparse_attn_bwd(prm, &qd, &kd, &vd, &od, &gd, lp, sl, B, T, ip, &dqd, &dkd, &dvd, ws.ptr, ws.bytes,
                                   current_stream(), fill);
    });
    return tuple3(dq, dk, dv);
}

// ---- the 4-bit cache and the windowed attention -------------------------------------------------------------------------
// These calls check shapes and devices as well: a tensor has the sizes that the library takes it to have and lies on
// the current device, whose stream the call goes to.
void expect(bool ok, const char *name, const char *what) {
    if (!ok) throw MarshalError(std::string(name) + what);
}
// the current device, asked for once in a call (asking costs as much as all other checks of a tensor)
thread_local int device_now;
const infllmv2_params *enter(PyObject *prm) {
    device_now = -1;
    return params(prm);
}
void here(const at::Tensor &t, const char *name) {
    if (t.is_cuda() && device_now < 0) device_now = c10::hip::getCurrentHIPStream().device_index();
    expect(t.is_cuda() && t.device().index() == device_now, name, " must be on the current device");
}
const at::Tensor &query(PyObject *o, const char *name, int64_t B, int64_t T, const infllmv2_params *prm) {       // B < 0: any
    const at::Tensor &t = bf16_4d(o, name);
    here(t, name);
    expect((B < 0 || t.size(0) == B) && t.size(1) >= T && q_shaped(t, prm), name, " must be [batch, tokens, n_q_heads, head_dim]");
    return t;
}
const at::Tensor &kv(PyObject *o, const char *name, int64_t B, int64_t T, const infllmv2_params *prm) {
    const at::Tensor &t = bf16_4d(o, name);
    here(t, name);
    expect((B < 0 || t.size(0) == B) && t.size(2) >= T && k_shaped(t, prm), name, " must be [batch, n_kv_heads, tokens, head_dim]");
    return t;
}
// (codes uint8 [B, Hkv, T, d / 2], scales uint8 [B, Hkv, T, d / 32])
infllmv2_quant_tensor quant(const at::Tensor &codes, const at::Tensor &scales) {
    return {codes.data_ptr(), scales.data_ptr(), codes.stride(0), codes.stride(1), codes.stride(2), scales.stride(0), scales.stride(1), scales.stride(2)};
}
infllmv2_quant_tensor quant(PyObject *o, const char *name, int64_t B, int64_t T, const infllmv2_params *prm, int64_t *batch = nullptr) {
    expect(PyTuple_Check(o) && PyTuple_GET_SIZE(o) == 2, name, " must be a pair (codes, scales)");
    const at::Tensor &codes = tensor(PyTuple_GET_ITEM(o, 0), name), &scales = tensor(PyTuple_GET_ITEM(o, 1), name);
    const at::Tensor *ts[2] = {&codes, &scales};
    for (int i = 0; i < 2; ++i) {
        const at::Tensor &t = *ts[i];
        expect(t.scalar_type() == at::kByte && t.dim() == 4 && t.stride(3) == 1, name, ": codes and scales must be 4-d uint8 tensors with a contiguous last axis");
        here(t, name);
        expect((B < 0 || t.size(0) == B) && t.size(1) == prm->n_kv_heads && t.size(2) >= T && t.size(3) == prm->head_dim / (i ? 32 : 2), name,
               " must be codes [batch, n_kv_heads, tokens, head_dim / 2], scales [batch, n_kv_heads, tokens, head_dim / 32]");
    }
    expect(codes.size(0) == scales.size(0), name, ": codes and scales differ in batch");
    if (batch) *batch = codes.size(0);
    return quant(codes, scales);
}
const int32_t *lengths(PyObject *o, int64_t B) {
    const int32_t *p = i32(o, "seqlens");
    here(THPVariable_Unpack(o), "seqlens");
    expect(THPVariable_Unpack(o).numel() == B, "seqlens", " must be [batch]");
    return p;
}
float *lse_of(const at::Tensor &t, int64_t n) {
    here(t, "lse");
    expect(t.scalar_type() == at::kFloat && t.is_contiguous() && t.numel() == n, "lse", " must be a contiguous fp32 device tensor of a value per row and head");
    return static_cast<float *>(t.data_ptr());
}
const int32_t *blocks(PyObject *o, int64_t n) {
    const int32_t *p = i32(o, "block_idx");
    here(THPVariable_Unpack(o), "block_idx");
    expect(THPVariable_Unpack(o).numel() == n, "block_idx", " must be [batch, n_kv_heads, queries, topk]");
    return p;
}
Workspace scratch(PyObject *o, size_t need, const at::Tensor &device_of) {
    if (o != Py_None) {
        here(tensor(o, "workspace"), "workspace");
        expect(tensor(o, "workspace").is_contiguous(), "workspace", " must be contiguous");
    }
    return Workspace(o, need, device_of);
}
// out and lse of an attention call: the caller's, or made here
struct Attended {
    Result out, lse;
    infllmv2_tensor od;
    float *lp;
    int32_t fill;
    Attended(PyObject *o, PyObject *l, const at::Tensor &q, int64_t T, at::IntArrayRef lse_shape, bool may_fill, const infllmv2_params *prm)
        : out(o), lse(l), fill(may_fill && out.make() && lse.make() && q.size(1) == T) {
        const bool whole = fill || (!may_fill && q.size(1) == T);        // every row is written
        int64_t n = 1;
        for (const int64_t x : lse_shape) n *= x;
        if (out.make()) out.own = whole ? at::empty_like(q) : at::zeros_like(q);
        if (lse.make()) lse.own = whole ? at::empty(lse_shape, like(q, at::kFloat)) : at::zeros(lse_shape, like(q, at::kFloat));
        od = rows(out.make() ? out.own : query(out.given, "out", q.size(0), T, prm));
        lp = lse_of(lse.make() ? lse.own : tensor(lse.given, "lse"), n);
    }
};
int32_t capacity(PyObject *o) {
    const int32_t T = integer(o);
    expect(T >= 0, "max_seqlen", " must not be negative");
    return T;
}

// (prm, k, v, seqlens, max_seqlen, (kq, vq) | None, n_new_tokens, QuantCache) -> (kq, vq)
PyObject *quantize_kv(Args a) {
    const infllmv2_params *prm = enter(a[0]);
    const int32_t T = capacity(a[4]), n_new = integer(a[6]);
    const at::Tensor &k = kv(a[1], "k", -1, T, prm), &v = kv(a[2], "v", k.size(0), T, prm);
    const int64_t B = k.size(0);
    const bool make = a[5] == Py_None;
    const int32_t fill = make && n_new <= 0 && k.size(2) == T;      // the call clears the rows behind a sequence itself
    at::Tensor own[4];                                    // codes and scales of K, of V
    infllmv2_quant_tensor kq, vq;
    if (make) {
        for (int i = 0; i < 4; ++i) {
            const at::IntArrayRef::value_type shape[4] = {B, k.size(1), k.size(2), k.size(3) / (i & 1 ? 32 : 2)};
            own[i] = fill ? at::empty(shape, like(k, at::kByte)) : at::zeros(shape, like(k, at::kByte));
        }
        kq = quant(own[0], own[1]);
        vq = quant(own[2], own[3]);
    } else {
        expect(PyTuple_Check(a[5]) && PyTuple_GET_SIZE(a[5]) == 2, "kq, vq", " must both be given");
        kq = quant(PyTuple_GET_ITEM(a[5], 0), "kq", B, T, prm);
        vq = quant(PyTuple_GET_ITEM(a[5], 1), "vq", B, T, prm);
    }
    const infllmv2_tensor kd = cache(k), vd = cache(v);
    const int32_t *sl = lengths(a[3], B);
    run("infllmv2_quantize_kv",
        [&] { return lib.quantize_kv(prm, &kd, &vd, sl, static_cast<int32_t>(B), T, n_new, &kq, &vq, current_stream(), fill); });
    if (!make) {
        Py_INCREF(a[5]);
        return a[5];
    }
    PyObject *r = PyTuple_New(2);
    for (int i = 0; i < 2; ++i) {                         // (codes, scales) twice, as binding.QuantCache
        PyObject *codes = THPVariable_Wrap(own[2 * i]), *scales = THPVariable_Wrap(own[2 * i + 1]);
        PyObject *pair = PyObject_CallFunctionObjArgs(a[7], codes, scales, nullptr);
        Py_DECREF(codes);
        Py_DECREF(scales);
        if (!pair) {
            Py_DECREF(r);
            throw python_error();
        }
        PyTuple_SET_ITEM(r, i, pair);
    }
    return r;
}

// (prm, kq, vq, seqlens, max_seqlen, k | None, v | None, n_new_tokens)
PyObject *dequantize_kv(Args a) {
    const infllmv2_params *prm = enter(a[0]);
    const int32_t T = capacity(a[4]), n_new = integer(a[7]);
    int64_t B;
    const infllmv2_quant_tensor kq = quant(a[1], "kq", -1, T, prm, &B), vq = quant(a[2], "vq", B, T, prm);
    Result k(a[5]), v(a[6]);
    const int32_t fill = k.make() && v.make() && n_new <= 0;
    const at::IntArrayRef::value_type shape[4] = {B, prm->n_kv_heads, T, prm->head_dim};
    const at::Tensor &codes = THPVariable_Unpack(PyTuple_GET_ITEM(a[1], 0));
    for (Result *r : {&k, &v})
        if (r->make()) r->own = fill ? at::empty(shape, like(codes, at::kBFloat16)) : at::zeros(shape, like(codes, at::kBFloat16));
    const infllmv2_tensor kd = cache(k.make() ? k.own : kv(k.given, "k", B, T, prm)), vd = cache(v.make() ? v.own : kv(v.given, "v", B, T, prm));
    const int32_t *sl = lengths(a[3], B);
    run("infllmv2_dequantize_kv",
        [&] { return lib.dequantize_kv(prm, &kq, &vq, sl, static_cast<int32_t>(B), T, n_new, &kd, &vd, current_stream(), fill); });
    return tuple2(k, v);
}

// (prm, k_new, v_new, kq, vq, seqlens, max_seqlen, ck | None)
PyObject *append_kv_quant(Args a) {
    const infllmv2_params *prm = enter(a[0]);
    const int32_t T = capacity(a[6]);
    const at::Tensor &kn = kv(a[1], "k_new", -1, 0, prm);
    const int64_t B = kn.size(0), n = kn.size(2);
    const at::Tensor &vn = kv(a[2], "v_new", B, n, prm);
    expect(vn.size(2) == n, "v_new", " must have the rows of k_new");
    const infllmv2_quant_tensor kq = quant(a[3], "kq", B, T, prm), vq = quant(a[4], "vq", B, T, prm);
    infllmv2_tensor ck{};
    if (a[7] != Py_None) {
        const bool some = prm->kernel_size > 0 && prm->kernel_stride > 0 && T >= prm->kernel_size;
        ck = cache(kv(a[7], "ck", B, some ? (T - prm->kernel_size) / prm->kernel_stride + 1 : 0, prm));
    }
    const infllmv2_tensor knd = cache(kn), vnd = cache(vn);
    const int32_t *sl = lengths(a[5], B);
    run("infllmv2_append_kv_quant", [&] {
        return lib.append_kv_quant(prm, &knd, &vnd, &kq, &vq, a[7] != Py_None ? &ck : nullptr, sl, static_cast<int32_t>(B), T,
                                   static_cast<int32_t>(n), current_stream());
    });
    Py_RETURN_NONE;
}

// (prm, q, kq, vq, seqlens, max_seqlen, block_idx, out | None, lse | None, workspace | None)
PyObject *sparse_attn_decode_quant(Args a) {
    const infllmv2_params *prm = enter(a[0]);
    const int32_t T = capacity(a[5]);
    const at::Tensor &q = query(a[1], "q", -1, 1, prm);
    expect(q.size(1) == 1, "q", " must have one row per sequence");
    const int32_t B = static_cast<int32_t>(q.size(0));
    const infllmv2_quant_tensor kq = quant(a[2], "kq", B, T, prm), vq = quant(a[3], "vq", B, T, prm);
    const int32_t *sl = lengths(a[4], B), *ip = blocks(a[6], static_cast<int64_t>(B) * prm->n_kv_heads * prm->topk);
    Attended r(a[7], a[8], q, 1, {B, prm->n_q_heads}, false, prm);
    const Workspace ws = scratch(a[9], a[9] == Py_None ? lib.workspace_bytes(INFLLMV2_OP_ATTN_DECODE, prm, B, T) : 0, q);
    const infllmv2_tensor qd = rows(q);
    run("infllmv2_sparse_attn_decode_quant", [&] {
        return lib.sparse_attn_decode_quant(prm, &qd, &kq, &vq, sl, B, T, ip, &r.od, r.lp, ws.ptr, ws.bytes, current_stream());
    });
    return tuple2(r.out, r.lse);
}

// (prm, q, kq, vq, seqlens, max_seqlen, block_idx, tree_mask | None, out | None, lse | None, workspace | None)
PyObject *sparse_attn_verify_quant(Args a) {
    const infllmv2_params *prm = enter(a[0]);
    const int32_t T = capacity(a[5]);
    const at::Tensor &q = query(a[1], "q", -1, 1, prm);
    const int32_t B = static_cast<int32_t>(q.size(0)), n = static_cast<int32_t>(q.size(1));
    const infllmv2_quant_tensor kq = quant(a[2], "kq", B, T, prm), vq = quant(a[3], "vq", B, T, prm);
    const int32_t *sl = lengths(a[4], B), *ip = blocks(a[6], static_cast<int64_t>(B) * prm->n_kv_heads * n * prm->topk);
    const uint64_t *mask = tree_mask(a[7], B, n);
    if (mask) here(tensor(a[7], "tree_mask"), "tree_mask");
    Attended r(a[8], a[9], q, n, {B, n, prm->n_q_heads}, false, prm);
    const Workspace ws = scratch(a[10], a[10] == Py_None ? lib.verify_workspace_bytes(INFLLMV2_OP_ATTN_VERIFY, prm, B, T, n) : 0, q);
    const infllmv2_tensor qd = rows(q);
    run("infllmv2_sparse_attn_verify_quant", [&] {
        return lib.sparse_attn_verify_quant(prm, &qd, &kq, &vq, sl, B, T, n, mask, ip, &r.od, r.lp, ws.ptr, ws.bytes, current_stream());
    });
    return tuple2(r.out, r.lse);
}

// (prm, n_sink, window, q, k, v, seqlens, max_seqlen, out | None, lse | None, workspace | None)
PyObject *window_attn_prefill(Args a) {
    const infllmv2_params *prm = enter(a[0]);
    const int32_t sink = integer(a[1]), window = integer(a[2]), T = capacity(a[7]);
    const at::Tensor &q = query(a[3], "q", -1, T, prm);
    const int32_t B = static_cast<int32_t>(q.size(0));
    const infllmv2_tensor kd = cache(kv(a[4], "k", B, T, prm)), vd = cache(kv(a[5], "v", B, T, prm));
    const int32_t *sl = lengths(a[6], B);
    Attended r(a[8], a[9], q, T, {B, T, prm->n_q_heads}, true, prm);
    const Workspace ws = scratch(a[10], a[10] == Py_None ? lib.window_workspace_bytes(INFLLMV2_OP_WINDOW_PREFILL, prm, sink, window, B, T) : 0, q);
    const infllmv2_tensor qd = rows(q);
    run("infllmv2_window_attn_prefill", [&] {
        return lib.window_attn_prefill(prm, sink, window, &qd, &kd, &vd, sl, B, T, &r.od, r.lp, ws.ptr, ws.bytes, current_stream(), r.fill);
    });
    return tuple2(r.out, r.lse);
}

// (prm, n_sink, window, q, k, v, out, dout, lse, seqlens, max_seqlen, dq | None, dk | None, dv | None, workspace | None)
PyObject *window_attn_bwd(Args a) {
    const infllmv2_params *prm = enter(a[0]);
    const int32_t sink = integer(a[1]), window = integer(a[2]), T = capacity(a[10]);
    const at::Tensor &q = query(a[3], "q", -1, T, prm);
    const int32_t B = static_cast<int32_t>(q.size(0));
    const at::Tensor &k = kv(a[4], "k", B, T, prm), &v = kv(a[5], "v", B, T, prm);
    const infllmv2_tensor od = rows(query(a[6], "out", B, T, prm)), gd = rows(query(a[7], "dout", B, T, prm));
    const float *lp = lse_of(tensor(a[8], "lse"), static_cast<int64_t>(B) * T * prm->n_q_heads);
    const int32_t *sl = lengths(a[9], B);
    Result dq(a[11]), dk(a[12]), dv(a[13]);
    const bool fill = dq.make() && dk.make() && dv.make() && q.size(1) == T && k.size(2) == T && v.size(2) == T;   // (as in the forward)
    if (dq.make()) dq.own = fill ? at::empty_like(q) : at::zeros_like(q);
    if (dk.make()) dk.own = fill ? at::empty_like(k) : at::zeros_like(k);
    if (dv.make()) dv.own = fill ? at::empty_like(v) : at::zeros_like(v);
    // (made here: what this call uses; the caller's: as large as the header asks)
    const Workspace ws = scratch(a[14], a[14] == Py_None ? lib.window_bwd_scratch_bytes(prm, sink, window, B, T) : 0, q);
    expect(a[14] == Py_None || ws.bytes >= lib.window_workspace_bytes(INFLLMV2_OP_WINDOW_BWD, prm, sink, window, B, T), "workspace",
           " must hold infllmv2_window_workspace_bytes");
    const infllmv2_tensor qd = rows(q), kd = cache(k), vd = cache(v), dqd = rows(dq.make() ? dq.own : query(dq.given, "dq", B, T, prm)),
                          dkd = cache(dk.make() ? dk.own : kv(dk.given, "dk", B, T, prm)),
                          dvd = cache(dv.make() ? dv.own : kv(dv.given, "dv", B, T, prm));
    run("infllmv2_window_attn_bwd", [&] {
        return lib.window_attn_bwd(prm, sink, window, &qd, &kd, &vd, &od, &gd, lp, sl, B, T, &dqd, &dkd, &dvd, ws.ptr, ws.bytes,
                                   current_stream(), fill);
    });
    return tuple3(dq, dk, dv);
}

// (prm, n_sink, window, q, k, v, seqlens, max_seqlen, out | None, lse | None, workspace | None); k, v of either kind
template <bool kQuant>
PyObject *window_decode(Args a) {
    const infllmv2_params *prm = enter(a[0]);
    const int32_t sink = integer(a[1]), window = integer(a[2]), T = capacity(a[7]);
    const at::Tensor &q = query(a[3], "q", -1, 1, prm);
    expect(q.size(1) == 1, "q", " must have one row per sequence");
    const int32_t B = static_cast<int32_t>(q.size(0));
    const int32_t *sl = lengths(a[6], B);
    Attended r(a[8], a[9], q, 1, {B, prm->n_q_heads}, false, prm);
    const Workspace ws = scratch(a[10], a[10] == Py_None ? lib.window_workspace_bytes(INFLLMV2_OP_WINDOW_DECODE, prm, sink, window, B, T) : 0, q);
    const infllmv2_tensor qd = rows(q);
    if constexpr (kQuant) {
        const infllmv2_quant_tensor kq = quant(a[4], "kq", B, T, prm), vq = quant(a[5], "vq", B, T, prm);
        run("infllmv2_window_attn_decode_quant", [&] {
            return lib.window_attn_decode_quant(prm, sink, window, &qd, &kq, &vq, sl, B, T, &r.od, r.lp, ws.ptr, ws.bytes, current_stream());
        });
    } else {
        const infllmv2_tensor kd = cache(kv(a[4], "k", B, T, prm)), vd = cache(kv(a[5], "v", B, T, prm));
        run("infllmv2_window_attn_decode", [&] {
            return lib.window_attn_decode(prm, sink, window, &qd, &kd, &vd, sl, B, T, &r.od, r.lp, ws.ptr, ws.bytes, current_stream());
        });
    }
    return tuple2(r.out, r.lse);
}
PyObject *window_attn_decode(Args a) { return window_decode<false>(a); }
PyObject *window_attn_decode_quant(Args a) { return window_decode<true>(a); }

// (path, error class): the library every later call goes through
PyObject *bind(Args a) {
    const char *path = PyUnicode_AsUTF8(a[0]);
    if (!path) throw python_error();
    Py_INCREF(a[1]);
    Py_XSETREF(g_error, a[1]);
    void *handle = dlopen(path, RTLD_NOW | RTLD_LOCAL);
    if (!handle) throw MarshalError(std::string("cannot load ") + path + ": " + dlerror());
    Library l;
    symbol(handle, "infllmv2_status_string", l.status_string);
    symbol(handle, "infllmv2_workspace_bytes", l.workspace_bytes);
    symbol(handle, "infllmv2_verify_workspace_bytes", l.verify_workspace_bytes);
    symbol(handle, "infllmv2_append_kv", l.append_kv);
    symbol(handle, "infllmv2_sparse_attn_decode", l.sparse_attn_decode);
    symbol(handle, "infllmv2_decode_step", l.decode_step);
    symbol(handle, "infllmv2_append_kv_verify", l.append_kv_verify);
    symbol(handle, "infllmv2_select_blocks_verify", l.select_blocks_verify);
    symbol(handle, "infllmv2_sparse_attn_verify", l.sparse_attn_verify);
    symbol(handle, "infllmv2_verify_step", l.verify_step);
    symbol(handle, "infllmv2i_compress_keys", l.compress_keys);
    symbol(handle, "infllmv2i_select_blocks", l.select_blocks);
    symbol(handle, "infllmv2i_sparse_attn_prefill", l.sparse_attn_prefill);
    symbol(handle, "infllmv2i_sparse_attn_bwd", l.sparse_attn_bwd);
    symbol(handle, "infllmv2_append_kv_quant", l.append_kv_quant);
    symbol(handle, "infllmv2_sparse_attn_decode_quant", l.sparse_attn_decode_quant);
    symbol(handle, "infllmv2_sparse_attn_verify_quant", l.sparse_attn_verify_quant);
    symbol(handle, "infllmv2_window_workspace_bytes", l.window_workspace_bytes);
    symbol(handle, "infllmv2_window_attn_decode", l.window_attn_decode);
    symbol(handle, "infllmv2_window_attn_decode_quant", l.window_attn_decode_quant);
    symbol(handle, "infllmv2i_quantize_kv", l.quantize_kv);
    symbol(handle, "infllmv2i_dequantize_kv", l.dequantize_kv);
    symbol(handle, "infllmv2i_window_attn_prefill", l.window_attn_prefill);
    symbol(handle, "infllmv2i_window_attn_bwd", l.window_attn_bwd);
    symbol(handle, "infllmv2i_window_bwd_scratch_bytes", l.window_bwd_scratch_bytes);
    lib = l;
    Py_RETURN_NONE;
}

template <PyObject *(*F)(Args), int N>
PyObject *entry(PyObject *, Args a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != N) {
        PyErr_Format(PyExc_TypeError, "expected %d arguments, got %zd", N, n);
        return nullptr;
    }
    try {
        return F(a);
    } catch (const MarshalError &e) {
        PyErr_SetString(g_error ? g_error : PyExc_RuntimeError, e.what());
        return nullptr;
    }
    END_HANDLE_TH_ERRORS
}

#define METHOD(name, n) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(entry<name, n>)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {
    METHOD(bind, 2),
    METHOD(compress_keys, 6),
    METHOD(append_kv, 8),
    METHOD(append_kv_verify, 8),
    METHOD(select_blocks, 8),
    METHOD(select_blocks_verify, 7),
    METHOD(sparse_attn_prefill, 10),
    METHOD(sparse_attn_decode, 10),
    METHOD(sparse_attn_verify, 11),
    METHOD(decode_step, 13),
    METHOD(verify_step, 14),
    METHOD(sparse_attn_bwd, 14),
    METHOD(quantize_kv, 8),
    METHOD(dequantize_kv, 8),
    METHOD(append_kv_quant, 8),
    METHOD(sparse_attn_decode_quant, 10),
    METHOD(sparse_attn_verify_quant, 11),
    METHOD(window_attn_prefill, 11),
    METHOD(window_attn_bwd, 15),
    METHOD(window_attn_decode, 11),
    METHOD(window_attn_decode_quant, 11),
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal() { return PyModule_Create(&module); }
