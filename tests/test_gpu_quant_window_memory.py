"""What the windowed and 4-bit calls do to memory beside their results: scratch, and rows that lie far apart."""
import ctypes

import pytest
import torch

import test_gpu_quant_window as base
from paper_2506_07900_amd import binding
from paper_2506_07900_amd.binding import CParams, CTensor

pytestmark = pytest.mark.gpu

D = base.D


def scratch_bytes(prm, n_sink, window, batch, tokens):
    fn = binding.load_library().infllmv2i_window_bwd_scratch_bytes
    fn.restype, fn.argtypes = ctypes.c_size_t, [ctypes.POINTER(CParams)] + [ctypes.c_int32] * 4
    return fn(ctypes.byref(prm.c()), n_sink, window, batch, tokens)


# spans of several lengths, one span, first tokens' tiles with many spans, ragged sequences
@pytest.mark.parametrize("G,H,lengths,n_sink,window", [
    (8, 2, [4096, 3333], 4, 1000), (4, 1, [4096], 4, 256), (16, 2, [1000] * 8, 0, 1000), (16, 1, [4000], 0, 1), (2, 3, [700, 0, 65], 300, 100), (1, 1, [40], 0, 9)])
def test_window_bwd_stays_within_its_scratch(G, H, lengths, n_sink, window):
    gen = torch.Generator(device="cuda").manual_seed(G + window)
    B, T = len(lengths), max(lengths)
    prm = binding.Params(G * H, H)
    k, v = base.random_cache(gen, B, H, T, lengths)
    q, dout, sl = base.normal(gen, B, T, G * H, D), base.normal(gen, B, T, G * H, D), base.lengths_tensor(lengths)
    out, lse = binding.window_attn_prefill(prm, n_sink, window, q, k, v, sl, T)
    used = scratch_bytes(prm, n_sink, window, B, T)
    torch.cuda.synchronize()
    torch.cuda.reset_peak_memory_stats()
    before = torch.cuda.memory_allocated()
    want = binding.window_attn_bwd(prm, n_sink, window, q, k, v, out, dout, lse, sl, T)
    peak = torch.cuda.max_memory_allocated() - before
    assert peak <= used + 2 * (q.nbytes + k.nbytes + v.nbytes) + (8 << 20)      # scratch, results, the allocator's rounding
    # the call with exactly that much, filled with NaNs, between two guards
    guard = 1 << 20
    ws = torch.full((guard + used + guard,), 255, dtype=torch.uint8, device="cuda")
    got = [torch.full_like(x, 9.0) for x in want]
    t = lambda x: ctypes.byref(CTensor(x.data_ptr(), x.stride(0), x.stride(1), x.stride(2)))
    r = lambda x: ctypes.byref(CTensor(x.data_ptr(), x.stride(0), x.stride(2), x.stride(1)))
    lib = binding.load_library()
    fn = lib.infllmv2i_window_attn_bwd
    fn.restype, fn.argtypes = ctypes.c_int32, lib.infllmv2_window_attn_bwd.argtypes + [ctypes.c_int32]
    assert fn(ctypes.byref(prm.c()), n_sink, window, r(q), t(k), t(v), r(out), r(dout), lse.data_ptr(), sl.data_ptr(), B, T, r(got[0]), t(got[1]), t(got[2]),
              ws.data_ptr() + guard, used, torch.cuda.current_stream().cuda_stream, 1) == 0
    assert all(torch.equal(x, y) for x, y in zip(got, want))
    assert (ws[:guard] == 255).all() and (ws[guard + used:] == 255).all()


def spread(x, strides):
    """x's values at these element strides in memory of its own: rows of D as far apart as a call takes"""
    size = sum((n - 1) * s for n, s in zip(x.shape, strides)) + 1
    y = torch.empty(size, dtype=x.dtype, device="cuda").as_strided(x.shape, strides)
    y.copy_(x)
    return y


FAR = 1 << 23                                                      # the longest token stride, elements


# rows of 16 MiB: a tile's lie up to 2 GiB apart; 32 rows to a workgroup, by halves, many workgroups; key-value heads behind each other beyond 4 GiB
@pytest.mark.parametrize("G,H,T,n_sink,window", [(4, 2, 130, 3, 40), (16, 2, 600, 0, 600), (16, 4, 300, 40, 100), (1, 1, 140, 0, 140)])
def test_rows_as_far_apart_as_the_calls_take_them(G, H, T, n_sink, window):
    gen = torch.Generator(device="cuda").manual_seed(T)
    prm = binding.Params(G * H, H)
    k, v = base.random_cache(gen, 1, H, T, [T])
    q, dout, sl = base.normal(gen, 1, T, G * H, D), base.normal(gen, 1, T, G * H, D), base.lengths_tensor([T])
    out, lse = binding.window_attn_prefill(prm, n_sink, window, q, k, v, sl, T)
    grads = binding.window_attn_bwd(prm, n_sink, window, q, k, v, out, dout, lse, sl, T)
    last = binding.window_attn_decode(prm, n_sink, window, q[:, -1:], k, v, sl, T)
    head = (1 << 29) // G - D                                      # (D less, so that no head's rows meet another's)
    wide = lambda x: spread(x, (8, FAR, head, 1))               # of queries
    cache = lambda x: spread(x, (8, (1 << 31) + D if H == 2 and T < 200 else D, FAR, 1))
    qf, gf, kf, vf = wide(q), wide(dout), cache(k), cache(v)
    of = wide(torch.zeros_like(q))
    z = torch.empty_like(lse)
    binding.window_attn_prefill(prm, n_sink, window, qf, kf, vf, sl, T, out=of, lse=z)
    assert torch.equal(of, out) and torch.equal(z, lse)
    assert all(torch.equal(x, y) for x, y in zip(binding.window_attn_decode(prm, n_sink, window, qf[:, -1:], kf, vf, sl, T), last))
    far = [wide(torch.zeros_like(q)), cache(torch.zeros_like(k)), cache(torch.zeros_like(v))]
    binding.window_attn_bwd(prm, n_sink, window, qf, kf, vf, of, gf, z, sl, T, dq=far[0], dk=far[1], dv=far[2])
    assert all(torch.equal(x, y) for x, y in zip(far, grads))
    vf[0, H - 1, 1, 5] = float("inf")                              # rows that are taken again
    v[0, H - 1, 1, 5] = float("inf")
    assert all(torch.equal(x, y) for x, y in zip(binding.window_attn_prefill(prm, n_sink, window, qf, kf, vf, sl, T, out=of, lse=z),
                                                 binding.window_attn_prefill(prm, n_sink, window, q, k, v, sl, T)))


def test_quantised_rows_as_far_apart_as_the_calls_take_them():
    G, H, T, topk = 16, 2, 100, 3
    gen = torch.Generator(device="cuda").manual_seed(1)
    prm = binding.Params(G * H, H, topk=topk)
    k, v = base.random_cache(gen, 1, H, T, [T])
    q, sl = base.normal(gen, 1, 1, G * H, D), base.lengths_tensor([T])
    kq, vq = binding.quantize_kv(prm, k, v, sl, T)
    far = 1 << 26                                                  # bytes from a row to the next; all four arrays and heads between them
    block = torch.empty(T * far, dtype=torch.uint8, device="cuda")
    at = lambda width, first: block.as_strided((1, H, T, width), (T * far, 256, far, 1), first)
    kf, vf = binding.QuantCache(at(64, 0), at(4, 64)), binding.QuantCache(at(64, 128), at(4, 192))
    binding.quantize_kv(prm, k, v, sl, T, kf, vf)
    for x, y in zip((*kf, *vf), (*kq, *vq)):
        assert torch.equal(x, y)
    idx = torch.tensor([0, 1, -1], dtype=torch.int32, device="cuda").expand(1, H, 1, topk).contiguous()
    for call in (lambda k, v: binding.window_attn_decode_quant(prm, 4, 50, q, k, v, sl, T),
                 lambda k, v: binding.sparse_attn_decode_quant(prm, q, k, v, sl, T, idx), lambda k, v: binding.dequantize_kv(prm, k, v, sl, T)):
        assert all(torch.equal(x, y) for x, y in zip(call(kf, vf), call(kq, vq)))
