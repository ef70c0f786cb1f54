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
