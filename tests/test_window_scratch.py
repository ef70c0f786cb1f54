"""CPU checks of the windowed backward's two workspace sizes: the bound that callers of the C ABI allocate, which holds for all smaller calls,
and what a call uses, which the binding allocates."""
import ctypes
import os

import pytest

from paper_2506_07900_amd import binding
from paper_2506_07900_amd.binding import CParams, CTensor

WORKSPACE = -3
FAKE = 0x10000   # non-null, 256-byte aligned; never dereferenced because validation fails first


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(binding.LIB_PATH):
        from paper_2506_07900_amd import build
        build.build()
    lib = binding.load_library()
    lib.infllmv2i_window_bwd_scratch_bytes.restype = ctypes.c_size_t
    lib.infllmv2i_window_bwd_scratch_bytes.argtypes = [ctypes.POINTER(CParams)] + [ctypes.c_int32] * 4
    return lib


def params(hq, hkv):
    return CParams(head_dim=128, n_q_heads=hq, n_kv_heads=hkv, block_size=64, kernel_size=32, kernel_stride=16, topk=16, n_init_blocks=1,
                   n_local_blocks=2, softmax_scale=128 ** -0.5)


@pytest.mark.parametrize("hq,hkv", [(1, 1), (4, 1), (16, 2), (32, 2), (64, 8)])
def test_scratch_is_within_the_bound(lib, hq, hkv):
    prm = params(hq, hkv)
    for batch in (1, 2, 7):
        for tokens in (1, 33, 128, 129, 1000, 4096, 4097, 32768, 131072):
            bound = lib.infllmv2_window_workspace_bytes(binding.OP_WINDOW_BWD, ctypes.byref(prm), 0, 1, batch, tokens)
            for sink, window in ((0, 1), (0, 100000), (4, 256), (64, 4096), (600, 33)):
                used = lib.infllmv2i_window_bwd_scratch_bytes(ctypes.byref(prm), sink, window, batch, tokens)
                assert batch * tokens * hq * 8 <= used <= bound            # two floats for every row, at least
    P = ctypes.byref(prm)
    assert lib.infllmv2i_window_bwd_scratch_bytes(P, 0, 1, 0, 64) == 0 and lib.infllmv2i_window_bwd_scratch_bytes(P, 0, 1, 1, 0) == 0
    assert lib.infllmv2i_window_bwd_scratch_bytes(P, -1, 1, 1, 64) == 0 and lib.infllmv2i_window_bwd_scratch_bytes(P, 0, 0, 1, 64) == 0
    assert lib.infllmv2i_window_bwd_scratch_bytes(None, 0, 1, 1, 64) == 0


def test_scratch_of_ordinary_calls(lib):
    # (heads, key-value heads, sequences, tokens, first tokens, window) -> at most so many MB; the bounds are 538, 134, 679 and 539
    for (hq, hkv, batch, tokens, sink, window), most in (((16, 2, 2, 4096, 4, 1000), 72), ((4, 1, 1, 4096, 4, 256), 37), ((32, 2, 1, 32768, 64, 4096), 420),
                                                         ((16, 1, 1, 16384, 0, 1), 53)):
        assert lib.infllmv2i_window_bwd_scratch_bytes(ctypes.byref(params(hq, hkv)), sink, window, batch, tokens) <= most * 10 ** 6


def test_what_either_call_refuses(lib):
    # the internal call one byte less than it uses, the public one less than the bound, though the plan would fit
    prm, (batch, tokens, sink, window) = params(16, 2), (2, 4096, 4, 1000)
    used = lib.infllmv2i_window_bwd_scratch_bytes(ctypes.byref(prm), sink, window, batch, tokens)
    x = ctypes.byref(CTensor(FAKE, 1 << 20, 1 << 16, 128))
    call = lambda fn, size, *fill: fn(ctypes.byref(prm), sink, window, x, x, x, x, x, FAKE, FAKE, batch, tokens, x, x, x, FAKE, size, None, *fill)
    inner = lib.infllmv2i_window_attn_bwd
    inner.restype, inner.argtypes = ctypes.c_int32, lib.infllmv2_window_attn_bwd.argtypes + [ctypes.c_int32]
    assert call(inner, used - 1, 0) == WORKSPACE
    assert call(lib.infllmv2_window_attn_bwd, used) == WORKSPACE
