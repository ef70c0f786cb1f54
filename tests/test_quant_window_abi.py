"""CPU checks of the 4-bit cache's and the windowed attention's entry points: what they refuse, before any HIP call."""
import ctypes
import os

import pytest
import torch

from paper_2506_07900_amd import binding
from paper_2506_07900_amd.binding import CParams, CQuantTensor, CTensor

INVALID, UNSUPPORTED, WORKSPACE = -1, -2, -3
FAKE = 0x10000   # non-null, 256-byte aligned; never dereferenced because validation fails first


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(binding.LIB_PATH):
        from paper_2506_07900_amd import build
        build.build()
    return binding.load_library()


def params(**kw):
    p = dict(head_dim=128, n_q_heads=32, n_kv_heads=2, block_size=64, kernel_size=32, kernel_stride=16, topk=16, n_init_blocks=1,
             n_local_blocks=2, softmax_scale=128 ** -0.5)
    p.update(kw)
    return CParams(**p)


def dense(ptr=FAKE, sb=1 << 20, sh=1 << 16, st=128):
    return CTensor(ptr, sb, sh, st)


def packed(codes=FAKE, scales=FAKE, sb=1 << 20, sh=1 << 16, st=64, eb=1 << 16, eh=1 << 12, et=4):
    return CQuantTensor(codes, scales, sb, sh, st, eb, eh, et)


def refs(args):
    return [ctypes.byref(x) if isinstance(x, ctypes.Structure) else x for x in args]


# name -> arguments that pass every check, with an empty batch: nothing is launched.  Positions of seqlens, batch, max_seqlen follow.
CALLS = {
    "quantize_kv": ([params(), dense(), dense(), FAKE, 0, 4096, 0, packed(), packed(), None], 3),
    "dequantize_kv": ([params(), packed(), packed(), FAKE, 0, 4096, 0, dense(), dense(), None], 3),
    "append_kv_quant": ([params(), dense(), dense(), packed(), packed(), dense(), FAKE, 0, 4096, 4, None], 6),
    "sparse_attn_decode_quant": ([params(), dense(), packed(), packed(), FAKE, 0, 4096, FAKE, dense(), FAKE, FAKE, 1 << 40, None], 4),
    "sparse_attn_verify_quant": ([params(), dense(), packed(), packed(), FAKE, 0, 4096, 4, None, FAKE, dense(), FAKE, FAKE, 1 << 40, None], 4),
    "window_attn_prefill": ([params(), 4, 256, dense(), dense(), dense(), FAKE, 0, 4096, dense(), FAKE, FAKE, 1 << 40, None], 6),
    "window_attn_bwd": ([params(), 4, 256, dense(), dense(), dense(), dense(), dense(), FAKE, FAKE, 0, 4096, dense(), dense(), dense(), FAKE,
                         1 << 40, None], 9),
    "window_attn_decode": ([params(), 4, 256, dense(), dense(), dense(), FAKE, 0, 4096, dense(), FAKE, FAKE, 1 << 40, None], 6),
    "window_attn_decode_quant": ([params(), 4, 256, dense(), packed(), packed(), FAKE, 0, 4096, dense(), FAKE, FAKE, 1 << 40, None], 6),
}


@pytest.mark.parametrize("name", sorted(CALLS))
def test_refusals(lib, name):
    good, at_lengths = CALLS[name]
    fn = getattr(lib, "infllmv2_" + name)
    call = lambda **kw: fn(*refs([kw.get("a%d" % i, x) for i, x in enumerate(good)]))
    assert call() == 0                                             # an empty batch: nothing to do
    assert call(a0=None) == INVALID
    assert call(a0=params(head_dim=64)) == UNSUPPORTED
    assert call(a0=params(n_q_heads=64)) == UNSUPPORTED            # G = 32
    assert call(a0=params(softmax_scale=0.0)) == INVALID
    assert call(**{"a%d" % at_lengths: None}) == INVALID
    assert call(**{"a%d" % (at_lengths + 1): -1}) == INVALID
    assert call(**{"a%d" % (at_lengths + 1): 65536}) == UNSUPPORTED
    assert call(**{"a%d" % (at_lengths + 2): -1}) == INVALID
    assert call(**{"a%d" % (at_lengths + 2): (1 << 30) + 1}) == UNSUPPORTED
    for i, x in enumerate(good):
        if isinstance(x, CTensor):
            if not (name == "append_kv_quant" and i == 5):         # ck may be left out
                assert call(**{"a%d" % i: None}) == INVALID
            for bad in (dense(ptr=None), dense(ptr=FAKE + 8), dense(st=100), dense(sb=-128), dense(sh=4)):
                assert call(**{"a%d" % i: bad}) == INVALID, i
        elif isinstance(x, CQuantTensor):
            assert call(**{"a%d" % i: None}) == INVALID
            for bad in (packed(codes=None), packed(scales=None), packed(codes=FAKE + 8), packed(scales=FAKE + 2), packed(st=72), packed(sh=8),
                        packed(sb=-64), packed(et=2), packed(eh=6), packed(eb=-4)):
                assert call(**{"a%d" % i: bad}) == INVALID, i
    if name.startswith("window"):
        assert call(a1=-1) == INVALID and call(a2=0) == INVALID and call(a2=-5) == INVALID
        assert call(a1=0) == 0 and call(a1=2 ** 31 - 1) == 0 and call(a2=2 ** 31 - 1) == 0
    if name in ("sparse_attn_decode_quant", "sparse_attn_verify_quant", "window_attn_decode_quant"):
        for i in [i for i, x in enumerate(good) if isinstance(x, CQuantTensor)]:
            assert call(**{"a%d" % i: packed(st=(1 << 26) + 16)}) == UNSUPPORTED and call(**{"a%d" % i: packed(et=(1 << 26) + 4)}) == UNSUPPORTED
            assert call(**{"a%d" % i: packed(st=1 << 26, et=1 << 26, sb=1 << 40, eh=1 << 40)}) == 0
    if name in ("window_attn_prefill", "window_attn_bwd"):         # tiles' rows have 32-bit offsets
        far, wide = dense(st=(1 << 23) + 8), dense(sh=1 << 26)
        assert call(a4=far) == UNSUPPORTED and call(a5=far) == UNSUPPORTED and call(a4=dense(st=1 << 23)) == 0
        assert call(a4=wide) == 0                                  # heads of k and v: 64-bit
        if name == "window_attn_bwd":
            assert call(a3=far) == UNSUPPORTED and call(a7=far) == UNSUPPORTED and call(a3=wide) == UNSUPPORTED and call(a7=wide) == UNSUPPORTED
            assert call(a6=far) == 0                               # out: 64-bit
    if name == "append_kv_quant":
        assert call(a5=None) == 0
        assert call(a9=0) == INVALID and call(a9=65) == UNSUPPORTED
    if name == "sparse_attn_verify_quant":
        assert call(a7=0) == INVALID and call(a7=65) == UNSUPPORTED and call(a8=FAKE + 4) == INVALID
        assert call(a5=16384, a7=4) == UNSUPPORTED                 # more than 65535 rows
        assert call(a9=None) == INVALID and call(a11=None) == INVALID
    if name == "sparse_attn_decode_quant":
        assert call(a7=None) == INVALID and call(a9=None) == INVALID


def test_workspaces(lib):
    P = ctypes.byref(params())
    size = lib.infllmv2_window_workspace_bytes
    pre, bwd, dec = binding.OP_WINDOW_PREFILL, binding.OP_WINDOW_BWD, binding.OP_WINDOW_DECODE
    assert size(99, P, 4, 256, 1, 4096) == 0 and size(bwd, P, -1, 256, 1, 4096) == 0 and size(bwd, P, 4, 0, 1, 4096) == 0
    assert size(bwd, P, 4, 256, 1, -1) == 0 and size(bwd, None, 4, 256, 1, 4096) == 0
    assert size(bwd, P, 4, 256, 1, 4096) >= 4096 * 32 * 8          # a log-sum-exp and <dout, out> per row
    # what suffices for a backward call suffices for any with a shorter cache or fewer sequences, whatever the window
    for b in (1, 3, 8):
        sizes = [size(bwd, P, 4, 256, b, t) for t in (1, 127, 128, 129, 1000, 4096, 4097, 32768, 131072)]
        assert sizes == sorted(sizes) and len({size(bwd, P, s, w, b, 4096) for s in (0, 100, 5000) for w in (1, 300, 9000)}) == 1
    for w in (1, 300, 100000):
        sizes = [[size(dec, P, 4, w, b, t) for t in (1, 127, 1000, 4096, 4097, 32768, 131072)] for b in (1, 2, 3, 8, 40, 64, 300, 1000)]
        assert all(x == sorted(x) for x in sizes) and all(list(x) == sorted(x) for x in zip(*sizes))
    for op, name in ((pre, "window_attn_prefill"), (dec, "window_attn_decode"), (dec, "window_attn_decode_quant"), (bwd, "window_attn_bwd")):
        need = size(op, P, 4, 256, 2, 4096)
        args, at = CALLS[name]
        args = list(args)
        args[at + 1] = 2
        if need:
            for ws, n in ((None, 0), (FAKE, need - 1), (FAKE + 16, need)):
                args[-3:-1] = [ws, n]
                assert getattr(lib, "infllmv2_" + name)(*refs(args)) == WORKSPACE, name
    for name, need in (("sparse_attn_decode_quant", lib.infllmv2_workspace_bytes(binding.OP_ATTN_DECODE, P, 2, 4096)),
                       ("sparse_attn_verify_quant", lib.infllmv2_verify_workspace_bytes(binding.OP_ATTN_VERIFY, P, 2, 4096, 4))):
        args, at = CALLS[name]
        args = list(args)
        args[at + 1] = 2
        args[-3:-1] = [FAKE, need - 1]
        assert getattr(lib, "infllmv2_" + name)(*refs(args)) == WORKSPACE


def test_struct_layout():
    assert ctypes.sizeof(CQuantTensor) == 64


def test_binding_refuses_what_is_no_device_tensor(lib):
    prm = binding.Params(4, 1)
    k = torch.zeros((1, 1, 64, 128), dtype=torch.bfloat16)
    sl = torch.zeros(1, dtype=torch.int32)
    c = binding.QuantCache(torch.zeros((1, 1, 64, 64), dtype=torch.uint8), torch.zeros((1, 1, 64, 4), dtype=torch.uint8))
    q = torch.zeros((1, 64, 4, 128), dtype=torch.bfloat16)
    for call in (lambda: binding.quantize_kv(prm, k, k, sl, 64), lambda: binding.dequantize_kv(prm, c, c, sl, 64),
                 lambda: binding.quantize_kv(prm, k, k, sl, 64, kq=c), lambda: binding.append_kv_quant(prm, k, k, c, c, sl, 64),
                 lambda: binding.window_attn_prefill(prm, 0, 8, q, k, k, sl, 64), lambda: binding.window_attn_decode(prm, 0, 8, q, k, k, sl, 64),
                 lambda: binding.dequantize_kv(prm, c.codes, c, sl, 64), lambda: binding.sparse_attn_decode_quant(prm, q, c, c, sl, 64, sl)):
        with pytest.raises(binding.InfLLMv2Error):
            call()
