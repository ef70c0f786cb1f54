"""CPU checks of the entry points of rotary positions and the cache in pages: the rotation's table, and what they refuse, before any HIP call."""
import ctypes
import math
import os
import sys

import pytest
import torch

from paper_2506_07900_amd import binding
from paper_2506_07900_amd.binding import CPages, CRopeConfig, CRotation, CTensor

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
from test_quant_window_abi import FAKE, INVALID, UNSUPPORTED, WORKSPACE, dense, params, refs  # noqa: E402


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(binding.LIB_PATH):
        from paper_2506_07900_amd import build
        build.build()
    return binding.load_library()


def pages(k=None, v=None, table=FAKE, stride=64, size=64, count=100):
    return CPages(k or dense(sb=1 << 16, sh=1 << 13), v or dense(sb=1 << 16, sh=1 << 13), table, stride, size, count)


def rotation(dim=128, inter=0, amplitude=1.0, steps=FAKE):
    return CRotation(dim, inter, amplitude, steps)


# name -> arguments that pass every check, with an empty batch: nothing is launched
CALLS = {
    "rope": [params(), rotation(), dense(), dense(), None, FAKE, 0, 4096, dense(), dense(), None],
    "rope_bwd": [params(), rotation(), dense(), dense(), FAKE, FAKE, 0, 4096, dense(), dense(), None],
    "paged_append": [params(), rotation(), dense(), dense(), dense(), pages(), None, None, FAKE, 0, 4096, 4, dense(), None],
    "paged_attn": [params(), dense(), pages(), None, FAKE, 0, 4096, 4, dense(), FAKE, FAKE, 1 << 40, None],
    "paged_attn_weights": [params(), dense(), FAKE, pages(), FAKE, FAKE, 0, 4096, 4, FAKE, 4096, FAKE, FAKE, 1 << 40, None],
    "paged_evict": [params(), FAKE, 4096, pages(), FAKE, 0, 4096, 1000, 4, 100, pages(), FAKE, FAKE, FAKE, FAKE, 1 << 40, None],
}
LENGTHS = {"rope": 5, "rope_bwd": 5, "paged_append": 8, "paged_attn": 4, "paged_attn_weights": 5, "paged_evict": 4}
OPTIONAL = {("rope", 4), ("rope_bwd", 4), ("paged_append", 6), ("paged_append", 7), ("paged_attn", 3), ("paged_attn_weights", 4), ("paged_attn_weights", 9),
            ("paged_evict", 12)}


def call(lib, name, **at):
    args = list(CALLS[name])
    for i, x in at.items():
        args[int(i[1:])] = x
    return getattr(lib, "infllmv2_" + name)(*refs(args))


@pytest.mark.parametrize("name", sorted(CALLS))
def test_refusals(lib, name):
    args, at = CALLS[name], LENGTHS[name]
    go = lambda **kw: call(lib, name, **kw)                       # noqa: E731
    assert go() == 0
    assert go(_0=None) == INVALID
    assert go(**{"_%d" % at: None}) == INVALID                    # seqlens
    assert go(**{"_%d" % (at + 1): -1}) == INVALID and go(**{"_%d" % (at + 2): -1}) == INVALID
    assert go(**{"_%d" % (at + 1): 65536}) == UNSUPPORTED
    assert go(**{"_%d" % (at + 2): (1 << 30) + 1}) == UNSUPPORTED
    assert go(_0=params(head_dim=64)) == UNSUPPORTED and go(_0=params(n_q_heads=24)) == UNSUPPORTED
    for i, x in enumerate(args):
        if isinstance(x, CTensor):
            for bad in (dense(0), dense(FAKE + 8), dense(st=4), dense(sh=-8), dense(sb=12)):
                assert go(**{"_%d" % i: bad}) == INVALID, i
        if isinstance(x, CPages):
            assert go(**{"_%d" % i: None}) == INVALID
            for bad in (pages(k=dense(FAKE + 2)), pages(v=dense(0)), pages(table=None), pages(size=0), pages(size=-16), pages(count=-1), pages(stride=-1),
                        pages(stride=15)):
                assert go(**{"_%d" % i: bad}) == INVALID, i
            for bad in (pages(size=48), pages(size=8), pages(size=2048), pages(k=dense(st=(1 << 23) + 8)), pages(v=dense(st=1 << 24))):
                assert go(**{"_%d" % i: bad}) == UNSUPPORTED, i
        if isinstance(x, CRotation):
            for bad in (rotation(0), rotation(-16), rotation(steps=None), rotation(steps=FAKE + 8), rotation(amplitude=math.nan), rotation(amplitude=math.inf)):
                assert go(**{"_%d" % i: bad}) == INVALID
            for bad in (rotation(144), rotation(20), rotation(2)):
                assert go(**{"_%d" % i: bad}) == UNSUPPORTED
        if x == FAKE and i != at and (name, i) not in OPTIONAL and not (i == len(args) - 3):
            assert go(**{"_%d" % i: None}) == INVALID, i


def test_more_refusals(lib):
    for name in ("rope", "rope_bwd"):                             # an input without its output
        assert call(lib, name, _2=None) == INVALID and call(lib, name, _8=None) == INVALID and call(lib, name, _3=None) == INVALID
        assert call(lib, name, _2=None, _8=None) == 0 and call(lib, name, _3=None, _9=None) == 0
        assert call(lib, name, _1=None) == INVALID
    assert call(lib, "paged_append", _4=None) == INVALID and call(lib, "paged_append", _12=None) == INVALID
    assert call(lib, "paged_append", _1=None) == INVALID          # queries without a rotation
    assert call(lib, "paged_append", _1=None, _4=None, _12=None) == 0
    for name, i in (("paged_append", 11), ("paged_attn", 7), ("paged_attn_weights", 8)):
        assert call(lib, name, **{"_%d" % i: 0}) == INVALID
        assert call(lib, name, **{"_%d" % i: (1 << 24) + 1}) == UNSUPPORTED
        assert call(lib, name, _0=params(n_q_heads=128, n_kv_heads=8), **{"_%d" % i: 1 << 24}) == UNSUPPORTED
    for name in ("paged_attn", "paged_attn_weights"):
        assert call(lib, name, _1=dense(st=(1 << 23) + 8)) == UNSUPPORTED and call(lib, name, _1=dense(sh=1 << 26)) == UNSUPPORTED
    assert call(lib, "paged_attn_weights", _10=4095) == INVALID
    assert call(lib, "paged_evict", _2=4095) == INVALID
    for budget, first, recent, want in ((0, 0, 0, INVALID), (10, 6, 5, INVALID), (10, -1, 5, INVALID), (10, 5, -1, INVALID), (10, 5, 5, 0),
                                        (2 ** 31 - 1, 2 ** 31 - 1, 2 ** 31 - 1, INVALID), (5000, 0, 0, 0), (4096, 0, 0, 0)):
        assert call(lib, "paged_evict", _7=budget, _8=first, _9=recent) == want
    # the kept rows' table: for the budget, or for all rows there can be
    for budget, stride, want in ((1000, 16, 0), (1000, 15, INVALID), (1 << 20, 64, 0), (1 << 20, 63, INVALID)):
        assert call(lib, "paged_evict", _7=budget, _10=pages(stride=stride)) == want
    # a workspace that is missing, small or crooked, where one is needed
    need = lib.infllmv2_paged_workspace_bytes(binding.OP_PAGED_ATTN, ctypes.byref(params()), 1, 4096, 4)
    assert need > 0
    for ws, size in ((None, need), (FAKE, need - 1), (FAKE + 128, need)):
        assert call(lib, "paged_attn", _5=1, _10=ws, _11=size) == WORKSPACE


def test_eviction_of_long_sequences_needs_a_workspace(lib):
    one = lambda b, t: lib.infllmv2_paged_workspace_bytes(binding.OP_PAGED_EVICT, ctypes.byref(params()), b, t, 1)   # noqa: E731
    assert one(1, 16384) == 0 and one(1, 16385) > 0 and one(0, 100000) == 0
    got = [one(2, t) for t in (1, 16385, 20480, 20481, 262143, 262144, 262145, 524288, 524289, 1 << 20, (1 << 20) + 1, 1 << 30)]
    assert got == sorted(got)
    assert one(1, (1 << 30) + 1) == 0


@pytest.mark.parametrize("op", [binding.OP_PAGED_ATTN, binding.OP_PAGED_WEIGHTS, binding.OP_PAGED_EVICT])
def test_workspaces_grow_with_every_size(lib, op):
    sizes = [1, 2, 3, 7, 16, 17, 64, 255, 256, 257, 511, 512, 513, 600, 1024, 5000, 65535]
    for hq, hkv in ((32, 2), (4, 4), (1, 1)):
        need = lambda b, t, n: lib.infllmv2_paged_workspace_bytes(op, ctypes.byref(params(n_q_heads=hq, n_kv_heads=hkv)), b, t, n)   # noqa: E731
        for fixed in (1, 16, 300, 5000):
            for f in (lambda x: need(x, 4096, fixed), lambda x: need(fixed, x, 16), lambda x: need(fixed, 20000, x)):
                got = [f(x) for x in sizes]
                assert got == sorted(got)
    assert lib.infllmv2_paged_workspace_bytes(op, ctypes.byref(params(head_dim=64)), 1, 100, 1) == 0
    assert lib.infllmv2_paged_workspace_bytes(op, ctypes.byref(params()), -1, 100, 1) == 0
    assert lib.infllmv2_paged_workspace_bytes(99, ctypes.byref(params()), 1, 100, 1) == 0


# ---- the rotation's table ---------------------------------------------------------------------------------------------

def table(lib, rot, scaling=0, base=10000.0, factor=1.0, original=0, fast=32.0, slow=1.0, amplitude=0.0, factors=None):
    arr = None if factors is None else (ctypes.c_double * len(factors))(*factors)
    cfg = CRopeConfig(rot, scaling, original, base, factor, fast, slow, amplitude, arr)
    steps, amp = (ctypes.c_uint64 * 64)(), ctypes.c_float()
    status = lib.infllmv2_rope_table(ctypes.byref(cfg), steps, ctypes.byref(amp))
    return status, list(steps)[:max(0, rot // 2)], amp.value


def turns(rot, base=10000.0):
    """turns per position, from logarithms in 64 bits.  The exponent, up to 9.3 in size, takes three roundings of 2^-53 of itself (the logarithm, the quotient, their
    product), and an absolute error of the exponent is a relative one of the result: 28 x 2^-53, with the exponential, the division by 2 pi and two more operations
    of the callers 33 x 2^-53 < 2^-47"""
    return [math.exp(-2.0 * j / rot * math.log(base)) / (2 * math.pi) for j in range(rot // 2)]


def near(steps, want):
    # (and a step is a whole number of 2^-64 turns)
    assert all(abs(s * 2.0 ** -64 - w) <= 2.0 ** -47 * w + 2.0 ** -65 for s, w in zip(steps, want)) and len(steps) == len(want)


def test_table(lib):
    for rot in (16, 32, 96, 128):
        status, steps, amp = table(lib, rot)
        assert status == 0 and amp == 1.0
        near(steps, turns(rot))
        status, steps, amp = table(lib, rot, binding.ROPE_SCALINGS["linear"], factor=3.0)
        near(steps, [x / 3 for x in turns(rot)])
        status, steps, amp = table(lib, rot, binding.ROPE_SCALINGS["ntk"], factor=4.0, amplitude=0.5)
        assert amp == 0.5
        near(steps, turns(rot, 10000.0 * 4.0 ** (rot / (rot - 2))))
        status, steps, amp = table(lib, rot, binding.ROPE_SCALINGS["yarn"], factor=8.0, original=4096)
        keep = [min(1, max(0, (4096 * x - 1) / 31)) for x in turns(rot)]
        near(steps, [x * (k + (1 - k) / 8) for x, k in zip(turns(rot), keep)])
        assert amp == pytest.approx(0.1 * math.log(8) + 1, rel=2 ** -23)
        factors = [1 + j / 7 for j in range(rot // 2)]
        status, steps, amp = table(lib, rot, binding.ROPE_SCALINGS["factors"], factor=8.0, original=4096, factors=factors)
        near(steps, [x / f for x, f in zip(turns(rot), factors)])
        assert amp == pytest.approx(math.sqrt(1 + math.log(8) / math.log(4096)), rel=2 ** -23)


def test_table_of_more_than_a_turn(lib):
    status, steps, _ = table(lib, 16, binding.ROPE_SCALINGS["factors"], factor=2.0, original=100, factors=[0.01] + [1.0] * 7)
    want = 100 / (2 * math.pi)
    assert status == 0 and abs(steps[0] * 2.0 ** -64 - (want - math.floor(want))) < 2.0 ** -46


def test_table_refusals(lib):
    S = binding.ROPE_SCALINGS
    for rot in (0, -16):
        assert table(lib, rot)[0] == INVALID
    for rot in (2, 24, 144):
        assert table(lib, rot)[0] == UNSUPPORTED
    for kw in (dict(scaling=5), dict(scaling=-1), dict(base=1.0), dict(base=math.nan), dict(base=math.inf), dict(amplitude=-1.0), dict(amplitude=math.nan),
               dict(scaling=S["linear"], factor=0.5), dict(scaling=S["ntk"], factor=math.nan), dict(scaling=S["yarn"], factor=2.0),
               dict(scaling=S["yarn"], factor=2.0, original=100, fast=1.0), dict(scaling=S["yarn"], factor=2.0, original=100, slow=-1.0),
               dict(scaling=S["factors"], factor=2.0, original=100), dict(scaling=S["factors"], factor=2.0, original=0, factors=[1.0] * 64),
               dict(scaling=S["factors"], factor=2.0, original=100, factors=[0.0] + [1.0] * 63),
               dict(scaling=S["factors"], factor=2.0, original=100, factors=[math.nan] + [1.0] * 63)):
        assert table(lib, 128, **kw)[0] == INVALID, kw
    steps, amp = (ctypes.c_uint64 * 64)(), ctypes.c_float()
    assert lib.infllmv2_rope_table(None, steps, ctypes.byref(amp)) == INVALID
    cfg = CRopeConfig(128, 0, 0, 10000.0, 1.0, 32.0, 1.0, 0.0, None)
    assert lib.infllmv2_rope_table(ctypes.byref(cfg), None, ctypes.byref(amp)) == INVALID
    assert lib.infllmv2_rope_table(ctypes.byref(cfg), steps, None) == INVALID


def test_binding_checks(lib):
    with pytest.raises(binding.InfLLMv2Error, match="scaling"):
        binding.rope_table(128, scaling="other", device="cpu")
    with pytest.raises(binding.InfLLMv2Error, match="pair_factors"):
        binding.rope_table(128, scaling="factors", pair_factors=[1.0], device="cpu")
    with pytest.raises(binding.InfLLMv2Error, match="rope_table"):
        binding.rope_table(20, device="cpu")
    r = binding.rope_table(64, interleaved=True, device="cpu")
    assert r.steps.shape == (32,) and r.steps.dtype == torch.int64 and r.interleaved and r.rot_dim == 64
    prm, x, y = binding.Params(8, 2), torch.zeros(1, 4, 8, 128, dtype=torch.bfloat16), torch.zeros(1, 2, 4, 128, dtype=torch.bfloat16)
    with pytest.raises(binding.InfLLMv2Error):                    # not on a device
        binding.rope(prm, r, x, y, torch.tensor([4], dtype=torch.int32), 4)
    cache = binding.PagedCache(torch.zeros(3, 2, 16, 128, dtype=torch.bfloat16), torch.zeros(3, 2, 16, 128, dtype=torch.bfloat16),
                               torch.zeros(1, 1, dtype=torch.int32))
    for f in (lambda: binding.paged_attn(prm, x, cache, torch.tensor([4], dtype=torch.int32), 4),
              lambda: binding.paged_append(prm, y, y, cache, torch.tensor([4], dtype=torch.int32), 4),
              lambda: binding.paged_attn(prm, None, cache, None, 4)):
        with pytest.raises(binding.InfLLMv2Error):
            f()


def test_c_structures(tmp_path):
    """ctypes' mirrors have the header's layout"""
    import subprocess
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    want = {"infllmv2_pages": CPages, "infllmv2_rope_config": CRopeConfig, "infllmv2_rotation": CRotation}
    lines = ['#include <stdio.h>', '#include <stddef.h>', '#include "infllmv2.h"', "int main(void) {"]
    for name, cls in want.items():
        lines.append('printf("%%zu ", sizeof(%s));' % name)
        lines += ['printf("%%zu ", offsetof(%s, %s));' % (name, f[0]) for f in cls._fields_]
    src = tmp_path / "layout.c"
    src.write_text("\n".join(lines + ["return 0; }"]))
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-std=c99", "-I", os.path.join(root, "include"), str(src), "-o", str(exe)], check=True)
    got = [int(x) for x in subprocess.run([str(exe)], stdout=subprocess.PIPE, check=True, text=True).stdout.split()]
    assert got == [x for cls in want.values() for x in [ctypes.sizeof(cls)] + [getattr(cls, f[0]).offset for f in cls._fields_]]
