"""Windowed attention, forward and backward, of large scores that the last channels alone make.

The units at a window's edge test their scores behind a branch: a maximum or a probability that lacked the product's last part would be far off here, where that part is the whole score.
"""
import pytest
import torch

import test_gpu_quant_window as base
from paper_2506_07900_amd import binding

pytestmark = pytest.mark.gpu

D, HALF = base.D, base.HALF
# workgroups of 32 rows, of two halves, of many rows
FORMS = [(4, 1, [777, 300], 4, 256), (16, 1, [700, 40], 5, 600), (2, 8, [4200], 33, 70)]


def inputs(G, H, lengths, size):
    """channels 112 .. 127 of queries and keys: small whole numbers times a power of two, so that products and their sums are exact in 32 bits"""
    gen = torch.Generator(device="cuda").manual_seed(len(lengths) + G)
    B, T = len(lengths), max(lengths)
    whole = lambda *shape: torch.randint(-8, 9, shape, generator=gen, device="cuda")             # noqa: E731
    q, k = (torch.zeros(s, dtype=torch.bfloat16, device="cuda") for s in ((B, T, G * H, D), (B, H, T, D)))
    q[..., 112:] = (whole(B, T, G * H, 16) * size).bfloat16()
    k[..., 112:] = whole(B, H, T, 16).bfloat16()
    return q, k, base.normal(gen, B, H, T, D), base.normal(gen, B, T, G * H, D)


@pytest.mark.parametrize("size", [0.125, 16.0])
@pytest.mark.parametrize("G,H,lengths,n_sink,window", FORMS)
def test_window_of_scores_from_the_last_channels(G, H, lengths, n_sink, window, size):
    q, k, v, dout = inputs(G, H, lengths, size)
    T, prm, sl = max(lengths), binding.Params(G * H, H), base.lengths_tensor(lengths)
    for _ in range(5):
        out, lse = binding.window_attn_prefill(prm, n_sink, window, q, k, v, sl, T)
        grads = binding.window_attn_bwd(prm, n_sink, window, q, k, v, out, dout, lse, sl, T)
        assert all(bool(torch.isfinite(x).all()) for x in (out, lse) + tuple(grads))
    for b, n in enumerate(lengths):
        seen = base.window_seen(torch.arange(n, device="cuda"), n, n_sink, window)
        for h in range(H):
            sums = None
            for hq in range(h * G, (h + 1) * G):
                x = [y.double() for y in (q[b, :n, hq], k[b, h, :n], v[b, h, :n])]
                want, z, mag, large = base.attend(*x, seen, prm.softmax_scale)
                # a score is off by its scale's rounding, its reference's and its own, 2^-24 of the largest each, and so are the sum's: a probability by 2^-21 of it at most
                tol = (1.0625 * HALF + 2.0 ** -21 * large[:, None]) * (mag + want.abs()) + 1e-30
                off = (out[b, :n, hq].double() - want).abs()
                assert bool((off <= tol).all()), ("out", float((off / tol).max()))
                off = (lse[b, :n, hq].double() - z).abs() - (2.0 ** -17 * large + 2.0 ** -20 + 2.0 ** -23 * z.abs())
                assert bool((off <= 0).all()), ("lse", float(off.max()))
                r = base.bwd_reference(*x, *(y.double() for y in (out[b, :n, hq], dout[b, :n, hq], lse[b, :n, hq])), seen, prm.softmax_scale)
                tol = 1.0625 * r[3] + HALF * r[0].abs() + 1e-30
                off = (grads[0][b, :n, hq].double() - r[0]).abs()
                assert bool((off <= tol).all()), ("dq", float((off / tol).max()))
                part = r[1:3] + r[4:6]
                sums = part if sums is None else [a + c for a, c in zip(sums, part)]
            for name, got, want, err in (("dk", grads[1], sums[0], sums[2]), ("dv", grads[2], sums[1], sums[3])):
                tol = 1.0625 * err + HALF * want.abs() + 1e-30
                off = (got[b, h, :n].double() - want).abs()
                assert bool((off <= tol).all()), (name, float((off / tol).max()))
