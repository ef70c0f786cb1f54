"""The 4-bit cache and the windowed attention against plain 64-bit computations of their definitions.

Tolerances, derived from the roundings of the calls (half a step of bf16 is 2^-8 of a value):
  outputs     a probability is rounded to bf16 once, the output once: 2^-8 (sum p |v| + |o|), a sixteenth more for the fp32 sums
              and the scores' own rounding (a dot product of 128 exact products is off by at most 2^-17 of the sum of their sizes, which moves a
              probability by that much: 2^-13 at sizes of 16)
  log-sum-exp 2^-17 of the largest logit's sum of sizes, and 2^-20 for the sum's, the exponentials' and the logarithm's roundings, and the result's
              own rounding
  dv          as an output: 2^-8 (sum p |dout| + |dv|)
  dq, dk      ds is rounded to bf16 once and the result once: 2^-8 (sum |ds| |k| + |dq|); ds itself comes from a difference of two fp32 sums, off by
              2^-17 of their terms' sizes
  4 bits      exact: codes, exponents and values are equal
"""
import math

import numpy as np
import pytest
import torch

from paper_2506_07900_amd import binding

pytestmark = pytest.mark.gpu

D = 128
HALF = 2.0 ** -8
GARBAGE = float("nan")


def normal(gen, *shape, scale=1.0):
    return (torch.randn(shape, generator=gen, device="cuda") * scale).bfloat16()


def lengths_tensor(lengths):
    return torch.tensor(lengths, dtype=torch.int32, device="cuda")


# ---- the format -------------------------------------------------------------------------------------------------

VALUES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def encode(x):
    """[.., 128] floats -> codes [.., 64], exponents [.., 4], values [.., 128], by search in 64 bits"""
    x = np.asarray(x, np.float64)
    g = x.reshape(-1, 32)
    finite = np.isfinite(g).all(-1)
    most = np.where(finite, np.abs(np.where(np.isfinite(g), g, 0.0)).max(-1), 1.0)
    frac, e = np.frexp(np.where(most > 0, most, 1.0))              # 0.5 <= frac < 1
    e = np.where(most > 0, np.where(frac >= 0.875, e, e - 1), -1000)
    byte = np.where(finite, np.clip(e + 127 - 2, 2, 252), 255)
    unit = np.where(finite, 2.0 ** (np.minimum(byte, 254) - 127.0), 1.0)
    y = np.abs(np.where(finite[:, None], g, 0.0)) / unit[:, None]
    gap = np.abs(y[..., None] - VALUES)
    odd = np.arange(8) % 2
    index = np.lexsort((np.broadcast_to(odd, gap.shape), gap), axis=-1)[..., 0]
    sign = np.where(finite[:, None], np.signbit(g), False)
    code = (index + 8 * sign).astype(np.uint8)
    value = np.where(finite[:, None], VALUES[index] * unit[:, None] * np.where(sign, -1.0, 1.0), np.nan)
    code = code.reshape(*x.shape[:-1], 64, 2)
    return code[..., 0] | (code[..., 1] << 4), byte.astype(np.uint8).reshape(*x.shape[:-1], 4), value.reshape(x.shape)


def values_of(c):
    """QuantCache -> fp64 values on its device"""
    nibble = torch.stack((c.codes & 15, c.codes >> 4), -1).flatten(-2).long()
    table = torch.tensor(np.concatenate((VALUES, -VALUES)), device=c.codes.device)
    scale = torch.where(c.scales == 255, math.nan, torch.exp2(c.scales.double() - 127))
    return table[nibble] * scale.repeat_interleave(32, -1)


def test_every_number_is_rounded_to_the_nearest_code():
    # all 65536 bit patterns, in groups of neighbours (equal exponents: all ties), shuffled within 2^12 of each other (exponents that
    # differ by a few), and one large number per group of the others
    bits = torch.arange(65536, dtype=torch.int32)
    order = torch.cat([torch.randperm(4096, generator=torch.Generator().manual_seed(i)) + 4096 * i for i in range(16)])
    large = bits.clone().reshape(-1, 32)
    finite = (large & 0x7f80) < 0x7d80                             # (four binades above: still a number)
    large[:, 5] = torch.where(finite.all(-1), (large[:, 5] & 0x7f80) + 0x200 + (large[:, 7] & 0x7f), large[:, 5])
    for x in (bits, bits[order], large.reshape(-1)):
        k = torch.from_numpy(x.numpy().astype(np.uint16).view(np.int16)).view(torch.bfloat16).reshape(1, 1, 512, D)
        prm = binding.Params(1, 1)
        kq, vq = binding.quantize_kv(prm, k.cuda(), (-k).cuda(), lengths_tensor([512]), 512)
        want = encode(k.double().numpy())
        minus = encode((-k).double().numpy())
        for got, ref in ((kq, want), (vq, minus)):
            assert np.array_equal(got.scales.cpu().numpy(), ref[1])
            assert np.array_equal(got.codes.cpu().numpy(), ref[0])
        back, backv = binding.dequantize_kv(prm, kq, vq, lengths_tensor([512]), 512)
        assert np.array_equal(back.double().cpu().numpy(), want[2], equal_nan=True)
        assert np.array_equal(backv.double().cpu().numpy(), minus[2], equal_nan=True)
        # nothing is clipped, so a value is off by half the grid's widest step (4 to 6) at most; but for magnitudes above 1.75 x 2^127, which the next
        # larger exponent would read back as infinite: up to 8 units become 6
        ok = np.isfinite(want[2])
        err = np.abs(k.double().numpy() - want[2])[ok].reshape(-1)
        byte = np.repeat(want[1].astype(float), 32, -1).reshape(k.shape)[ok].reshape(-1)
        assert (err <= 2.0 ** (byte - 127) * np.where(byte == 252, 2, 1)).all()


@pytest.mark.parametrize("lengths,n_new", [([1], 0), ([0, 5, 64, 65, 200], 0), ([777, 0, 33], 0), ([777, 3, 0], 7), ([128], 200), ([300, 299], 64)])
def test_quantize_rows(lengths, n_new):
    gen = torch.Generator(device="cuda").manual_seed(sum(lengths) + n_new)
    B, H, T = len(lengths), 3, max(max(lengths), 1)
    prm = binding.Params(6, 3)
    # heads and tokens in another order in memory than in the tensor
    k = normal(gen, B, T + 5, H, D).transpose(1, 2)
    v = normal(gen, H, B, T + 5, D).transpose(0, 1)
    for b, n in enumerate(lengths):
        k[b, :, n:], v[b, :, n:] = GARBAGE, GARBAGE
    base = [torch.randint(0, 255, (B, H, T + 2, w), dtype=torch.uint8, generator=gen, device="cuda") for w in (80, 8, 64, 4)]
    kq = binding.QuantCache(base[0][..., 16:80], base[1][..., 4:8])
    vq = binding.QuantCache(base[2], base[3])
    before = [x.clone() for x in base]
    sl = lengths_tensor(lengths)
    binding.quantize_kv(prm, k, v, sl, T, kq, vq, n_new_tokens=n_new)
    kb = normal(gen, B, H, T + 1, D)
    vb = normal(gen, B, T + 1, H, D).transpose(1, 2)
    kept = kb.clone(), vb.clone()
    binding.dequantize_kv(prm, kq, vq, sl, T, kb, vb, n_new_tokens=n_new)
    made = binding.quantize_kv(prm, k, v, sl, T)                   # results made by the call: rows behind a sequence are 0
    read = binding.dequantize_kv(prm, *made, sl, T)
    want = encode(k.double().cpu().numpy()), encode(v.double().cpu().numpy())
    for (codes, scales, values), got, back, old, make, rd in zip(want, (kq, vq), (kb, vb), kept, made, read):
        for b, n in enumerate(lengths):
            lo = max(0, n - n_new) if n_new > 0 else 0
            assert np.array_equal(got.codes[b, :, lo:n].cpu().numpy(), codes[b, :, lo:n])
            assert np.array_equal(got.scales[b, :, lo:n].cpu().numpy(), scales[b, :, lo:n])
            assert np.array_equal(back[b, :, lo:n].double().cpu().numpy(), values[b, :, lo:n])
            assert torch.equal(back[b, :, :lo], old[b, :, :lo]) and torch.equal(back[b, :, n:], old[b, :, n:])
            assert np.array_equal(make.codes[b, :, :n].cpu().numpy(), codes[b, :, :n]) and not make.codes[b, :, n:].any()
            assert not make.scales[b, :, n:].any() and not rd[b, :, n:].any()
            assert np.array_equal(rd[b, :, :n].double().cpu().numpy(), values[b, :, :n])
    for x, y, (lo_c, hi_c) in zip(base, before, ((16, 80), (4, 8), (0, 64), (0, 4))):
        for b, n in enumerate(lengths):
            lo = max(0, n - n_new) if n_new > 0 else 0
            x[b, :, lo:n, lo_c:hi_c] = y[b, :, lo:n, lo_c:hi_c]
        assert torch.equal(x, y)                                   # nothing else was written


@pytest.mark.parametrize("n", [1, 2, 5, 16, 17, 33, 64])
@pytest.mark.parametrize("with_ck", [True, False])
def test_append(n, with_ck):
    # lengths around the completion of a kernel, a sequence that is too short for n rows, one longer than the cache
    lengths = [n, n + 15, n + 31, n + 32, 256, 255, 200, max(0, n - 1), 300]
    gen = torch.Generator(device="cuda").manual_seed(n)
    B, H, T = len(lengths), 2, 256
    prm = binding.Params(8, 2)
    k, v = normal(gen, B, H, T, D), normal(gen, B, H, T, D, scale=3.0)
    sl = lengths_tensor(lengths)
    old = [max(0, min(x, T) - n) for x in lengths]
    kq, vq = binding.quantize_kv(prm, k, v, lengths_tensor(old), T)
    ck = torch.full((B, H, 15, D), 7.0, dtype=torch.bfloat16, device="cuda")
    before = [x.clone() for x in (*kq, *vq)], ck.clone()
    new = normal(gen, B, n, H, D).transpose(1, 2), normal(gen, B, H, n + 1, D)[:, :, :n]
    binding.append_kv_quant(prm, *new, kq, vq, sl, T, ck=ck if with_ck else None)
    for b, length in enumerate(lengths):
        if length < n or length > T:
            for x, y in zip((*kq, *vq), before[0]):
                assert torch.equal(x[b], y[b])
            assert torch.equal(ck[b], before[1][b])
            continue
        whole_k, whole_v = k[b, :, :length].clone(), v[b, :, :length].clone()
        whole_k[:, length - n:], whole_v[:, length - n:] = new[0][b], new[1][b]
        for got, x in ((kq, whole_k), (vq, whole_v)):
            codes, scales, _ = encode(x.double().cpu().numpy())
            assert np.array_equal(got.codes[b, :, :length].cpu().numpy(), codes)
            assert np.array_equal(got.scales[b, :, :length].cpu().numpy(), scales)
            assert not got.codes[b, :, length:].any() and not got.scales[b, :, length:].any()
    if with_ck:                                                    # the kernels of the cache as it is read back
        inside = lengths_tensor([x if n <= x <= T else 0 for x in lengths])
        kb, _ = binding.dequantize_kv(prm, kq, vq, inside, T)
        want = before[1].clone()
        binding.compress_keys(prm, kb, inside, T, ck=want, n_new_tokens=n)
        assert torch.equal(ck.view(torch.int16), want.view(torch.int16))


# ---- attention --------------------------------------------------------------------------------------------------

def attend(q, k, v, seen, scale):
    """q [R, D], k, v [K, D], seen [R, K] in fp64 -> out, lse, and the sizes their tolerances are measured in"""
    s = (q @ k.t().contiguous()) * scale
    size = (q.abs() @ k.abs().t().contiguous()) * scale
    s = torch.where(seen, s, -math.inf)
    top = s.amax(-1, keepdim=True)
    p = torch.exp(s - torch.where(top == -math.inf, 0.0, top))
    total = p.sum(-1, keepdim=True)
    w = p / torch.where(total > 0, total, 1.0)
    v = torch.where(seen.any(0)[:, None], v, 0.0)
    lse = (torch.where(top == -math.inf, 0.0, top) + torch.log(total))[:, 0]
    return w @ v, lse, w @ v.abs(), torch.where(seen, size, 0.0).amax(-1)


def check(got, got_lse, want):
    o, lse, mag, size = want
    got, got_lse = got.double(), got_lse.double()
    tol = 1.0625 * HALF * (mag + o.abs()) + 1e-30
    assert ((got - o).abs() <= tol).all(), float(((got - o).abs() / tol).max())
    empty = lse == -math.inf
    assert torch.equal(got_lse == -math.inf, empty)
    tol = 2.0 ** -17 * size + 2.0 ** -20 + 2.0 ** -23 * lse.abs()
    diff = torch.where(empty, 0.0, (got_lse - lse).abs())
    assert (diff <= torch.where(empty, 1.0, tol)).all(), float(diff.max())


def window_seen(pos, length, n_sink, window, device="cuda"):
    t, i = torch.arange(length, device=device)[None], pos[:, None]
    return (t <= i) & ((t < n_sink) | (i - t < window))


def random_cache(gen, B, H, T, lengths, spoil=True):
    k, v = normal(gen, B, H, T, D), normal(gen, B, T, H, D).transpose(1, 2)
    if spoil:
        for b, n in enumerate(lengths):
            k[b, :, n:], v[b, :, n:] = GARBAGE, GARBAGE
    return k, v


def quant_of(prm, k, v, lengths):
    """the cache in 4 bits; rows behind a sequence stand for NaN"""
    kq, vq = binding.quantize_kv(prm, k, v, lengths_tensor(lengths), k.shape[2])
    for c in (kq, vq):
        for b, n in enumerate(lengths):
            c.codes[b, :, n:], c.scales[b, :, n:] = 0x77, 255
    return kq, vq


DECODE_CASES = [  # G, Hkv, lengths, n_sink, window
    (16, 2, [1, 2, 31, 32, 33, 64, 65, 0], 4, 40),
    (1, 3, [100, 1, 97], 0, 1),
    (2, 1, [500, 77], 33, 64),
    (4, 1, [2000], 4, 256),
    (8, 2, [1999, 1, 640], 100, 10000),
    (16, 1, [5000, 4097, 4096], 64, 4096),
    (16, 4, [333] * 5, 400, 7),
    (16, 2, [30011], 128, 8192),
]


@pytest.mark.parametrize("G,H,lengths,n_sink,window", DECODE_CASES)
@pytest.mark.parametrize("quant", [False, True])
def test_window_decode(G, H, lengths, n_sink, window, quant):
    gen = torch.Generator(device="cuda").manual_seed(G * 1000 + window)
    B, T = len(lengths), max(lengths) + 3
    prm = binding.Params(G * H, H)
    k, v = random_cache(gen, B, H, T, lengths, spoil=False)
    masked = [(min(n_sink, n), max(min(n_sink, n), n - window)) for n in lengths]     # rows no query sees
    q = normal(gen, B, G * H, 1, D).transpose(1, 2)
    sl = lengths_tensor(lengths)
    if quant:
        kq, vq = quant_of(prm, k, v, lengths)
        for b, (lo, hi) in enumerate(masked):
            for c in (kq, vq):
                c.scales[b, :, lo:hi] = 255
        out, lse = binding.window_attn_decode_quant(prm, n_sink, window, q, kq, vq, sl, T)
        k64, v64 = values_of(kq), values_of(vq)
    else:
        for b, (lo, hi) in enumerate(masked):
            k[b, :, lo:hi], v[b, :, lo:hi] = GARBAGE, math.inf
            k[b, :, lengths[b]:], v[b, :, lengths[b]:] = math.inf, GARBAGE
        out, lse = binding.window_attn_decode(prm, n_sink, window, q, k, v, sl, T)
        k64, v64 = k.double(), v.double()
    assert out.shape == (B, 1, G * H, D) and lse.shape == (B, G * H)
    for b, n in enumerate(lengths):
        for h in range(H):
            rows = slice(h * G, (h + 1) * G)
            if n == 0:
                assert not out[b, 0, rows].any() and (lse[b, rows] == -math.inf).all()
                continue
            seen = window_seen(torch.tensor([n - 1], device="cuda"), n, n_sink, window).expand(G, n)
            at = seen[0].nonzero()[:, 0]
            check(out[b, 0, rows], lse[b, rows], attend(q[b, 0, rows].double(), k64[b, h, at], v64[b, h, at], seen[:, at], prm.softmax_scale))


def block_lists(gen, lengths, H, n, topk, holes):
    idx = torch.full((len(lengths), H, n, topk), -1, dtype=torch.int32)
    rng = np.random.default_rng(int(torch.randint(0, 1 << 30, (1,), generator=gen, device="cuda")))
    for b, length in enumerate(lengths):
        for h in range(H):
            for i in range(n):
                own = max(0, length - n + i) // 64
                some = rng.permutation(own + 1)[:topk]
                if len(some) and own not in some:
                    some[0] = own
                if holes:
                    some = some[rng.random(len(some)) < 0.7]
                some = np.sort(some)
                idx[b, h, i, :len(some)] = torch.from_numpy(some.astype(np.int32))
                if holes and topk > len(some):
                    idx[b, h, i, topk - 1] = 1 << 25               # a block far behind the query: skipped
    return idx.cuda()


@pytest.mark.parametrize("G,H,lengths,topk,holes", [
    (16, 2, [1, 63, 64, 65, 1000, 0], 8, False), (1, 2, [777, 3], 3, True), (2, 3, [4000], 64, False), (4, 1, [130, 2048, 517], 5, True),
    (8, 2, [9000, 64], 16, False), (16, 1, [20000] * 3, 64, True), (16, 2, [5000] * 40, 12, False)])
def test_sparse_decode_quant(G, H, lengths, topk, holes):
    gen = torch.Generator(device="cuda").manual_seed(G + topk)
    B, T = len(lengths), max(lengths)
    prm = binding.Params(G * H, H, topk=topk)
    k, v = random_cache(gen, B, H, T, lengths, spoil=False)
    kq, vq = quant_of(prm, k, v, lengths)
    q = normal(gen, B, 1, G * H, D)
    idx = block_lists(gen, lengths, H, 1, topk, holes)
    out, lse = binding.sparse_attn_decode_quant(prm, q, kq, vq, lengths_tensor(lengths), T, idx)
    k64, v64 = values_of(kq), values_of(vq)
    for b, n in enumerate(lengths):
        for h in range(H):
            rows = slice(h * G, (h + 1) * G)
            chosen = [j for j in idx[b, h, 0].tolist() if 0 <= j < (n + 63) // 64]
            at = torch.tensor([t for j in chosen for t in range(64 * j, min(n, 64 * j + 64))], dtype=torch.long, device="cuda")
            if len(at) == 0:
                assert not out[b, 0, rows].any() and (lse[b, rows] == -math.inf).all()
                continue
            seen = torch.ones((G, len(at)), dtype=torch.bool, device="cuda")
            check(out[b, 0, rows], lse[b, rows], attend(q[b, 0, rows].double(), k64[b, h, at], v64[b, h, at], seen, prm.softmax_scale))


@pytest.mark.parametrize("G,H,lengths,n,topk,kind", [
    (16, 2, [300, 70, 16, 15], 16, 8, "tree"), (4, 1, [1000, 999], 2, 16, "chain"), (8, 2, [640, 641], 64, 3, "random"),
    (1, 2, [500], 5, 8, "empty"), (16, 1, [4096, 64, 63], 64, 12, "tree"), (2, 1, [333], 33, 4, "random")])
def test_sparse_verify_quant(G, H, lengths, n, topk, kind):
    gen = torch.Generator(device="cuda").manual_seed(n + topk)
    rng = np.random.default_rng(n)
    B, T = len(lengths), max(lengths) + 1
    prm = binding.Params(G * H, H, topk=topk)
    k, v = random_cache(gen, B, H, T, lengths, spoil=False)
    kq, vq = quant_of(prm, k, v, lengths)
    q = normal(gen, B, n, G * H, D)
    idx = block_lists(gen, lengths, H, n, topk, True)
    words = np.zeros((B, n), np.uint64)
    for b in range(B):
        for t in range(n):
            if kind == "tree":
                words[b, t] = (words[b, rng.integers(0, t)] if t else np.uint64(0)) | np.uint64(1) << np.uint64(t)
            elif kind == "random":                                 # any bits, those from n on ignored
                words[b, t] = rng.integers(0, 1 << 64, dtype=np.uint64)
    mask = None if kind == "chain" else torch.from_numpy(words.view(np.int64)).cuda()
    if kind == "empty":                                            # lists of the drafted tokens' own block only, masks of nothing
        idx[:] = -1
        idx[..., 0] = (torch.tensor(lengths) // 64).int().cuda()[:, None, None]
        lengths = [length // 64 * 64 + n for length in lengths]
        T = max(T, max(lengths))
        k, v = random_cache(gen, B, H, T, lengths, spoil=False)
        kq, vq = quant_of(prm, k, v, lengths)
    out, lse = binding.sparse_attn_verify_quant(prm, q, kq, vq, lengths_tensor(lengths), T, idx, tree_mask=mask)
    k64, v64 = values_of(kq), values_of(vq)
    for b, length in enumerate(lengths):
        for h in range(H):
            rows = slice(h * G, (h + 1) * G)
            for i in range(n):
                if length < n:
                    assert not out[b, i, rows].any() and (lse[b, i, rows] == -math.inf).all()
                    continue
                first, ts = length - n, []
                for j in idx[b, h, i].tolist():
                    for t in range(64 * j, min(64 * j + 64, length)) if j >= 0 else ():
                        if (t <= first + i) if mask is None else (t < first or int(words[b, i]) >> (t - first) & 1):
                            ts.append(t)
                if not ts:
                    assert not out[b, i, rows].any() and (lse[b, i, rows] == -math.inf).all()
                    continue
                at = torch.tensor(ts, device="cuda")
                seen = torch.ones((G, len(at)), dtype=torch.bool, device="cuda")
                check(out[b, i, rows], lse[b, i, rows], attend(q[b, i, rows].double(), k64[b, h, at], v64[b, h, at], seen, prm.softmax_scale))


# 63 to 66, 512 and 514 rows, units of 16, 17, 40 and 41: the sizes at which a row changes from one workgroup to several
@pytest.mark.parametrize("G,H,lengths,n_sink,window", [
    (16, 2, [1200 + 3 * i for i in range(32)] + [0, 1], 4, 1000), (16, 1, [1300] * 63, 0, 1200), (4, 2, [1300, 31, 900] * 11, 0, 1217),
    (8, 2, [700, 0] * 16, 0, 1250), (2, 4, [90 + i for i in range(128)], 1, 64), (1, 2, [200 + i % 7 for i in range(257)], 33, 97),
    (16, 1, [2000], 0, 480), (16, 1, [2000], 0, 481)])
@pytest.mark.parametrize("quant", [False, True])
def test_window_decode_rows_and_units(G, H, lengths, n_sink, window, quant):
    test_window_decode(G, H, lengths, n_sink, window, quant)


@pytest.mark.parametrize("G,H,lengths,n,topk,kind", [
    (16, 2, [900, 70], 16, 20, "tree"), (4, 2, [1700, 65], 16, 21, "random"), (16, 1, [800, 799], 31, 12, "tree"), (2, 8, [500, 40, 16], 22, 5, "chain")])
def test_sparse_verify_quant_rows_and_units(G, H, lengths, n, topk, kind):
    test_sparse_verify_quant(G, H, lengths, n, topk, kind)


@pytest.mark.parametrize("G,H,lengths,topk,holes", [(16, 2, [3000, 1, 0, 700] * 8, 20, True), (16, 2, [100 + 9 * i for i in range(260)], 4, False), (8, 1, [900], 8, True), (8, 1, [900], 9, True)])
def test_sparse_decode_quant_rows_and_units(G, H, lengths, topk, holes):
    test_sparse_decode_quant(G, H, lengths, topk, holes)


PREFILL_CASES = [  # G, Hkv, lengths, n_sink, window
    (1, 1, [1], 0, 1), (16, 2, [1, 7, 8, 9, 0], 1, 3), (1, 2, [300, 129, 128], 0, 1), (2, 1, [500], 4, 50),
    (4, 1, [777], 4, 256), (8, 2, [640, 333], 64, 100), (16, 2, [700, 1], 100, 64), (16, 1, [513], 600, 5),
    (4, 3, [400, 65], 0, 100000), (8, 1, [1500], 33, 1000), (2, 2, [1100], 130, 129), (16, 1, [1030], 0, 512),
    (16, 4, [1100, 3], 4, 100), (2, 8, [4200], 33, 70), (16, 8, [650], 0, 100000),
]


@pytest.mark.parametrize("G,H,lengths,n_sink,window", PREFILL_CASES)
def test_window_prefill(G, H, lengths, n_sink, window):
    gen = torch.Generator(device="cuda").manual_seed(G * 100 + window)
    B, T = len(lengths), max(lengths) + 2
    prm = binding.Params(G * H, H)
    k, v = random_cache(gen, B, H, T, lengths)
    q = normal(gen, B, G * H, T, D).transpose(1, 2)
    for b, n in enumerate(lengths):
        q[b, n:] = GARBAGE
    sl = lengths_tensor(lengths)
    out, lse = binding.window_attn_prefill(prm, n_sink, window, q, k, v, sl, T)
    own = torch.full((B, T + 1, G * H + 1, D), 9.0, dtype=torch.bfloat16, device="cuda")
    own_lse = torch.full((B, T, G * H), 9.0, dtype=torch.float32, device="cuda")
    binding.window_attn_prefill(prm, n_sink, window, q, k, v, sl, T, out=own[:, :, 1:], lse=own_lse)
    for b, n in enumerate(lengths):
        assert not out[b, n:].any() and not lse[b, n:].any()       # made by the call: cleared
        assert (own[b, n:] == 9).all() and (own[b, :, 0] == 9).all() and (own_lse[b, n:] == 9).all()   # the caller's: left alone
        assert torch.equal(own[b, :n, 1:], out[b, :n]) and torch.equal(own_lse[b, :n], lse[b, :n])
        for hq in range(G * H):
            if n:
                seen = window_seen(torch.arange(n, device="cuda"), n, n_sink, window)
                check(out[b, :n, hq], lse[b, :n, hq],
                      attend(q[b, :n, hq].double(), k[b, hq // G, :n].double(), v[b, hq // G, :n].double(), seen, prm.softmax_scale))


# around 64 and 128 workgroups of 128 rows and walks of 512 keys, and more runs of rows than XCDs
@pytest.mark.parametrize("G,H,lengths,n_sink,window", [(4, 1, [2049], 0, 511), (4, 1, [2049], 0, 512), (4, 1, [2080], 9, 503), (4, 1, [4096], 0, 600), (4, 1, [4097], 0, 600), (16, 2, [1000] * 8, 0, 1000)])
def test_window_prefill_rows_and_walks(G, H, lengths, n_sink, window):
    test_window_prefill(G, H, lengths, n_sink, window)


# workgroups by halves: up to 256 of them, walks of 512 keys or more, one tile and odd numbers of tiles among them
HALVES = [(4, 1, [5000], 0, 700), (16, 1, [700, 40, 64], 5, 600), (16, 2, [65, 900, 0, 1], 70, 500), (2, 4, [2048, 1985], 0, 513), (16, 2, [1200, 63], 100, 1100), (16, 2, [1200, 63], 99, 1100)]


@pytest.mark.parametrize("G,H,lengths,n_sink,window", HALVES)
def test_window_prefill_by_halves(G, H, lengths, n_sink, window):
    test_window_prefill(G, H, lengths, n_sink, window)


@pytest.mark.parametrize("G,H,lengths,n_sink,window", HALVES)
def test_window_bwd_by_halves(G, H, lengths, n_sink, window):
    test_window_bwd(G, H, lengths, n_sink, window)


def test_window_prefill_of_large_values():
    # values near bf16's largest: their sums overflow 32 bits before they are divided, their means do not
    gen = torch.Generator(device="cuda").manual_seed(6)
    n, prm = 300, binding.Params(4, 2)
    k, v = random_cache(gen, 1, 2, n, [n], spoil=False)
    v = (v.float().clamp(-1, 1) * 3e38).bfloat16()
    q = normal(gen, 1, n, 4, D)
    out, lse = binding.window_attn_prefill(prm, 4, 50, q, k, v, lengths_tensor([n]), n)
    seen = window_seen(torch.arange(n, device="cuda"), n, 4, 50)
    for hq in range(4):
        check(out[0, :, hq], lse[0, :, hq], attend(q[0, :, hq].double(), k[0, hq // 2].double(), v[0, hq // 2].double(), seen, prm.softmax_scale))


def bwd_reference(q, k, v, out, dout, lse, seen, scale):
    """one head in fp64 -> (dq, dk, dv) and their tolerances"""
    s = (q @ k.t().contiguous()) * scale
    p = torch.where(seen, torch.exp(s - lse[:, None]), 0.0)
    dp = dout @ v.t().contiguous()
    d = (dout * out).sum(-1, keepdim=True)
    ds = p * (dp - d)
    rough = p * (dout.abs() @ v.abs().t().contiguous() + (dout * out).abs().sum(-1, keepdim=True))
    move = 2.0 ** -17 * (q.abs() @ k.abs().t().contiguous()) * scale + 2.0 ** -22 * lse.abs()[:, None]   # of a probability
    t = lambda x: x.t().contiguous()
    err = HALF * ds.abs() + 2.0 ** -16 * rough + move * ds.abs()
    errp = (HALF + move) * p
    return ((ds @ k) * scale, t(ds) @ q * scale, t(p) @ dout,
            (err @ k.abs()) * scale, t(err) @ q.abs() * scale, t(errp) @ dout.abs())


BWD_CASES = PREFILL_CASES + [(16, 2, [1200, 900], 4, 100), (4, 1, [2100], 200, 1500)]


@pytest.mark.parametrize("G,H,lengths,n_sink,window", BWD_CASES)
def test_window_bwd(G, H, lengths, n_sink, window):
    gen = torch.Generator(device="cuda").manual_seed(G * 10 + window)
    B, T = len(lengths), max(lengths) + 2
    prm = binding.Params(G * H, H)
    k, v = random_cache(gen, B, H, T, lengths)
    q, dout = normal(gen, B, G * H, T, D).transpose(1, 2), normal(gen, B, T, G * H, D)
    for b, n in enumerate(lengths):
        q[b, n:], dout[b, n:] = GARBAGE, GARBAGE
    sl = lengths_tensor(lengths)
    out, lse = binding.window_attn_prefill(prm, n_sink, window, q, k, v, sl, T)
    for b, n in enumerate(lengths):
        out[b, n:], lse[b, n:] = GARBAGE, GARBAGE
    grads = binding.window_attn_bwd(prm, n_sink, window, q, k, v, out, dout, lse, sl, T)
    again = [torch.full_like(x, 9.0) for x in grads]
    need = binding.window_workspace_bytes(binding.OP_WINDOW_BWD, prm, n_sink, window, B, T)
    ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
    binding.window_attn_bwd(prm, n_sink, window, q, k, v, out, dout, lse, sl, T, dq=again[0], dk=again[1], dv=again[2], workspace=ws)
    for b, n in enumerate(lengths):
        assert not grads[0][b, n:].any() and not grads[1][b, :, n:].any() and not grads[2][b, :, n:].any()
        assert (again[0][b, n:] == 9).all() and (again[1][b, :, n:] == 9).all() and (again[2][b, :, n:] == 9).all()
        assert torch.equal(again[0][b, :n], grads[0][b, :n])       # results repeat
        assert all(torch.equal(x[b, :, :n], y[b, :, :n]) for x, y in zip(again[1:], grads[1:]))
        if n == 0:
            continue
        seen = window_seen(torch.arange(n, device="cuda"), n, n_sink, window)
        for h in range(H):
            sums = None
            for hq in range(h * G, (h + 1) * G):
                x = [y.double() for y in (q[b, :n, hq], k[b, h, :n], v[b, h, :n], out[b, :n, hq], dout[b, :n, hq], lse[b, :n, hq])]
                r = bwd_reference(*x, seen, prm.softmax_scale)
                tol = 1.0625 * r[3] + HALF * r[0].abs() + 1e-30
                diff = (grads[0][b, :n, hq].double() - r[0]).abs()
                assert (diff <= tol).all(), ("dq", float((diff / tol).max()))
                part = r[1:3] + r[4:6]
                sums = part if sums is None else [a + c for a, c in zip(sums, part)]
            for name, got, want, err in (("dk", grads[1], sums[0], sums[2]), ("dv", grads[2], sums[1], sums[3])):
                tol = 1.0625 * err + HALF * want.abs() + 1e-30
                diff = (got[b, h, :n].double() - want).abs()
                assert (diff <= tol).all(), (name, float((diff / tol).max()))


@pytest.mark.parametrize("G,H,lengths,n_sink,window", [(4, 1, [2049], 0, 511), (4, 1, [2080], 9, 503), (4, 1, [4097], 0, 600), (16, 2, [1000] * 8, 0, 1000), (2, 1, [1100, 1, 0, 515] * 3, 0, 1100)])
def test_window_bwd_rows_and_walks(G, H, lengths, n_sink, window):
    test_window_bwd(G, H, lengths, n_sink, window)


@pytest.mark.parametrize("G,H,n,n_sink,window,at", [(16, 2, 200, 4, 20, 70), (1, 1, 400, 0, 129, 255), (4, 2, 3000, 3, 100, 1), (8, 4, 1500, 0, 64, 1499), (16, 4, 1100, 70, 33, 1000)])
def test_window_prefill_keeps_what_is_not_finite_where_it_is_seen(G, H, n, n_sink, window, at):
    gen = torch.Generator(device="cuda").manual_seed(n)
    prm = binding.Params(G * H, H)
    k, v = random_cache(gen, 1, H, n, [n])
    q = normal(gen, 1, n, G * H, D)
    v[0, 0, at, 5], v[0, H - 1, at, 127] = math.inf, GARBAGE
    out, lse = binding.window_attn_prefill(prm, n_sink, window, q, k, v, lengths_tensor([n]), n)
    seen = window_seen(torch.arange(n, device="cuda"), n, n_sink, window)
    hit = seen[:, at]
    for hq in range(G * H):
        h = hq // G
        clean = torch.nan_to_num(v[0, h].double(), nan=0.0, posinf=0.0)
        want = attend(q[0, :, hq].double(), k[0, h].double(), clean, seen, prm.softmax_scale)
        check(out[0, ~hit, hq], lse[0, ~hit, hq], [x[~hit] for x in want])
        finite = torch.isfinite(out[0, :, hq])
        bad = [c for c, hh in ((5, 0), (127, H - 1)) if hh == h]
        assert not finite[hit][:, bad].any() and finite[~hit].all()
        rest = [c for c in range(D) if c not in bad]               # the other channels of the same value: whole
        check(out[0, hit, hq][:, rest], lse[0, hit, hq], [x[hit][:, rest] if x.dim() == 2 else x[hit] for x in want])


# ---- as they are used ---------------------------------------------------------------------------------------------

@pytest.mark.parametrize("G,H,n,n_sink,window,at", [(16, 2, 700, 0, 600, 50), (16, 2, 700, 3, 513, 127), (4, 1, 5000, 0, 700, 4000)])
def test_halves_keep_what_is_not_finite_where_it_is_seen(G, H, n, n_sink, window, at):
    test_window_prefill_keeps_what_is_not_finite_where_it_is_seen(G, H, n, n_sink, window, at)


def test_gradients_are_differences():
    # a loss <out, w> along random directions: the calls' gradients against central differences of the definition in 64 bits
    G, H, n, n_sink, window = 4, 2, 90, 3, 17
    gen = torch.Generator(device="cuda").manual_seed(5)
    prm = binding.Params(G * H, H)
    q, w = normal(gen, 1, n, G * H, D), normal(gen, 1, n, G * H, D)
    k, v = random_cache(gen, 1, H, n, [n], spoil=False)
    sl = lengths_tensor([n])
    seen = window_seen(torch.arange(n, device="cuda"), n, n_sink, window)

    def loss(q, k, v):
        total = 0.0
        for hq in range(G * H):
            o, *_ = attend(q[0, :, hq], k[0, hq // G], v[0, hq // G], seen, prm.softmax_scale)
            total = total + (o * w[0, :, hq].double()).sum()
        return float(total)

    out, lse = binding.window_attn_prefill(prm, n_sink, window, q, k, v, sl, n)
    grads = binding.window_attn_bwd(prm, n_sink, window, q, k, v, out, w, lse, sl, n)
    x = [q.double(), k.double(), v.double()]
    for i, g in enumerate(grads):
        for _ in range(4):
            d = torch.randn(x[i].shape, generator=gen, device="cuda", dtype=torch.float64)
            h = 1e-4                                               # central: error h^2 of the third derivative, 64-bit rounding 1e-16 / h
            at = lambda s: loss(*[y + s * d if j == i else y for j, y in enumerate(x)])
            slope = (at(h) - at(-h)) / (2 * h)
            # a gradient's elements are rounded independently, 2^-8 of each at most (two roundings of 2^-9 on average): their sum along d is
            # off by that of the root of the sum of squares, five times over
            tol = 5 * 2.0 ** -8 * float((g.double() * d).norm()) + 1e-3
            assert abs(float((g.double() * d).sum()) - slope) <= tol, (i, float((g.double() * d).sum()), slope, tol)


def serve(prm, gen, lengths, steps, graph):
    """a prompt, its cache in 4 bits, then decode steps on it: append, select, attend; checked against the path's own calls on the cache read
    back.  Returns the outputs."""
    B, H, Hq, T = len(lengths), prm.n_kv_heads, prm.n_q_heads, max(lengths) + steps
    k, v = random_cache(gen, B, H, T, lengths, spoil=False)
    q = normal(gen, B, T, Hq, D)
    sl = lengths_tensor(lengths)
    ck = torch.zeros((B, H, binding.num_kernels(T, prm), D), dtype=torch.bfloat16, device="cuda")
    binding.compress_keys(prm, k, sl, T, ck=ck)
    idx = binding.select_blocks(prm, binding.MODE_PREFILL, q, ck, sl, T)
    binding.sparse_attn_prefill(prm, q, k, v, sl, T, idx)
    kq, vq = binding.quantize_kv(prm, k, v, sl, T)
    new = [normal(gen, steps, B, H, 1, D) for _ in range(2)]
    queries = normal(gen, steps, B, 1, Hq, D)
    ws = torch.empty(max(binding.workspace_bytes(op, prm, B, T) for op in (binding.OP_SELECT_DECODE, binding.OP_ATTN_DECODE)),
                     dtype=torch.uint8, device="cuda")
    now = [torch.empty_like(x[0]) for x in (*new, queries)]
    bufs = dict(out=torch.empty((B, 1, Hq, D), dtype=torch.bfloat16, device="cuda"),
                lse=torch.empty((B, Hq), dtype=torch.float32, device="cuda"), workspace=ws)
    block_idx = torch.empty((B, H, 1, prm.topk), dtype=torch.int32, device="cuda")

    def step():
        sl.add_(1)
        binding.append_kv_quant(prm, now[0], now[1], kq, vq, sl, T, ck=ck)
        binding.select_blocks(prm, binding.MODE_DECODE, now[2], ck, sl, T, block_idx=block_idx, workspace=ws)
        binding.sparse_attn_decode_quant(prm, now[2], kq, vq, sl, T, block_idx, **bufs)

    captured = None
    if graph:
        saved = [x.clone() for x in (sl, ck, *kq, *vq)]
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            for x, y in zip(now, (*new, queries)):
                x.copy_(y[0])
            step()
        torch.cuda.current_stream().wait_stream(side)
        captured = torch.cuda.CUDAGraph()
        with torch.cuda.graph(captured, stream=side):
            step()
        for x, y in zip((sl, ck, *kq, *vq), saved):
            x.copy_(y)
    results = []
    for i in range(steps):
        for x, y in zip(now, (*new, queries)):
            x.copy_(y[i])
        captured.replay() if captured else step()
        kb, vb = binding.dequantize_kv(prm, kq, vq, sl, T)         # the program's own work between the steps
        want, want_lse = binding.sparse_attn_decode(prm, now[2], kb, vb, sl, T, block_idx)
        # both round probabilities to bf16 (2^-8 of |o| <= sum p |v|) and the result; |v| of N(0,1) in 4 bits is at most 6
        assert (bufs["out"].float() - want.float()).abs().max() <= 4 * HALF * 6
        assert (bufs["lse"] - want_lse).abs().max() <= 1e-4
        own = (sl - 1) // 64
        assert torch.equal(block_idx.amax(-1)[:, :, 0], own[:, None].expand(-1, H).to(torch.int32))
        results.append([x.clone() for x in (bufs["out"], bufs["lse"], block_idx, ck, *kq, *vq)])
    return results


@pytest.mark.parametrize("hq,hkv,lengths,topk", [(32, 2, [777, 1300], 8), (4, 1, [4090], 16), (2, 2, [100, 40, 63], 3)])
def test_a_prompt_and_decode_steps_on_the_4_bit_cache(hq, hkv, lengths, topk):
    prm = binding.Params(hq, hkv, topk=topk)
    eager = serve(prm, torch.Generator(device="cuda").manual_seed(3), lengths, 18, False)
    replayed = serve(prm, torch.Generator(device="cuda").manual_seed(3), lengths, 18, True)
    for a, b in zip(eager, replayed):
        assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_verification_step_on_the_4_bit_cache():
    # append and verify n drafted tokens; without a mask it is n decode steps
    prm = binding.Params(8, 2, topk=8)
    gen = torch.Generator(device="cuda").manual_seed(9)
    lengths, n, T = [500, 37], 7, 512
    k, v = random_cache(gen, 2, 2, T, lengths, spoil=False)
    new = [normal(gen, 2, 2, n, D) for _ in range(2)]
    q = normal(gen, 2, n, 8, D)
    ck = binding.compress_keys(prm, k, lengths_tensor(lengths), T)
    one, two = [[binding.QuantCache(*(y.clone() for y in x)) for x in binding.quantize_kv(prm, k, v, lengths_tensor(lengths), T)] + [ck.clone()] for _ in range(2)]
    sl = lengths_tensor([x + n for x in lengths])
    binding.append_kv_quant(prm, *new, one[0], one[1], sl, T, ck=one[2])
    idx = binding.select_blocks_verify(prm, q, one[2], sl, T)
    out, lse = binding.sparse_attn_verify_quant(prm, q, one[0], one[1], sl, T, idx)
    for i in range(n):
        at = lengths_tensor([x + i + 1 for x in lengths])
        binding.append_kv_quant(prm, new[0][:, :, i:i + 1], new[1][:, :, i:i + 1], two[0], two[1], at, T, ck=two[2])
        qi = q[:, i:i + 1]
        di = binding.select_blocks(prm, binding.MODE_DECODE, qi, two[2], at, T)
        assert torch.equal(di, idx[:, :, i:i + 1])
        o, z = binding.sparse_attn_decode_quant(prm, qi, two[0], two[1], at, T, di)
        assert (o[:, 0].float() - out[:, i].float()).abs().max() <= 4 * HALF * 6 and (z - lse[:, i]).abs().max() <= 1e-5
    for x, y in zip((*one[0], *one[1], one[2]), (*two[0], *two[1], two[2])):
        assert torch.equal(x, y)


def test_window_training_step_captured():
    # forward and backward in one graph, replayed with new inputs, eager work and synchronisations in between
    prm = binding.Params(16, 2)
    gen = torch.Generator(device="cuda").manual_seed(2)
    B, T, n_sink, window = 2, 900, 4, 200
    sl = lengths_tensor([900, 650])
    x = [normal(gen, B, T, 16, D), normal(gen, B, 2, T, D), normal(gen, B, 2, T, D), normal(gen, B, T, 16, D)]

    def both(q, k, v, dout):
        out, lse = binding.window_attn_prefill(prm, n_sink, window, q, k, v, sl, T)
        return (out, lse, *binding.window_attn_bwd(prm, n_sink, window, q, k, v, out, dout, lse, sl, T))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        both(*x)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        got = both(*x)
    for i in range(4):
        for y in x:
            y.normal_(generator=gen)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, both(*x))), i


def test_two_streams_at_once():
    # calls on two streams with workspaces of their own, and results and scratch made by the call on each
    prm = binding.Params(16, 1)
    gen = torch.Generator(device="cuda").manual_seed(4)
    T, sl = 2048, lengths_tensor([2048])
    sets = [(normal(gen, 1, T, 16, D), *random_cache(gen, 1, 1, T, [T])) for _ in range(2)]

    def work(q, k, v):
        kq, vq = binding.quantize_kv(prm, k, v, sl, T)
        out, lse = binding.window_attn_prefill(prm, 4, 500, q, k, v, sl, T)
        last = q[:, -1:]
        return [out, lse, *binding.window_attn_bwd(prm, 4, 500, q, k, v, out, q, lse, sl, T), *kq, *vq,
                *binding.window_attn_decode(prm, 4, 500, last, k, v, sl, T), *binding.window_attn_decode_quant(prm, 4, 500, last, kq, vq, sl, T)]

    want = [work(*s) for s in sets]
    streams = [torch.cuda.Stream() for _ in sets]
    torch.cuda.synchronize()
    for _ in range(3):
        got = []
        for s, st in zip(sets, streams):
            with torch.cuda.stream(st):
                got.append(work(*s))
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for x, y in zip(got, want) for a, b in zip(x, y))


def test_caches_beyond_32_bits():
    # a cache whose last head lies 4 GiB and more behind the first: offsets of heads and sequences are 64-bit
    prm = binding.Params(2, 2)
    gen = torch.Generator(device="cuda").manual_seed(8)
    T, n = 9_000_000, 100
    k = torch.zeros((1, 2, T, D), dtype=torch.bfloat16, device="cuda")     # 4.6 GB
    k[:, :, :n], k[:, :, T - n:] = normal(gen, 1, 2, n, D), normal(gen, 1, 2, n, D)
    q = normal(gen, 1, 1, 2, D)
    sl = lengths_tensor([T])
    seen = torch.ones((1, 2 * n), dtype=torch.bool, device="cuda")
    kq, vq = binding.quantize_kv(prm, k, k, sl, T)
    for out, lse, src in ((*binding.window_attn_decode(prm, n, n, q, k, k, sl, T), k),
                          (*binding.window_attn_decode_quant(prm, n, n, q, kq, vq, sl, T), None)):
        for h in range(2):
            x = values_of(binding.QuantCache(*(torch.cat((y[0, h, :n], y[0, h, T - n:])) for y in kq))) if src is None else \
                torch.cat((k[0, h, :n], k[0, h, T - n:])).double()
            check(out[0, 0, h:h + 1], lse[0, h:h + 1], attend(q[0, 0, h:h + 1].double(), x, x, seen, prm.softmax_scale))


def test_caches_of_no_rows():
    """max_seqlen 0: nothing is seen; where results have no memory the call is refused, as everywhere."""
    gen = torch.Generator(device="cuda").manual_seed(4)
    prm = binding.Params(8, 2, topk=4)
    k, v = normal(gen, 3, 2, 64, D), normal(gen, 3, 2, 64, D)
    q, sl = normal(gen, 3, 1, 8, D), lengths_tensor([5, 0, -1])
    kq, vq = binding.quantize_kv(prm, k, v, sl, 0)
    assert not kq.codes.any() and not vq.scales.any()
    assert not any(x.any() for x in binding.dequantize_kv(prm, kq, vq, sl, 0, k=torch.zeros_like(k), v=torch.zeros_like(v)))
    idx = torch.zeros((3, 2, 1, 4), dtype=torch.int32, device="cuda")
    for out, lse in (binding.window_attn_decode(prm, 0, 8, q, k, v, sl, 0), binding.window_attn_decode(prm, 3, 8, q, k, v, sl, 0),
                     binding.window_attn_decode_quant(prm, 3, 8, q, kq, vq, sl, 0), binding.sparse_attn_decode_quant(prm, q, kq, vq, sl, 0, idx)):
        assert not out.any() and (lse == -math.inf).all()
    qs = normal(gen, 3, 64, 8, D)
    for call in (lambda: binding.dequantize_kv(prm, kq, vq, sl, 0), lambda: binding.window_attn_prefill(prm, 0, 8, qs, k, v, sl, 0)):
        with pytest.raises(binding.InfLLMv2Error):
            call()


def test_refusals_of_the_binding():
    prm = binding.Params(4, 1)
    gen = torch.Generator(device="cuda").manual_seed(1)
    T = 64
    q, k, v = normal(gen, 1, T, 4, D), normal(gen, 1, 1, T, D), normal(gen, 1, 1, T, D)
    sl = lengths_tensor([T])
    kq, vq = binding.quantize_kv(prm, k, v, sl, T)
    idx = torch.zeros((1, 1, 1, prm.topk), dtype=torch.int32, device="cuda")
    one = q[:, :1]
    lse = torch.zeros((1, T, 4), device="cuda")
    QC = binding.QuantCache
    bad = [
        lambda: binding.quantize_kv(prm, k, v, sl, T + 1),                                   # longer than the cache
        lambda: binding.quantize_kv(prm, k, v.float(), sl, T),
        lambda: binding.quantize_kv(prm, k, v[:, :, :T - 1], sl, T),
        lambda: binding.quantize_kv(prm, k, v, sl.long(), T),
        lambda: binding.quantize_kv(prm, k, v, lengths_tensor([T, T]), T),
        lambda: binding.quantize_kv(prm, k, v, sl, -1),
        lambda: binding.quantize_kv(prm, k, v, sl, T, QC(kq.codes[..., :32], kq.scales), vq),
        lambda: binding.quantize_kv(prm, k, v, sl, T, kq),
        lambda: binding.dequantize_kv(prm, QC(kq.codes, kq.scales.int()), vq, sl, T),
        lambda: binding.dequantize_kv(prm, QC(kq.codes.cpu(), kq.scales), vq, sl, T),
        lambda: binding.dequantize_kv(prm, kq, vq, sl, T, k=k[..., :64]),
        lambda: binding.append_kv_quant(prm, k[:, :, :2], v[:, :, :1], kq, vq, sl, T),
        lambda: binding.append_kv_quant(prm, k[:, :, :0], v[:, :, :0], kq, vq, sl, T),
        lambda: binding.append_kv_quant(prm, k[:, :, :1], v[:, :, :1], kq, vq, sl, T, ck=k[:, :, :2]),
        lambda: binding.sparse_attn_decode_quant(prm, q, kq, vq, sl, T, idx),                # more than one row
        lambda: binding.sparse_attn_decode_quant(prm, one, kq, vq, sl, T, idx[..., :3]),
        lambda: binding.sparse_attn_decode_quant(prm, one, kq, vq, sl, T, idx, out=q[:, :, :2]),
        lambda: binding.sparse_attn_verify_quant(prm, q[:, :3], kq, vq, sl, T, idx),
        lambda: binding.window_attn_prefill(prm, -1, 8, q, k, v, sl, T),
        lambda: binding.window_attn_prefill(prm, 0, 0, q, k, v, sl, T),
        lambda: binding.window_attn_prefill(prm, 0, 8, q[:, :T - 1], k, v, sl, T),
        lambda: binding.window_attn_prefill(prm, 0, 8, q, k, v, sl, T, lse=lse[:, :, :2]),
        lambda: binding.window_attn_prefill(prm, 0, 1 << 31, q, k, v, sl, T),
        lambda: binding.window_attn_bwd(prm, 0, 8, q, k, v, q, q, lse.half(), sl, T),
        lambda: binding.window_attn_bwd(prm, 0, 8, q, k, v, q, q, lse, sl, T, workspace=torch.empty(256, dtype=torch.uint8, device="cuda")),
        lambda: binding.window_attn_decode(prm, 0, 8, q, k, v, sl, T),
        lambda: binding.window_attn_decode_quant(prm, 0, 8, one, k, v, sl, T),
    ]
    for i, call in enumerate(bad):
        with pytest.raises(binding.InfLLMv2Error):
            call()
            pytest.fail("call %d was not refused" % i)
    # a sequence that claims to be longer than max_seqlen is clamped to it, a negative length is none
    out, _ = binding.window_attn_prefill(prm, 0, 8, q, k, v, sl, T)
    assert torch.equal(binding.window_attn_prefill(prm, 0, 8, q, k, v, lengths_tensor([1000]), T)[0], out)
    assert not binding.window_attn_prefill(prm, 0, 8, q, k, v, lengths_tensor([-5]), T)[0].any()
    assert torch.equal(binding.window_attn_decode(prm, 0, 8, one, k, v, lengths_tensor([1000]), T)[0],
                       binding.window_attn_decode(prm, 0, 8, one, k, v, sl, T)[0])
