"""Rotary positions and the cache in pages against plain 64-bit computations of their definitions.

Tolerances, derived from the roundings of the calls (half a step of bf16 is 2^-8 of a value):
  rotation    the result is rounded once: 2^-8 |y|; cosine, sine, their products with the amplitude and the sum are off by a few 2^-24 each: 2^-20 (|a| + |b|)
  attention   a probability is rounded to bf16 once, the output once: 2^-8 (sum p |v| + |o|), a sixteenth more for the fp32 sums and the scores' own
              rounding (a dot product of 128 exact products is off by at most 2^-17 of the sum of their sizes, which moves a probability by that much)
  log-sum-exp 2^-17 of the largest logit's sum of sizes, and 2^-20 for the sum's, the exponentials' and the logarithm's roundings, and the result's
              own rounding
  weights     each term by its score's 2^-17, by 2^-22 of the score and the log-sum-exp (their products with log2 e) and by the exponential's 2^-22; a sum of
              N terms by N / 32 + 8 additions of 2^-24
  copies, choices   equal
"""
import math

import pytest
import torch

from paper_2506_07900_amd import binding

pytestmark = pytest.mark.gpu

D = 128
HALF = 2.0 ** -8
NAN = float("nan")
SCALE = D ** -0.5


def gen_of(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def normal(gen, *shape, scale=1.0):
    return (torch.randn(shape, generator=gen, device="cuda") * scale).bfloat16()


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


# ---- pages -------------------------------------------------------------------------------------------------------

def make_pages(gen, lengths, hkv, page, spare=2, fill=NAN):
    """-> PagedCache with pages in random order; unused rows, pages and table entries hold what must not matter"""
    counts = [(x + page - 1) // page for x in lengths]
    total = sum(counts) + spare
    order = torch.randperm(total, generator=torch.Generator().manual_seed(int(gen.initial_seed()))).int()
    table = torch.full((len(lengths), max(1, max(counts))), total - 1, dtype=torch.int32)
    at = 0
    for b, n in enumerate(counts):
        table[b, :n] = order[at:at + n]
        at += n
    k, v = (torch.full((total, hkv, page, D), fill, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    return binding.PagedCache(k, v, table.cuda())


def rows_of(cache, pool, b, length):
    """[Hkv, length, D] of a sequence"""
    page = pool.shape[2]
    n = (length + page - 1) // page
    return pool[cache.table[b, :n].long()].transpose(0, 1).reshape(pool.shape[1], n * page, D)[:, :length]


def write_rows(cache, pool, b, rows):
    """rows [Hkv, length, D] into the pages of sequence b"""
    page = pool.shape[2]
    t = torch.arange(rows.shape[1], device="cuda")
    pool[cache.table[b].long()[t // page], :, t % page] = rows.transpose(0, 1)


def filled(gen, lengths, hkv, page, heavy=False, **kw):
    cache = make_pages(gen, lengths, hkv, page, **kw)
    for b, n in enumerate(lengths):
        for pool in (cache.k, cache.v):
            x = normal(gen, hkv, n, D)
            if heavy and pool is cache.k:
                x = (x.float() * torch.exp(0.7 * torch.randn((hkv, n, 1), generator=gen, device="cuda"))).bfloat16()
            write_rows(cache, pool, b, x)
    return cache


# ---- rotary positions ----------------------------------------------------------------------------------------------

def frequencies(rot, base=10000.0, scaling="none", factor=1.0, original_len=0, pair_factors=None, beta_fast=32.0, beta_slow=1.0):
    """radians per position, and the amplitude"""
    j = torch.arange(rot // 2, dtype=torch.float64)
    if scaling == "ntk":
        base = base * factor ** (rot / (rot - 2))
    f = base ** (-2 * j / rot)
    amplitude = 1.0
    if scaling == "linear":
        f = f / factor
    elif scaling == "yarn":
        keep = ((original_len * f / (2 * math.pi) - beta_slow) / (beta_fast - beta_slow)).clamp(0, 1)
        f = f * (keep + (1 - keep) / factor)
        amplitude = 0.1 * math.log(factor) + 1
    elif scaling == "factors":
        f = f / torch.tensor(pair_factors, dtype=torch.float64)
        amplitude = math.sqrt(1 + math.log(factor) / math.log(original_len))
    return f, amplitude


def rotated64(x, position, f, amplitude, interleaved, back=False):
    """x [rows, heads, D] fp64 on the CPU or GPU, position [rows] -> values, and |a| + |b| of each element's pair times the amplitude"""
    x = x.double()
    rot = 2 * len(f)
    angle = torch.remainder(position.double()[:, None] * f.to(x.device), 2 * math.pi)[:, None]
    c, s = amplitude * torch.cos(angle), amplitude * torch.sin(angle) * (-1 if back else 1)
    y, size = x.clone(), torch.zeros_like(x)
    i, j = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, rot // 2), slice(rot // 2, rot))
    a, b = x[..., i], x[..., j]
    y[..., i], y[..., j] = a * c - b * s, b * c + a * s
    size[..., i] = size[..., j] = amplitude * (a.abs() + b.abs())
    return y, size


ROTATIONS = [
    dict(rot_dim=128), dict(rot_dim=128, interleaved=True), dict(rot_dim=64, interleaved=True), dict(rot_dim=16), dict(rot_dim=96, scaling="linear", factor=3.5),
    dict(rot_dim=32, interleaved=True, scaling="ntk", factor=8.0), dict(rot_dim=128, scaling="yarn", factor=16.0, original_len=4096),
    dict(rot_dim=64, scaling="factors", factor=4.0, original_len=2048, pair_factors=[1.0 + 0.1 * j for j in range(32)]),
    dict(rot_dim=112, base=500000.0),
]


def plain_table(kw):
    kw = {k: v for k, v in kw.items() if k not in ("interleaved", "rot_dim")}
    return kw


def far_positions(gen, b, t):
    """small, large, negative and the extreme ones.  (A product with a frequency in 64 bits is off by 2^-53 of it: 2^-22 at 2^31.)"""
    p = torch.randint(-2 ** 31, 2 ** 31 - 1, (b, t), generator=gen, device="cuda")
    p[:, ::3] = torch.randint(0, 5000, p[:, ::3].shape, generator=gen, device="cuda")
    p[:, ::7] = torch.randint(0, 1 << 20, p[:, ::7].shape, generator=gen, device="cuda")
    flat = p.view(-1)
    for i, x in enumerate([2 ** 31 - 1, -2 ** 31, 0, -1][:flat.numel()]):
        flat[i] = x
    return p.int()


def close_rotation(got, want, size):
    assert bool(((got.double() - want).abs() <= HALF * want.abs() + 2.0 ** -20 * size).all())


@pytest.mark.parametrize("kw", ROTATIONS, ids=lambda kw: "%s_%d%s" % (kw.get("scaling", "none"), kw["rot_dim"], "i" if kw.get("interleaved") else ""))
@pytest.mark.parametrize("hq,hkv,t,lengths,far", [(32, 2, 70, [70, 33, 1], True), (4, 4, 5, [5], False), (1, 1, 1, [1, 0], True), (16, 1, 4500, [4500], False), (32, 2, 4000, [4000], False)])
def test_rotation(kw, hq, hkv, t, lengths, far):
    gen, b = gen_of(t + kw["rot_dim"]), len(lengths)
    prm, rope = binding.Params(hq, hkv), binding.rope_table(**kw)
    f, amplitude = frequencies(kw["rot_dim"], **plain_table(kw))
    assert rope.amplitude == pytest.approx(amplitude, rel=2 ** -23)
    q, k = normal(gen, b, t, hq, D), normal(gen, b, hkv, t, D)
    positions = far_positions(gen, b, t) if far else None
    for call, back in ((binding.rope, False), (binding.rope_bwd, True)):
        qo, ko = call(prm, rope, q, k, i32(lengths), t, positions=positions)
        for i, n in enumerate(lengths):
            p = positions[i, :n] if far else torch.arange(n, device="cuda")
            for got, x in ((qo[i], q[i]), (ko[i].transpose(0, 1), k[i].transpose(0, 1))):
                want, size = rotated64(x[:n], p, f, amplitude, kw.get("interleaved", False), back)
                close_rotation(got[:n], want, size)
                assert bool((got[:n, :, kw["rot_dim"]:] == x[:n, :, kw["rot_dim"]:]).all())
                assert not bool(got[n:].any())                   # (made by the call: rows behind a sequence are zeros)


def test_rotation_layouts():
    """slices of one projection, in place, queries or keys alone, given outputs whose other rows stay"""
    gen = gen_of(3)
    b, t, hq, hkv = 2, 40, 8, 2
    prm, rope, sl = binding.Params(hq, hkv), binding.rope_table(64), i32([40, 17])
    qkv = normal(gen, b, t, hq + 2 * hkv, D)
    q, k = qkv[:, :, :hq], qkv[:, :, hq:hq + hkv].transpose(1, 2)
    want_q, want_k = binding.rope(prm, rope, q.contiguous(), k.contiguous(), sl, t)
    for given in ((q, k), (q, None), (None, k)):
        got = binding.rope(prm, rope, *given, sl, t)
        assert (got[0] is None) == (given[0] is None) and (got[1] is None) == (given[1] is None)
        assert got[0] is None or torch.equal(got[0], want_q)
        assert got[1] is None or torch.equal(got[1], want_k)
    before = qkv.clone()
    out = binding.rope(prm, rope, q, k, sl, t, q_out=q, k_out=k)
    assert out[0] is q and out[1] is k
    for i, n in enumerate([40, 17]):
        assert torch.equal(q[i, :n], want_q[i, :n]) and torch.equal(k[i, :, :n], want_k[i, :, :n])
        assert torch.equal(qkv[i, n:], before[i, n:])
    assert torch.equal(qkv[:, :, hq + hkv:], before[:, :, hq + hkv:])


def test_rotation_gradient_is_the_transposed_map():
    """<rope(x), y> = <x, rope_bwd(y)> for every x, y, and differences of the forward: the map is linear.  With x and y of few bits, the sums' errors are the
    results' roundings: 2^-8 of each product's size."""
    gen = gen_of(5)
    t, hq, hkv = 129, 4, 2
    prm, sl = binding.Params(hq, hkv), i32([t])
    for kw in ROTATIONS:
        rope = binding.rope_table(**kw)
        x, y = normal(gen, 1, t, hq, D), normal(gen, 1, t, hq, D)
        fx = binding.rope(prm, rope, x, None, sl, t)[0].double()
        by = binding.rope_bwd(prm, rope, y, None, sl, t)[0].double()
        left, right = (fx * y.double()).sum(-1), (x.double() * by).sum(-1)
        size = (fx * y.double()).abs().sum(-1) + (x.double() * by).abs().sum(-1)
        small = 2.0 ** -19 * rope.amplitude * (x.double().abs().amax(-1) * y.double().abs().sum(-1) * 2)
        assert bool(((left - right).abs() <= HALF * size + small).all())
        # plain autograd of the definition
        f, amplitude = frequencies(kw["rot_dim"], **plain_table(kw))
        z = x[0].double().requires_grad_()
        rotated64(z, torch.arange(t, device="cuda"), f, amplitude, kw.get("interleaved", False))[0].backward(y[0].double())
        _, size = rotated64(y[0], torch.arange(t, device="cuda"), f, amplitude, kw.get("interleaved", False))
        close_rotation(by[0], z.grad, size)


# ---- the append ------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("page", [16, 32, 64, 256])
@pytest.mark.parametrize("hq,hkv,lengths,counts,n", [(32, 2, [100, 17, 5, 64], [7, 0, 5, 1], 7), (4, 1, [1], None, 1), (8, 8, [300, 257], [33, 70], 70),
                                                     (2, 1, [4300], None, 4200),
                                                     (32, 2, [4200], None, 4000)])
def test_append(page, hq, hkv, lengths, counts, n):
    gen, b, cap = gen_of(page + n), len(lengths), max(lengths)
    prm, rope = binding.Params(hq, hkv), binding.rope_table(64, interleaved=True)
    cache = make_pages(gen, lengths, hkv, page)
    before = [x.clone() for x in (cache.k, cache.v)]
    k_new, v_new, q = normal(gen, b, hkv, n, D), normal(gen, b, hkv, n, D), normal(gen, b, n, hq, D)
    new = counts or [n] * b
    positions = torch.randint(0, 1 << 20, (b, n), generator=gen, device="cuda").int()
    for use_rope, pos in ((False, None), (True, None), (True, positions)):
        cache.k.copy_(before[0])
        cache.v.copy_(before[1])
        got = binding.paged_append(prm, k_new, v_new, cache, i32(lengths), cap, n_new=None if counts is None else i32(counts),
                                   rope=rope if use_rope else None, positions=pos, q=q if use_rope else None)
        assert (got is None) == (not use_rope)
        want = [x.clone() for x in before]
        for i, (length, m) in enumerate(zip(lengths, new)):
            first = length - m
            keys = k_new[i:i + 1, :, :m]
            if use_rope and m:
                p = (torch.arange(first, length, device="cuda").int()[None] if pos is None else pos[i:i + 1, :m]).contiguous()
                qo, keys = binding.rope(prm, rope, q[i:i + 1, :m], keys, i32([m]), m, positions=p)
                assert torch.equal(got[i, :m], qo[0])
            if use_rope:
                assert not bool(got[i, m:].any())
            t = torch.arange(first, length, device="cuda")
            at = cache.table[i].long()[t // page]
            want[0][at, :, t % page] = keys[0].transpose(0, 1)
            want[1][at, :, t % page] = v_new[i, :, :m].transpose(0, 1)
        for x, y in ((cache.k, want[0]), (cache.v, want[1])):
            assert torch.equal(x.view(torch.int16), y.view(torch.int16))


def test_counts_of_new_tokens_outside_their_range():
    """more than there are rows for: all of them; less than none: none"""
    gen = gen_of(31)
    prm, lengths = binding.Params(4, 2), [300, 200, 100]
    for n in (2, 6, 40):
        cache = filled(gen, lengths, 2, 16)
        q, k = normal(gen, 3, n, 4, D), normal(gen, 3, 2, n, D)
        got, want = [], []
        for counts, results in (([1000, -7, -2 ** 31], got), ([n, 0, 0], want)):
            c = cache._replace(k=cache.k.clone(), v=cache.v.clone())
            binding.paged_append(prm, k, k, c, i32(lengths), 300, n_new=i32(counts))
            out, lse = binding.paged_attn(prm, q, c, i32(lengths), 300, n_new=i32(counts))
            results += [c.k.view(torch.int16), c.v.view(torch.int16), out, lse,
                        binding.paged_attn_weights(prm, q, lse, c, i32(lengths), 300, n_new=i32(counts))]
        assert all(torch.equal(x, y) for x, y in zip(got, want))


def test_c_calls_without_what_is_optional():
    """the C entry points with null pointers for what they may do without"""
    import ctypes
    from paper_2506_07900_amd.binding import CPages, CTensor
    gen, lib = gen_of(32), binding.load_library()
    prm, length, budget = binding.Params(4, 2), 500, 100
    cache, to = filled(gen, [length], 2, 16), make_pages(gen, [budget], 2, 16, fill=0.0)
    w, sl = torch.rand((1, 2, length), generator=gen, device="cuda"), i32([length])
    kept, lengths = torch.zeros((1, 2, budget), dtype=torch.int32, device="cuda"), i32([0])

    def pages(c):
        d = [CTensor(x.data_ptr(), x.stride(0), x.stride(1), x.stride(2)) for x in c[:2]]
        return CPages(d[0], d[1], c.table.data_ptr(), c.table.shape[1], c.k.shape[2], c.k.shape[0])

    stream = ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
    p, f, t = prm.c(), pages(cache), pages(to)
    assert lib.infllmv2_paged_evict(ctypes.byref(p), w.data_ptr(), length, ctypes.byref(f), sl.data_ptr(), 1, length, budget, 4, 10, ctypes.byref(t), kept.data_ptr(),
                                    None, lengths.data_ptr(), None, 0, stream) == 0
    first = to.k.clone()
    ref = binding.paged_evict(prm, w, cache, sl, length, budget, 4, 10, to)
    assert torch.equal(kept, ref[0]) and torch.equal(lengths, ref[2]) and torch.equal(first, to.k)
    q = normal(gen, 1, 1, 4, D)
    _, lse = binding.paged_attn(prm, q, cache, sl, length)
    out = torch.zeros((1, 2, length), device="cuda")
    qd = CTensor(q.data_ptr(), q.stride(0), q.stride(2), q.stride(1))
    assert lib.infllmv2_paged_attn_weights(ctypes.byref(p), ctypes.byref(qd), lse.data_ptr(), ctypes.byref(f), None, sl.data_ptr(), 1, length, 1, None, length, out.data_ptr(),
                                           None, 0, stream) == 0
    assert torch.equal(out, binding.paged_attn_weights(prm, q, lse, cache, sl, length))


def test_append_skips():
    """sequences shorter than what is new, longer than the bound, rows without a page"""
    gen = gen_of(9)
    prm = binding.Params(4, 2)
    cache = make_pages(gen, [40, 40, 40, 40], 2, 16, fill=0.0)
    total = cache.k.shape[0]
    cache.table[2, 1], cache.table[3, 2] = -1, total
    k_new, v_new = normal(gen, 4, 2, 24, D), normal(gen, 4, 2, 24, D)
    binding.paged_append(prm, k_new, v_new, cache, i32([23, 41, 40, 40]), 40)
    want = torch.zeros_like(cache.k)
    for b in (2, 3):
        for t in range(24):
            row = 16 + t
            p = int(cache.table[b, row // 16])
            if 0 <= p < total:
                want[p, :, row % 16] = k_new[b, :, t]
    assert torch.equal(cache.k, want)


# ---- attention ---------------------------------------------------------------------------------------------------------

def seen_rows(cache, b, length):
    """rows of a sequence that have a page"""
    page, total = cache.k.shape[2], cache.k.shape[0]
    t = torch.arange(length, device="cuda")
    p = cache.table[b].long()[t // page]
    return (p >= 0) & (p < total)


def attention64(q, k, v, first, there):
    """q [n, Hq, D], k, v [Hkv, L, D] -> out, lse, tolerance of out, of lse; row i sees rows 0 .. first + i that are there"""
    n, hq = q.shape[:2]
    group = hq // k.shape[0]
    t = torch.arange(k.shape[1], device="cuda")
    seen = (t[None] <= first + torch.arange(n, device="cuda")[:, None]) & there[None]
    out, lse, tol, ltol = (torch.zeros((n, hq) + x, dtype=torch.float64, device="cuda") for x in ((D,), (), (D,), ()))
    for h in range(hq):
        kk, vv = k[h // group].double(), v[h // group].double()
        x = torch.where(seen, q[:, h].double() @ kk.t() * SCALE, -math.inf)
        size = torch.where(seen, q[:, h].double().abs() @ kk.abs().t() * SCALE, 0.0).amax(-1)
        lse[:, h] = torch.logsumexp(x, -1)
        p = torch.where(seen, torch.exp(x - torch.where(torch.isinf(lse[:, h]), 0.0, lse[:, h])[:, None]), 0.0)
        vv = torch.where(there[:, None], vv, 0.0)
        out[:, h] = p @ vv
        tol[:, h] = HALF * (p @ vv.abs() + out[:, h].abs()) * 17 / 16
        ltol[:, h] = 2.0 ** -17 * size + 2.0 ** -20 + 2.0 ** -23 * lse[:, h].abs().nan_to_num(posinf=0.0)
    return out, lse, tol, ltol


def check_attention(prm, cache, q, lengths, counts, out, lse, rows=None):
    for b, (length, n) in enumerate(zip(lengths, counts)):
        if length < n:
            assert not bool(out[b, :n].any()) and bool((lse[b, :n] == -math.inf).all())
            continue
        if n == 0:
            continue
        there = seen_rows(cache, b, length)
        safe = cache._replace(table=cache.table.clamp(0, cache.k.shape[0] - 1))
        k, v = (torch.where(there[None, :, None], rows_of(safe, x, b, length), 0) for x in (cache.k, cache.v))
        want, z, tol, ltol = attention64(q[b, :n], k, v, length - n, there)
        assert bool(torch.isfinite(out[b, :n]).all())
        far = ((out[b, :n].double() - want).abs() - tol)
        assert bool((far <= 0).all()), (b, float(far.max()))
        none = z == -math.inf
        assert bool((lse[b, :n][none] == -math.inf).all())
        off = (lse[b, :n].double() - z).abs()[~none] - ltol[~none]
        assert bool((off <= 0).all()), (b, float(off.max()))


ATTENTION = [
    # hq, hkv, page, lengths, counts, n, heavy
    (32, 2, 64, [1], None, 1, False),
    (32, 2, 64, [777, 64, 65, 1, 63], None, 1, True),
    (1, 1, 16, [33, 500], None, 1, False),
    (8, 1, 256, [9001], None, 1, False),
    (8, 2, 32, [2049, 100], None, 1, False),
    (4, 4, 16, [300, 17, 40], [3, 0, 7], 9, False),
    (8, 8, 64, [100, 129], None, 16, True),
    (4, 1, 16, [777, 4], [4, 2], 4, False),
    (16, 1, 32, [1031, 37], [37, 20], 37, False),
    (32, 2, 64, [555], None, 2, False),
    (2, 1, 16, [200], None, 200, False),
    (4, 2, 64, [1000, 700, 64], [300, 1, 64], 300, True),
    (8, 2, 128, [5000], None, 129, False),
    (32, 2, 16, [2100], None, 333, False),
    (16, 16, 32, [150], None, 100, False),
    # as many tiles as fill the chip with workgroups of one group; keys in parts by eight, four, one wavefront each
    (16, 16, 64, [801, 800, 513, 799, 800, 700, 801, 650], [700, 700, 513, 1, 0, 700, 699, 650], 700, True),
    (4, 1, 1024, [20000], None, 1, True),
    (16, 1, 16, [9000, 20], None, 1, False),
    (8, 1, 64, [1200, 321], None, 2, False),
    (32, 2, 32, [6000, 300], [40, 17], 40, True),
    # ragged batches, dealt by units; more sequences than lanes
    (4, 2, 16, [1 + (37 * i * i) % 901 for i in range(69)] + [3000], None, 1, False),
    (2, 1, 64, [4 + (53 * i) % 700 for i in range(130)], [(3 * i) % 5 for i in range(130)], 4, False),
    (16, 1, 32, [9000, 40, 2000, 33, 5000, 1, 700], None, 1, True),
    (8, 2, 64, [3000, 2990, 2980, 2991], [1, 2, 0, 1], 2, False),
]


@pytest.mark.parametrize("hq,hkv,page,lengths,counts,n,heavy", ATTENTION)
def test_attention(hq, hkv, page, lengths, counts, n, heavy):
    gen, b, cap = gen_of(len(lengths) + n), len(lengths), max(lengths)
    prm = binding.Params(hq, hkv)
    cache = filled(gen, lengths, hkv, page, heavy)
    q = normal(gen, b, n, hq, D)
    new = counts or [n] * b
    out, lse = binding.paged_attn(prm, q, cache, i32(lengths), cap, n_new=None if counts is None else i32(counts))
    check_attention(prm, cache, q, lengths, new, out, lse)
    for i, m in enumerate(new):
        assert not bool(out[i, m:].any()) and not bool(lse[i, m:].any())
    # given tensors keep the rows behind a sequence's new tokens, and a longer bound and table change nothing that is promised
    wide = cache._replace(table=torch.cat((cache.table, cache.table.new_full((b, 70), -5)), 1).contiguous())
    given, given_lse = torch.full_like(q, 7.0), torch.full((b, n, hq), 7.0, device="cuda")
    binding.paged_attn(prm, q, wide, i32(lengths), cap + 70, n_new=None if counts is None else i32(counts), out=given, lse=given_lse)
    check_attention(prm, wide, q, lengths, new, given, given_lse)
    for i, m in enumerate(new):
        assert bool((given[i, m:] == 7).all()) and bool((given_lse[i, m:] == 7).all())
    again = binding.paged_attn(prm, q, cache, i32(lengths), cap, n_new=None if counts is None else i32(counts))
    assert torch.equal(out, again[0]) and torch.equal(lse, again[1])


@pytest.mark.parametrize("hq,hkv,n", [(16, 1, 1), (4, 1, 3), (8, 2, 20), (4, 2, 150)])
def test_attention_without_pages_and_short_sequences(hq, hkv, n):
    gen = gen_of(n)
    prm = binding.Params(hq, hkv)
    lengths = [400, 300, n - 1, 350, n]
    cache = filled(gen, [max(1, x) for x in lengths], hkv, 16)
    total = cache.k.shape[0]
    cache.table[0, 3], cache.table[0, 4], cache.table[0, 24] = -1, total, 2 ** 31 - 1
    cache.table[1, :] = -1                                        # sees nothing
    cache.table[3, 21] = -2 ** 31
    q = normal(gen, 5, n, hq, D)
    out, lse = binding.paged_attn(prm, q, cache, i32(lengths), 400)
    check_attention(prm, cache, q, lengths, [n] * 5, out, lse)
    assert not bool(out[1].any()) and bool((lse[1] == -math.inf).all())
    # lengths above the bound are taken as the bound
    out2, lse2 = binding.paged_attn(prm, q, cache, i32([500, 400, n - 1, 400, n]), 350)
    ref = binding.paged_attn(prm, q, cache, i32([350, 350, n - 1, 350, n]), 350)
    assert torch.equal(out2, ref[0]) and torch.equal(lse2, ref[1])


@pytest.mark.parametrize("hq,hkv,n", [(16, 1, 1), (2, 1, 6), (4, 1, 4), (8, 2, 40), (1, 1, 300)])
def test_attention_values_that_are_not_finite(hq, hkv, n):
    """an infinity or a NaN reaches the rows that see it and no others; a score that is NaN or +inf makes its row NaN"""
    gen = gen_of(100 + n)
    prm, length = binding.Params(hq, hkv), n + 90
    first = length - n
    cache = filled(gen, [length], hkv, 16)
    q = normal(gen, 1, n, hq, D)
    ref, ref_lse = binding.paged_attn(prm, q, cache, i32([length]), length)
    # values, of the last new token's and of one in the middle
    v = cache.v.clone()
    rows = sorted({length - 1, first + n // 2})
    for j, t in enumerate(rows):
        at = int(cache.table[0, t // 16])
        v[at, :, t % 16, 5 + j] = [math.inf, NAN][j]
        v[at, :, t % 16, 77] = -math.inf
    out, lse = binding.paged_attn(prm, q, cache._replace(v=v), i32([length]), length)
    assert torch.equal(lse, ref_lse)
    for i in range(n):
        sees = [t <= first + i for t in rows]
        odd = torch.zeros(D, dtype=torch.bool, device="cuda")
        for j, s in enumerate(sees):
            if s:
                odd[5 + j] = odd[77] = True
        assert bool((~torch.isfinite(out[0, i, :, odd])).all())
        assert torch.equal(out[0, i][:, ~odd], ref[0, i][:, ~odd])
    if sees[0] and len(rows) == 2:
        assert bool((out[0, n - 1, :, 5] == math.inf).all()) or bool(torch.isnan(out[0, n - 1, :, 5]).all())
    # keys: NaN
    k = cache.k.clone()
    t = first + n // 2
    k[int(cache.table[0, t // 16]), :, t % 16, 3] = NAN
    out, lse = binding.paged_attn(prm, q, cache._replace(k=k), i32([length]), length)
    for i in range(n):
        if t <= first + i:
            assert bool(torch.isnan(out[0, i]).all()) and bool(torch.isnan(lse[0, i]).all())
        else:
            assert torch.equal(out[0, i], ref[0, i]) and torch.equal(lse[0, i], ref_lse[0, i])


@pytest.mark.parametrize("hq,hkv,n,length", [(16, 1, 1, 3000), (8, 2, 40, 700), (4, 4, 1, 200000), (2, 1, 300, 300)])
def test_attention_of_values_near_the_largest(hq, hkv, n, length):
    """values of one size and sign keep their mean"""
    gen = gen_of(length)
    prm = binding.Params(hq, hkv)
    cache = filled(gen, [length], hkv, 64)
    big = torch.finfo(torch.bfloat16).max
    for value in (big, -big, 1e-25):
        v = torch.full_like(cache.v, value)
        q = normal(gen, 1, n, hq, D)
        out, _ = binding.paged_attn(prm, q, cache._replace(v=v), i32([length]), length)
        want = float(v.view(-1)[0])
        assert bool(((out.double() - want).abs() <= 2 * HALF * 17 / 16 * abs(want)).all())


def test_attention_of_equal_and_extreme_scores():
    prm = binding.Params(4, 1)
    gen = gen_of(8)
    for n, length in ((1, 1000), (50, 1000)):
        cache = filled(gen, [length], 1, 16)
        q = normal(gen, 1, n, 4, D)
        zero, _ = binding.paged_attn(prm, torch.zeros_like(q), cache, i32([length]), length)
        check_attention(prm, cache, torch.zeros_like(q), [length], [n], zero, _)
        big = (q.float() * 3000).bfloat16()                       # scores of tens of thousands: one key takes all
        out, lse = binding.paged_attn(prm, big, cache, i32([length]), length)
        check_attention(prm, cache, big, [length], [n], out, lse)


@pytest.mark.parametrize("hq,hkv,n,length,batch", [(32, 2, 1, 3000, 8), (4, 1, 4, 300, 2), (8, 2, 60, 2500, 1), (16, 16, 600, 700, 10), (32, 2, 500, 4000, 1)])
def test_attention_of_large_scores(hq, hkv, n, length, batch):
    """scores of thousands: a maximum that lacked some of a product would leave exponentials that overflow"""
    prm, gen = binding.Params(hq, hkv), gen_of(n)
    cache = filled(gen, [length] * batch, hkv, 64)
    for size in (300, 3000):
        q = (normal(gen, batch, n, hq, D).float() * size).bfloat16()
        out, lse = binding.paged_attn(prm, q, cache, i32([length] * batch), length)
        assert bool(torch.isfinite(out).all()) and bool(torch.isfinite(lse).all())
        check_attention(prm, cache, q[:1], [length], [n], out[:1], lse[:1])


def test_attention_of_many_tiles_with_odd_values_and_pages():
    """the form for many tiles: what a hidden infinity, a missing page and a row without any leave alone"""
    gen = gen_of(55)
    hq, hkv, n, b = 16, 16, 640, 10
    prm, lengths = binding.Params(hq, hkv), [700 - 3 * i for i in range(b)]
    cache = filled(gen, lengths, hkv, 16)
    q = normal(gen, b, n, hq, D)
    cache.table[3, 7], cache.table[4, 0], cache.table[5, :] = -1, 2 ** 30, -7
    out, lse = binding.paged_attn(prm, q, cache, i32(lengths), 700)
    check_attention(prm, cache, q, lengths, [n] * b, out, lse)
    v = cache.v.clone()
    t = lengths[0] - 100
    v[int(cache.table[0, t // 16]), :, t % 16, 9] = NAN
    again, _ = binding.paged_attn(prm, q, cache._replace(v=v), i32(lengths), 700)
    first = t - (lengths[0] - n)                                  # the first query that sees it
    assert torch.equal(again[1:], out[1:]) and torch.equal(again[0, :first], out[0, :first])
    assert bool(torch.isnan(again[0, first:, :, 9]).all())
    keep = torch.arange(D, device="cuda") != 9
    assert torch.equal(again[0, :, :, keep], out[0, :, :, keep])


CHUNKS = [
    # hq, hkv, page, lengths, counts, n: parts by what is there
    (16, 1, 32, [8 + (97 * i) % 900 for i in range(100)], [(5 * i) % 9 for i in range(100)], 8),
    (16, 1, 16, [4 + (53 * i) % 1200 for i in range(128)], [8 if i % 37 == 3 else 0 for i in range(128)], 8),
    (8, 2, 64, [9000, 50, 40, 3000, 257], [60, 50, 41, 0, 1], 60),
    (4, 1, 16, [5000, 3000], [1, 500], 500),
    (4, 2, 64, [700, 600], [0, 0], 100),
    (4, 2, 64, [90, 600, 3], [100, 0, 4], 100),
    (32, 2, 128, [4000], [9], 700),
    (16, 1, 64, [64 + 31 * i for i in range(65)], [8] * 65, 8),
    # no more tiles than compute units, without parts: three groups, and with fewer keys one
    (16, 16, 64, [801, 640, 500, 30], [300, 256, 1, 30], 300),
    (16, 16, 32, [440, 300, 299, 30], [300, 256, 300, 30], 300),
    (8, 2, 16, [512, 449, 448], [60, 60, 0], 60),
    (8, 2, 16, [513, 449, 448], [60, 60, 0], 60),
]


@pytest.mark.parametrize("hq,hkv,page,lengths,counts,n", CHUNKS)
def test_attention_of_few_tiles(hq, hkv, page, lengths, counts, n):
    gen, b, cap = gen_of(len(lengths) + n), len(lengths), max(lengths)
    prm = binding.Params(hq, hkv)
    cache = filled(gen, lengths, hkv, page)
    q = normal(gen, b, n, hq, D)
    out, lse = binding.paged_attn(prm, q, cache, i32(lengths), cap, n_new=i32(counts))
    check_attention(prm, cache, q, lengths, counts, out, lse)
    for i, m in enumerate(counts):
        assert not bool(out[i, m:].any()) and not bool(lse[i, m:].any())
    given, given_lse = torch.full_like(q, 7.0), torch.full((b, n, hq), 7.0, device="cuda")
    binding.paged_attn(prm, q, cache, i32(lengths), cap, n_new=i32(counts), out=given, lse=given_lse)
    for i, m in enumerate(counts):
        assert torch.equal(given[i, :m], out[i, :m]) and torch.equal(given_lse[i, :m], lse[i, :m])
        assert bool((given[i, m:] == 7).all()) and bool((given_lse[i, m:] == 7).all())


@pytest.mark.parametrize("cap", [700, 440])
def test_attention_of_as_many_tiles_as_compute_units_with_odd_values_and_pages(cap):
    gen = gen_of(cap)
    hq, hkv, n, b = 16, 16, 300, 4
    prm, lengths = binding.Params(hq, hkv), [cap - 3 * i for i in range(b)]
    cache = filled(gen, lengths, hkv, 16)
    q = normal(gen, b, n, hq, D)
    cache.table[2, 7], cache.table[3, :] = -1, -7
    out, lse = binding.paged_attn(prm, q, cache, i32(lengths), cap)
    check_attention(prm, cache, q, lengths, [n] * b, out, lse)
    v = cache.v.clone()
    t = cap - 100
    v[int(cache.table[0, t // 16]), :, t % 16, 9] = -math.inf
    again, _ = binding.paged_attn(prm, q, cache._replace(v=v), i32(lengths), cap)
    first = t - (cap - n)                                         # the first query that sees it
    assert torch.equal(again[1:], out[1:]) and torch.equal(again[0, :first], out[0, :first])
    assert bool((again[0, first:, :, 9] == -math.inf).all())
    keep = torch.arange(D, device="cuda") != 9
    assert torch.equal(again[0, :, :, keep], out[0, :, :, keep])


# ---- weights -------------------------------------------------------------------------------------------------------------

def weights64(q, lse, k, first, there):
    n, hq = q.shape[:2]
    group = hq // k.shape[0]
    t = torch.arange(k.shape[1], device="cuda")
    seen = (t[None] <= first + torch.arange(n, device="cuda")[:, None]) & there[None]
    total, tol = (torch.zeros(k.shape[:2], dtype=torch.float64, device="cuda") for _ in range(2))
    for h in range(hq):
        kk = k[h // group].double()
        x, size = q[:, h].double() @ kk.t() * SCALE, q[:, h].double().abs() @ kk.abs().t() * SCALE
        z = lse[:, h].double()[:, None]
        p = torch.where(seen & (z > -math.inf), torch.exp(x - z), 0.0)
        total[h // group] += p.sum(0)
        rel = 2.0 ** -17 * size + 2.0 ** -22 * (x.abs() + z.abs().nan_to_num(posinf=0.0)) + 2.0 ** -22
        tol[h // group] += (p * rel).sum(0)
    return total, tol + total * 2.0 ** -24 * (n * group / 32 + 8)


@pytest.mark.parametrize("hq,hkv,page,lengths,counts,n,heavy", ATTENTION)
def test_weights(hq, hkv, page, lengths, counts, n, heavy):
    gen, b, cap = gen_of(len(lengths) + n), len(lengths), max(lengths)
    prm = binding.Params(hq, hkv)
    cache = filled(gen, lengths, hkv, page, heavy)
    if b > 1 and lengths[0] > 64:
        cache.table[0, 1] = -1
    q = normal(gen, b, n, hq, D)
    new = counts or [n] * b
    n_new = None if counts is None else i32(counts)
    _, lse = binding.paged_attn(prm, q, cache, i32(lengths), cap, n_new=n_new)
    had = torch.rand((b, hkv, cap + 9), generator=gen, device="cuda")
    got = binding.paged_attn_weights(prm, q, lse, cache, i32(lengths), cap, n_new=n_new, weights=had)
    alone = binding.paged_attn_weights(prm, q, lse, cache, i32(lengths), cap, n_new=n_new)
    assert got.shape == had.shape and alone.shape == (b, hkv, cap)
    for i, (length, m) in enumerate(zip(lengths, new)):
        first, there = length - m, seen_rows(cache, i, length)
        safe = cache._replace(table=cache.table.clamp(min=0))
        k = torch.where(there[None, :, None], rows_of(safe, cache.k, i, length), 0)
        want, tol = weights64(q[i, :m], lse[i, :m], k, first, there)
        assert bool(((alone[i, :, :length].double() - want).abs() <= tol).all())
        before = had[i, :, :length].double().clone()
        before[:, first:] = 0
        assert bool(((got[i, :, :length].double() - want - before).abs() <= tol + 2.0 ** -23 * (want + before)).all())
        assert not bool(got[i, :, length:].any())                # (made by the call)
    # in place, and entries behind a sequence stay
    mine = had.clone()
    assert binding.paged_attn_weights(prm, q, lse, cache, i32(lengths), cap, n_new=n_new, weights=mine, weights_out=mine) is mine
    for i, length in enumerate(lengths):
        assert torch.equal(mine[i, :, :length], got[i, :, :length]) and torch.equal(mine[i, :, length:], had[i, :, length:])


@pytest.mark.parametrize("hq,hkv,n", [(16, 1, 1), (8, 2, 40)])
def test_weights_of_short_sequences_and_nan(hq, hkv, n):
    gen = gen_of(n)
    prm = binding.Params(hq, hkv)
    lengths = [200, n - 1, 150]
    cache = filled(gen, [max(1, x) for x in lengths], hkv, 16)
    q = normal(gen, 3, n, hq, D)
    _, lse = binding.paged_attn(prm, q, cache, i32(lengths), 200)
    had = torch.rand((3, hkv, 200), generator=gen, device="cuda")
    out = torch.full_like(had, 3.0)
    k = cache.k.clone()
    t = 200 - n                                                   # the first new token's own row: NaN for all that see it
    k[int(cache.table[0, t // 16]), 0, t % 16, 0] = NAN
    binding.paged_attn_weights(prm, q, lse, cache._replace(k=k), i32(lengths), 200, weights=had, weights_out=out)
    ref = binding.paged_attn_weights(prm, q, lse, cache, i32(lengths), 200, weights=had)
    assert bool((out[1] == 3).all())
    assert bool(torch.isnan(out[0, 0, t]))
    rest = torch.ones(200, dtype=torch.bool, device="cuda")
    rest[t] = False
    assert torch.equal(out[0, 0, rest], ref[0, 0, rest]) and torch.equal(out[2, :, :150], ref[2, :, :150])


# ---- eviction -------------------------------------------------------------------------------------------------------------

def choice(w, length, budget, first, recent):
    if length <= budget:
        return list(range(length))
    def key(t):
        return (0.0, 0.0) if math.isnan(w[t]) else (1.0, -w[t])
    mid = sorted(range(first, length - recent), key=lambda t: key(t) + (t,))[:budget - first - recent]
    return sorted(list(range(first)) + mid + list(range(length - recent, length)))


EVICTIONS = [
    # lengths, budget, first, recent, page, page of the others, kind
    ([1000, 5, 0, 333], 100, 4, 30, 16, 64, "random"),
    ([5000], 4999, 0, 0, 64, 16, "ties"),
    ([5000, 4097], 1, 0, 0, 256, 256, "ties"),
    ([777, 128], 128, 64, 64, 32, 32, "random"),
    ([9001, 8192], 4501, 64, 2000, 16, 128, "odd"),
    ([3000, 2000], 512, 1, 0, 16, 16, "equal"),
    ([300], 400, 4, 100, 16, 16, "random"),
    ([70001], 20000, 4, 1, 64, 64, "random"),
    ([140000], 3, 1, 1, 64, 64, "small"),
    ([40000], 35000, 4, 9000, 64, 64, "random"),
]


@pytest.mark.parametrize("lengths,budget,first,recent,page,to_page,kind", EVICTIONS)
def test_eviction(lengths, budget, first, recent, page, to_page, kind):
    gen, hkv = gen_of(budget), 2
    prm, b, cap = binding.Params(8, hkv), len(lengths), max(lengths)
    cache = filled(gen, [max(1, x) for x in lengths], hkv, page)
    to = make_pages(gen, [min(budget, cap)] * b, hkv, to_page, fill=7.0)
    w = torch.rand((b, hkv, cap + 3), generator=gen, device="cuda")
    if kind == "ties":
        w = (w * 4).floor()
    elif kind == "equal":
        w = torch.zeros_like(w)
        w[:, :, ::2] = -0.0
    elif kind == "small":
        w = w * 1e-42
    elif kind == "odd":
        pick = torch.rand(w.shape, generator=gen, device="cuda")
        w = torch.where(pick < 0.1, NAN, torch.where(pick < 0.2, math.inf, torch.where(pick < 0.3, -math.inf, torch.where(pick < 0.6, -w, w))))
        w[0, 0, 100] = torch.tensor(-1, dtype=torch.int32).view(torch.float32)                  # a NaN with its sign bit set
    before = [x.clone() for x in to[:2]]
    kept, wo, so = binding.paged_evict(prm, w, cache, i32(lengths), cap, budget, first, recent, to)
    want_pools = [x.clone() for x in before]
    for i, length in enumerate(lengths):
        m = min(length, budget)
        assert int(so[i]) == m
        for h in range(hkv):
            rows = choice(w[i, h].tolist(), length, budget, first, recent)
            assert kept[i, h].tolist() == rows + [-1] * (budget - m)
            at = torch.tensor(rows, dtype=torch.long, device="cuda")
            assert torch.equal(wo[i, h, :m].view(torch.int32), w[i, h, at].view(torch.int32)) and not bool(wo[i, h, m:].any())
            j = torch.arange(m, device="cuda")
            dst = to.table[i].long()[j // to_page]
            for pool, src in ((want_pools[0], cache.k), (want_pools[1], cache.v)):
                if m:
                    pool[dst, h, j % to_page] = rows_of(cache, src, i, length)[h, at]
    for got, want in zip(to[:2], want_pools):
        assert torch.equal(got.view(torch.int16), want.view(torch.int16))


@pytest.mark.parametrize("cap", [12000, 20000])
def test_eviction_of_ties_in_many_workgroups(cap):
    """more numbers with the first digit than a run's list takes: all wavefronts have to go on alike, in every workgroup"""
    gen, hkv, b, budget = gen_of(9), 4, 128, 3001
    prm = binding.Params(4, hkv)
    lengths = [cap - 37 * i for i in range(b)]
    cache = make_pages(gen, [16] * b, hkv, 16)
    cache = binding.PagedCache(cache.k, cache.v, torch.full((b, cap // 16), -1, dtype=torch.int32, device="cuda"))
    to = binding.PagedCache(cache.k, cache.v, torch.full((b, budget // 16 + 1), -1, dtype=torch.int32, device="cuda"))
    w = 1.0 + torch.randint(0, 3, (b, hkv, cap), generator=gen, device="cuda").float() * 2.0 ** -23      # (equal but for their last bits)
    hidden = torch.arange(cap, device="cuda") >= torch.tensor(lengths, device="cuda")[:, None, None]
    want = torch.where(hidden, -1.0, w).sort(dim=-1, descending=True, stable=True).indices[:, :, :budget].sort(dim=-1).values.int()
    for _ in range(20):
        assert torch.equal(binding.paged_evict(prm, w, cache, i32(lengths), cap, budget, 0, 0, to)[0], want)


@pytest.mark.parametrize("kind", ["equal", "ties", "odd", "random"])
@pytest.mark.parametrize("lengths,cap,budget,first,recent", [([20000, 900, 0, 4097], 20000, 1000, 4, 30), ([40001, 16384], 40001, 12000, 0, 0), ([90000], 90000, 89999, 64, 0),
                                                             ([300001, 262145, 5], 300001, 1, 0, 0), ([270000], 400000, 100000, 10, 60000), ([600000], 600000, 600000 - 4096, 0, 0),
                                                             ([16385, 3], 16385, 16384, 8000, 8383)])
def test_eviction_in_parts(lengths, cap, budget, first, recent, kind):
    gen, hkv, b, page = gen_of(cap + budget), 2, len(lengths), 64
    prm = binding.Params(2, hkv)
    pools = [torch.zeros((4, hkv, page, D), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    cache, to = (binding.PagedCache(*pools, torch.full((b, (n + page - 1) // page), -1, dtype=torch.int32, device="cuda")) for n in (cap, budget))
    w = torch.rand((b, hkv, cap + 5), generator=gen, device="cuda")
    if kind == "equal":
        w = torch.full_like(w, 0.25)
    elif kind == "ties":
        w = (w * 5).floor() - 2.0
    elif kind == "odd":
        w = torch.where(w < 0.2, -math.inf, torch.where(w < 0.3, math.inf, torch.where(w < 0.4, NAN, (w - 0.7) * 1e-39)))
    kept, wo, so = binding.paged_evict(prm, w, cache, i32(lengths), cap, budget, first, recent, to)
    for i, length in enumerate(lengths):
        m = min(length, budget)
        assert int(so[i]) == m
        key = w[i, :, :length].nan_to_num(nan=math.inf, posinf=3e38, neginf=-3e38)      # (a NaN above infinity; no number here is near them)
        if length > budget:
            fixed = torch.zeros_like(key)
            fixed[:, :first], fixed[:, length - recent:] = 1.0, 1.0
            order = key.sort(dim=-1, descending=True, stable=True).indices
            order = order.gather(1, fixed.gather(1, order).sort(dim=-1, descending=True, stable=True).indices)       # those that stay in any case before all others
            want = order[:, :budget].sort(dim=-1).values.int()
        else:
            want = torch.cat((torch.arange(m, device="cuda"), torch.full((budget - m,), -1, device="cuda"))).int().expand(hkv, budget)
        assert torch.equal(kept[i], want)
        assert torch.equal(wo[i, :, :m].view(torch.int32), w[i].gather(1, want[:, :m].long()).view(torch.int32)) and not bool(wo[i, :, m:].any())


def test_eviction_with_rows_without_pages():
    gen = gen_of(1)
    prm = binding.Params(2, 1)
    cache, to = filled(gen, [100], 1, 16), make_pages(gen, [50], 1, 16, fill=7.0)
    cache.table[0, 1], to.table[0, 2] = -1, 1000
    w = torch.rand((1, 1, 100), generator=gen, device="cuda")
    kept, wo, so = binding.paged_evict(prm, w, cache, i32([100]), 100, 50, 0, 0, to)
    assert kept[0, 0].tolist() == choice(w[0, 0].tolist(), 100, 50, 0, 0)
    for j, t in enumerate(kept[0, 0].tolist()):
        if 32 <= j < 48:
            continue
        got = to.k[int(to.table[0, j // 16]), 0, j % 16]
        if 16 <= t < 32:
            assert bool((got == 7).all())
        else:
            assert torch.equal(got, cache.k[int(cache.table[0, t // 16]), 0, t % 16])


# ---- as they are used -------------------------------------------------------------------------------------------------------

def test_serving_run():
    """prompts in pieces, ragged; an eviction; single tokens after it, eagerly and in a replayed graph, against the definitions on plain tensors"""
    gen = gen_of(77)
    hq, hkv, page, cap, budget, b = 16, 2, 16, 420, 200, 2
    prm, rope = binding.Params(hq, hkv), binding.rope_table(128, scaling="yarn", factor=4.0, original_len=128)
    f, amplitude = frequencies(128, scaling="yarn", factor=4.0, original_len=128)
    cache, to = make_pages(gen, [cap] * b, hkv, page), make_pages(gen, [budget + 40] * b, hkv, page)
    lengths = [0, 0]
    total = torch.zeros((b, hkv, cap), device="cuda")
    for counts in ([100, 33], [150, 150], [0, 1], [77, 200]):
        n = max(counts)
        lengths = [x + y for x, y in zip(lengths, counts)]
        sl, n_new = i32(lengths), i32(counts)
        k, v, q = normal(gen, b, hkv, n, D), normal(gen, b, hkv, n, D), normal(gen, b, n, hq, D)
        q = binding.paged_append(prm, k, v, cache, sl, cap, n_new=n_new, rope=rope, q=q, q_out=q)
        out, lse = binding.paged_attn(prm, q, cache, sl, cap, n_new=n_new)
        check_attention(prm, cache, q, lengths, counts, out, lse)
        before = total.clone()
        binding.paged_attn_weights(prm, q, lse, cache, sl, cap, n_new=n_new, weights=total, weights_out=total)
        for i in range(b):
            want, tol = weights64(q[i, :counts[i]], lse[i, :counts[i]], rows_of(cache, cache.k, i, lengths[i]), lengths[i] - counts[i],
                                  seen_rows(cache, i, lengths[i]))
            assert bool(((total[i, :, :lengths[i]].double() - before[i, :, :lengths[i]].double() - want).abs() <= tol + 2.0 ** -22 * total[i, :, :lengths[i]]).all())
    kept, moved, sl = binding.paged_evict(prm, total, cache, sl, cap, budget, 4, 64, to)
    assert sl.tolist() == [min(x, budget) for x in lengths]
    # single tokens: positions go on where the rows did not
    total = torch.cat((moved, torch.zeros((b, hkv, 40), device="cuda")), -1).contiguous()
    cap2 = budget + 40
    q, k, v = torch.zeros((b, 1, hq, D), dtype=torch.bfloat16, device="cuda"), *(torch.zeros((b, hkv, 1, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    positions, qr = i32([[x] for x in lengths]), torch.zeros_like(q)
    out, lse = torch.zeros_like(q), torch.zeros((b, 1, hq), device="cuda")
    ws = torch.empty(max(256, binding.paged_workspace_bytes(binding.OP_PAGED_ATTN, prm, b, cap2, 1)), dtype=torch.uint8, device="cuda")

    def step():
        binding.paged_append(prm, k, v, to, sl, cap2, rope=rope, positions=positions, q=q, q_out=qr)
        binding.paged_attn(prm, qr, to, sl, cap2, out=out, lse=lse, workspace=ws)
        binding.paged_attn_weights(prm, qr, lse, to, sl, cap2, weights=total, weights_out=total)

    graph = torch.cuda.CUDAGraph()
    held = None
    for i in range(12):
        sl += 1
        for x in (q, k, v):
            x.copy_(normal(gen, *x.shape))
        if i == 5:
            held = (to.k.clone(), to.v.clone(), total.clone())
            with torch.cuda.graph(graph):
                step()
            assert torch.equal(to.k.view(torch.int16), held[0].view(torch.int16))              # (captured, not run)
        before = total.clone()
        graph.replay() if i >= 5 else step()
        torch.cuda.synchronize()
        now = sl.tolist()
        check_attention(prm, to, qr, now, [1] * b, out, lse)
        for j in range(b):
            at = int(to.table[j, (now[j] - 1) // page])
            want, size = rotated64(k[j].transpose(0, 1), positions[j], f, amplitude, False)
            close_rotation(to.k[at, :, (now[j] - 1) % page], want[0], size[0])
            want, tol = weights64(qr[j], lse[j], rows_of(to, to.k, j, now[j]), now[j] - 1, seen_rows(to, j, now[j]))
            assert bool(((total[j, :, :now[j]].double() - before[j, :, :now[j]].double() - want).abs() <= tol + 2.0 ** -22 * total[j, :, :now[j]]).all())
        positions += 1


def test_graphs_that_share_a_workspace_and_calls_side_by_side():
    """two captured graphs of different calls over one workspace, replayed in turn; and two streams with a workspace each"""
    gen = gen_of(12)
    prm = binding.Params(16, 2)
    cases = [(5000, 1), (3000, 40), (900, 300)]
    caches = [filled(gen, [length], 2, 32) for length, _ in cases]
    qs = [normal(gen, 1, n, 16, D) for _, n in cases]
    sls = [i32([length]) for length, _ in cases]
    need = max(max(binding.paged_workspace_bytes(op, prm, 1, length, n) for length, n in cases) for op in (binding.OP_PAGED_ATTN, binding.OP_PAGED_WEIGHTS))
    ws = torch.empty(max(need, 256), dtype=torch.uint8, device="cuda")

    def call(i, work):
        out, lse = binding.paged_attn(prm, qs[i], caches[i], sls[i], cases[i][0], workspace=work)
        return out, lse, binding.paged_attn_weights(prm, qs[i], lse, caches[i], sls[i], cases[i][0], workspace=work)

    want = [[x.clone() for x in call(i, ws)] for i in range(3)]
    graphs, got = [], []
    for i in range(3):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            got.append(call(i, ws))
        graphs.append(g)
    for turn in range(4):
        for i in (0, 1, 2, 1, 0):
            for x in got[i]:
                x.zero_()
            ws.fill_(255)                                         # (what it holds before does not matter)
            graphs[i].replay()
            torch.cuda.synchronize()
            assert all(torch.equal(x, y) for x, y in zip(got[i], want[i]))
    streams, works, side = [torch.cuda.Stream() for _ in range(2)], [torch.empty_like(ws) for _ in range(2)], [None, None]
    for turn in range(5):
        for j, i in ((0, 1), (1, 2)):
            with torch.cuda.stream(streams[j]):
                side[j] = call(i, works[j])
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for j, i in ((0, 1), (1, 2)) for x, y in zip(side[j], want[i]))


def test_eviction_and_attention_in_a_graph_whose_lengths_change():
    """captured once for the longest; what is replayed reads the lengths, counts and weights of its time, and nothing that an earlier replay left in the workspace"""
    gen = gen_of(77)
    hq, hkv, b, cap, n, budget, page = 16, 2, 3, 20000, 24, 700, 64
    prm = binding.Params(hq, hkv)
    cache = filled(gen, [cap] * b, hkv, page)
    to = make_pages(gen, [budget] * b, hkv, page, fill=0.0)
    q, w = normal(gen, b, n, hq, D), torch.rand((b, hkv, cap), generator=gen, device="cuda")
    sl, counts = i32([cap] * b), i32([n] * b)
    ws = [torch.empty(max(256, binding.paged_workspace_bytes(op, prm, b, cap, n)), dtype=torch.uint8, device="cuda") for op in (binding.OP_PAGED_ATTN, binding.OP_PAGED_WEIGHTS, binding.OP_PAGED_EVICT)]

    def run():
        out, lse = binding.paged_attn(prm, q, cache, sl, cap, n_new=counts, workspace=ws[0])
        weights = binding.paged_attn_weights(prm, q, lse, cache, sl, cap, n_new=counts, weights=w, workspace=ws[1])
        return (out, lse, weights) + tuple(binding.paged_evict(prm, weights, cache, sl, cap, budget, 4, 64, to, workspace=ws[2])) + (to.k, to.v)

    run()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = run()
    for lengths, new in (([cap, cap, cap], [n, n, n]), ([5, 16385, 900], [5, 0, 1]), ([0, 0, 3], [0, 1, 4]), ([19999, 700, 701], [1, 24, 24]), ([cap, 4100, 12], [n, 7, 12])):
        sl.copy_(i32(lengths))
        counts.copy_(i32(new))
        w.copy_(torch.rand(w.shape, generator=gen, device="cuda") * 4)
        for x in ws:
            x.fill_(255)
        to.k.zero_(), to.v.zero_()
        graph.replay()
        torch.cuda.synchronize()
        replayed = [x.clone() for x in got]
        for x in ws:
            x.fill_(0)
        to.k.zero_(), to.v.zero_()
        eager = run()
        for i, (x, y) in enumerate(zip(replayed, eager)):
            assert torch.equal(x, y), i
        kept, so = replayed[3], replayed[5]
        for i, length in enumerate(lengths):
            assert int(so[i]) == min(length, budget)
            for h in range(hkv):
                rows = choice(replayed[2][i, h].tolist(), length, budget, 4, 64)
                assert kept[i, h].tolist() == rows + [-1] * (budget - len(rows))


def test_another_stream_and_order():
    """calls go to the current stream"""
    gen = gen_of(4)
    prm = binding.Params(8, 2)
    cache = filled(gen, [3000], 2, 16)
    q = normal(gen, 1, 30, 8, D)
    want = binding.paged_attn(prm, q, cache, i32([3000]), 3000)
    side = torch.cuda.Stream()
    qs, sl = torch.zeros_like(q), i32([3000])
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        x = torch.randn((4096, 4096), device="cuda")
        for _ in range(10):
            x = x @ x * 1e-3
        qs.copy_(q)
        got = binding.paged_attn(prm, qs, cache, sl, 3000)
    side.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_far_pages_and_wide_strides():
    """pages beyond 4 GiB, rows and heads further apart than their sizes"""
    gen = gen_of(6)
    hkv, page, length = 2, 16, 1500
    need = (length + page - 1) // page
    step = (5 << 30) // (2 * need) // 8 * 8                       # elements from page to page
    pools = [torch.zeros(step * need + hkv * page * 512, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    k, v = (x.as_strided((need, hkv, page, D), (step, page * 512 - 256, 384, 1)) for x in pools)
    cache = binding.PagedCache(k, v, torch.randperm(need, generator=torch.Generator().manual_seed(1)).int().cuda()[None].contiguous())
    near = make_pages(gen, [length], hkv, page)
    near.table.copy_(cache.table)
    for x, y in ((k, near.k), (v, near.v)):
        rows = normal(gen, hkv, length, D)
        write_rows(cache, x, 0, rows)
        write_rows(near, y, 0, rows)
    for hq, n in ((32, 1), (8, 3), (8, 60)):
        prm = binding.Params(hq, hkv)
        buffer = normal(gen, 1, hq, n, 2 * D)
        q = buffer[:, :, :, :D].transpose(1, 2)                   # heads before tokens, rows twice as far apart
        out, lse = binding.paged_attn(prm, q, cache, i32([length]), length)
        ref = binding.paged_attn(prm, q.contiguous(), near, i32([length]), length)
        assert torch.equal(out, ref[0]) and torch.equal(lse, ref[1])
        assert torch.equal(binding.paged_attn_weights(prm, q, lse, cache, i32([length]), length), binding.paged_attn_weights(prm, q, lse, near, i32([length]), length))
        qo = torch.zeros_like(buffer)[:, :, :, :D].transpose(1, 2)
        kn = normal(gen, 1, hkv, n, D)
        rope = binding.rope_table(64)
        for c in (cache, near):
            binding.paged_append(prm, kn, kn, c, i32([length]), length, rope=rope, q=q, q_out=qo)
        assert torch.equal(rows_of(cache, k, 0, length), rows_of(near, near.k, 0, length)) and torch.equal(rows_of(cache, v, 0, length), rows_of(near, near.v, 0, length))
    w = torch.rand((1, hkv, length), generator=gen, device="cuda")
    to = make_pages(gen, [400], hkv, page, fill=0.0)
    a = binding.paged_evict(prm, w, cache, i32([length]), length, 400, 4, 100, to)
    first = to.k.clone()
    b = binding.paged_evict(prm, w, near, i32([length]), length, 400, 4, 100, to)
    assert torch.equal(a[0], b[0]) and torch.equal(first, to.k)
