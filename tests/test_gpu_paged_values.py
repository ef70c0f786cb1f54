"""The paged cache's calls on values that are not finite, where their answer is a number all the same."""
import math

import pytest
import torch

from paper_2506_07900_amd import binding
from test_gpu_paged import D, NAN, filled, gen_of, i32, make_pages, normal, rows_of, seen_rows, weights64

pytestmark = pytest.mark.gpu


# single tokens and chunks whose last 32 rows of (token, head) are filled and are not; several parts of a tile's rows
SHAPES = [(16, 1, 1, 300), (4, 1, 3, 90), (16, 1, 3, 200), (16, 1, 4, 200), (8, 2, 37, 300), (2, 1, 33, 129), (1, 1, 100, 100), (16, 1, 700, 900)]


@pytest.mark.parametrize("hq,hkv,n,length", SHAPES)
def test_weights_of_keys_whose_scores_are_minus_infinity(hq, hkv, n, length):
    """such a key gets nothing, wherever it lies: seen by all new tokens, or one of them itself"""
    prm, gen = binding.Params(hq, hkv), gen_of(n)
    cache = filled(gen, [length], hkv, 16)
    q = normal(gen, 1, n, hq, D)
    q[..., 3] = 1.0                                               # all queries go against the infinity
    at = sorted({0, length - 1, length // 2, max(0, length - n), max(0, length - n - 1)})
    for t in at:
        cache.k[int(cache.table[0, t // 16]), :, t % 16, 3] = -math.inf
    _, lse = binding.paged_attn(prm, q, cache, i32([length]), length)
    got = binding.paged_attn_weights(prm, q, lse, cache, i32([length]), length)
    had = torch.rand((1, hkv, length), generator=gen, device="cuda")
    more = binding.paged_attn_weights(prm, q, lse, cache, i32([length]), length, weights=had)
    k = rows_of(cache, cache.k, 0, length)
    k[:, at] = 0.0
    there = seen_rows(cache, 0, length)
    there[at] = False
    want, tol = weights64(q[0], lse[0], k, length - n, there)
    assert bool(torch.isfinite(got).all()) and not bool(got[0, :, at].any())
    assert bool(((got[0].double() - want).abs() <= tol).all())
    had[:, :, length - n:] = 0
    assert torch.equal(more, had + got)


@pytest.mark.parametrize("hq,hkv,n,length", SHAPES)
def test_weights_of_heads_without_a_sum(hq, hkv, n, length):
    """heads whose lse is -inf add nothing, whatever their queries are"""
    prm, gen = binding.Params(hq, hkv), gen_of(n + 1)
    cache = filled(gen, [length], hkv, 16)
    q = normal(gen, 1, n, hq, D)
    _, lse = binding.paged_attn(prm, q, cache, i32([length]), length)
    none = torch.rand((n, hq), generator=gen, device="cuda") < 0.3
    none[0, 0] = True
    lse[0][none] = -math.inf
    clean = torch.where(none[None, :, :, None], 0, q)
    want, tol = weights64(clean[0], lse[0], rows_of(cache, cache.k, 0, length), length - n, seen_rows(cache, 0, length))
    kinds = torch.randint(0, 3, (n, hq), generator=gen, device="cuda")
    for i, x in enumerate((NAN, math.inf, 3e38)):
        q[0][none & (kinds == i)] = x
    got = binding.paged_attn_weights(prm, q, lse, cache, i32([length]), length)
    assert bool(((got[0].double() - want).abs() <= tol).all())


def entries(cache, cap):
    """the table with as many entries as `cap` rows take, those behind the sequence's -1"""
    table = torch.full((1, (cap + cache.k.shape[2] - 1) // cache.k.shape[2]), -1, dtype=torch.int32, device="cuda")
    table[:, :cache.table.shape[1]] = cache.table
    return table


@pytest.mark.parametrize("cap,length,budget,first,recent", [(200, 200, 100, 4, 20), (200, 90, 100, 0, 0), (20000, 19990, 700, 40, 90)])
def test_eviction_of_rows_without_pages(cap, length, budget, first, recent):
    """what lay in the places of kept rows that have no page is seen by nobody: they hold zeros, and no result depends on it"""
    hkv, hq, page, found = 2, 8, 16, []
    prm = binding.Params(hq, hkv)
    for fill in (7.0, NAN, math.inf):
        gen = gen_of(cap)
        cache, to = filled(gen, [length], hkv, page), make_pages(gen, [budget], hkv, page, fill=fill)
        cache.table[0, 1], cache.table[0, 3], cache.table[0, (length - 1) // page] = -1, cache.k.shape[0], 1 << 30
        w = torch.rand((1, hkv, cap), generator=gen, device="cuda")
        w[:, :, 16:32] += 1.0                                     # they stay for their weight too
        kept, _, left = binding.paged_evict(prm, w, cache._replace(table=entries(cache, cap)), i32([length]), cap, budget, first, recent, to)
        m = min(length, budget)
        assert int(left[0]) == m
        there, safe = seen_rows(cache, 0, length), cache._replace(table=cache.table.clamp(0, cache.k.shape[0] - 1))
        for pool, new in ((cache.k, to.k), (cache.v, to.v)):
            rows, moved = rows_of(safe, pool, 0, length), rows_of(to, new, 0, m)
            for h in range(hkv):
                t = kept[0, h, :m].long()
                assert 0 < int((~there[t]).sum()) < m
                assert torch.equal(moved[h], torch.where(there[t][:, None], rows[h, t], 0))
        q = normal(gen, 1, 1, hq, D)
        found.append(binding.paged_attn(prm, q, to, left, budget))
    assert all(bool(torch.isfinite(x).all()) and torch.equal(x, y) for pair in found for x, y in zip(pair, found[0]))
