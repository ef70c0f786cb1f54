"""Calls of rotary positions and the cache in pages with so many rows that a launch of one dimension would have 2^32 threads and more."""
import pytest
import torch

from paper_2506_07900_amd import binding
from test_gpu_paged import D, filled, gen_of, i32, normal

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("hq,rows", [(1, (1 << 26) + 77), (9, (1 << 25) + 5)])
def test_rotation_of_many_rows(hq, rows):
    """17 and 77 GB, in place"""
    prm, rope = binding.Params(hq, hq), binding.rope_table(128)
    q = torch.ones((1, rows, hq, D), dtype=torch.bfloat16, device="cuda")
    assert binding.rope(prm, rope, q, None, i32([rows - 2]), rows, q_out=q)[0] is q
    at = torch.tensor([0, 1, 63, 64, 65, 77, 4096, rows // 2, (1 << 25) - 1, (1 << 25), (1 << 25) + 1, rows - 70, rows - 4, rows - 3], device="cuda")
    small = torch.ones((1, len(at), hq, D), dtype=torch.bfloat16, device="cuda")
    want = binding.rope(prm, rope, small, None, i32([len(at)]), len(at), positions=at.int()[None])[0]
    assert torch.equal(q[0, at], want[0]) and bool((q[0, rows - 2:] == 1).all())
    assert float((q[0].view(-1)[D * hq::1 << 20] == 1).float().mean()) < 0.05         # (a few come out as 1; of rows left out all are)
    del q
    torch.cuda.empty_cache()


@pytest.mark.parametrize("cap", [1 << 28, (1 << 28) + 128 * 1000])
def test_weights_of_many_rows(cap):
    """a bound of so many rows that 128 of them to a workgroup are 2^24 workgroups and more; 8.6 GB of weights"""
    hkv, group, n, lengths = 8, 16, 4, [3000]
    prm, gen = binding.Params(hkv * group, hkv), gen_of(7)
    cache = filled(gen, lengths, hkv, 1024)
    q = normal(gen, 1, n, hkv * group, D)
    _, lse = binding.paged_attn(prm, q, cache, i32(lengths), 3000)
    want = binding.paged_attn_weights(prm, q, lse, cache, i32(lengths), 3000)
    table = torch.zeros((1, cap // 1024 + 1), dtype=torch.int32, device="cuda")
    table[:, :3] = cache.table
    got = binding.paged_attn_weights(prm, q, lse, cache._replace(table=table), i32(lengths), cap)
    # (the sums' parts, and so their order, go by the bound: each of 64 numbers is added to what is before it, twice over)
    assert bool(((got[:, :, :3000] - want[:, :, :3000]).abs() <= 64 * 2.0 ** -23 * want[:, :, :3000]).all())
    assert not bool(got[:, :, 3000:].any())
    # its last tile, of the last head: a sequence that is as long as the bound shares its pages
    table[:] = cache.table[0, 0]
    n_new = i32([1])
    whole = torch.full((1, hkv, cap), -1.0, device="cuda")
    binding.paged_attn_weights(prm, q, torch.zeros_like(lse), cache._replace(table=table), i32([cap]), cap, n_new=n_new, weights_out=whole)
    x = (q[0, 0].view(hkv, group, D).double() @ cache.k[int(cache.table[0, 0])].double().transpose(1, 2)) * prm.softmax_scale      # [hkv, group, 1024]
    size = (q[0, 0].view(hkv, group, D).double().abs() @ cache.k[int(cache.table[0, 0])].double().abs().transpose(1, 2)) * prm.softmax_scale
    once, tol = x.exp().sum(1), (x.exp() * (2.0 ** -17 * size + 2.0 ** -22 * x.abs() + 2.0 ** -18)).sum(1)
    rows = whole[0, :, :cap // 1024 * 1024].view(hkv, -1, 1024)
    for piece in range(0, rows.shape[1], 32768):
        assert bool(((rows[:, piece:piece + 32768].double() - once[:, None]).abs() <= tol[:, None]).all())
    del got, whole, rows
    torch.cuda.empty_cache()
