"""CPU checks of how large the calls of rotary positions and the cache in pages may be: a launch has fewer than 2^32 threads along a dimension, and of more the runtime silently starts what is left
modulo 2^32."""
import pytest

from test_paged_abi import CALLS, LENGTHS, UNSUPPORTED, call, lib, pages, params  # noqa: F401


@pytest.mark.parametrize("name", ["rope", "rope_bwd"])
def test_rows_of_the_rotation(lib, name):  # noqa: F811
    at = LENGTHS[name]
    for hq, hkv, rows, want in ((1, 1, 1 << 30, 0), (4, 4, 1 << 30, 0), (8, 1, (1 << 29) + 1, UNSUPPORTED), (32, 2, (1 << 30) // 5, 0), (32, 2, (1 << 30) // 5 + 1, UNSUPPORTED)):
        assert call(lib, name, _0=params(n_q_heads=hq, n_kv_heads=hkv), **{"_%d" % (at + 2): rows}) == want, (hq, hkv, rows)


def test_workgroups_of_attention_and_weights(lib):  # noqa: F811
    wide = pages(stride=1 << 20, size=1024)
    one = lambda heads: params(n_q_heads=heads, n_kv_heads=heads)                                  # noqa: E731
    # with batches: nothing that passes is asked for
    assert call(lib, "paged_attn", _0=one(1024), _5=65535, _7=129) == UNSUPPORTED
    assert call(lib, "paged_attn", _0=one(129), _5=65535, _7=17) == UNSUPPORTED
    assert call(lib, "paged_attn_weights", _0=one(8), _3=wide, _6=129, _7=1 << 27, _10=1 << 27) == UNSUPPORTED
    assert call(lib, "paged_attn_weights", _0=one(2048), _3=wide, _6=65535, _7=1025, _10=1025) == UNSUPPORTED


def test_rows_to_keep(lib):  # noqa: F811
    for budget, want in (((1 << 30) - 64, 0), ((1 << 30) - 63, UNSUPPORTED), (1 << 30, UNSUPPORTED)):
        assert call(lib, "paged_evict", _7=budget) == want
    assert len(CALLS["paged_evict"]) == 17
