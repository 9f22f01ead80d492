"""The attention's limits that the host checks before a launch (no GPU needed)."""
import ctypes

import pytest

from test_attend_pins import attend_args, cache_struct


@pytest.fixture(scope="module")
def px():
    import paper_2607_22595_amd as m
    return m


@pytest.mark.parametrize("n_q,n_kv", [(8, 2), (64, 1), (17, 1)])
def test_rows_past_32_bits(px, n_q, n_kv):
    """Rows of a key head, up to the end of the last tile of 128, fit into 32 bits."""
    c = cache_struct(px, n_kv=n_kv)
    least = (2 ** 31 - 1 - 128) // (n_q // n_kv) + 1
    for T_max in (least, 2 ** 31 - 1):
        for name in ("xmix_paged_attention", "xmix_paged_attention_valid"):
            args = attend_args(px, c, T_max=T_max, n_q=n_q, q_stride=64 * n_q, out_stride=64 * n_q)
            if name.endswith("valid"):
                args.insert(len(args) - 1, None)
            assert getattr(px._lib, name)(*args) == px.XMIX_E_UNSUPPORTED
        assert px._lib.xmix_paged_attention_workspace(T_max, n_q, 5, ctypes.byref(c)) == 0
    assert px._lib.xmix_paged_attention_workspace(least - 1, n_q, 5, ctypes.byref(c)) > 0


def test_the_counted_call_refuses_what_the_plain_one_does(px):
    for kw, status in [(dict(q=None), px.XMIX_E_INVAL), (dict(window=-1), px.XMIX_E_INVAL),
                       (dict(scale=0.0), px.XMIX_E_INVAL), (dict(err=None), px.XMIX_E_INVAL),
                       (dict(ws=None), px.XMIX_E_WORKSPACE), (dict(ws_bytes=1), px.XMIX_E_WORKSPACE)]:
        args = attend_args(px, **kw)
        args.insert(len(args) - 1, 1 << 20)
        assert px._lib.xmix_paged_attention_valid(*args) == status, kw
