"""The oracle's attention of a serving step against facts other than itself, and
the calls' refusals that need no GPU."""
import ctypes
import math

import numpy as np
import pytest

import oracle


def bits(x):
    return (np.asarray(x, np.float32).view(np.uint32) >> 16).astype(np.uint16)


def grid(rng, *shape):
    """Values that bf16 holds exactly."""
    return rng.integers(-64, 65, shape).astype(np.float64) / 16.0


def test_rotation_is_a_rotation():
    rng = np.random.default_rng(0)
    x = rng.normal(size=(5, 2, 32)).astype(np.float32)
    f = 10000.0 ** (-np.arange(8) / 8)
    pos = np.array([0, 1, 7, 100000, -1], np.int32)
    for pairs in (False, True):
        y = oracle.norm_rope(x, pos, inv_freq=f, pairs=pairs)
        assert np.array_equal(y[0], x[0].astype(np.float64))          # position 0: the identity
        assert np.isnan(y[4]).all()                                   # padding: not written
        assert np.array_equal(y[:4, :, 16:], x[:4, :, 16:])           # past the rotated part
        np.testing.assert_allclose((y[:4] ** 2).sum(-1), (x[:4].astype(np.float64) ** 2).sum(-1))
        a = slice(0, 16, 2) if pairs else slice(0, 8)
        b = slice(1, 16, 2) if pairs else slice(8, 16)
        z = (x[2, :, a] + 1j * x[2, :, b].astype(np.float64)) * np.exp(7j * f)
        np.testing.assert_allclose(y[2][:, a] + 1j * y[2][:, b], z, rtol=1e-12, atol=1e-12)


def test_rotated_products_depend_on_the_distance_alone():
    rng = np.random.default_rng(1)
    q, k = rng.normal(size=(2, 1, 1, 64)).astype(np.float32)
    f = 500000.0 ** (-np.arange(32) / 32)
    dots = []
    for p in (0, 13, 4000):
        a = oracle.norm_rope(q, [p + 9], inv_freq=f)
        b = oracle.norm_rope(k, [p], inv_freq=f)
        dots.append(float((a * b).sum()))
    np.testing.assert_allclose(dots, dots[0], rtol=1e-9)


def test_norm_has_unit_mean_square():
    x = np.random.default_rng(2).normal(size=(3, 2, 48)).astype(np.float32)
    y = oracle.norm_rope(x, [0, 1, 2], weight=np.ones(48, np.float32))
    np.testing.assert_allclose((y ** 2).mean(-1), 1.0)
    w = np.arange(48, dtype=np.float32)
    np.testing.assert_allclose(oracle.norm_rope(x, [0, 1, 2], weight=w), y * w, rtol=1e-12)


def paged(rng, total, ps, n_kv, hd):
    """A cache of one request with `total` keys in shuffled pages, and its rows."""
    n = -(-total // ps)
    k, v = grid(rng, n + 2, n_kv, ps, hd), grid(rng, n + 2, n_kv, ps, hd)
    table = rng.permutation(n + 2)[:n].astype(np.int32)
    rows = [x[table].transpose(0, 2, 1, 3).reshape(-1, n_kv, hd)[:total] for x in (k, v)]
    return k, v, table[None], rows


@pytest.mark.parametrize("window", [0, 1, 5, 100])
def test_attention_matches_a_dense_softmax(window):
    rng = np.random.default_rng(3)
    n, total, n_q, n_kv, hd = 4, 37, 4, 2, 16
    k, v, table, (kr, vr) = paged(rng, total, 16, n_kv, hd)
    q = grid(rng, n, n_q, hd)
    out, lse, mag, _ = oracle.attend(bits(q), [0, n], [total], k, v, table, 0.3, window)
    for i in range(n):
        p = total - n + i
        see = np.arange(total) <= p
        if window:
            see &= np.arange(total) > p - window
        for g in range(n_q):
            s = 0.3 * kr[see, g // 2] @ q[i, g]
            w = np.exp(s - s.max())
            np.testing.assert_allclose(out[i, g], w @ vr[see, g // 2] / w.sum(), rtol=1e-10, atol=1e-12)
            np.testing.assert_allclose(lse[g, i], s.max() + math.log(w.sum()), rtol=1e-12)


def test_one_key_returns_its_value_and_no_key_zeros():
    rng = np.random.default_rng(4)
    k, v, table, (kr, vr) = paged(rng, 1, 16, 1, 16)
    q = grid(rng, 3, 2, 16)
    out, lse, _, _ = oracle.attend(bits(q), [0, 3], [1], k, v, table, 1.0)   # positions -2, -1, 0
    assert np.array_equal(out[2], np.broadcast_to(vr[0], (2, 16)))
    assert (out[:2] == 0).all() and np.isneginf(lse[:, :2]).all()


def test_equal_keys_give_the_mean():
    k = np.ones((2, 1, 16, 16))
    v = grid(np.random.default_rng(5), 2, 1, 16, 16)
    out, lse, _, _ = oracle.attend(bits(np.ones((1, 1, 16))), [0, 1], [20], k, v, [[1, 0]], 0.5)
    rows = np.concatenate([v[1, 0], v[0, 0]])[:20]
    np.testing.assert_allclose(out[0, 0], rows.mean(0))
    np.testing.assert_allclose(lse[0, 0], 8.0 + math.log(20))


def test_missing_pages_are_left_out():
    rng = np.random.default_rng(6)
    k, v, table, _ = paged(rng, 48, 16, 1, 16)
    q = bits(grid(rng, 1, 1, 16))
    broken = table.copy()
    broken[0, 1] = 99
    out = oracle.attend(q, [0, 1], [48], k, v, broken, 1.0)[0]
    short = oracle.attend(q, [0, 1], [32], k, v, table[:, [0, 2]], 1.0)[0]
    np.testing.assert_allclose(out, short, rtol=1e-12)


# ------------------------------------------------------------------- refusals

@pytest.fixture(scope="module")
def px():
    import paper_2607_22595_amd as m
    return m


P = 1 << 20  # an aligned address that no refused call looks at


def cache_struct(px, **kw):
    d = dict(k=P, v=P, pages=P, k_scale=None, v_scale=None, n_pages=4, page_size=16, n_kv=2,
             head_dim=64, R_max=3, max_pages=8, dt=px.XMIX_BF16)
    d.update(kw)
    return px.XmixKvCache(*[d[n] for n, _ in px.XmixKvCache._fields_])


BAD_CACHES = [dict(k=None), dict(v=None), dict(pages=None), dict(k=P + 2), dict(v=P + 8), dict(n_pages=0),
              dict(page_size=8), dict(page_size=24), dict(page_size=8192), dict(n_kv=0), dict(head_dim=8),
              dict(head_dim=72), dict(head_dim=272), dict(R_max=0), dict(max_pages=0),
              dict(max_pages=1 << 27), dict(dt=0), dict(dt=3), dict(k_scale=P), dict(dt=2),
              dict(dt=2, k_scale=P), dict(dt=2, v_scale=P)]


def norm_rope_args(px, **kw):
    d = dict(q=P, q_stride=256, n_q=4, k=P, k_stride=128, n_kv=2, dt=px.XMIX_BF16, head_dim=64, T_max=5,
             pos=P, q_w=P, k_w=P, eps=1e-6, rope=px.XmixRope(P, 64, 0), q_out=P, q_out_stride=256, k_out=P,
             k_out_stride=128, T_valid=None, stream=None)
    d.update(kw)
    if d["rope"] is not None:
        d["rope"] = ctypes.byref(d["rope"])
    return list(d.values())


def rope(px, freq=P, rot=64, pairing=0):
    return px.XmixRope(freq, rot, pairing)


def test_norm_rope_refusals(px):
    bad = [dict(q=None), dict(q_out=None), dict(k=None), dict(k_out=None), dict(n_kv=0), dict(pos=None),
           dict(n_q=0), dict(n_q=-1), dict(n_kv=-1), dict(T_max=0), dict(dt=2), dict(dt=7), dict(head_dim=0),
           dict(head_dim=40), dict(head_dim=264), dict(q=P + 8), dict(k=P + 2), dict(q_out=P + 4),
           dict(k_out=P + 8), dict(q_w=P + 8), dict(k_w=P + 2), dict(q_stride=252), dict(k_stride=-128),
           dict(q_out_stride=248), dict(k_out_stride=120), dict(eps=-1.0), dict(eps=math.nan),
           dict(rope=rope(px, None)), dict(rope=rope(px, P + 8)), dict(rope=rope(px, rot=8)),
           dict(rope=rope(px, rot=72)), dict(rope=rope(px, rot=80)), dict(rope=rope(px, pairing=2))]
    for kw in bad:
        assert px._lib.xmix_qk_norm_rope(*norm_rope_args(px, **kw)) == px.XMIX_E_INVAL, kw


def append_args(px, cache=None, **kw):
    d = dict(k=P, k_stride=128, v=P, v_stride=128, dt=px.XMIX_BF16, T_max=5, req=P, pos=P,
             rope=rope(px), cache=cache or cache_struct(px), err=P, T_valid=None, stream=None)
    d.update(kw)
    d["cache"] = ctypes.byref(d["cache"])
    if d["rope"] is not None:
        d["rope"] = ctypes.byref(d["rope"])
    return list(d.values())


def test_append_refusals(px):
    bad = [dict(k=None), dict(v=None), dict(req=None), dict(pos=None), dict(err=None), dict(T_max=0), dict(dt=2),
           dict(k=P + 8), dict(v=P + 2), dict(k_stride=124), dict(v_stride=-8), dict(rope=rope(px, rot=80))]
    for kw in bad:
        assert px._lib.xmix_kv_append(*append_args(px, **kw)) == px.XMIX_E_INVAL, kw
    for kw in BAD_CACHES:
        assert px._lib.xmix_kv_append(*append_args(px, cache_struct(px, **kw))) == px.XMIX_E_INVAL, kw
    args = append_args(px)
    args[9] = None
    assert px._lib.xmix_kv_append(*args) == px.XMIX_E_INVAL


def attend_args(px, cache=None, **kw):
    d = dict(q=P, q_stride=256, n_q=4, T_max=5, cu=P, kv_len=P, cache=cache or cache_struct(px), scale=0.125,
             window=0, max_q=5, out=P, out_stride=256, lse=P, err=P, ws=P, ws_bytes=1 << 40, stream=None)
    d.update(kw)
    d["cache"] = ctypes.byref(d["cache"])
    return list(d.values())


def test_attention_refusals(px):
    fn = px._lib.xmix_paged_attention
    bad = [dict(q=None), dict(cu=None), dict(kv_len=None), dict(out=None), dict(err=None), dict(T_max=0),
           dict(n_q=0), dict(n_q=3), dict(n_q=-2), dict(max_q=0), dict(window=-1), dict(scale=0.0),
           dict(scale=-1.0), dict(scale=math.nan), dict(scale=math.inf), dict(q=P + 8), dict(out=P + 2),
           dict(q_stride=252), dict(out_stride=248)]
    for kw in bad:
        assert fn(*attend_args(px, **kw)) == px.XMIX_E_INVAL, kw
    for kw in BAD_CACHES:
        assert fn(*attend_args(px, cache_struct(px, **kw))) == px.XMIX_E_INVAL, kw
    for kw in (dict(head_dim=32), dict(head_dim=96), dict(R_max=4097)):
        c = cache_struct(px, **kw)
        assert fn(*attend_args(px, c, q_stride=1024, out_stride=1024)) == px.XMIX_E_UNSUPPORTED, kw
        assert px._lib.xmix_paged_attention_workspace(5, 4, 5, ctypes.byref(c)) == 0


@pytest.mark.parametrize("max_q", [1, 3, 5, 300])
def test_attention_workspace(px, max_q):
    c = cache_struct(px)
    need = px._lib.xmix_paged_attention_workspace(300, 4, max_q, ctypes.byref(c))
    assert need < 1 << 28  # whatever the lengths
    if need:
        for kw in (dict(ws=None), dict(ws=P + 8), dict(ws_bytes=need - 1)):
            args = attend_args(px, T_max=300, max_q=max_q, **kw)
            assert px._lib.xmix_paged_attention(*args) == px.XMIX_E_WORKSPACE, kw


def test_descriptors_check_what_they_are_given(px):
    import torch
    with pytest.raises(TypeError):
        px.Rope(torch.zeros(8))
    with pytest.raises(TypeError):
        px.Rope(torch.zeros(2, 4, dtype=torch.float64))
    with pytest.raises(ValueError):
        px.Rope(torch.zeros(8, dtype=torch.float64))  # not on the GPU
    k = torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16)
    table = torch.zeros(3, 4, dtype=torch.int32)
    k8 = k.to(torch.float8_e4m3fn)
    for args, err in [((k.float(), k.float(), table), TypeError), ((k, k8, table), TypeError),
                      ((k, k[:3], table), ValueError), ((k[0], k[0], table), ValueError),
                      ((k, k, table.long()), ValueError), ((k, k, table[0]), ValueError),
                      ((k, k, table, torch.ones(2)), ValueError), ((k8, k8, table, torch.ones(3)), ValueError),
                      ((k8, k8, table, torch.ones(2).double()), ValueError), ((k, k, table), ValueError)]:
        with pytest.raises(err):
            px.KvCache(*args)
