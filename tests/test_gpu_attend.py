"""Attention of a serving step on the GPU against the oracle: norm and rotation of
heads, append to the paged cache, attention over its pages, and the three in a
row as a step runs them.

Tolerances count roundings, of half a step of the type each (bf16 2^-8, e4m3 2^-4
of the value, fp32 2^-24):
  heads      one rounding to the stored type; in fp32 before it a sum of head_dim
             squares, and products with a sine and cosine that are 1.2e-7 off
  attention  the weights exp(s - max) are rounded to bf16 (2^-8 of sum p |v|), the
             result once more (2^-8 of it); a score in fp32 is head_dim
             roundings of sum |q k| off, which the weights take as a factor
"""
import numpy as np
import pytest
import torch

import oracle

pytestmark = pytest.mark.gpu

BF, F32, E4 = torch.bfloat16, torch.float32, torch.float8_e4m3fn


@pytest.fixture(scope="module")
def px():
    import paper_2607_22595_amd as m
    return m


def i32(x):
    return torch.as_tensor(np.asarray(x), dtype=torch.int32).cuda()


def word():
    return torch.zeros(1, dtype=torch.int32, device="cuda")


def bits(t):
    t = t.detach().cpu().contiguous()
    return t.view(torch.int16).numpy().view(np.uint16) if t.dtype == BF else t.numpy()


def wide(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def same(a, b):
    v = {BF: torch.int16, F32: torch.int32, E4: torch.uint8}[a.dtype]
    return torch.equal(a.contiguous().view(v), b.contiguous().view(v))


def frequencies(rot, theta=500000.0):
    return theta ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)


# ------------------------------------------------------------- norm and rotation

def check_heads(got, ref, hd, half_step):
    slack = (2 * (hd + 16) * 2.0 ** -24 + 4e-7) * np.abs(ref).max(-1, keepdims=True)
    assert np.isfinite(got).all()
    assert (np.abs(got - ref) <= half_step * np.abs(ref) + slack).all()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("hd,rot,pairs,norm", [
    (128, 128, False, True), (128, 64, False, False), (64, 32, True, True), (64, 64, False, True),
    (256, 256, True, False), (256, 128, False, True), (96, 96, False, True), (80, 32, False, True),
    (16, 16, True, True), (16, 16, False, False), (48, 0, False, True), (240, 240, False, True),
    (112, 48, True, False)])
@pytest.mark.parametrize("T,n_q,n_kv", [(1, 1, 1), (7, 14, 2), (33, 40, 8)])
def test_norm_rope(px, dtype, hd, rot, pairs, norm, T, n_q, n_kv):
    g = torch.Generator().manual_seed(hd + rot + T)
    row = torch.randn(T, n_q + 2 * n_kv, hd, generator=g).to(dtype).cuda()
    q, k = row[:, :n_q], row[:, n_q:n_q + n_kv]
    w = [(1 + 0.3 * torch.randn(hd, generator=g)).to(dtype).cuda() if norm else None for _ in range(2)]
    pos = torch.randint(0, 1 << 17, (T,), generator=g, dtype=torch.int32)
    f = frequencies(rot) if rot else None
    rope = px.Rope(f.cuda(), px.XMIX_ROPE_PAIRS if pairs else px.XMIX_ROPE_HALF) if rot else None
    qo, ko = torch.zeros_like(q.contiguous()), torch.zeros_like(k.contiguous())
    px.xmix_qk_norm_rope(q, k, pos.cuda(), w[0], w[1], 1e-6, rope, qo, ko)
    for x, weight, out in ((q, w[0], qo), (k, w[1], ko)):
        ref = oracle.norm_rope(bits(x), pos.numpy(), None if weight is None else bits(weight), 1e-6,
                               None if f is None else f.numpy(), pairs)
        check_heads(wide(out), ref, hd, 2.0 ** -8 if dtype == BF else 2.0 ** -24)
    # in place, and queries alone: the same bits; values are not touched
    before = row.clone()
    px.xmix_qk_norm_rope(q, k, pos.cuda(), w[0], w[1], 1e-6, rope, q, k)
    assert same(q, qo) and same(k, ko) and same(row[:, n_q + n_kv:], before[:, n_q + n_kv:])
    alone = torch.zeros_like(qo)
    px.xmix_qk_norm_rope(before[:, :n_q], None, pos.cuda(), w[0], None, 1e-6, rope, alone, None)
    assert same(alone, qo)


def test_norm_rope_leaves_padding_and_keeps_zero_rows(px):
    T, n, hd = 9, 3, 64
    x = torch.randn(T, n, hd, generator=torch.Generator().manual_seed(1)).to(BF).cuda()
    x[4] = 0
    w = torch.ones(hd, dtype=BF, device="cuda")
    pos = i32([0, 1, -1, 3, 4, -7, 6, 7, 8])
    rope = px.Rope(frequencies(hd).cuda())
    out, out2 = torch.full_like(x, 9.0), torch.full_like(x, 9.0)
    px.xmix_qk_norm_rope(x, None, pos, w, None, 1e-6, rope, out, None)
    px.xmix_qk_norm_rope(x, None, pos, w, None, 1e-6, rope, out2, None, T_valid=i32([7]))
    assert (out[[2, 5]] == 9).all() and (out[4] == 0).all() and torch.isfinite(out).all()
    assert (out2[7:] == 9).all() and same(out2[:7], out[:7])


def test_far_positions_keep_their_angle(px):
    hd, pos = 64, [2 ** 31 - 1, 2 ** 30 + 12345, 10 ** 9 + 7]
    x = torch.randn(3, 2, hd, generator=torch.Generator().manual_seed(2)).cuda()
    f, out = frequencies(hd), torch.zeros(3, 2, hd, device="cuda")
    px.xmix_qk_norm_rope(x, None, i32(pos), None, None, 0.0, px.Rope(f.cuda()), out, None)
    ref = oracle.norm_rope(bits(x), pos, inv_freq=f.numpy())
    # 2^31 radians are known to 2^31 2^-53 in fp64: on either side another 2.4e-7 (twice rounded)
    assert np.abs(wide(out) - ref).max() <= 2e-6 * np.abs(ref).max()


# --------------------------------------------------------------------- append

def make_cache(px, g, n_pages, n_kv, ps, hd, R, max_pages, dtype=BF, table=None):
    k, v = [torch.randn(n_pages, n_kv, ps, hd, generator=g, device="cuda").to(dtype) for _ in range(2)]
    if table is None:
        table = torch.randperm(n_pages, generator=torch.Generator().manual_seed(5))[:R * max_pages]
        table = table.to(torch.int32).view(R, max_pages)
    s = [None, None] if dtype == BF else [0.02 + 0.05 * torch.rand(n_kv, generator=g, device="cuda") for _ in "kv"]
    return px.KvCache(k, v, torch.as_tensor(table, dtype=torch.int32).cuda(), *s)


def gpu_generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def slots(cache, req, pos):
    ps = cache.k.shape[2]
    page = cache.pages.cpu().numpy()[req, np.asarray(pos) // ps]
    return torch.as_tensor(page).long(), torch.as_tensor(np.asarray(pos) % ps).long()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("stored", [BF, E4])
@pytest.mark.parametrize("hd,rot,pairs,n_kv,ps", [(128, 128, False, 8, 16), (64, 0, False, 1, 32),
                                                  (64, 32, True, 3, 64), (256, 256, False, 2, 16),
                                                  (80, 80, False, 5, 16), (16, 16, True, 1, 128)])
def test_append(px, dtype, stored, hd, rot, pairs, n_kv, ps):
    g, R, per = gpu_generator(hd + ps), 5, 6
    cache = make_cache(px, g, R * per + 2, n_kv, ps, hd, R, per, stored)
    lens, ctx = [1, 7, 20, 3, 1], [0, 15, 31, per * ps - 3, 17]
    req = np.repeat(np.arange(R), lens)
    pos = np.concatenate([np.arange(c, c + n) for n, c in zip(lens, ctx)])
    T = len(req)
    row = torch.randn(T, 2 * n_kv + 1, hd, generator=g, device="cuda").to(dtype)
    row[:, :, 3] *= 100.0  # past what 8 bits hold
    k, v = row[:, :n_kv], row[:, n_kv:2 * n_kv]
    f = frequencies(rot) if rot else None
    rope = px.Rope(f.cuda(), px.XMIX_ROPE_PAIRS if pairs else px.XMIX_ROPE_HALF) if rot else None
    before = [cache.k.clone(), cache.v.clone()]
    err = word()
    px.xmix_kv_append(k, v, i32(req), i32(pos), rope, cache, err)
    page, slot = slots(cache, req, pos)
    for x, pages, scale, old, turned in ((k, cache.k, cache.k_scale, before[0], rope),
                                         (v, cache.v, cache.v_scale, before[1], None)):
        got = pages.float().cpu()[page, :, slot].double().numpy()
        ref = oracle.norm_rope(bits(x), pos, inv_freq=f.numpy() if turned else None, pairs=pairs)
        slack = 4e-7 * np.abs(ref).max(-1, keepdims=True)
        if scale is None:
            half, tiny = 2.0 ** -8, 0.0
        else:
            s = wide(scale)[:, None]
            ref, slack = np.clip(ref / s, -448, 448), slack / s
            half, tiny = 2.0 ** -4, 2.0 ** -10
        if turned is None:  # no arithmetic but the stored type's own: to the bit
            y = x.float().cpu()
            if scale is not None:
                y = (y / scale.cpu()[:, None]).clamp(-448, 448)
            assert np.array_equal(got, y.to(stored).double().numpy())
        assert (np.abs(got - ref) <= half * np.abs(ref) + tiny + slack).all()
        touched = torch.zeros(pages.shape[0], ps, dtype=torch.bool)
        touched[page, slot] = True
        rest = ~touched[:, None, :, None].expand(pages.shape)
        view = torch.uint8 if stored == E4 else torch.int16
        assert torch.equal(pages.view(view).cpu()[rest], old.view(view).cpu()[rest])
    assert err.item() == 0


@pytest.mark.parametrize("stored", [BF, E4])
def test_append_leaves_padding_and_reports_bad_slots(px, stored):
    g = gpu_generator(9)
    table = [[0, 1], [2, 9], [3, -1]]  # pages 9 and -1 are not there
    cache = make_cache(px, g, 4, 2, 16, 64, 3, 2, stored, table)
    row = torch.randn(9, 4, 64, generator=g, device="cuda").to(BF)
    k, v = row[:, :2], row[:, 2:]
    before = cache.k.clone(), cache.v.clone()
    good = (i32([0, 1, -1, 2, 0, 2, 1, 0, 2]), i32([0, 4, 5, 15, -1, -9, 3, 1, 0]))
    err = word()
    px.xmix_kv_append(k, v, *good, None, cache, err, T_valid=i32([7]))
    assert err.item() == 0
    changed = (cache.k.view(torch.uint8) != before[0].view(torch.uint8)).flatten(3).any(-1).any(1)
    assert changed.nonzero().tolist() == [[0, 0], [2, 3], [2, 4], [3, 15]]
    now = cache.k.clone(), cache.v.clone()
    for req, pos in ((3, 0), (2 ** 31 - 1, 0), (0, 32), (0, 2 ** 31 - 1), (1, 16), (2, 31)):
        err = word()
        px.xmix_kv_append(k[:1], v[:1], i32([req]), i32([pos]), None, cache, err)
        assert err.item() == px.XMIX_ERR_KV_SLOT, (req, pos)
    assert same(cache.k, now[0]) and same(cache.v, now[1])


def test_append_keeps_nan_and_saturates(px):
    cache = make_cache(px, gpu_generator(1), 1, 1, 16, 64, 1, 1, E4)
    cache.k_scale.fill_(0.5)
    cache.v_scale.fill_(2.0)
    x = torch.zeros(1, 1, 64, device="cuda")
    x[0, 0, :6] = torch.tensor([float("nan"), float("inf"), -float("inf"), 1e30, -230.0, 2.0 ** -9])
    px.xmix_kv_append(x, x, i32([0]), i32([3]), None, cache, word())
    k, v = cache.k[0, 0, 3].float().cpu(), cache.v[0, 0, 3].float().cpu()
    assert torch.isnan(k[0]) and k[1:6].tolist() == [448.0, -448.0, 448.0, -448.0, 2.0 ** -8]
    assert torch.isnan(v[0]) and v[1:6].tolist() == [448.0, -448.0, 448.0, -112.0, 0.0]


# ------------------------------------------------------------------ attention

def batch(px, seed, n, total, n_q, n_kv, hd, ps, stored=BF, pad=0, spare=2, outlier=True):
    """A batch of spans of n[r] tokens whose requests hold total[r] keys each."""
    g = gpu_generator(seed)
    count = [-(-max(t, 0) // ps) for t in total]
    order = torch.randperm(sum(count) + spare, generator=torch.Generator().manual_seed(seed))
    table, at = np.full((len(n), max(max(count), 1)), -1, np.int32), 0
    for r, c in enumerate(count):
        table[r, :c] = order[at:at + c]
        at += c
    cache = make_cache(px, g, len(order), n_kv, ps, hd, len(n), table.shape[1], stored, table)
    T = sum(n) + pad
    q = torch.randn(T, n_q, hd, generator=g, device="cuda")
    if outlier:
        q[..., 7] *= 8.0
    return dict(cache=cache, q=q.to(BF), cu=np.concatenate([[0], np.cumsum(n)]), kv_len=np.asarray(total),
                T=T, max_q=max(max(n), 1), scale=hd ** -0.5, window=0)


def attend(px, b, lse=True, **kw):
    """One call; the outputs start as 9 so that an untouched row shows."""
    b = dict(b, **kw)
    n_q = b["q"].shape[1]
    out = b.get("out")
    if out is None:
        out = torch.full(b["q"].shape, 9.0, dtype=BF, device="cuda")
    z = torch.full((n_q, b["T"]), 9.0, device="cuda") if lse else None
    ws = torch.full((px.paged_attention_workspace(b["T"], n_q, b["max_q"], b["cache"]),), 0xA5,
                    dtype=torch.uint8, device="cuda")
    err = word()
    px.xmix_paged_attention(b["q"], i32(b["cu"]), i32(b["kv_len"]), b["cache"], b["scale"], b["window"],
                            b["max_q"], out, z, err, ws)
    torch.cuda.synchronize()
    return out, z, err.item()


def reference(b):
    c = b["cache"]
    k, v = wide(c.k), wide(c.v)
    if c.k_scale is not None:
        k, v = k * wide(c.k_scale)[:, None, None], v * wide(c.v_scale)[:, None, None]
    return oracle.attend(bits(b["q"]), b["cu"], b["kv_len"], k, v, c.pages.cpu().numpy(),
                         float(np.float32(b["scale"])), b["window"])


def check_attention(got, ref, hd, rows=None):
    out, lse = wide(got[0]), wide(got[1])
    o, z, mag, big = ref
    if rows is not None:
        out, o, mag = out[rows], o[rows], mag[rows]
        lse, z, big = lse[:, rows], z[:, rows], big[:, rows]
    live = ~np.isnan(z)
    assert (lse[~live] == 9).all() and (out[~live.T] == 9).all()   # rows outside every span
    none = np.isneginf(z)
    assert np.isneginf(lse[none]).all() and (out[none.T] == 0).all()
    score = 2 * (hd + 4) * 2.0 ** -24 * big
    on = live & ~none
    assert np.isfinite(lse[on]).all()
    assert (np.abs(lse - z)[on] <= (score + 2.0 ** -20 + 2.0 ** -22 * np.abs(z))[on]).all()
    tol = (2.0 ** -8 * 1.01 * (np.abs(o) + mag) + (2 * score + 2.0 ** -18).T[..., None] * mag)
    assert (np.abs(out - o) <= tol)[on.T].all(), np.nanmax((np.abs(out - o) / tol)[on.T])


SPANS = {
    "one": ([1], [1]),
    "one_long": ([1], [3001]),
    "decode": ([1] * 9, [1, 2, 15, 16, 17, 63, 64, 65, 700]),
    "decode_gaps": ([1, 0, 1, 0, 0, 1], [40, 33, 1, 0, 5, 129]),
    "drafts": ([5, 2, 4, 8], [5, 300, 64, 72]),
    "chunk": ([130], [130]),
    "chunk_cached": ([70], [333]),
    "prompts": ([1, 31, 64, 129], [1, 31, 64, 129]),
    "mixed": ([1, 150, 1, 3, 1], [512, 200, 31, 77, 1]),
    "no_keys": ([3, 40, 1], [1, 17, 0]),
}


@pytest.mark.parametrize("stored", [BF, E4])
@pytest.mark.parametrize("heads", [(4, 1, 128), (8, 8, 64), (14, 2, 128), (16, 2, 64), (6, 2, 256), (20, 1, 64)])
@pytest.mark.parametrize("spans", list(SPANS))
def test_attention(px, spans, heads, stored):
    n, total = SPANS[spans]
    n_q, n_kv, hd = heads
    b = batch(px, len(spans) + hd, n, total, n_q, n_kv, hd, 16, stored, pad=3)
    got = attend(px, b)
    assert got[2] == 0
    check_attention(got, reference(b), hd)
    again = attend(px, b)
    assert same(got[0], again[0]) and same(got[1], again[1])
    assert same(attend(px, b, lse=False)[0], got[0])


@pytest.mark.parametrize("window", [1, 2, 17, 64, 100, 4096])
@pytest.mark.parametrize("spans", ["decode", "drafts", "chunk", "chunk_cached", "mixed", "no_keys"])
def test_attention_in_a_window(px, spans, window):
    n, total = SPANS[spans]
    b = dict(batch(px, window, n, total, 8, 2, 64, 32), window=window)
    got = attend(px, b)
    assert got[2] == 0
    check_attention(got, reference(b), 64)


@pytest.mark.parametrize("ps", [16, 64, 256, 4096])
@pytest.mark.parametrize("n,total", [([1, 1, 2], [4100, 31, 900]), ([200, 1], [777, 5000])])
def test_attention_page_sizes(px, ps, n, total):
    b = batch(px, ps, n, total, 4, 2, 128, ps)
    got = attend(px, b)
    assert got[2] == 0
    check_attention(got, reference(b), 128)


@pytest.mark.parametrize("stored", [BF, E4])
@pytest.mark.parametrize("n,total", [([1] * 3, [20011, 9000, 130]), ([1] * 300, [90] * 300),
                                     ([6] * 40, [200 + 7 * i for i in range(40)]), ([700, 600], [700, 2600])])
def test_attention_of_larger_batches(px, n, total, stored):
    b = batch(px, len(n), n, total, 8, 2, 128, 16, stored)
    got = attend(px, b)
    assert got[2] == 0
    check_attention(got, reference(b), 128)


@pytest.mark.parametrize("max_q", [2, 4, 8, 9, 64, 1000])
def test_a_larger_bound_on_the_spans_gives_the_same(px, max_q):
    b = batch(px, 3, [1, 2, 1], [70, 300, 5], 8, 2, 64, 16)
    got = attend(px, b, max_q=max_q)
    assert got[2] == 0
    check_attention(got, reference(b), 64)


@pytest.mark.parametrize("spans", ["decode", "drafts", "mixed"])
def test_rows_at_any_distance(px, spans):
    n, total = SPANS[spans]
    b = batch(px, 8, n, total, 8, 2, 64, 16)
    got = attend(px, b)
    row = torch.full((b["T"], 14, 64), 9.0, dtype=BF, device="cuda")
    row[:, 3:11] = b["q"]
    wide_out = torch.full((b["T"], 11, 64), 9.0, dtype=BF, device="cuda")
    attend(px, b, q=row[:, 3:11], out=wide_out[:, 2:10])
    assert same(wide_out[:, 2:10], got[0])
    assert (wide_out[:, :2] == 9).all() and (wide_out[:, 10:] == 9).all()


def poison(b, keep):
    """NaN and infinities in every slot that no token of `keep` {request: keys} sees."""
    c, bad = b["cache"], [float("nan"), float("inf"), -float("inf")]
    ps, table = c.k.shape[2], c.pages.cpu().numpy()
    seen = torch.zeros(c.k.shape[0], ps, dtype=torch.bool)
    for r, keys in keep.items():
        for j in keys:
            seen[table[r, j // ps], j % ps] = True
    hidden = ~seen.cuda()
    for x in (c.k, c.v):
        junk = torch.tensor(bad, device="cuda")[torch.randint(0, 3, x.shape, device="cuda")]
        x.copy_(torch.where(hidden[:, None, :, None], junk, x.float()).to(x.dtype))


@pytest.mark.parametrize("stored", [BF, E4])
@pytest.mark.parametrize("spans", ["one", "decode", "drafts", "chunk_cached", "mixed", "no_keys"])
def test_stale_slots_have_no_effect(px, spans, stored):
    n, total = SPANS[spans]
    b = batch(px, 12, n, total, 8, 2, 128, 16, stored)
    before = attend(px, b)
    poison(b, {r: range(t) for r, t in enumerate(total)})
    after = attend(px, b)
    assert same(before[0], after[0]) and same(before[1], after[1])


@pytest.mark.parametrize("stored", [BF, E4])
@pytest.mark.parametrize("n,total,at", [(5, 69, 2), (8, 8, 0), (90, 200, 17), (150, 150, 149), (64, 64, 40)])
def test_a_later_token_has_no_effect_on_an_earlier_one(px, n, total, at, stored):
    """NaN and infinities in the keys and values of the tokens after `at`."""
    b = batch(px, 13, [n], [total], 4, 2, 64, 16, stored)
    before = attend(px, b)
    poison(b, {0: range(total - n + at + 1)})
    after = attend(px, b)
    check_attention(after, reference(dict(b, cache=clean(b))), 64, rows=slice(0, at + 1))
    assert np.allclose(wide(after[0])[:at + 1], wide(before[0])[:at + 1], rtol=0.02, atol=0.02)
    if at + 1 < n:  # and they do reach those that see them
        assert not torch.isfinite(after[0][at + 1:].float()).all()


def clean(b):
    c = b["cache"]
    d = type(c).__new__(type(c))
    d.__dict__.update(c.__dict__)
    d.k, d.v = [torch.nan_to_num(x.float(), 0.0, 0.0, 0.0) for x in (c.k, c.v)]
    return d


def test_windowed_past_has_no_effect(px):
    b = dict(batch(px, 14, [3, 1], [90, 200], 4, 2, 64, 16), window=20)
    before = attend(px, b)
    poison(b, {0: range(90 - 3 - 19, 90), 1: range(180, 200)})
    after = attend(px, b)
    check_attention(after, reference(dict(b, cache=clean(b))), 64)
    assert same(before[1][:, 3:], after[1][:, 3:])


def test_infinite_values_that_are_seen_come_through(px):
    b = batch(px, 15, [4], [20], 2, 1, 64, 16)
    table = b["cache"].pages.cpu().numpy()
    b["cache"].v[table[0, 1], 0, 2, 5] = float("inf")   # key 18: seen by the last two tokens
    b["cache"].v[table[0, 0], 0, 3, 6] = float("-inf")  # key 3: seen by all
    out = attend(px, b)[0].float()
    assert torch.isfinite(out[:2, :, 5]).all() and (out[2:, :, 5] == float("inf")).all()
    assert (out[..., 6] == float("-inf")).all()
    rest = [c for c in range(64) if c not in (5, 6)]
    assert torch.isfinite(out[..., rest]).all()


def test_large_scores(px):
    """Scores of some thousands: one key carries each row, nothing overflows."""
    b = batch(px, 16, [1, 33], [50, 33], 4, 2, 128, 16)
    b["q"] = b["q"] * 300.0
    got = attend(px, b)
    check_attention(got, reference(b), 128)


def test_bad_spans_and_lengths_are_reported(px):
    base = batch(px, 17, [2, 3, 1], [20, 30, 40], 4, 2, 64, 16)
    good = attend(px, base)
    cap = base["cache"].pages.shape[1] * 16
    for cu, kv_len, max_q, dead in [
            ([0, 2, 5, 6], [20, -1, 40], 3, [1]), ([0, 2, 5, 6], [20, cap + 1, 40], 3, [1]),
            ([0, 2, 5, 6], [20, 2 ** 31 - 1, 40], 3, [1]), ([0, 2, 5, 6], [20, 30, 40], 2, [1]),
            ([0, 2, 5, 7], [20, 30, 40], 3, [2]), ([-1, 2, 5, 6], [20, 30, 40], 3, [0]),
            ([0, 2, 5, 4], [20, 30, 40], 3, [2]), ([2 ** 31 - 1, 2, 5, 6], [20, 30, 40], 3, [0])]:
        got = attend(px, base, cu=cu, kv_len=kv_len, max_q=max_q)
        assert got[2] == px.XMIX_ERR_KV_SPAN, (cu, kv_len)
        rows = [slice(0, 2), slice(2, 5), slice(5, 6)]
        for r in range(3):
            if r in dead:
                assert (got[0][rows[r]] == 9).all() and (got[1][:, rows[r]] == 9).all()
            else:
                check_attention((got[0][rows[r]], got[1][:, rows[r]]),
                                [x[rows[r]] if i in (0, 2) else x[:, rows[r]] for i, x in enumerate(reference(base))],
                                64)
    assert good[2] == 0


@pytest.mark.parametrize("n", [1, 3, 100])
def test_missing_pages_are_left_out(px, n):
    b = batch(px, 18, [n, 1], [200, 60], 4, 2, 64, 16)
    for bad in (-1, 1 << 30, b["cache"].k.shape[0]):
        b["cache"].pages[0, 2] = bad
        got = attend(px, b)
        assert got[2] == px.XMIX_ERR_KV_PAGE
        check_attention(got, reference(b), 64)
    b["cache"].pages[0, :] = -1
    got = attend(px, b)
    assert got[2] == px.XMIX_ERR_KV_PAGE
    check_attention(got, reference(b), 64)
    assert (got[0][:n] == 0).all()


@pytest.mark.parametrize("stored", [BF, E4])
def test_offsets_past_32_bits(px, stored):
    """Pages more than 2^32 bytes (and 2^31 values) into the cache."""
    n_kv, ps, hd = 8, 64, 128
    n_pages = (1 << 31) // (n_kv * ps * hd) + 600 if stored == BF else (1 << 32) // (n_kv * ps * hd) + 600
    k, v = [torch.zeros(n_pages, n_kv, ps, hd, dtype=stored, device="cuda") for _ in "kv"]
    used = torch.arange(n_pages - 8, n_pages, device="cuda")
    g = gpu_generator(19)
    for x in (k, v):
        x.view(torch.uint8)[used] = torch.randn(8, n_kv, ps, hd, generator=g, device="cuda").to(stored).view(torch.uint8)
    table = used.to(torch.int32).view(2, 4)
    cache = px.KvCache(k, v, table)
    q = torch.randn(3, 16, hd, generator=g, device="cuda").to(BF)
    b = dict(cache=cache, q=q, cu=[0, 1, 3], kv_len=[250, 131], T=3, max_q=2, scale=hd ** -0.5, window=0)
    got = attend(px, b)
    small = px.KvCache(k[n_pages - 8:], v[n_pages - 8:], i32(np.arange(8).reshape(2, 4)))
    want = attend(px, dict(b, cache=small))
    assert same(got[0], want[0]) and same(got[1], want[1])
    check_attention(want, reference(dict(b, cache=small)), hd)
    x = torch.randn(2, n_kv, hd, generator=g, device="cuda").to(BF)
    px.xmix_kv_append(x, x, i32([0, 1]), i32([250, 131]), None, cache, word())
    assert torch.equal(cache.k[n_pages - 5, :, 58].float(), x[0].to(stored).float())
    assert torch.equal(cache.v[n_pages - 2, :, 3].float(), x[1].to(stored).float())


def test_calls_on_streams_with_workspaces_of_their_own(px):
    """Two calls that overlap."""
    a, b = batch(px, 20, [1] * 8, [3000] * 8, 8, 2, 128, 16), batch(px, 21, [300], [900], 8, 2, 64, 16)
    want = [attend(px, x) for x in (a, b)]
    streams, outs = [torch.cuda.Stream(), torch.cuda.Stream()], []
    torch.cuda.synchronize()
    for _ in range(5):
        for x, s in zip((a, b), streams):
            with torch.cuda.stream(s):
                out, z = torch.zeros_like(x["q"]), torch.zeros((8, x["T"]), device="cuda")
                ws = torch.empty(px.paged_attention_workspace(x["T"], 8, x["max_q"], x["cache"]),
                                 dtype=torch.uint8, device="cuda")
                px.xmix_paged_attention(x["q"], i32(x["cu"]), i32(x["kv_len"]), x["cache"], x["scale"], 0,
                                        x["max_q"], out, z, word(), ws)
                outs.append((out, z))
    torch.cuda.synchronize()
    for i, (out, z) in enumerate(outs):
        assert same(out, want[i % 2][0]) and same(z, want[i % 2][1])


# --------------------------------------------------------------- the binding

def test_binding_refusals(px):
    b = batch(px, 22, [1, 2], [40, 50], 4, 2, 64, 16)
    c, q, z = b["cache"], b["q"], torch.zeros(4, 3, device="cuda")
    cu, kv, err, out = i32(b["cu"]), i32(b["kv_len"]), word(), torch.zeros_like(b["q"])
    ws = torch.zeros(max(px.paged_attention_workspace(3, 4, 2, c), 1), dtype=torch.uint8, device="cuda")
    args = dict(q=q, cu_seqlens=cu, kv_len=kv, cache=c, scale=0.1, window=0, max_q=2, out=out, lse_out=z,
                err_word=err, ws=ws)
    px.xmix_paged_attention(**args)
    for kw, e in [(dict(q=q.float()), AssertionError), (dict(q=q.cpu()), ValueError), (dict(q=q[:, :3]), AssertionError),
                  (dict(q=q[:2]), AssertionError), (dict(q=q.transpose(1, 2)), ValueError), (dict(q=q[..., :32]), ValueError),
                  (dict(cu_seqlens=cu[:2]), AssertionError), (dict(cu_seqlens=cu.long()), AssertionError),
                  (dict(kv_len=kv[:1]), AssertionError), (dict(kv_len=kv.float()), AssertionError),
                  (dict(cache=None), AttributeError), (dict(cache=px.Ring(4, 32)), (TypeError, AttributeError)),
                  (dict(scale=-1.0), px.XmixError), (dict(scale="x"), TypeError), (dict(window=-1), px.XmixError),
                  (dict(max_q=0), px.XmixError), (dict(out=out[:, :, :32]), ValueError),
                  (dict(out=torch.zeros(4, 4, 64, dtype=BF, device="cuda")), AssertionError),
                  (dict(out=out[:1].expand(3, 4, 64)), px.XmixError), (dict(lse_out=z.t()), ValueError),
                  (dict(lse_out=torch.zeros(3, 4, device="cuda")), AssertionError), (dict(err_word=None), px.XmixError)]:
        with pytest.raises(e):
            px.xmix_paged_attention(**dict(args, **kw))
    x = torch.zeros(3, 2, 64, dtype=BF, device="cuda")
    args = dict(k=x, v=x, req_of_token=i32([0, 0, 1]), pos_of_token=i32([1, 2, 3]), rope=None, cache=c, err_word=err)
    px.xmix_kv_append(**args)
    for kw, e in [(dict(k=x.float()), AssertionError), (dict(v=x[:2]), AssertionError), (dict(k=x.half()), TypeError),
                  (dict(k=x[:, :1], v=x[:, :1]), AssertionError), (dict(req_of_token=i32([0, 1])), AssertionError),
                  (dict(pos_of_token=i32([1, 2])), AssertionError), (dict(err_word=None), px.XmixError),
                  (dict(rope=c), TypeError), (dict(rope=px.Rope(frequencies(128).cuda())), px.XmixError)]:
        with pytest.raises(e):
            px.xmix_kv_append(**dict(args, **kw))
    w = torch.ones(64, dtype=BF, device="cuda")
    args = dict(q=q, k=x, pos_of_token=i32([0, 1, 2]), q_weight=w, k_weight=w, eps=1e-6, rope=None,
                q_out=out, k_out=torch.zeros_like(x))
    px.xmix_qk_norm_rope(**args)
    for kw, e in [(dict(k=x.float()), AssertionError), (dict(q_weight=w[:32]), AssertionError),
                  (dict(k_weight=w.float()), AssertionError), (dict(k=None), px.XmixError), (dict(k_out=None), px.XmixError),
                  (dict(eps=-1.0), px.XmixError), (dict(pos_of_token=i32([0, 1])), AssertionError),
                  (dict(q_out=out[:2]), AssertionError), (dict(q=q.double()), TypeError)]:
        with pytest.raises(e):
            px.xmix_qk_norm_rope(**dict(args, **kw))
    torch.cuda.synchronize()
