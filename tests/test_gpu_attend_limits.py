"""Attention operators at the ends of what they allow: more tokens than one row of
a grid holds, batches of many kinds in one call, objects of another device."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


@pytest.fixture(scope="module")
def px():
    import paper_2607_22595_amd as m
    return m


def i32(x):
    return torch.as_tensor(np.asarray(x), dtype=torch.int32).cuda()


def same(a, b):
    return torch.equal(a.contiguous().view(torch.int16), b.contiguous().view(torch.int16))


def test_more_tokens_than_a_grid_has_in_one_dimension(px):
    """2^24 workgroups of 256 threads are 2^32 threads."""
    T, hd = 2 ** 24 + 3, 16
    x = torch.zeros(T, 1, hd, dtype=BF, device="cuda")
    x[:] = torch.arange(1, hd + 1, device="cuda").to(BF)
    pos = torch.zeros(T, dtype=torch.int32, device="cuda")
    w = torch.ones(hd, dtype=BF, device="cuda")
    few = torch.zeros(3, 1, hd, dtype=BF, device="cuda")
    px.xmix_qk_norm_rope(x[:3], None, pos[:3], w, None, 0.0, None, few, None)
    cache = px.KvCache(*[torch.zeros(2, 1, 16, hd, dtype=BF, device="cuda") for _ in "kv"], i32([[0, 1]]))
    req = torch.full((T,), -1, dtype=torch.int32, device="cuda")
    req[[0, 2 ** 20, T - 1]] = 0
    pos[[2 ** 20, T - 1]] = i32([1, 31])
    err = i32([0])
    px.xmix_kv_append(x, x, req, pos, None, cache, err)
    assert int(err.item()) == 0
    rows = torch.stack([cache.k[0, 0, 0], cache.k[0, 0, 1], cache.k[1, 0, 15]])
    assert same(rows, x[:3, 0]) and int((cache.v != 0).any(-1).sum()) == 3
    px.xmix_qk_norm_rope(x, None, pos, w, None, 0.0, None, x, None)
    assert bool((x == few[0]).all())


def test_objects_of_another_device_are_refused(px):
    hd = 64
    x = torch.zeros(1, 1, hd, dtype=BF, device="cuda")
    cache = px.KvCache(*[torch.zeros(1, 1, 16, hd, dtype=BF, device="cuda") for _ in "kv"], i32([[0]]))
    rope = px.Rope(torch.ones(hd // 2, dtype=torch.float64, device="cuda"))
    ws = torch.zeros(px.paged_attention_workspace(1, 1, 1, cache), dtype=torch.uint8, device="cuda")
    zero, one, err = i32([0]), i32([1]), i32([0])

    def norm():
        px.xmix_qk_norm_rope(x, None, zero, None, None, 0.0, rope, x, None)

    def append():
        px.xmix_kv_append(x, x, zero, zero, rope, cache, err)

    def attend():
        px.xmix_paged_attention(x, i32([0, 1]), one, cache, 1.0, 0, 1, x.clone(), None, err, ws)

    for call in (norm, append, attend):
        call()
    rope.device = torch.device("cuda", 1)
    for call in (norm, append):
        with pytest.raises(ValueError, match="device"):
            call()
    rope.device, cache.device = x.device, torch.device("cuda", 1)
    for call in (append, attend):
        with pytest.raises(ValueError, match="device"):
            call()


def soft_rows(q, k, v, scale, pos, window):
    """Rows [n, group, hd] over keys [len, hd] in 64 bits; the positions are pos."""
    s = np.einsum("ngh,lh->ngl", q, k) * scale
    j = np.arange(k.shape[0])
    see = (j[None] <= pos[:, None]) & ((window == 0) | (j[None] > pos[:, None] - window))
    s = np.where(see[:, None], s, -np.inf)
    top = np.where(see.any(1)[:, None, None], s.max(-1, keepdims=True), 0.0)
    p = np.exp(s - top)
    total = p.sum(-1, keepdims=True)
    return np.einsum("ngl,lh->ngh", p / np.where(total == 0, 1, total), v), p


@pytest.mark.parametrize("window", [0, 100])
@pytest.mark.parametrize("hd,n_kv,group", [(64, 2, 8), (128, 1, 4), (256, 2, 5), (128, 3, 16), (64, 1, 17)])
def test_rows_and_tiles_in_one_call(px, hd, n_kv, group, window):
    """A batch whose requests are row units (up to 16 rows), tiles, cut and whole ones
    of both, and empty ones in between; NaN in the pages that nobody owns."""
    n = [1, 0, 200, 2, 1, 37, 0, 1, 3, 1, 129, 1]
    ln = [1, 50, 900, 2500, 4000, 37, 9, 0, 70, 1203, 2000, 16]
    R, ps, T = len(n), 32, sum(n) + 3
    g = torch.Generator(device="cuda").manual_seed(hd + group)
    per = [-(-x // ps) for x in ln]
    pages = np.full((R, max(per)), 0, dtype=np.int32)
    at = 1
    for r, c in enumerate(per):
        pages[r, :c] = np.arange(at, at + c)[::-1]
        at += c
    k, v = [torch.randn(at, n_kv, ps, hd, generator=g, device="cuda").to(BF) for _ in "kv"]
    k[0], v[0] = float("nan"), float("nan")
    cache = px.KvCache(k, v, i32(pages))
    q = torch.randn(T, n_kv * group, hd, generator=g, device="cuda").to(BF)
    cu, err = i32(np.concatenate([[0], np.cumsum(n)])), i32([0])
    out = torch.full_like(q, 7.0)
    ws = torch.full((px.paged_attention_workspace(T, n_kv * group, 200, cache),), 0xFF, dtype=torch.uint8,
                    device="cuda")
    scale = hd ** -0.5
    px.xmix_paged_attention(q, cu, i32(ln), cache, scale, window, 200, out, None, err, ws)
    assert int(err.item()) == 0 and bool((out[sum(n):] == 7).all())
    wide = [x.float().cpu().numpy().astype(np.float64) for x in (q, k, v, out)]
    lo = 0
    for r in range(R):
        for h in range(n_kv):
            kk, vv = [x[pages[r, :per[r]], h].reshape(-1, hd)[:ln[r]] for x in wide[1:3]]
            rows = slice(lo, lo + n[r])
            heads = slice(h * group, (h + 1) * group)
            pos = ln[r] - n[r] + np.arange(n[r])
            got = wide[3][rows, heads]
            if n[r] == 0:
                continue
            if ln[r] == 0:
                assert (got == 0).all()
                continue
            ref, p = soft_rows(wide[0][rows, heads], kk, vv, scale, pos, window)
            # weights to bf16 (2^-8 of each, on sum p |v|), one rounding of the result, and
            # scores of up to 60 in fp32 (hd terms of 2^-24 each, on every weight)
            size = np.einsum("ngl,lh->ngh", p / np.maximum(p.sum(-1, keepdims=True), 1e-300), np.abs(vv))
            bound = (2.0 ** -8 + 4 * hd * 2.0 ** -24 * 60) * size + 2.0 ** -8 * np.abs(ref) + 1e-6
            assert (np.abs(got - ref) <= bound).all(), (r, h)
        lo += n[r]
    again = torch.full_like(q, 7.0)
    ws.fill_(0x5A)
    px.xmix_paged_attention(q, cu, i32(ln), cache, scale, window, 200, again, None, err, ws)
    assert same(out, again)


@pytest.mark.parametrize("dtype", [BF, torch.float32])
def test_scaled_values_are_the_rounded_quotients(px, dtype):
    """Keys and values of every exponent over scales from 2^-80 to 2^80 and ones that
    are no powers of two, to the bit (signs of zeros too)."""
    n_kv, hd, T, ps = 16, 64, 512, 16
    rng = np.random.default_rng(4)
    x = rng.normal(size=(T, n_kv, hd)) * 2.0 ** rng.integers(-20, 20, (T, n_kv, 1))
    scale = np.float32(rng.uniform(1, 2, n_kv) * 2.0 ** np.linspace(-80, 80, n_kv))
    scale[[3, 8]] = 0.0375, 1.0
    x = x * scale[:, None].astype(np.float64) * 2.0 ** rng.integers(-6, 7, (T, 1, 1))
    x[::7] = rng.normal(size=x[::7].shape) * 2.0 ** rng.integers(-120, 120, x[::7].shape)
    x[0], x[1], x[2], x[3] = 0.0, -0.0, 3e38, -1e-38
    x[4] = (rng.integers(-448, 449, (n_kv, hd)) / 16.0) * scale[:, None]  # ties among them
    k = torch.as_tensor(x).to(dtype).cuda()
    s = torch.as_tensor(scale).cuda()
    pages = torch.arange(T // ps, dtype=torch.int32, device="cuda")[None].contiguous()
    cache = px.KvCache(*[torch.zeros(T // ps, n_kv, ps, hd, device="cuda").to(torch.float8_e4m3fn) for _ in "kv"],
                       pages, s, s)
    err = i32([0])
    px.xmix_kv_append(k, k, i32(np.zeros(T)), i32(np.arange(T)), None, cache, err)
    want = (k.float().cpu() / s.cpu()[:, None]).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
    for got in (cache.k, cache.v):
        rows = got.view(torch.uint8).cpu().transpose(1, 2).reshape(T, n_kv, hd)
        assert torch.equal(rows, want)
    assert int(err.item()) == 0


def test_more_workgroups_than_a_row_of_the_grid(px):
    """Heads that take a workgroup a token, past 2^20 tokens."""
    T, n, hd = 2 ** 20 + 3, 16, 256
    x = torch.randn(1, n, hd, generator=torch.Generator().manual_seed(3)).to(BF).cuda()
    q = x.expand(T, n, hd)
    pos = torch.arange(T, dtype=torch.int32, device="cuda") % 7
    w = torch.ones(hd, dtype=BF, device="cuda")
    few, out = torch.zeros(7, n, hd, dtype=BF, device="cuda"), torch.empty(T, n, hd, dtype=BF, device="cuda")
    rope = px.Rope(1.0 / 10.0 ** torch.arange(hd // 2, dtype=torch.float64, device="cuda"))
    px.xmix_qk_norm_rope(q[:7], None, pos[:7], w, None, 1e-6, rope, few, None)
    px.xmix_qk_norm_rope(q, None, pos, w, None, 1e-6, rope, out, None)
    whole = T // 7 * 7
    assert bool((out[:whole].view(-1, 7, n, hd) == few).all()) and same(out[whole:], few[:T - whole])
    cache = px.KvCache(*[torch.zeros(2, 8, 16, hd, dtype=BF, device="cuda") for _ in "kv"], i32([[0, 1]]))
    req = torch.full((T,), -1, dtype=torch.int32, device="cuda")
    req[[1, 2 ** 20, T - 1]] = 0
    pos[[1, 2 ** 20, T - 1]] = i32([5, 6, 30])
    err = i32([0])
    px.xmix_kv_append(q[:, :8], q[:, 8:], req, pos, None, cache, err)
    for got, want in ((cache.k, x[0, :8]), (cache.v, x[0, 8:])):
        for page, slot in ((0, 5), (0, 6), (1, 14)):
            assert same(got[page, :, slot], want)
        assert int((got != 0).any(-1).sum()) == 3 * 8
    assert int(err.item()) == 0
