"""Pages behind a window: a cache that gives them away and marks their entries gets no
error, and a page with one key that some token sees still sets it."""
import numpy as np
import pytest
import torch

from test_gpu_attend import SPANS, attend, batch, check_attention, reference, same

pytestmark = pytest.mark.gpu
BF, E4 = torch.bfloat16, torch.float8_e4m3fn

CASES = dict(SPANS, far=([1, 2, 1], [500, 333, 64]), cut=([1], [3001]), prompt=([200], [777]))


@pytest.fixture(scope="module")
def px():
    import paper_2607_22595_amd as m
    return m


def first_seen(n, total, window):
    """The first key that some token of a span sees."""
    return max(0, total - n - window + 1)


@pytest.mark.parametrize("hd,n_q,n_kv,ps,stored", [(64, 8, 2, 16, BF), (64, 8, 2, 32, E4), (128, 20, 1, 16, E4),
                                                   (256, 4, 2, 32, BF)])
@pytest.mark.parametrize("window", [1, 20, 33, 49, 130])
@pytest.mark.parametrize("spans", ["decode", "drafts", "chunk_cached", "mixed", "no_keys", "far", "cut", "prompt"])
def test_pages_behind_the_window(px, spans, window, hd, n_q, n_kv, ps, stored):
    n, total = CASES[spans]
    b = dict(batch(px, window, n, total, n_q, n_kv, hd, ps, stored), window=window)
    before = attend(px, b)
    assert before[2] == 0
    n_pages, table = b["cache"].k.shape[0], b["cache"].pages.cpu().numpy().copy()
    for bad in (-1, n_pages, 2 ** 31 - 1):
        t = table.copy()
        for r, (a, c) in enumerate(zip(n, total)):
            t[r, :first_seen(a, c, window) // ps] = bad
        b["cache"].pages.copy_(torch.as_tensor(t))
        got = attend(px, b)
        assert got[2] == 0, bad
        assert same(got[0], before[0]) and same(got[1], before[1])
    # one more is a page that somebody needs: the first seen, and the last
    for which in (0, 1):
        t = table.copy()
        some = False
        for r, (a, c) in enumerate(zip(n, total)):
            if a and c:
                t[r, first_seen(a, c, window) // ps if which == 0 else (c - 1) // ps] = -1
                some = True
        b["cache"].pages.copy_(torch.as_tensor(t))
        got = attend(px, b)
        assert some and got[2] == px.XMIX_ERR_KV_PAGE
        if ps == 16 and hd == 64:
            check_attention(got, reference(b), hd)
