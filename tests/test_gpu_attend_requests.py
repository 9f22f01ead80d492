"""Batches of more requests than the planning workgroup has threads, up to the limit:
most of them with a token or none, in every form of the plan."""
import numpy as np
import pytest
import torch

from test_gpu_attend import attend, batch, check_attention, reference, same

pytestmark = pytest.mark.gpu
BF, E4 = torch.bfloat16, torch.float8_e4m3fn


@pytest.fixture(scope="module")
def px():
    import paper_2607_22595_amd as m
    return m


def spans(R, kind):
    """Single tokens; a few rows each, up to four tiles; prompts and chunks of many tiles,
    in a launch that is long enough for the queue.  Empty spans between them, at both
    ends and in long runs."""
    rng = np.random.default_rng(R)
    n = rng.choice([0, 1], R, p=[0.6, 0.4])
    total = n + rng.integers(0, 90, R)
    some = rng.permutation(R)
    if kind == "tiles":
        for r in some[:30]:
            n[r] = rng.integers(2, 61)
            total[r] = n[r] + rng.integers(0, 150)
    if kind == "queue":
        for r in some[:40]:
            n[r] = total[r] = rng.integers(100, 330)
        for r in some[40:44]:
            n[r] = rng.integers(66, 200)
            total[r] = n[r] + rng.integers(500, 1500)
        n[some[44:60]] = total[some[44:60]] = 3
    total[some[60:70]] = 0                      # rows without a key, and requests without either
    n[R // 3:R // 3 + R // 8] = 0
    n[:2], n[-3:] = 0, 0
    n[-1], total[-1] = 1, 77                    # the last request has a row
    return n.tolist(), total.tolist()


@pytest.mark.parametrize("kind,n_q,n_kv,hd,stored", [("rows", 4, 2, 64, BF), ("rows", 8, 1, 128, E4),
                                                     ("tiles", 8, 1, 64, BF), ("queue", 16, 2, 64, BF),
                                                     ("queue", 32, 4, 64, E4), ("queue", 8, 2, 256, BF)])
@pytest.mark.parametrize("R", [1024, 1025, 2049, 4095, 4096])
def test_many_requests(px, R, kind, n_q, n_kv, hd, stored):
    n, total = spans(R, kind)
    b = batch(px, R + hd, n, total, n_q, n_kv, hd, 16, stored, pad=3)
    got = attend(px, b)
    assert got[2] == 0
    check_attention(got, reference(b), hd)
    again = attend(px, b)
    assert same(got[0], again[0]) and same(got[1], again[1])


@pytest.mark.parametrize("kind,n_q,n_kv", [("rows", 4, 2), ("tiles", 8, 1), ("queue", 16, 2)])
def test_a_bad_request_among_many(px, kind, n_q, n_kv):
    """Behind the threads' first requests; the others are computed."""
    n, total = spans(4096, kind)
    b = batch(px, 5, n, total, n_q, n_kv, 64, 16)
    ref = reference(b)
    live = [r for r in range(1100, 4096) if n[r]]
    for r, bad in ((live[0], -1), (live[-1], b["cache"].pages.shape[1] * 16 + 1), (live[len(live) // 2], 2 ** 31 - 1)):
        kv_len = np.array(total)
        kv_len[r] = bad
        got = attend(px, b, kv_len=kv_len)
        assert got[2] == px.XMIX_ERR_KV_SPAN
        lo, hi = int(b["cu"][r]), int(b["cu"][r + 1])
        assert bool((got[0][lo:hi] == 9).all()) and bool((got[1][:, lo:hi] == 9).all())
        for rows in (slice(0, lo), slice(hi, b["T"])):
            check_attention(got, ref, 64, rows=rows)
