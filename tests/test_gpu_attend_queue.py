"""Launches long enough that the short units are queued, not dealt: prompts from their
first token on, alone and among other requests, the same bits whoever takes a unit."""
import numpy as np
import pytest
import torch

from test_gpu_attend import attend, batch, check_attention, i32, reference, same

pytestmark = pytest.mark.gpu
BF, E4 = torch.bfloat16, torch.float8_e4m3fn


@pytest.fixture(scope="module")
def px():
    import paper_2607_22595_amd as m
    return m


def prompts(kind):
    rng = np.random.default_rng(7)
    n = [int(x) for x in rng.integers(150, 420, 18)]
    total = list(n)
    if kind == "all_short":        # every tile has few blocks
        n = total = [int(x) for x in rng.integers(60, 200, 40)]
    if kind == "among_others":     # single tokens, a chunk over cached keys, empty requests
        n[3:3], total[3:3] = [1, 0, 1, 90], [700, 5, 3, 1200]
        n[12:12], total[12:12] = [0, 1, 2, 3], [0, 1, 999, 3]
    if kind == "one":
        n = total = [2600]
    return n, total


@pytest.mark.parametrize("stored,window", [(BF, 0), (E4, 0), (BF, 130)])
@pytest.mark.parametrize("kind,n_q,n_kv,hd", [("prompts", 32, 4, 64), ("among_others", 32, 4, 64),
                                              ("all_short", 32, 8, 64), ("one", 16, 8, 64),
                                              ("prompts", 32, 4, 128), ("prompts", 16, 2, 256)])
def test_queued_units(px, kind, n_q, n_kv, hd, stored, window):
    n, total = prompts(kind)
    b = batch(px, hd + len(n), n, total, n_q, n_kv, hd, 32, stored, pad=5)
    b["window"] = window
    got = attend(px, b)
    assert got[2] == 0
    check_attention(got, reference(b), hd)
    for _ in range(3):
        again = attend(px, b)
        assert same(got[0], again[0]) and torch.equal(got[1], again[1])


def test_a_captured_long_launch(px):
    """Replays, between them other lengths and a workspace that something else has used."""
    n, total = prompts("among_others")
    b = batch(px, 3, n, total, 32, 4, 64, 32)
    cu, ln = i32(b["cu"]), i32(b["kv_len"])
    out, err = torch.zeros_like(b["q"]), i32([0])
    ws = torch.full((px.paged_attention_workspace(b["T"], 32, b["max_q"], b["cache"]),), 0xEE,
                    dtype=torch.uint8, device="cuda")

    def call():
        px.xmix_paged_attention(b["q"], cu, ln, b["cache"], b["scale"], 0, b["max_q"], out, None, err, ws)

    call()
    torch.cuda.synchronize()
    full = out.clone()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    few = cu.clone().clamp_(max=int(b["cu"][4]))     # the first requests alone: a short launch
    for rep in range(4):
        ws.fill_(0x33 + rep)
        out.fill_(0.0)
        keep = cu.clone()
        cu.copy_(few)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert bool((out[int(b["cu"][4]):] == 0).all())
        cu.copy_(keep)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert same(out, full) and int(err.item()) == 0
