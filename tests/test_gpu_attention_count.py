"""The device count of valid tokens in the attention: rows at or past it are left as
they are, what lies before them in the same span keeps its position and its result."""
import numpy as np
import pytest
import torch

import synth
from test_gpu_attend import SPANS, batch, check_attention, clean, i32, poison, reference, same, word

pytestmark = pytest.mark.gpu
BF, E4 = torch.bfloat16, torch.float8_e4m3fn

CASES = dict(SPANS, long=([300, 1, 0, 700, 2], [300, 90, 4, 1500, 2]),
             queued=([1] + [260] * 18 + [3], [70] + [260] * 18 + [200]))


@pytest.fixture(scope="module")
def px():
    import paper_2607_22595_amd as m
    return m


def call(px, b, count, out, z, err, ws):
    px.xmix_paged_attention(b["q"], b["cu_"], b["len_"], b["cache"], b["scale"], b["window"], b["max_q"], out, z,
                            err, ws, T_valid=count)


def buffers(px, b):
    n_q = b["q"].shape[1]
    b["cu_"], b["len_"] = i32(b["cu"]), i32(b["kv_len"])
    ws = torch.full((px.paged_attention_workspace(b["T"], n_q, b["max_q"], b["cache"]),), 0xA5, dtype=torch.uint8,
                    device="cuda")
    return torch.empty_like(b["q"]), torch.empty((n_q, b["T"]), device="cuda"), word(), ws


def counts(cu, T):
    """Between spans, inside of them, none, all, and what is outside of [0, T]."""
    inside = [int(c) + 1 for c in cu[:-1]] + [int(c) - 1 for c in cu[1:]]
    return sorted({c for c in [0, int(cu[1]), int(cu[-1]) // 2, T, T + 9, 2 ** 31 - 1, -1, -2 ** 31] + inside})


@pytest.mark.parametrize("window", [0, 33])
@pytest.mark.parametrize("hd,n_q,n_kv,stored", [(64, 8, 2, BF), (128, 4, 1, E4), (256, 6, 2, BF)])
@pytest.mark.parametrize("spans", ["one", "decode_gaps", "drafts", "chunk_cached", "mixed", "no_keys", "long"])
def test_rows_past_the_count(px, spans, hd, n_q, n_kv, stored, window):
    n, total = CASES[spans]
    b = dict(batch(px, 40 + window, n, total, n_q, n_kv, hd, 16, stored, pad=2), window=window)
    ref = reference(b)
    out, z, err, ws = buffers(px, b)
    for count in counts(b["cu"], b["T"]):
        out.fill_(9.0), z.fill_(9.0)
        call(px, b, i32([count]), out, z, err, ws)
        live = min(max(count, 0), b["T"])
        assert bool((out[live:] == 9).all()) and bool((z[:, live:] == 9).all()), count
        check_attention((out, z), ref, hd, rows=slice(0, live))
    assert err.item() == 0


@pytest.mark.parametrize("spans", ["drafts", "chunk_cached", "long", "queued"])
def test_what_lies_past_the_count_is_not_read(px, spans):
    """NaN and infinities in the queries, keys and values of the tokens left out, and
    no pages for those of them that have pages of their own."""
    n, total = CASES[spans]
    b = batch(px, 51, n, total, 32, 4, 64, 16)
    r = int(np.argmax(np.cumsum(n) > sum(n) // 2))       # the request that is cut
    count = int(b["cu"][r]) + max(n[r] // 2, 1)
    kept = [min(a, max(0, count - int(c))) for a, c in zip(n, b["cu"])]
    keys = [t - (a - k) if k else 0 for t, a, k in zip(total, n, kept)]
    poison(b, {i: range(k) for i, k in enumerate(keys)})
    b["q"][count:] = float("nan")
    table = b["cache"].pages.cpu().numpy()
    for i, k in enumerate(keys):
        table[i, -(-k // 16):] = -7
    b["cache"].pages.copy_(torch.as_tensor(table))
    out, z, err, ws = buffers(px, b)
    out.fill_(9.0), z.fill_(9.0)
    call(px, b, i32([count]), out, z, err, ws)
    assert err.item() == 0
    assert bool((out[count:] == 9).all()) and bool((z[:, count:] == 9).all())
    cut = dict(b, cache=clean(b), cu=np.minimum(b["cu"], count),
               kv_len=np.array(keys))
    cut["q"] = torch.nan_to_num(b["q"].float(), 0.0).to(BF)
    check_attention((out, z), reference(cut), 64, rows=slice(0, count))


def test_a_captured_call_follows_the_count(px):
    n, total = CASES["queued"]
    b = batch(px, 52, n, total, 32, 4, 64, 32)
    out, z, err, ws = buffers(px, b)
    count = i32([b["T"]])
    call(px, b, count, out, z, err, ws)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call(px, b, count, out, z, err, ws)
    want = torch.empty_like(out)
    for rep, c in enumerate((sum(n), 700, 1, 0, 3000, sum(n))):
        count.fill_(c)
        want.fill_(9.0), out.fill_(9.0)
        call(px, b, i32([c]), want, z, err, ws)
        torch.cuda.synchronize()
        ws.fill_(0x21 + rep)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert same(out, want) and bool((out[c:] == 9).all()) and err.item() == 0


@pytest.mark.parametrize("make", ["c2", "c4"])
def test_a_step_whose_count_alone_is_lowered(px, make):
    """The captured step, the spans as they were: rows past the count keep what they hold."""
    from paper_2607_22595_amd.hookstep import HookStep
    if make == "c2":
        wl = synth.with_attention(synth.make("c2", d=512, T=48, n_layers=2), 8, 2, ctx_hi=100)
    else:
        wl = synth.make("c4", d=512, T=400, R=5, len_lo=3, len_hi=200, m=1024, k=16)
        wl = synth.with_attention(wl, 8, 2, ctx_lo=0, ctx_hi=90, page_size=32)
    step = HookStep(wl)
    step.run()
    torch.cuda.synchronize()
    full = [lay.attention.q_rot.clone() for lay in step.layers]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step.run()
    for count in (wl.T_max // 3, 1, wl.T_max - 2, 0, wl.T_max):
        step.T_valid.fill_(count)
        for lay in step.layers:
            lay.h.fill_(3.0)
            lay.attention.q_rot[count:] = float("nan")
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        for lay, q in zip(step.layers, full):
            assert bool((lay.h[count:] == 3).all())
            assert bool(torch.isfinite(lay.h[:count].float()).all())
            assert not bool((lay.h[:count] == 3).all(-1).any())
            assert same(lay.attention.q_rot[:count], q[:count])
        assert step.err.item() == 0
