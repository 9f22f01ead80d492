"""The attention in front of a layer's hooks, as HookStep runs it: heads normed and
rotated, keys and values appended, attention over the cache, then the hook step on
its output.  Every stage against the oracle on the GPU's own input of that stage;
the whole step captured and replayed."""
import numpy as np
import pytest
import torch

import oracle
import synth
from parity import check_steer, torch_bits
from test_gpu_attend import check_attention, check_heads, frequencies, i32, same, wide

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def px():
    import paper_2607_22595_amd as m
    return m


def decode(norm, window=0):
    wl = synth.make("c2", d=1024, T=70, n_layers=2)
    wl.T_valid = 66
    wl.req[66:] = -1
    return synth.with_attention(wl, 16, 4, ctx_hi=300, norm=norm, window=window)


def prefill(norm, window=0):
    wl = synth.make("c4", d=512, T=400, R=5, len_lo=3, len_hi=200, m=1024, k=16)
    return synth.with_attention(wl, 8, 2, ctx_lo=0, ctx_hi=90, page_size=32, rot_dim=32, norm=norm, window=window)


def host(step, li, spec):
    """What one layer's stages should give, from the GPU's inputs of each stage."""
    a, wl = step.layers[li].attention, step.wl
    pos = step.pos.cpu().numpy()
    live = pos >= 0
    q = oracle.norm_rope(torch_bits(a.q.contiguous()), pos, spec.q_weight, spec.eps, spec.inv_freq)
    k = oracle.norm_rope(torch_bits(a.k.contiguous()), pos, spec.k_weight, spec.eps, spec.inv_freq)
    check_heads(wide(a.q_rot)[live], q[live], spec.head_dim, 2.0 ** -8)
    ps = spec.k_pages.shape[2]
    page, slot = spec.pages[wl.req[live], pos[live] // ps], pos[live] % ps
    check_heads(wide(a.cache.k)[page, :, slot], k[live], spec.head_dim, 2.0 ** -8)
    assert np.array_equal(wide(a.cache.v)[page, :, slot], wide(a.v)[live])
    return oracle.attend(torch_bits(a.q_rot), wl.cu_seqlens, step.kv_len.cpu().numpy(), wide(a.cache.k),
                         wide(a.cache.v), spec.pages, float(np.float32(spec.head_dim ** -0.5)), spec.window)


@pytest.mark.parametrize("norm", [True, False])
@pytest.mark.parametrize("make,window", [(decode, 0), (decode, 40), (prefill, 0), (prefill, 50)])
def test_attention_in_front_of_the_hooks(px, make, window, norm):
    from paper_2607_22595_amd.hookstep import HookStep
    wl = make(norm, window)
    step = HookStep(wl)
    assert "L0/norm_rope" in step.stage_names() and "L0/attention" in step.stage_names()
    step.run(only=None)
    torch.cuda.synchronize()
    assert step.err.item() == 0
    full = [lay.h.clone() for lay in step.layers]
    # the attention's own output: the same stages without the hooks
    for li, L in enumerate(wl.layers):
        step.layers[li].h.fill_(9.0)
        for name in ("norm_rope", "kv_append", "attention"):
            step.run(only=f"L{li}/{name}")
        torch.cuda.synchronize()
        n_q, hd = L.attention.n_q, L.attention.head_dim
        out = step.layers[li].attention.out.clone()
        lse = torch.full((n_q, wl.T_max), 9.0, device="cuda")
        a = step.layers[li].attention
        px.xmix_paged_attention(a.q_rot, step.cu, step.kv_len, a.cache, hd ** -0.5, window, step.max_q, a.out, lse,
                                step.err, step.attention_ws)
        assert same(out, a.out)
        check_attention((out, lse), host(step, li, L.attention), hd)
        # the hooks read and write what the attention made
        tok_mask = step.route.tok_mask.cpu().numpy().view(np.uint32)
        before = torch_bits(out.view(wl.T_max, -1))
        if L.steer:
            want = oracle.steer(before, tok_mask, wl.req, np.stack([s.v for s in L.steer]),
                                [s.bit for s in L.steer], wl.alpha)
            on = (tok_mask & sum(1 << s.bit for s in L.steer)) != 0
            live = step.pos.cpu().numpy() >= 0
            check_steer(torch_bits(full[li])[live], want[live], before[live], on[live])
        p = step.layers[li].probes[0]
        logit, _ = oracle.probe_token(before, tok_mask, np.stack([q.w for q in L.probes if q.mode == "token"]),
                                      np.array([q.b for q in L.probes if q.mode == "token"], np.float32), p.bits)
        on = (tok_mask & (1 << p.bits[0])) != 0
        got = p.logit.cpu().numpy()[0]
        assert np.allclose(got[on], logit[0, on], rtol=1e-3, atol=1e-2)


def test_step_is_captured_and_replayed(px):
    """New lengths, positions and projections between replays, each against the eager run."""
    from paper_2607_22595_amd.hookstep import HookStep
    wl = decode(True)
    step = HookStep(wl)
    step.run()
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    g = px.Graph(lambda: step.run(stream), stream)
    assert g.kernel_nodes >= 2 * 5
    gen = torch.Generator(device="cuda").manual_seed(3)
    pages = step.layers[0].attention.cache.pages.shape[1] * 16
    for trial in range(4):
        ctx = torch.randint(0, 200, (wl.R_max,), generator=gen, device="cuda", dtype=torch.int32)
        room = (step.layers[0].attention.cache.pages >= 0).sum(1).to(torch.int32) * 16
        ctx = torch.minimum(ctx, room - 1).clamp_min(0)
        assert int(ctx.max()) < pages
        n = torch.diff(step.cu)
        step.kv_len.copy_(ctx + n)
        live = step.pos >= 0
        step.pos.copy_(torch.where(live, ctx[step.req.clamp_min(0).long()], step.pos))
        for lay in step.layers:
            lay.attention.q.copy_(torch.randn(lay.attention.q.shape, generator=gen, device="cuda"))
            lay.attention.v.copy_(torch.randn(lay.attention.v.shape, generator=gen, device="cuda"))
        step.reset()
        step.run()
        torch.cuda.synchronize()
        want = [lay.h.clone() for lay in step.layers] + [lay.attention.cache.k.clone() for lay in step.layers]
        for lay in step.layers:
            lay.h.copy_(lay.h_in)
        step.attention_ws.random_(0, 256, generator=gen)
        torch.cuda.synchronize()
        g.launch()
        g.stream.synchronize()
        got = [lay.h for lay in step.layers] + [lay.attention.cache.k for lay in step.layers]
        assert all(same(x, y) for x, y in zip(got, want)), trial
        assert step.err.item() == 0
    g.close()


def test_two_graphs_share_a_workspace(px):
    """Captured calls of different sizes on one stream with one workspace."""
    from test_gpu_attend import attend, batch, word
    calls = [batch(px, 30, [1] * 20, [700] * 20, 8, 2, 128, 16), batch(px, 31, [90, 200], [300, 200], 8, 2, 128, 16)]
    want = [attend(px, c) for c in calls]
    need = max(px.paged_attention_workspace(c["T"], 8, c["max_q"], c["cache"]) for c in calls)
    ws = torch.randint(0, 256, (need,), dtype=torch.uint8, device="cuda")
    stream, graphs, outs = torch.cuda.Stream(), [], []
    for c in calls:
        out, z, cu, kv = torch.zeros_like(c["q"]), torch.zeros((8, c["T"]), device="cuda"), i32(c["cu"]), i32(c["kv_len"])
        torch.cuda.synchronize()
        keep = (cu, kv, word())
        graphs.append(px.Graph(lambda c=c, out=out, z=z, k=keep: px.xmix_paged_attention(
            c["q"], k[0], k[1], c["cache"], c["scale"], 0, c["max_q"], out, z, k[2], ws, stream), stream))
        outs.append((out, z, keep))
    for _ in range(4):
        for out, z, _ in outs:
            out.zero_(), z.zero_()
        torch.cuda.synchronize()
        for g in graphs:
            g.launch()
        stream.synchronize()
        for (out, z, _), w in zip(outs, want):
            assert same(out, w[0]) and same(z, w[1])


def test_redirecting_a_captured_cache(px):
    """A captured step pointed at another layer's pages and tables."""
    from test_gpu_attend import attend, batch, word
    a = batch(px, 33, [1, 4, 1], [50, 90, 7], 4, 2, 64, 16)
    b = batch(px, 34, [1, 4, 1], [50, 90, 7], 4, 2, 64, 16)
    want = attend(px, dict(b, q=a["q"]))
    out, z, err = torch.zeros_like(a["q"]), torch.zeros((4, 6), device="cuda"), word()
    cu, kv = i32(a["cu"]), i32(a["kv_len"])
    ws = torch.empty(px.paged_attention_workspace(6, 4, 4, a["cache"]), dtype=torch.uint8, device="cuda")
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    g = px.Graph(lambda: px.xmix_paged_attention(a["q"], cu, kv, a["cache"], a["scale"], 0, 4, out, z, err, ws, stream),
                 stream)
    for x in ("k", "v", "pages"):
        assert g.redirect(getattr(a["cache"], x), getattr(b["cache"], x)) >= 1
    g.launch()
    g.stream.synchronize()
    assert same(out, want[0]) and same(z, want[1])
