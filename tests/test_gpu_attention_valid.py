"""A captured step with attention replayed with fewer valid tokens: what the device
count leaves out is neither normed, nor appended, nor attended to."""
import numpy as np
import pytest
import torch

import synth

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("norm", [True, False])
def test_fewer_valid_tokens_in_a_replay(norm):
    from paper_2607_22595_amd.hookstep import HookStep
    wl = synth.with_attention(synth.make("c2", d=512, T=48, n_layers=2), 8, 2, ctx_hi=100, norm=norm)
    step = HookStep(wl)
    step.run()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step.run()
    n = 20
    pos = step.pos.cpu().numpy()
    for rep in range(3):
        step.T_valid.fill_(n)
        step.cu.copy_(torch.arange(len(step.cu), dtype=torch.int32).clamp(max=n))
        for lay in step.layers:
            a = lay.attention
            lay.h.fill_(3.0)
            a.q_rot.fill_(3.0)
            a.cache.k.fill_(0.5)
            a.cache.v.fill_(0.5)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert step.err.item() == 0
        for L, lay in zip(wl.layers, step.layers):
            a, ps = lay.attention, L.attention.k_pages.shape[2]
            assert bool((lay.h[n:] == 3).all()) and bool((a.q_rot[n:] == 3).all())
            assert not bool((lay.h[:n] == 3).all(-1).any()) and not bool((a.q_rot[:n] == 3).all(-1).any())
            page = L.attention.pages[np.arange(48), pos[:48] // ps]
            at = torch.as_tensor(page).long(), torch.as_tensor(pos[:48] % ps).long()
            for cached in (a.cache.k, a.cache.v):
                rows = cached.cpu()[at[0], :, at[1]]
                assert bool((rows[n:] == 0.5).all()) and not bool((rows[:n] == 0.5).all(-1).any())
                assert int((cached != 0.5).any(-1).sum()) == n * 2
