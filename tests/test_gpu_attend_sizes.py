"""Sizes of the attention's arguments: what is shorter than the kernels read is refused
before a launch, by the binding itself; key counts up to the last one below 2^31, and
scales at the ends of fp32."""
import numpy as np
import pytest
import torch

from test_gpu_attend import BF, E4, SPANS, attend, batch, check_attention, i32, reference, word

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def px():
    import paper_2607_22595_amd as m
    return m


@pytest.mark.parametrize("short", [0, 1, 2, 4])
def test_span_starts_of_another_length(px, short):
    """Three requests have four of them."""
    b = batch(px, 60, [1, 2, 1], [40, 50, 3], 4, 2, 64, 16)
    cu = torch.zeros(short + (short > 3), dtype=torch.int32, device="cuda")
    ws = torch.zeros(px.paged_attention_workspace(4, 4, 2, b["cache"]), dtype=torch.uint8, device="cuda")
    out = torch.zeros_like(b["q"])
    with pytest.raises(AssertionError, match="wrong size"):
        px.xmix_paged_attention(b["q"], cu, i32(b["kv_len"]), b["cache"], 0.1, 0, 2, out, None, word(), ws)
    with pytest.raises(AssertionError, match="wrong size"):
        px._paged_attention(b["q"], cu, i32(b["kv_len"]), b["cache"], 3, 4, 64, 0.1, 0, 2, out, None, word(), ws,
                            None, None)
    torch.cuda.synchronize()


@pytest.mark.parametrize("stored", [BF, E4])
@pytest.mark.parametrize("n,hd,n_q,n_kv", [(1, 128, 4, 1), (5, 64, 8, 2), (200, 128, 4, 1), (200, 64, 8, 2), (3, 256, 2, 1)])
def test_key_counts_next_to_two_to_the_31(px, n, hd, n_q, n_kv, stored):
    """The last keys that a table of pages of 16 can hold, in a window: the same as those
    of a short request with the same last pages."""
    last, window = 80, 1000
    b = dict(batch(px, 61, [n], [last * 16], n_q, n_kv, hd, 16, stored), window=window)
    ref = reference(b)
    c = b["cache"]
    max_pages = 2 ** 27 - 1
    table = torch.full((1, max_pages), -1, dtype=torch.int32, device="cuda")
    table[:, -last:] = c.pages
    far = px.KvCache(c.k, c.v, table, c.k_scale, c.v_scale)
    got = attend(px, dict(b, cache=far, kv_len=np.array([max_pages * 16])))
    assert got[2] == 0
    check_attention(got, ref, hd)
    x = torch.randn(1, n_kv, hd, device="cuda").to(BF)
    err, pos = word(), max_pages * 16 - 1
    px.xmix_kv_append(x, x, i32([0]), i32([pos]), None, far, err)
    at = int(table[0, -1])
    scale = 1.0 if c.v_scale is None else c.v_scale[:, None]
    assert torch.equal(c.v[at, :, 15].float(), (x[0].float() / scale).to(stored).float()) and err.item() == 0


@pytest.mark.parametrize("spans", ["decode", "drafts", "chunk_cached", "mixed"])
@pytest.mark.parametrize("stored,k_scale,scale", [(E4, 1e-20, 1e-30), (BF, None, 2.0 ** -149), (BF, None, 1e-30),
                                                  (E4, 1e-38, 1.0), (E4, 1e30, 1e20), (BF, None, 3e38)])
def test_scales_at_the_ends_of_fp32(px, spans, stored, k_scale, scale):
    """Products far below 1: every key that is seen weighs the same.  Past the other end
    only queries of zeros have scores that are numbers."""
    n, total = SPANS[spans]
    b = dict(batch(px, 62, n, total, 8, 2, 64, 16, stored), scale=scale)
    if k_scale is not None:
        b["cache"].k_scale.fill_(k_scale)
    if scale > 1:
        b["q"].zero_()
    got = attend(px, b)
    assert got[2] == 0
    check_attention(got, reference(b), 64)


@pytest.mark.parametrize("kw", [dict(window=2 ** 32 + 5), dict(window=2 ** 31), dict(max_q=2 ** 32 + 2)])
def test_a_window_and_a_bound_of_more_than_32_bits(px, kw):
    """A window of 2^32 + 5 keys is not one of 5."""
    b = batch(px, 63, [1, 2], [40, 50], 4, 2, 64, 16)
    ws = torch.zeros(px.paged_attention_workspace(3, 4, 2, b["cache"]), dtype=torch.uint8, device="cuda")
    args = dict(dict(scale=0.1, window=0, max_q=2), **kw)
    with pytest.raises(OverflowError):
        px.xmix_paged_attention(b["q"], i32(b["cu"]), i32(b["kv_len"]), b["cache"], out=torch.zeros_like(b["q"]),
                                lse_out=None, err_word=word(), ws=ws, **args)


@pytest.mark.parametrize("count", [0, 2])
def test_a_count_of_valid_tokens_is_one_number(px, count):
    """An empty tensor has no address: it would stand for every row."""
    b = batch(px, 64, [1, 2], [40, 50], 4, 2, 64, 16)
    c, live = b["cache"], torch.ones(count, dtype=torch.int32, device="cuda")
    x = torch.zeros(3, 2, 64, dtype=BF, device="cuda")
    out = torch.full_like(b["q"], 9.0)
    ws = torch.zeros(px.paged_attention_workspace(3, 4, 2, c), dtype=torch.uint8, device="cuda")
    before = c.k.clone()
    with pytest.raises(AssertionError, match="wrong size"):
        px.xmix_qk_norm_rope(b["q"], None, i32([0, 1, 2]), None, None, 0.0, None, out, None, T_valid=live)
    with pytest.raises(AssertionError, match="wrong size"):
        px.xmix_kv_append(x, x, i32([0, 1, 1]), i32([0, 1, 2]), None, c, word(), T_valid=live)
    with pytest.raises(AssertionError, match="wrong size"):
        px.xmix_paged_attention(b["q"], i32(b["cu"]), i32(b["kv_len"]), c, 0.1, 0, 2, out, None, word(), ws,
                                T_valid=live)
    torch.cuda.synchronize()
    assert bool((out == 9).all()) and torch.equal(c.k, before)
