"""Sizes of the attention's arguments: what is shorter than the kernels read is refused
before a launch, by the binding itself."""
import pytest
import torch

from test_gpu_attend import batch, i32, word

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
