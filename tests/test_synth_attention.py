"""Workloads with an attention: a request's tokens are the rows of its span."""
import numpy as np
import pytest

import synth


def small(**kw):
    return synth.make("c2", d=64, T=12, n_layers=1, **kw)


def test_tokens_that_are_not_in_their_span_are_refused():
    """Positions are counted from a span's first row: a row of another request would be
    given a wrong one, below zero even, and its keys another request's slots."""
    for req in (np.arange(12)[::-1], np.r_[0, 0, np.arange(2, 12)], np.r_[np.arange(11), 40]):
        wl = small()
        wl.req = req.astype(np.int32)
        with pytest.raises(ValueError, match="span"):
            synth.with_attention(wl, 4, 2)
        assert wl.cu_seqlens is None and wl.layers[0].attention is None
    wl = synth.make("c4", d=64, T=40, R=3, len_lo=3, len_hi=20, m=64, k=4)
    wl.req = np.roll(wl.req, 1)
    with pytest.raises(ValueError, match="span"):
        synth.with_attention(wl, 4, 2)


def test_padding_and_spans_are_taken():
    wl = small()
    wl.T_valid = 9
    wl.req[9:] = 3        # past the valid tokens anything may stand
    wl.req[4] = -1        # and a token of no request within them
    synth.with_attention(wl, 4, 2)
    assert wl.cu_seqlens.tolist() == list(range(10)) + [9] * 3
    wl = synth.make("c4", d=64, T=40, R=3, len_lo=3, len_hi=20, m=64, k=4)
    cu = wl.cu_seqlens.copy()
    synth.with_attention(wl, 4, 2)
    assert np.array_equal(wl.cu_seqlens, cu)
