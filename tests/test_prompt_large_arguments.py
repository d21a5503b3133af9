"""CPU checks that numbers past the C structures' 32 bits are refused, not wrapped."""
import pytest

import paper_2502_21079_amd as ad
from paper_2502_21079_amd.prompt import _bias_ref


@pytest.mark.parametrize("offset", [1 << 28, -(1 << 28), 1 << 32, (1 << 32) + 7, -(1 << 32), 1 << 70])
def test_query_offsets(offset):
    with pytest.raises(ad.AdaspaError):
        _bias_ref(32, 128, True, False, offset, True)


@pytest.mark.parametrize("offset", [0, -5, (1 << 28) - 1, "end"])
def test_query_offsets_that_fit(offset):
    r = _bias_ref(32, 128, True, True, offset, True)._obj
    assert (r.q_offset, r.queries_at_end) == ((0, 1) if offset == "end" else (offset, 0))


@pytest.mark.parametrize("q,k", [((1, 1, (1 << 32) + 5, 64), (1, 1, 9, 64)), ((1, 1, 5, 64), (1, 1, (1 << 32) + 9, 64)),
                                 (((1 << 32) + 1, 1, 5, 64), ((1 << 32) + 1, 1, 9, 64)),
                                 ((1, 1, 5, (1 << 32) + 64), (1, 1, 9, (1 << 32) + 64))])
def test_sizes(q, k):
    for size in (ad.cross_attn_workspace, ad.cross_attn_bwd_workspace):
        with pytest.raises(ad.AdaspaError):
            size(q, k)
    with pytest.raises(ad.AdaspaError):
        ad.rel_bias_attn_workspace(q, k, 32)
