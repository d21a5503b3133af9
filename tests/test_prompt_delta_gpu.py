"""How close dq comes to its rounding at d 128 where an order mask leaves rows with
2,049 to 4,096 keys to see."""
import math

import pytest
import torch

import paper_2502_21079_amd as ad
from _prompt_ref import reference
from test_prompt_edges_gpu import off_by
from test_prompt_gpu import BF, HF, make, table_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dt", [BF, HF])
@pytest.mark.parametrize("H,Lq,Lk,offset", [(12, 2100, 2100, 0), (12, 3000, 3000, 0), (12, 4095, 4095, 0),
                                            (12, 1100, 4000, 2500), (110, 5, 4095, "end"),
                                            (110, 5, 4096, 4091), (100, 130, 3500, "end")])
def test_dq_of_rows_that_see_many_keys(H, Lq, Lk, offset, dt):
    """The last rows, which see every key: the error of a delta from the rounded output
    grows with the keys, dS's rounding and the final one do not."""
    q, k, v, g = make(1, H, 1, Lq, Lk, 128, dt, seed=16)
    v = v + 0.5
    table = table_of(32, H, dt)
    kw = dict(causal=True, bidirectional=False, q_offset=offset)
    out, lse = ad.rel_bias_attn(q, k, v, table, **kw)
    dq = ad.rel_bias_attn_bwd(g, q, k, v, table, out, lse, **kw)[0]
    h, rows = (slice(1, 2), slice(Lq - 300, Lq)) if Lq > 300 else (slice(1, 31), slice(0, Lq))
    first = (Lk - Lq if offset == "end" else offset) + rows.start
    ref = reference(q[:, h, rows], k, v, dout=g[:, h, rows], table=table[:, h], causal=True, bidirectional=False,
                    q_offset=first)["dq"][0]
    assert off_by(dq[:, h, rows], ref) < 1.1 * math.sqrt(2) * off_by(ref.to(dt), ref)


@pytest.mark.parametrize("offset", [0, 2500, "end"])
def test_a_workspace_of_the_named_size_serves_every_offset(offset):
    """Sizes are asked for without an offset."""
    q, k, v, g = make(1, 110, 1, 5, 4095, 128, BF, seed=17)
    table = table_of(32, 110, BF)
    kw = dict(causal=True, bidirectional=False)
    out, lse = ad.rel_bias_attn(q, k, v, table, q_offset=offset, **kw)
    ws = torch.empty(ad.rel_bias_attn_bwd_workspace(q.shape, k.shape, 32, **kw), dtype=torch.uint8, device="cuda")
    want = ad.rel_bias_attn_bwd(g, q, k, v, table, out, lse, q_offset=offset, **kw)
    got = ad.rel_bias_attn_bwd(g, q, k, v, table, out, lse, q_offset=offset, workspace=ws, **kw)
    for x, y in zip(got, want):
        assert torch.equal(x, y)
