"""Edges of the prompt side's attentions on the GPU: bias tables that hide keys
with the type's lowest value or an infinity, order masks over several samples and
ranges, how close dq comes to its rounding, a second differentiation."""
import math

import pytest
import torch

import paper_2502_21079_amd as ad
from _prompt_ref import reference
from test_prompt_gpu import BF, HF, lens_of, make, mask_of, run_bias, table_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("L,D", [(90, 64), (300, 64), (100, 128), (700, 128)])
@pytest.mark.parametrize("dt,low", [(torch.float32, torch.finfo(torch.float32).min), (BF, torch.finfo(BF).min),
                                    (HF, torch.finfo(HF).min), (torch.float32, -math.inf), (BF, -1e9)])
def test_a_bucket_that_hides_keys(L, D, dt, low):
    """Keys of a bucket at the type's lowest value, far below the others, or at
    minus infinity have weight 0 and no gradient."""
    q, k, v, g = make(2, 2, 2, L, L, D, HF if dt is HF else BF, seed=4)
    table = table_of(8, 2, dt, seed=1)
    table[[1, 6], 0] = low
    run_bias(q, k, v, g, table, max_distance=40)
    out, lse = ad.rel_bias_attn(q, k, v, table, max_distance=40)
    dt_ = ad.rel_bias_attn_bwd(g, q, k, v, table, out, lse, max_distance=40)[3]
    assert (dt_[[1, 6], 0] == 0).all()


@pytest.mark.parametrize("low", [torch.finfo(torch.float32).min, -math.inf])
def test_a_table_that_hides_every_key(low):
    """Values past -2.3e38 count as minus infinity: rows of such a head are empty."""
    q, k, v, g = make(1, 2, 2, 150, 170, 64, BF)
    table = table_of(8, 2)
    table[:, 1] = low
    out, lse = ad.rel_bias_attn(q, k, v, table, max_distance=40)
    assert (out[:, 1] == 0).all() and (lse[:, 1] == -math.inf).all() and torch.isfinite(lse[:, 0]).all()
    for x in ad.rel_bias_attn_bwd(g, q, k, v, table, out, lse, max_distance=40)[:3]:
        assert (x[:, 1] == 0).all() and torch.isfinite(x).all()


@pytest.mark.parametrize("B,H,Hk", [(1, 3, 3), (8, 2, 1), (5, 4, 2)])
@pytest.mark.parametrize("Lq,Lk,offset", [(300, 300, 0), (140, 900, "end"), (700, 650, -100), (2, 400, "end")])
def test_order_masks_over_samples(B, H, Hk, Lq, Lk, offset):
    """Launches of several tiles a head, whose order goes by length: numbers of
    heads and samples that do and do not divide by the XCDs."""
    D = 128 if B == 5 else 64
    q, k, v, g = make(B, H, Hk, Lq, Lk, D, BF, "blhd", seed=7)
    run_bias(q, k, v, g, table_of(16, H), max_distance=100, bidirectional=False, causal=True, q_offset=offset,
             key_lens=lens_of(B, Lk, "some"), key_mask=mask_of(B, Lk, "some"))


def off_by(x, ref):
    return ((x.double() - ref).norm() / ref.norm()).item()


@pytest.mark.parametrize("dt", [BF, HF])
@pytest.mark.parametrize("Lq,Lk,causal", [(900, 700, False), (300, 300, True), (700, 700, True), (9000, 200, False)])
def test_dq_is_as_good_as_its_rounding(Lq, Lk, causal, dt):
    """At d 128, values with a mean of their own per channel, as in use: the
    output's rounding then weighs most.  dq's error is its final rounding, r, and
    delta's, which is that of the output: no larger than r, since the values' spread,
    which dS is made of, is three times their mean.  Together at most sqrt(2) r."""
    H = 3 if Lk > 256 or causal else 8
    q, k, v, g = make(1, H, H, Lq, Lk, 128, dt, seed=12)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(5)
    v = (v.float() + 0.3 * torch.randn(1, H, 1, 128, generator=gen, device="cuda")).to(dt)
    if causal:
        table = table_of(32, H, dt)
        kw = dict(bidirectional=False, causal=True, max_distance=500)
        out, lse = ad.rel_bias_attn(q, k, v, table, **kw)
        dq = ad.rel_bias_attn_bwd(g, q, k, v, table, out, lse, **kw)[0]
        ref = reference(q, k, v, dout=g, table=table, **kw)["dq"][0]
    else:
        out, lse = ad.cross_attn(q, k, v)
        dq = ad.cross_attn_bwd(g, q, k, v, out, lse)[0]
        ref = reference(q, k, v, dout=g)["dq"][0]
    assert off_by(dq, ref) < math.sqrt(2) * off_by(ref.to(dt), ref)


def test_a_second_differentiation_is_refused():
    q, k, v, g = make(1, 2, 2, 40, 30, 64, BF)
    q.requires_grad_(True)
    for out in (ad.cross_attention(q, k, v), ad.rel_bias_attention(q, k, v, table_of(32, 2))):
        dq, = torch.autograd.grad(out, q, g, create_graph=True)
        with pytest.raises(RuntimeError):
            dq.float().sum().backward()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Lq,Lk", [(40, 90001), (300, 40000)])
def test_fp16_weights_of_very_many_keys(Lq, Lk, D):
    """Weights below fp16's smallest normal number (6e-5) keep their bits on the way
    to dv: its error is that of its weights' rounding and its own, independent and
    of one size, the second larger where dv itself is small.  A tenth on top is for
    the weights' rounding being uneven within a binade."""
    q, k, v, g = make(1, 2, 2, Lq, Lk, D, HF, seed=13)
    out, lse = ad.cross_attn(q, k, v)
    _, dk, dv = ad.cross_attn_bwd(g, q, k, v, out, lse)
    ref = reference(q, k, v, dout=g)
    assert off_by(dv, ref["dv"][0]) < 1.1 * math.sqrt(2) * off_by(ref["dv"][0].to(HF), ref["dv"][0])
    table = torch.zeros(8, 2, device="cuda")
    out, lse = ad.rel_bias_attn(q, k, v, table, max_distance=40)
    dv = ad.rel_bias_attn_bwd(g, q, k, v, table, out, lse, max_distance=40)[2]
    assert off_by(dv, ref["dv"][0]) < 1.1 * math.sqrt(2) * off_by(ref["dv"][0].to(HF), ref["dv"][0])


@pytest.mark.parametrize("dt", [BF, HF])
@pytest.mark.parametrize("bias,Lq,Lk", [(False, 1200, 9000), (True, 4300, 4300)])
def test_dq_over_very_many_keys(bias, Lq, Lk, dt):
    """d 128, more rows than the keys are split for.  An error of delta would weigh
    the more the more keys there are: its share of dq leans towards q, dq's own terms
    cancel.  With delta exact the error is dS's rounding and the final one, as before."""
    H = 3 if bias else 12
    q, k, v, g = make(1, H, 1, Lq, Lk, 128, dt, seed=14)
    v = v + 0.5
    if bias:
        table = table_of(32, H, dt)
        out, lse = ad.rel_bias_attn(q, k, v, table, causal=True)
        dq = ad.rel_bias_attn_bwd(g, q, k, v, table, out, lse, causal=True)[0]
        rows = slice(4000, 4300)
    else:
        out, lse = ad.cross_attn(q, k, v)
        dq = ad.cross_attn_bwd(g, q, k, v, out, lse)[0]
        rows = slice(500, 800)
    h = slice(1, 2)
    kw = dict(table=table[:, h], causal=True, q_offset=rows.start) if bias else {}
    ref = reference(q[:, h, rows], k, v, dout=g[:, h, rows], **kw)["dq"][0]
    assert off_by(dq[:, h, rows], ref) < 1.1 * math.sqrt(2) * off_by(ref.to(dt), ref)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Lq,Lk", [(1, 1), (8, 8), (6, 17), (64, 64), (33, 40), (64, 1), (65, 64), (1, 64)])
def test_backward_of_tiny_problems(Lq, Lk, D):
    """Up to 64 queries and keys, one of each more, with masks, shared heads and an
    order mask; and every gradient within sqrt(2) times its final rounding: that, and
    an error of delta or of the forward call's lse that is no larger."""
    dt = HF if Lq % 2 else BF
    q, k, v, g = make(3, 4, 2, Lq, Lk, D, dt, "blhd", seed=15)
    table = table_of(8, 4, dt)
    run_bias(q, k, v, g, table, max_distance=20, key_lens=lens_of(3, Lk, "empty"), key_mask=mask_of(3, Lk, "some"))
    run_bias(q, k, v, g, table, max_distance=20, causal=True)
    if min(Lq, Lk) > 5 and max(Lq, Lk) <= 64:
        kw = dict(max_distance=20)
        out, lse = ad.rel_bias_attn(q, k, v, table, **kw)
        ref = reference(q, k, v, dout=g, table=table, **kw)
        for name, x in zip(("dq", "dk", "dv"), ad.rel_bias_attn_bwd(g, q, k, v, table, out, lse, **kw)):
            assert off_by(x, ref[name][0]) < math.sqrt(2) * off_by(ref[name][0].to(dt), ref[name][0]), name
