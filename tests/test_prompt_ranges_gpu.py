"""Cross attention and relative position bias on the GPU at the sizes where a
call takes another way through the kernels: keys of a head kept on chip, keys
or queries divided into ranges that are joined afterwards, problems that one
launch holds whole; each with lengths, masks, shared heads and empty rows,
against the plain 64-bit form."""
import math

import pytest
import torch

import paper_2502_21079_amd as ad
from _prompt_ref import check, reference
from test_prompt_gpu import BF, HF, lens_of, make, mask_of, run_bias, run_cross, table_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D,Lk", [(64, 1), (64, 64), (64, 65), (64, 226), (64, 512), (64, 513), (128, 9), (128, 100),
                                  (128, 256), (128, 257)])
@pytest.mark.parametrize("hide", ["none", "lens", "both"])
def test_many_rows_over_few_keys(D, Lk, hide):
    """Rows enough for every CU's waves: up to 512 keys at d 64 and 256 at d 128
    stay on chip, one key more does not."""
    B, H, Hk, Lq = 3, 8, 4, 6011
    dt, layout = (HF, "blhd") if Lk % 2 else (BF, "bhld")
    q, k, v, g = make(B, H, Hk, Lq, Lk, D, dt, layout, seed=D)
    kw = {}
    if hide != "none":
        kw["key_lens"] = lens_of(B, Lk, "empty")
    if hide == "both":
        kw["key_mask"] = mask_of(B, Lk, "empty")
    out, lse = run_cross(q, k, v, g, **kw)
    if hide != "none":
        assert (out[-1] == 0).all() and (lse[-1] == -math.inf).all()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_keys_on_chip_may_hold_anything_where_masked(D, bad):
    B, H, Lq, Lk = 2, 8, 9001, 200
    q, k, v, g = make(B, H, H, Lq, Lk, D, BF, seed=8)
    lens = torch.tensor([Lk, 70], dtype=torch.int32, device="cuda")
    mask = mask_of(B, Lk, "some")
    kw = dict(key_lens=lens, key_mask=mask)
    hidden = (~mask | (torch.arange(Lk, device="cuda") >= lens.view(2, 1))).view(2, 1, Lk, 1)
    a = ad.cross_attn(q, k, v, **kw)
    ga = ad.cross_attn_bwd(g, q, k, v, *a, **kw)
    k2, v2 = k.masked_fill(hidden, bad), v.masked_fill(hidden, bad)
    b = ad.cross_attn(q, k2, v2, **kw)
    gb = ad.cross_attn_bwd(g, q, k2, v2, *b, **kw)
    for x, y in zip(a + ga, b + gb):
        assert torch.equal(x, y)
    for x in gb[1:]:
        assert (x.masked_select(hidden) == 0).all()


@pytest.mark.parametrize("Lq,Lk", [(1, 1024), (7, 1500), (32, 2500), (33, 1300), (90, 4000), (250, 1100)])
@pytest.mark.parametrize("H,Hk", [(2, 2), (6, 1)])
@pytest.mark.parametrize("hide", ["none", "both"])
def test_few_rows_over_many_keys(Lq, Lk, H, Hk, hide):
    """The keys are split: few rows and many ranges, more rows and few ranges."""
    B, D = 2, 64 if (Lq + H) % 2 else 128
    q, k, v, g = make(B, H, Hk, Lq, Lk, D, BF if Lq % 2 else HF, "blhd" if H == 6 else "bhld", seed=2)
    kw = dict(key_lens=lens_of(B, Lk, "empty"), key_mask=mask_of(B, Lk, "some")) if hide == "both" else {}
    run_cross(q, k, v, g, **kw)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Lq,Lk,offset", [(3100, 3100, 0), (1500, 3300, "end"), (3200, 3100, -700), (300, 1500, 5)])
def test_order_mask_with_split_keys(Lq, Lk, D, offset):
    """Ranges that lie past all of a row's keys, and rows before every key."""
    q, k, v, g = make(1, 2, 1, Lq, Lk, D, BF, seed=4)
    run_bias(q, k, v, g, table_of(32, 2), max_distance=128, bidirectional=False, causal=True, q_offset=offset)


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("Lq,Lk", [(13, 2000), (700, 1900)])
def test_bias_with_split_keys_and_masks(Lq, Lk, causal):
    B = 3
    q, k, v, g = make(B, 2, 2, Lq, Lk, 64, HF, "blhd", seed=6)
    run_bias(q, k, v, g, table_of(16, 2, HF), max_distance=300, bidirectional=not causal, causal=causal,
             q_offset="end" if causal else 0, key_lens=lens_of(B, Lk, "some"), key_mask=mask_of(B, Lk, "some"))


@pytest.mark.parametrize("D,Lq,Lk", [(64, 256, 256), (64, 257, 256), (64, 256, 257), (64, 31, 256), (64, 256, 1),
                                     (128, 128, 128), (128, 129, 128), (128, 128, 129), (128, 97, 33)])
@pytest.mark.parametrize("far", [128, 256, 257])
def test_backward_of_small_problems(D, Lq, Lk, far):
    """A head's queries and keys on chip, up to 256 (d 64) or 128 (d 128) of
    each and distances to 256; one more takes the general way."""
    B, H, Hk = 2, 6, 3
    q, k, v, g = make(B, H, Hk, Lq, Lk, D, BF if Lk % 2 else HF, "blhd" if Lq % 2 else "bhld", seed=far)
    causal = far == 256
    run_bias(q, k, v, g, table_of(32, H), max_distance=far, bidirectional=not causal, causal=causal,
             key_lens=lens_of(B, Lk, "some"), key_mask=mask_of(B, Lk, "some" if Lk > 1 else "none"))


@pytest.mark.parametrize("G,Lq,Lk", [(1, 3000, 40), (4, 1100, 300), (2, 5000, 700)])
@pytest.mark.parametrize("D", [64, 128])
def test_split_queries(G, Lq, Lk, D):
    """Few key tiles: the queries are split, and dk and dv joined."""
    B = 2
    q, k, v, g = make(B, G, 1, Lq, Lk, D, HF, "bhld", seed=9)
    run_cross(q, k, v, g, key_lens=lens_of(B, Lk, "empty"))


def rel(x, ref):
    return ((x.double() - ref).norm() / ref.norm()).item()


@pytest.mark.parametrize("D,Lq,Lk", [(64, 20, 9000), (128, 20, 9000), (64, 230, 250), (128, 120, 100), (64, 700, 900)])
def test_gradients_do_not_carry_the_outputs_rounding(D, Lq, Lk):
    """Steep scores, where dS = P (dP - delta) cancels.  dq and dk are sums of
    terms dS x with dS rounded to u = 2^-9 of its size, independently, and are
    rounded by u once more: the errors add up as the terms do, so the relative
    error of the whole is at most sqrt(2) u; 2 u leaves a margin for fp32's part.
    The table's gradient holds no rounded term: u, and the same margin again.  A
    delta formed from the rounded output would add errors of its own, which the
    rows' keys have in common."""
    u = 2.0 ** -9
    q, k, v, g = make(2, 2, 2, Lq, Lk, D, BF, seed=11, std=3.0)
    out, lse = ad.cross_attn(q, k, v)
    dq, dk, dv = ad.cross_attn_bwd(g, q, k, v, out, lse)
    ref = reference(q, k, v, dout=g)
    assert rel(dq, ref["dq"][0]) < 2 * u
    assert rel(dk, ref["dk"][0]) < 2 * u
    table = table_of(32, 2, BF)
    kw = dict(max_distance=128, bidirectional=True)
    out, lse = ad.rel_bias_attn(q, k, v, table, **kw)
    dq, dk, dv, dt = ad.rel_bias_attn_bwd(g, q, k, v, table, out, lse, **kw)
    ref = reference(q, k, v, dout=g, table=table, **kw)
    assert rel(dq, ref["dq"][0]) < 2 * u
    assert rel(dk, ref["dk"][0]) < 2 * u
    assert rel(dt, ref["dtable"][0]) < 2 * u


@pytest.mark.parametrize("B,H,Lq,Lk,causal", [(1, 6, 3300, 3300, True), (1, 6, 3300, 3300, False),
                                              (2, 2, 200, 2000, False), (1, 2, 700, 900, True)])
def test_workspaces_of_the_named_sizes(B, H, Lq, Lk, causal):
    """A caller's workspaces, of just the named sizes, give the results of the
    call's own; one byte less is refused."""
    q, k, v, g = make(B, H, H, Lq, Lk, 64, BF, seed=3)
    table = table_of(32, H)
    kw = dict(bidirectional=not causal, causal=causal)
    out, lse = ad.rel_bias_attn(q, k, v, table, **kw)
    grads = ad.rel_bias_attn_bwd(g, q, k, v, table, out, lse, **kw)
    sizes = [f(q.shape, k.shape, 32, **kw) for f in (ad.rel_bias_attn_workspace, ad.rel_bias_attn_bwd_workspace)]
    ws = [torch.empty(n, dtype=torch.uint8, device="cuda") for n in sizes]
    again = ad.rel_bias_attn(q, k, v, table, workspace=ws[0], **kw)
    again += ad.rel_bias_attn_bwd(g, q, k, v, table, *again, workspace=ws[1], **kw)
    for x, y in zip((out, lse) + grads, again):
        assert torch.equal(x, y)
    if sizes[0] > 16:
        with pytest.raises(ad.AdaspaError):
            ad.rel_bias_attn(q, k, v, table, workspace=ws[0][:-1], **kw)
    with pytest.raises(ad.AdaspaError):
        ad.rel_bias_attn_bwd(g, q, k, v, table, out, lse, workspace=ws[1][:-1], **kw)
