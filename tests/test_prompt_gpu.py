"""Cross attention and attention with a relative position bias on the GPU, with
their backward passes, against a plain 64-bit form: types, layouts, lengths
from none to long, shared key heads, masks that leave rows empty, strides."""
import math

import pytest
import torch

import paper_2502_21079_amd as ad
from _prompt_ref import check, reference

pytestmark = pytest.mark.gpu
BF, HF = torch.bfloat16, torch.float16


def make(B, H, Hk, Lq, Lk, D, dt, layout="bhld", seed=0, std=1.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 7919 + Lq * 31 + Lk)

    def t(h, n, s=1.0):
        if layout == "bhld":
            x = torch.randn(B, h, n, D, generator=g, device="cuda")
        else:
            x = torch.randn(B, n, h, D, generator=g, device="cuda").transpose(1, 2)
        return (x * s).to(dt)
    return t(H, Lq, std), t(Hk, Lk), t(Hk, Lk), t(H, Lq)


def lens_of(B, Lk, kind):
    if kind == "none":
        return None
    n = [max(0, Lk - b * ((Lk + 2) // 3)) for b in range(B)]
    if kind == "empty":
        n[-1] = 0
    return torch.tensor(n, dtype=torch.int32, device="cuda")


def mask_of(B, Lk, kind, seed=3):
    if kind == "none":
        return None
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    m = torch.rand(B, Lk, generator=g, device="cuda") > 0.3
    if kind == "empty":
        m[0] = False
    return m


def run_cross(q, k, v, g, bwd=True, **kw):
    out, lse = ad.cross_attn(q, k, v, **kw)
    torch.cuda.synchronize()
    ref = reference(q, k, v, dout=g if bwd else None, **kw)
    check(lse, ref["lse"], "lse")
    check(out, ref["out"], "out")
    if bwd:
        grads = ad.cross_attn_bwd(g, q, k, v, out, lse, **kw)
        torch.cuda.synchronize()
        for name, x in zip(("dq", "dk", "dv"), grads):
            check(x, ref[name], name)
    return out, lse


LENGTHS = [(1, 1), (1, 63), (5, 64), (33, 65), (127, 200), (130, 1), (300, 77), (129, 513), (1, 3001), (64, 1999),
           (2100, 226), (777, 256), (513, 257)]


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Lq,Lk", LENGTHS)
def test_cross_lengths(Lq, Lk, D):
    dt, layout = (BF, "bhld") if (Lq + Lk) % 2 else (HF, "blhd")
    q, k, v, g = make(2, 3, 3, Lq, Lk, D, dt, layout)
    run_cross(q, k, v, g)


@pytest.mark.parametrize("H,Hk", [(4, 1), (6, 2), (8, 8)])
@pytest.mark.parametrize("lens,mask", [("some", "none"), ("empty", "none"), ("none", "some"), ("empty", "some"),
                                       ("none", "empty")])
def test_cross_masks_and_shared_heads(H, Hk, lens, mask):
    B, Lq, Lk, D = 3, 70, 190, 64 if H == 6 else 128
    q, k, v, g = make(B, H, Hk, Lq, Lk, D, HF if H == 4 else BF, "blhd" if H == 8 else "bhld", seed=H)
    out, lse = run_cross(q, k, v, g, key_lens=lens_of(B, Lk, lens), key_mask=mask_of(B, Lk, mask))
    if lens == "empty":
        assert (out[-1] == 0).all() and (lse[-1] == -math.inf).all()


@pytest.mark.parametrize("Lq,Lk", [(7, 100), (300, 150), (3, 2000), (2500, 256), (2500, 130)])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_masked_keys_may_hold_anything(Lq, Lk, D, bad):
    """Infinities and NaN behind a mask or past a sample's keys change nothing,
    and get no gradient."""
    q, k, v, g = make(2, 2, 2, Lq, Lk, D, BF, seed=5)
    lens = torch.tensor([Lk, Lk - 37], dtype=torch.int32, device="cuda")
    mask = mask_of(2, Lk, "some")
    kw = dict(key_lens=lens, key_mask=mask)
    hidden = ~mask | (torch.arange(Lk, device="cuda") >= lens.view(2, 1))
    a = ad.cross_attn(q, k, v, **kw)
    ga = ad.cross_attn_bwd(g, q, k, v, *a, **kw)
    k2, v2 = k.clone(), v.clone()
    k2.masked_fill_(hidden.view(2, 1, Lk, 1), bad)
    v2.masked_fill_(hidden.view(2, 1, Lk, 1), bad)
    b = ad.cross_attn(q, k2, v2, **kw)
    gb = ad.cross_attn_bwd(g, q, k2, v2, *b, **kw)
    for x, y in zip(a + ga, b + gb):
        assert torch.equal(x, y)
    for x in gb[1:]:
        assert (x.masked_select(hidden.view(2, 1, Lk, 1)) == 0).all()


def test_lengths_outside_the_cache_are_clamped():
    q, k, v, _ = make(3, 2, 2, 40, 90, 64, BF)
    a = ad.cross_attn(q, k, v, key_lens=torch.tensor([90, 0, 90], dtype=torch.int32, device="cuda"))
    b = ad.cross_attn(q, k, v, key_lens=torch.tensor([1 << 30, -5, 91], dtype=torch.int32, device="cuda"))
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_zero_lengths():
    q, k, v, g = make(2, 2, 2, 5, 0, 64, BF)
    out, lse = ad.cross_attn(q, k, v)
    assert (out == 0).all() and (lse == -math.inf).all()
    dq, dk, dv = ad.cross_attn_bwd(g, q, k, v, out, lse)
    assert (dq == 0).all() and dk.shape == k.shape and dv.shape == v.shape
    q, k, v, g = make(2, 2, 2, 0, 9, 64, BF)
    out, lse = ad.cross_attn(q, k, v)
    assert out.shape == q.shape and lse.shape == (2, 2, 0)
    dq, dk, dv = ad.cross_attn_bwd(g, q, k, v, out, lse)
    assert (dk == 0).all() and (dv == 0).all()
    table = torch.randn(8, 2, device="cuda")
    out, lse = ad.rel_bias_attn(q, k, v, table)
    assert (ad.rel_bias_attn_bwd(g, q, k, v, table, out, lse)[3] == 0).all()
    q, k, v, g = make(0, 2, 2, 4, 9, 64, BF)
    assert ad.cross_attn(q, k, v)[0].shape == q.shape


def test_strided_and_broadcast_inputs():
    """Slices of a fused projection, and one sample's states read by all."""
    B, H, Lq, Lk, D = 3, 4, 150, 99, 64
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    kv = torch.randn(B, Lk, 2, H, D, generator=g, device="cuda").to(BF)
    qx = torch.randn(B, Lq, H, 3, D, generator=g, device="cuda").to(BF)
    q, k, v = qx[:, :, :, 1].transpose(1, 2), kv[:, :, 0].transpose(1, 2), kv[:, :, 1].transpose(1, 2)
    do = torch.randn(B, H, Lq, D, generator=g, device="cuda").to(BF)
    run_cross(q, k, v, do)
    run_cross(q, k[:1].expand(B, -1, -1, -1), v[:1].expand(B, -1, -1, -1), do)
    # Every second token of a longer sequence, and outputs given by the caller.
    out = torch.full((B, Lq, H, D), 7.0, dtype=BF, device="cuda")
    ad.cross_attn(q, k[:, :, ::2], v[:, :, ::2], out=out.transpose(1, 2))
    check(out.transpose(1, 2), reference(q, k[:, :, ::2], v[:, :, ::2])["out"], "out")


@pytest.mark.parametrize("dt", [BF, HF])
@pytest.mark.parametrize("std", [8.0, 60.0])
def test_steep_scores(dt, std):
    """Scores that rise by far more than the reference's slack, rows whose
    weight sits on one key, and scores far below zero."""
    q, k, v, g = make(1, 2, 2, 200, 700, 128, dt, seed=9, std=std)
    k = k * torch.linspace(0.05, 1.0, 700, device="cuda").view(1, 1, -1, 1)
    run_cross(q, k.to(dt), v, g, bwd=False)
    run_cross(q.abs(), -k.abs().to(dt), v, g, bwd=False)


def test_overflowing_rows_stay_their_own():
    """A row with an infinite query is NaN as in the formula, its neighbours are
    what they were."""
    q, k, v, _ = make(1, 2, 2, 50, 120, 64, BF)
    a = ad.cross_attn(q, k, v)[0]
    q2 = q.clone()
    q2[0, 1, 17, 3] = math.inf
    b = ad.cross_attn(q2, k, v)[0]
    assert torch.isnan(b[0, 1, 17]).all()
    b[0, 1, 17] = a[0, 1, 17]
    assert torch.equal(a, b)


def test_long_keys_past_32_bits():
    """A cache of more than 2^32 bytes per sample: token stride 24,576 bytes x
    180,000 tokens, values only where the lengths reach."""
    B, H, Lk, D = 1, 96, 180000, 128
    pool = torch.empty(Lk, H, D, dtype=BF, device="cuda")
    g = torch.Generator(device="cuda")
    g.manual_seed(4)
    pool[:, -1].copy_(torch.randn(Lk, D, generator=g, device="cuda"))
    k = pool[:, -1:].unsqueeze(0).transpose(1, 2)
    q = torch.randn(B, 1, 3, D, generator=g, device="cuda").to(BF)
    do = torch.randn(B, 1, 3, D, generator=g, device="cuda").to(BF)
    out, lse = ad.cross_attn(q, k, k)
    ref = reference(q, k.contiguous(), k.contiguous(), dout=do)
    check(out, ref["out"], "out")
    check(lse, ref["lse"], "lse")
    dk, dv = torch.empty(B, 1, Lk, D, dtype=BF, device="cuda"), torch.empty(B, 1, Lk, D, dtype=BF, device="cuda")
    grads = ad.cross_attn_bwd(do, q, k, k, out, lse, dk=dk, dv=dv)
    for name, x in zip(("dq", "dk", "dv"), grads):
        check(x, ref[name], name)


# --- relative position bias ----------------------------------------------------

def run_bias(q, k, v, g, table, bwd=True, **kw):
    out, lse = ad.rel_bias_attn(q, k, v, table, **kw)
    torch.cuda.synchronize()
    ref = reference(q, k, v, dout=g if bwd else None, table=table, **kw)
    check(lse, ref["lse"], "lse")
    check(out, ref["out"], "out")
    if bwd:
        grads = ad.rel_bias_attn_bwd(g, q, k, v, table, out, lse, **kw)
        torch.cuda.synchronize()
        for name, x in zip(("dq", "dk", "dv", "dtable"), grads):
            check(x, ref[name], name)
    return out, lse


def table_of(n, H, dt=torch.float32, seed=0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed + 100)
    return torch.randn(n, H, generator=g, device="cuda").to(dt)


@pytest.mark.parametrize("both", [True, False])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Lq,Lk", [(1, 1), (2, 70), (65, 64), (130, 131), (400, 400), (1000, 333), (333, 1000),
                                   (700, 701)])
def test_bias_lengths(Lq, Lk, D, both):
    q, k, v, g = make(2, 3, 3, Lq, Lk, D, BF if Lq % 2 else HF, "blhd" if Lk % 2 else "bhld", seed=2)
    run_bias(q, k, v, g, table_of(32, 3, torch.float32 if both else q.dtype), bidirectional=both)


@pytest.mark.parametrize("n,far,both", [(4, 2, True), (2, 2, False), (8, 64, True), (64, 500, False),
                                        (512, 1024, True), (256, 1024, False), (32, 20, True)])
def test_bias_bucket_plans(n, far, both):
    q, k, v, g = make(1, 2, 2, 300, 1300, 64, BF, seed=n)
    run_bias(q, k, v, g, table_of(n, 2), max_distance=far, bidirectional=both, q_offset=500)


@pytest.mark.parametrize("offset", [0, 37, -40, "end"])
@pytest.mark.parametrize("H,Hk", [(2, 2), (6, 2)])
@pytest.mark.parametrize("Lq,Lk", [(1, 500), (200, 200), (130, 300), (300, 130)])
def test_bias_causal(Lq, Lk, H, Hk, offset):
    """Order masks, with offsets that leave rows empty; shared key heads; a
    sample's own lengths."""
    q, k, v, g = make(3, H, Hk, Lq, Lk, 64, HF, seed=H)
    run_bias(q, k, v, g, table_of(16, H, HF), max_distance=60, bidirectional=False, causal=True, q_offset=offset,
             key_lens=lens_of(3, Lk, "empty"))


def test_bias_causal_and_both_ways_with_masks():
    q, k, v, g = make(2, 4, 4, 260, 260, 128, BF, seed=8)
    run_bias(q, k, v, g, table_of(32, 4, BF), causal=True, key_mask=mask_of(2, 260, "empty"), scale=1.0 / 16)
    run_bias(q, k, v, g, table_of(32, 4, BF), key_mask=mask_of(2, 260, "some"), key_lens=lens_of(2, 260, "some"))


def test_bias_of_zero_is_cross_attention():
    q, k, v, _ = make(2, 4, 4, 200, 300, 128, BF)
    a, la = ad.cross_attn(q, k, v)
    b, lb = ad.rel_bias_attn(q, k, v, torch.zeros(32, 4, device="cuda"))
    assert torch.allclose(a.float(), b.float(), atol=2 ** -8, rtol=2 ** -7)
    assert torch.allclose(la, lb, atol=1e-5, rtol=1e-5)


# --- gradients against differences ----------------------------------------------

def test_gradients_against_differences():
    """Central differences of the kernels' own forward pass along the gradient:
    sum(dout * out) moves by |gradient| per unit step.  fp16 outputs carry
    2^-11; over 2 x 2 x 96 x 64 values that noise is about 0.05 in the sum,
    against a change of several units."""
    B, H, Lq, Lk, D = 2, 2, 96, 120, 64
    q, k, v, g = make(B, H, H, Lq, Lk, D, HF, seed=6)
    table = table_of(32, H)
    loss = lambda *a: float((ad.rel_bias_attn(*a)[0].double() * g.double()).sum())  # noqa: E731
    out, lse = ad.rel_bias_attn(q, k, v, table)
    grads = ad.rel_bias_attn_bwd(g, q, k, v, table, out, lse)
    args = [q, k, v, table]
    for i, gr in enumerate(grads):
        d = gr.double() / gr.double().norm()
        step = 2.0 if i < 3 else 0.25
        up, down = list(args), list(args)
        up[i] = (args[i].double() + step * d).to(args[i].dtype)
        down[i] = (args[i].double() - step * d).to(args[i].dtype)
        moved = up[i].double() - down[i].double()          # what rounding left of the step
        want = float((gr.double() * moved).sum())
        got = loss(*up) - loss(*down)
        assert abs(got - want) <= 0.05 * abs(want) + 0.2, (i, got, want)


def test_autograd_functions():
    q, k, v, g = make(2, 4, 2, 150, 90, 64, BF, "blhd")
    lens = lens_of(2, 90, "some")
    for x in (q, k, v):
        x.requires_grad_(True)
    out = ad.cross_attention(q, k, v, key_lens=lens)
    out.backward(g)
    ref = reference(q.detach(), k.detach(), v.detach(), dout=g, key_lens=lens)
    for name, x in (("dq", q), ("dk", k), ("dv", v)):
        check(x.grad, ref[name], name)
        x.grad = None
    table = table_of(32, 4).requires_grad_(True)
    out = ad.rel_bias_attention(q, k, v, table, max_distance=40, key_lens=lens)
    (out * 2).sum().backward()                              # an expanded gradient
    two = torch.full_like(out, 2.0)
    ref = reference(q.detach(), k.detach(), v.detach(), dout=two, table=table.detach(), max_distance=40, key_lens=lens)
    for name, x in (("dq", q), ("dk", k), ("dv", v), ("dtable", table)):
        check(x.grad, ref[name], name)


# --- the same bits, other streams, graphs -----------------------------------------

def test_results_repeat_bit_for_bit():
    q, k, v, g = make(2, 6, 2, 700, 300, 128, BF, seed=3)
    table = table_of(32, 6)

    def once():
        a = ad.cross_attn(q, k, v)
        b = ad.rel_bias_attn(q, k, v, table)
        return a + b + ad.cross_attn_bwd(g, q, k, v, *a) + ad.rel_bias_attn_bwd(g, q, k, v, table, *b)
    first = once()
    for _ in range(3):
        for x, y in zip(first, once()):
            assert torch.equal(x, y)


def test_another_stream():
    q, k, v, g = make(1, 4, 4, 1, 9000, 128, BF)
    want = ad.cross_attn(q, k, v)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = ad.cross_attn(q, k, v)
    s.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_graph_replays_match_eager_calls():
    q, k, v, g = make(2, 4, 4, 3, 5000, 64, BF)
    table = table_of(32, 4)
    kw = dict(bidirectional=False, causal=True, q_offset="end",
              key_lens=torch.tensor([5000, 4000], dtype=torch.int32, device="cuda"))
    ws = torch.empty(max(256, ad.rel_bias_attn_workspace(q.shape, k.shape, 32, bidirectional=False)),
                     dtype=torch.uint8, device="cuda")
    wb = torch.empty(ad.rel_bias_attn_bwd_workspace(q.shape, k.shape, 32, bidirectional=False), dtype=torch.uint8,
                     device="cuda")
    out, lse = torch.empty_like(q), torch.empty(2, 4, 3, device="cuda")
    ad.rel_bias_attn(q, k, v, table, out=out, lse=lse, workspace=ws, **kw)
    ad.rel_bias_attn_bwd(g, q, k, v, table, out, lse, workspace=wb, **kw)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ad.rel_bias_attn(q, k, v, table, out=out, lse=lse, workspace=ws, **kw)
        grads = ad.rel_bias_attn_bwd(g, q, k, v, table, out, lse, workspace=wb, **kw)
    for i in range(4):
        q.copy_(torch.randn_like(q, dtype=torch.float32))
        kw["key_lens"].copy_(torch.tensor([5000 - 700 * i, 100 + i], dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        a = ad.rel_bias_attn(q, k, v, table, **kw)
        b = ad.rel_bias_attn_bwd(g, q, k, v, table, *a, **kw)
        for x, y in zip((out, lse) + tuple(grads), a + b):
            assert torch.equal(x, y)


# --- refusals ---------------------------------------------------------------------

def test_refusals():
    q, k, v, g = make(2, 4, 2, 300, 9, 64, BF)
    table = table_of(32, 4)
    out, lse = ad.cross_attn(q, k, v)
    err = pytest.raises(ad.AdaspaError)
    lens = torch.ones(2, dtype=torch.int32, device="cuda")
    for call in (
            lambda: ad.cross_attn(q.float(), k.float(), v.float()),
            lambda: ad.cross_attn(q, k.half(), v),
            lambda: ad.cross_attn(q.cpu(), k, v),
            lambda: ad.cross_attn(q[0], k, v),
            lambda: ad.cross_attn(q[:1], k, v),
            lambda: ad.cross_attn(q[:, :3], k, v),
            lambda: ad.cross_attn(q[..., :32], k[..., :32], v[..., :32]),
            lambda: ad.cross_attn(q, k, v[:, :, :5]),
            lambda: ad.cross_attn(q.transpose(2, 3).contiguous().transpose(2, 3), k, v),
            lambda: ad.cross_attn(q, k, v, key_lens=lens.long()),
            lambda: ad.cross_attn(q, k, v, key_lens=lens[:1]),
            lambda: ad.cross_attn(q, k, v, key_lens=lens.cpu()),
            lambda: ad.cross_attn(q, k, v, key_mask=torch.ones(2, 8, dtype=torch.bool, device="cuda")),
            lambda: ad.cross_attn(q, k, v, key_mask=torch.ones(2, 9, device="cuda")),
            lambda: ad.cross_attn(q, k, v, scale=math.nan),
            lambda: ad.cross_attn(q, k, v, out=out[:, :2]),
            lambda: ad.cross_attn(q, k, v, out=out[:1].expand(2, -1, -1, -1)),
            lambda: ad.cross_attn(q, k, v, lse=lse[:1]),
            lambda: ad.cross_attn_bwd(g[:1], q, k, v, out, lse),
            lambda: ad.cross_attn_bwd(g, q, k, v, out, lse.double()),
            lambda: ad.cross_attn_bwd(g, q, k, v, out, lse, dk=torch.empty_like(q)),
            lambda: ad.cross_attn_bwd(g, q, k, v, out, lse, workspace=torch.empty(8, device="cuda")),
            lambda: ad.rel_bias_attn(q, k, v, table[:, :2]),
            lambda: ad.rel_bias_attn(q, k, v, table.double()),
            lambda: ad.rel_bias_attn(q, k, v, table.half()),
            lambda: ad.rel_bias_attn(q, k, v, table[:31]),
            lambda: ad.rel_bias_attn(q, k, v, table, max_distance=8),
            lambda: ad.rel_bias_attn(q, k, v, table, max_distance=5000),
            lambda: ad.rel_bias_attn(q, k, v, table, q_offset=1 << 29)):
        with err:
            call()
