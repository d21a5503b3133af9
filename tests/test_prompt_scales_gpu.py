"""fp16 gradients on the GPU away from unit variance: output gradients as a mean over
many elements gives them or as a loss scale makes them, rows of very different size,
values of another size."""
import math

import pytest
import torch

import paper_2502_21079_amd as ad
from _prompt_ref import reference
from test_prompt_gpu import HF, make, table_of

pytestmark = pytest.mark.gpu


def off_by(x, ref):
    return ((x.double() - ref).norm() / ref.norm()).item()


def roundings(ref):
    """Relative error of a result's rounding to fp16 as it is, and were none of it subnormal."""
    up = ref * (8.0 / ref.abs().max())
    return off_by(ref.to(HF), ref), off_by(up.float().to(HF).double(), up)


def grads(q, k, v, g, bias, **kw):
    if not bias:
        out, lse = ad.cross_attn(q, k, v, **kw)
        return ad.cross_attn_bwd(g, q, k, v, out, lse, **kw), reference(q, k, v, dout=g, **kw)
    table = table_of(32, q.shape[1])
    out, lse = ad.rel_bias_attn(q, k, v, table, **kw)
    return ad.rel_bias_attn_bwd(g, q, k, v, table, out, lse, **kw), reference(q, k, v, dout=g, table=table, **kw)


# The ways through the backward kernels: queries and keys of a head on chip (the
# smallest and others), the general one, keys of a head kept on chip (walked twice and
# once), split keys, delta first.
WAYS = [(True, 6, 6, 50, 60, 64), (True, 6, 6, 50, 60, 128), (True, 4, 4, 200, 230, 64), (True, 6, 6, 120, 100, 128),
        (True, 2, 2, 700, 900, 64), (True, 2, 2, 700, 900, 128), (False, 4, 2, 700, 900, 64), (False, 4, 2, 700, 900, 128),
        (False, 8, 8, 9001, 60, 64), (False, 8, 8, 9001, 100, 128), (False, 8, 8, 9001, 200, 64),
        (False, 8, 8, 9001, 200, 128), (False, 6, 3, 40, 9000, 64), (False, 6, 3, 40, 9000, 128),
        (False, 12, 1, 1200, 5000, 128)]


def near_its_rounding(x, ref, name):
    """dS is rounded to 11 bits, independently of the result's rounding: sqrt(r^2 + r0^2),
    and a tenth for delta's share and chance."""
    r, r0 = roundings(ref)
    assert torch.isfinite(x).all(), name
    assert off_by(x, ref) < 1.1 * math.sqrt(r * r + r0 * r0), (name, off_by(x, ref), r, r0)


@pytest.mark.parametrize("size", [1e-3, 1e-4, 1e-5])
@pytest.mark.parametrize("bias,H,Hk,Lq,Lk,D", WAYS)
def test_small_output_gradients(bias, H, Hk, Lq, Lk, D, size):
    q, k, v, g = make(1, H, Hk, Lq, Lk, D, HF, seed=31)
    got, ref = grads(q, k, v, (g.float() * size).to(HF), bias)
    for name, x in zip(("dq", "dk"), got):
        near_its_rounding(x, ref[name][0], name)


@pytest.mark.parametrize("bias,H,Hk,Lq,Lk,D", WAYS)
def test_small_values(bias, H, Hk, Lq, Lk, D):
    """Values a hundredth of unit size (smaller ones leave outputs that are subnormal
    themselves) under small output gradients."""
    q, k, v, g = make(1, H, Hk, Lq, Lk, D, HF, seed=32)
    got, ref = grads(q, k, (v.float() * 1e-2).to(HF), (g.float() * 1e-3).to(HF), bias)
    for name, x in zip(("dq", "dk"), got):
        near_its_rounding(x, ref[name][0], name)


@pytest.mark.parametrize("bias,H,Lq,D", [(True, 6, 60, 64), (True, 6, 60, 128), (True, 6, 200, 64), (True, 6, 120, 128),
                                         (True, 6, 300, 64), (True, 6, 300, 128), (False, 8, 9001, 64),
                                         (False, 8, 9001, 128), (False, 6, 1000, 64), (False, 6, 1000, 128)])
@pytest.mark.parametrize("Lk", [4, 70])
def test_output_gradients_under_a_loss_scale(bias, H, Lq, D, Lk):
    """dP reaches ten times fp16's largest number, dq and dk (times a small scale) do not."""
    q, k, v, g = make(1, H, H, Lq, Lk, D, HF, seed=33)
    got, ref = grads(q, k, v, (g.float() * 12000.0).to(HF), bias, scale=2.0 ** -9)
    for name, x in zip(("dq", "dk"), got):
        near_its_rounding(x, ref[name][0], name)


@pytest.mark.parametrize("bias,H,Hk,Lq,Lk,D", WAYS)
def test_rows_and_keys_of_different_sizes(bias, H, Hk, Lq, Lk, D):
    """Output gradients of 1e-4 to 100 from row to row (dq row by row of one size),
    values of 1e-2 to 10 from key to key (dk of every key as good as the whole)."""
    q, k, v, g = make(1, H, Hk, Lq, Lk, D, HF, seed=34)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(8)
    step = torch.randint(0, 7, (Lq,), generator=gen, device="cuda")
    g = (g.float() * 10.0 ** (step - 4.0).view(1, 1, Lq, 1)).to(HF)
    got, ref = grads(q, k, v, g, bias)
    for s in range(7):
        rows = (step == s).nonzero().flatten()
        if rows.numel():
            x, z = got[0][:, :, rows].double(), ref["dq"][0][:, :, rows]
            r, r0 = roundings(z)
            # Few rows: a quarter for chance.
            assert off_by(x, z) < 1.25 * math.sqrt(r * r + r0 * r0), (s, off_by(x, z), r, r0)
    near_its_rounding(got[1], ref["dk"][0], "dk")
    q, k, v, g = make(1, H, Hk, Lq, Lk, D, HF, seed=35)
    v = (v.float() * 10.0 ** (torch.randint(0, 4, (Lk,), generator=gen, device="cuda") - 2.0).view(1, 1, Lk, 1)).to(HF)
    got, ref = grads(q, k, v, (g.float() * 1e-3).to(HF), bias)
    for name, x in zip(("dq", "dk"), got):
        near_its_rounding(x, ref[name][0], name)
