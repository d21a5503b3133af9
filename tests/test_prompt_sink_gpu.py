"""fp16 on the GPU where one key's weight is far above all others and its value small."""
import math

import pytest
import torch

import paper_2502_21079_amd as ad
from _prompt_ref import reference
from test_prompt_edges_gpu import off_by
from test_prompt_gpu import HF

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("H,D", [(16, 128), (24, 64)])
@pytest.mark.parametrize("place", [5, 70003])
@pytest.mark.parametrize("logit,mean", [(16.0, 0.5), (18.0, 0.5), (16.0, 0.0)])
def test_a_dominant_key_of_small_value(H, D, place, logit, mean):
    """100,000 keys of unit-variance scores beside one at ``logit`` whose value is
    zero: the others' weights, 2^-23 to 2^-26 of the largest, make the output.  Its
    error is their rounding and its own, each as large as the latter at most."""
    Lq, Lk = 2100, 100000
    gen = torch.Generator(device="cuda")
    gen.manual_seed(41)
    u = torch.randn(D, generator=gen, device="cuda")
    u *= D ** 0.5 / u.norm()
    q = (u + 0.2 * torch.randn(1, H, Lq, D, generator=gen, device="cuda")).to(HF)
    k = torch.randn(1, 1, Lk, D, generator=gen, device="cuda")
    v = (torch.randn(1, 1, Lk, D, generator=gen, device="cuda") + mean)
    k[:, :, place] = u * (logit * D ** -0.5)
    v[:, :, place] = 0.0
    k, v = k.to(HF), v.to(HF)
    out, lse = ad.cross_attn(q, k, v)
    h, rows = slice(3, 4), slice(1000, 1100)
    ref = reference(q[:, h, rows], k, v)
    assert off_by(out[:, h, rows], ref["out"][0]) < 1.1 * math.sqrt(2) * off_by(ref["out"][0].to(HF), ref["out"][0])
    assert (lse[:, h, rows].double() - ref["lse"][0]).abs().max() < 1e-4
