"""fp16 on the GPU: dv of keys that no query gives more than a millionth of its weight is
as good as that of the others."""
import math

import pytest
import torch

from test_prompt_gpu import HF
from test_prompt_scales_gpu import WAYS, grads, off_by

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bias,H,Hk,Lq,Lk,D", WAYS)
def test_dv_of_keys_with_little_weight(bias, H, Hk, Lq, Lk, D):
    """A third of the keys 9 below the others in score: weights of 1e-6 and less, times
    output gradients of 100.  Weights are rounded to 11 bits and dv once more: sqrt(2) r,
    and a tenth for chance."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(51)
    u = torch.randn(D, generator=gen, device="cuda")
    u *= D ** 0.5 / u.norm()
    n = lambda h, L: torch.randn(1, h, L, D, generator=gen, device="cuda")  # noqa: E731
    q, k, v, g = (u + 0.3 * n(H, Lq)).to(HF), n(Hk, Lk), n(Hk, Lk).to(HF), (100.0 * n(H, Lq)).to(HF)
    far = torch.arange(Lk, device="cuda") % 3 == 1
    k = torch.where(far.view(1, 1, Lk, 1), k - u * (9.0 * D ** -0.5), k).to(HF)
    got, ref = grads(q, k, v, g, bias)
    for which in (far, ~far):
        z = ref["dv"][0][:, :, which]
        assert off_by(got[2][:, :, which], z) < 1.1 * math.sqrt(2) * off_by(z.to(HF), z), bool(which[1])
