"""Query heads that share key heads under a position bias without an order mask, where
the keys are divided into ranges: few rows over many keys, forward and backward,
against the plain 64-bit form."""
import pytest

from test_prompt_gpu import BF, HF, lens_of, make, mask_of, run_bias, table_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("both", [True, False])
@pytest.mark.parametrize("D,dt", [(64, HF), (128, BF)])
@pytest.mark.parametrize("H,Hk,Lq,Lk,offset", [(4, 2, 1, 3001, 3000), (6, 1, 20, 2500, "end"), (8, 4, 33, 2111, 700),
                                               (4, 1, 130, 1999, 0)])
def test_shared_heads_over_split_keys(H, Hk, Lq, Lk, offset, D, dt, both):
    q, k, v, g = make(2, H, Hk, Lq, Lk, D, dt, "blhd", seed=23)
    run_bias(q, k, v, g, table_of(32, H, dt), bidirectional=both, q_offset=offset, key_lens=lens_of(2, Lk, "some"),
             key_mask=mask_of(2, Lk, "some"))
