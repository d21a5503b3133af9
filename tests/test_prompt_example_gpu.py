"""The prompt-conditioning example runs the operators together: it learns, and
the sample without a prompt is left alone."""
import os
import runpy

import pytest
import torch

pytestmark = pytest.mark.gpu
EXAMPLE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples",
                       "prompt_conditioning.py")


@pytest.mark.parametrize("tokens,prompt", [(320, 48), (520, 65)])
def test_example(tokens, prompt):
    losses, before, out = runpy.run_path(EXAMPLE)["run"](steps=30, tokens=tokens, prompt=prompt)
    assert losses[-1] < 0.5 * losses[0]
    assert torch.isfinite(out.float()).all()
    assert torch.equal(out[1], before[1])          # no prompt: the attention's output is 0
    assert not torch.equal(out[0], before[0])
