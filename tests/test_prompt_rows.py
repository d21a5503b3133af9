"""CPU check of the copy that a gradient gets where the kernels cannot read it as it lies."""
import pytest
import torch

from paper_2502_21079_amd.prompt import _rows

X = torch.arange(2 * 3 * 4 * 64).float().to(torch.bfloat16).view(2, 3, 4, 64)


@pytest.mark.parametrize("t", [X, X.transpose(1, 2), X[:, :, ::2], X[:1].expand(2, -1, -1, -1)])
def test_readable_gradients_are_taken_as_they_lie(t):
    assert _rows(t) is t


@pytest.mark.parametrize("skip", [1, 2, 4, 7])
def test_a_contiguous_view_at_an_odd_offset_is_copied(skip):
    """A slice of one flat buffer of gradients."""
    flat = torch.zeros(X.numel() + 8, dtype=X.dtype)
    flat[skip:skip + X.numel()] = X.flatten()
    t = flat[skip:skip + X.numel()].view(X.shape)
    assert t.is_contiguous() and t.data_ptr() % 16 != 0
    assert _rows(t).data_ptr() % 16 == 0 and torch.equal(_rows(t), X)


@pytest.mark.parametrize("t", [X.transpose(2, 3).contiguous().transpose(2, 3), X[..., :1].expand(-1, -1, -1, 64),
                               torch.as_strided(torch.zeros(1 << 23, dtype=X.dtype).expand(1 << 23), (1, 1, 1, 64),
                                                (64, 64, 64, 0))])
def test_other_orders_are_copied(t):
    y = _rows(t)
    assert y.is_contiguous() and y.data_ptr() % 16 == 0 and torch.equal(y, t)


def test_tokens_further_apart_than_a_tile_of_them_may_be_are_copied():
    t = torch.as_strided(torch.zeros((1 << 23) + 64, dtype=X.dtype), (1, 1, 2, 64), (0, 0, 1 << 23, 1))
    assert _rows(t).is_contiguous()


@pytest.mark.gpu
def test_autograd_takes_a_gradient_at_an_odd_offset():
    import paper_2502_21079_amd as ad
    g = torch.Generator(device="cuda")
    g.manual_seed(2)
    q, k = (torch.randn(2, 3, n, 64, generator=g, device="cuda").to(torch.bfloat16) for n in (4, 9))
    flat = torch.zeros(X.numel() + 8, dtype=X.dtype, device="cuda")
    flat[1:1 + X.numel()] = torch.randn(X.numel(), generator=g, device="cuda").to(X.dtype)
    do, got = flat[1:1 + X.numel()].view(X.shape), []
    for grad in (do, do.clone()):
        x = q.clone().requires_grad_(True)
        ad.cross_attention(x, k, k).backward(grad)
        got.append(x.grad)
    assert torch.equal(*got) and got[0].abs().max() > 0
