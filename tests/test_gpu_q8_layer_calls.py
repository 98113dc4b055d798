"""dp.NormLinear on the GPU: refused calls, and the gradients that a caller has in hand."""
import numpy as np
import pytest
import torch

from oracle import q8 as plain

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    import paper_2506_16235_b200 as nsml
    from paper_2506_16235_b200 import dp


def rand(rows, cols, seed, scale=1.0, dtype=torch.bfloat16):
    return (torch.randn(rows, cols, generator=torch.Generator().manual_seed(seed)) * scale).to(dtype).cuda()


def layer(n, k, fill=0.0):
    bucket = torch.full((dp.NormLinear.size(n, k),), fill, device="cuda")
    return dp.NormLinear(rand(n, k, 2, k ** -0.5, torch.float32), torch.ones(k, device="cuda"), bucket), bucket


def test_a_refused_backward_can_be_made_again():
    m, n, k = 40, 24, 48
    x, dy, dh = rand(m, k, 3), rand(m, n, 4, 1e-3), rand(m, k, 5, 1e-3)
    block, bucket = layer(n, k, 0.5)
    block.forward(x)
    want = block.backward(dy, dh, zero_first=False)
    block, again = layer(n, k, 0.5)
    block.forward(x)
    for bad_dy, bad_dh in ((dy.half(), None), (dy[:, :16], dh), (dy, dh.half()), (dy, dh[:, 1:]), (dy, dh.cpu()), (dy.cpu(), dh)):
        with pytest.raises((TypeError, ValueError)):
            block.backward(bad_dy, bad_dh, zero_first=False)
        assert bool((again == 0.5).all())
    assert torch.equal(block.backward(dy, dh, zero_first=False), want) and torch.equal(again, bucket)
    with pytest.raises(RuntimeError, match="forward"):
        block.backward(dy, dh)


def f64(t):
    return t.detach().cpu().double().numpy()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("m,n,k", [(1, 5, 16), (37, 13, 40), (300, 257, 131), (6, 50257, 24)])
def test_a_gradient_laid_out_and_typed_like_the_layers_output(m, n, k, dtype):
    block, bucket = layer(n, k)
    x, residual = rand(m, k, 3, dtype=dtype), rand(m, k, 4, dtype=dtype)
    y, h = block.forward(x, residual)
    dy, dh = torch.empty_like(y).copy_(rand(m, n, 5, 1e-3, dtype)), torch.empty_like(h).copy_(rand(m, k, 6, 1e-3, dtype))
    assert y.dtype is h.dtype is dtype and y.is_contiguous()
    dx = block.backward(dy, dh)
    assert dx.dtype is dtype
    taken = f64(dy.bfloat16())  # float32 is rounded to bfloat16 for the products
    rstd, normed = plain.rms_norm(f64(h), f64(block.norm_weight), 1e-5)
    want_dx, want_dwn = plain.rms_norm_backward(taken @ f64(block.weight), f64(h), rstd, f64(block.norm_weight), f64(dh))
    # rows in 8 bits are off by at most 2^-7 of their largest value per element: less than 4 * 2^-7 of a Gaussian row's root mean square
    for got, want in ((dx, want_dx), (block.grad_weight, taken.T @ normed), (block.grad_norm_weight, want_dwn)):
        assert np.linalg.norm(f64(got) - want) <= 4 * 2.0 ** -7 * np.linalg.norm(want)


def test_the_copy_changes_nothing_but_the_layout():
    m, n, k = 70, 48, 40
    x, dy = rand(m, k, 3), rand(m, n, 4, 1e-3)
    shifted = torch.empty(m * (n + 3) + 1, dtype=torch.bfloat16, device="cuda")[1:].view(m, n + 3)[:, :n].copy_(dy)
    results = []
    for gradient in (dy, shifted):
        block, bucket = layer(n, k)
        block.forward(x)
        results.append((block.backward(gradient), bucket))
    assert torch.equal(results[0][0], results[1][0]) and torch.equal(results[0][1], results[1][1])
