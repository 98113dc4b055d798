"""dp.NormLinear on the GPU: refused calls, and the gradients that a caller has in hand."""
import pytest
import torch

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
