"""dp.NormLinear on the GPU: the layer's forward and backward pass against plain 64-bit NumPy, micro-batches, and a step with the
gradient exchange behind it."""
import numpy as np
import pytest
import torch

from oracle import q8 as plain

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    import paper_2506_16235_b200 as nsml
    from paper_2506_16235_b200 import dp


def f64(t):
    return t.detach().cpu().double().numpy()


def rand(rows, cols, seed, scale=1.0, dtype=torch.bfloat16):
    return (torch.randn(rows, cols, generator=torch.Generator().manual_seed(seed)) * scale).to(dtype).cuda()


def layer(n, k, bucket_dtype=torch.float32, offset=3):
    bucket = torch.full((offset + dp.NormLinear.size(n, k) + 2,), 9.0, dtype=bucket_dtype, device="cuda")
    norm_weight = (1.0 + 0.1 * torch.randn(k, generator=torch.Generator().manual_seed(1))).cuda()
    return dp.NormLinear(rand(n, k, 2, k ** -0.5, torch.float32), norm_weight, bucket, offset), bucket


def near(got, want, by=0.03):
    """Rows in 8 bits are off by at most 2^-7 of their largest value per element; the products of Gaussian rows by less than
    that over their root mean square, 4 * 2^-7, relative to the result."""
    assert np.linalg.norm(f64(got) - want) <= by * np.linalg.norm(want)


@pytest.mark.parametrize("m,n,k", [(1, 8, 16), (5, 24, 100), (300, 256, 384), (513, 136, 771)])
def test_layer(m, n, k):
    block, bucket = layer(n, k)
    x, residual, dy, dh = rand(m, k, 3), rand(m, k, 4), rand(m, n, 5, 1e-3), rand(m, k, 6, 1e-3)
    y, h = block.forward(x, residual)
    dx = block.backward(dy, dh)
    kept = f64((x.float() + residual.float()).bfloat16())
    assert np.array_equal(f64(h), kept)
    rstd, normed = plain.rms_norm(kept, f64(block.norm_weight), 1e-5)
    near(y, normed @ f64(block.weight).T)
    want_dx, want_dwn = plain.rms_norm_backward(f64(dy) @ f64(block.weight), kept, rstd, f64(block.norm_weight), f64(dh))
    near(dx, want_dx)
    near(block.grad_weight, f64(dy).T @ normed)
    near(block.grad_norm_weight, want_dwn)
    assert bool((bucket[:3] == 9.0).all()) and bool((bucket[-2:] == 9.0).all())


@pytest.mark.parametrize("bucket_dtype", [torch.float32, torch.bfloat16])
def test_micro_batches_add_up(bucket_dtype):
    m, n, k = 96, 64, 80
    block, _ = layer(n, k, bucket_dtype)
    x, dy = rand(2 * m, k, 3), rand(2 * m, n, 5, 1e-3)
    parts = []
    for i in range(2):
        block.forward(x[i * m:(i + 1) * m])
        block.backward(dy[i * m:(i + 1) * m])
        parts.append((f64(block.grad_weight), f64(block.grad_norm_weight)))
    for i in range(2):
        block.forward(x[i * m:(i + 1) * m])
        block.backward(dy[i * m:(i + 1) * m], zero_first=i == 0)
    half = torch.finfo(bucket_dtype).eps / 2
    for got, a, b in zip((block.grad_weight, block.grad_norm_weight), *parts):
        # the parts are reproducible; the second one has been rounded on its own, the sum of both once
        assert np.all(np.abs(f64(got) - (a + b)) <= 2.1 * half * (np.abs(a) + np.abs(b)))


def test_layer_and_exchange():
    m, n, k = 200, 128, 96
    block, bucket = layer(n, k, offset=0)
    exchange, dense = dp.GradientExchange(bucket.numel(), bits=8, ratio_init=0.1, ratio_max=0.1), torch.empty_like(bucket)
    x, dy = rand(m, k, 3), rand(m, n, 5, 1e-3)
    for _ in range(2):
        block.forward(x)
        block.backward(dy)
        exchange.step(bucket, dense)
        kept = nsml.nsml_k_of(bucket.numel(), exchange.ratio)
        assert int((dense != 0).sum()) <= kept
        top = bucket.abs().topk(kept // 2).indices
        # a code of 127 steps of the block's largest value: half a step each
        assert bool(((dense[top] - bucket[top]).abs() <= bucket.abs().max() / 254 * 1.001).all())
        block.weight -= 0.1 * block.grad_weight
        block.pack()


def test_refusals():
    block, bucket = layer(16, 32)
    with pytest.raises(RuntimeError, match="forward"):
        block.backward(rand(4, 16, 1))
    with pytest.raises(ValueError, match="room"):
        dp.NormLinear(block.weight, block.norm_weight, bucket, offset=40)
    block.forward(rand(4, 32, 1))
    block.backward(rand(4, 16, 1))
    with pytest.raises(RuntimeError, match="forward"):  # what was kept is gone
        block.backward(rand(4, 16, 1))


def test_status_of_every_product():
    block, _ = layer(16, 32)
    for ws in (*block.workspaces, block.norm_workspace):
        ws.fill_(0x55)
    block.forward(rand(4, 32, 1))
    block.backward(rand(4, 16, 1))
    assert [nsml.nsml_last_status(ws) for ws in (*block.workspaces, block.norm_workspace)] == [0, 0, 0, 0]
