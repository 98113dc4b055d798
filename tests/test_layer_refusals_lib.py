"""dp.NormLinear.backward: what it refuses it refuses before it has written or freed anything (no GPU: a stand-in takes the calls)."""
import pytest
import torch

from paper_2506_16235_b200 import dp

M, N, K = 4, 16, 32


class Calls:
    """Stands in for the library: notes which operator was called, in order."""

    def __init__(self, fail_at=None):
        self.made, self.fail_at = [], fail_at

    def __getattr__(self, name):
        def call(*args, **kwargs):
            if name == self.fail_at:
                raise RuntimeError("refused by the library")
            self.made.append(name)

        return call


def layer(fail_at=None):
    block = object.__new__(dp.NormLinear)
    block.nsml = Calls(fail_at)
    block.codes, block.scales = torch.zeros(N, K, dtype=torch.int8), torch.zeros(N)
    block.grad_weight, block.grad_norm_weight, block.norm_weight = torch.zeros(N, K), torch.zeros(K), torch.ones(K)
    block.workspaces, block.norm_workspace = (None, None, None), None
    block.kept = torch.zeros(M, K, dtype=torch.int8), torch.zeros(M), torch.zeros(M), (torch.zeros(M, K, dtype=torch.int8), torch.zeros(M))
    return block


def bf16(*shape):
    return torch.zeros(*shape, dtype=torch.bfloat16)


@pytest.mark.parametrize("error,dy,dh", [
    (TypeError, torch.zeros(M, N, dtype=torch.float16), None), (TypeError, torch.zeros(M, N, dtype=torch.int8), None),
    (ValueError, bf16(M, N + 8), None), (ValueError, bf16(M + 1, N), None), (ValueError, bf16(M * N), None), (ValueError, bf16(N, M).t(), None),
    (TypeError, bf16(M, N), torch.zeros(M, K, dtype=torch.float16)), (ValueError, bf16(M, N), bf16(M, K + 1)), (ValueError, bf16(M, N), bf16(M, N)),
    (ValueError, bf16(M, N), bf16(K, M).t()), (ValueError, bf16(M, N), bf16(1, K).expand(M, K)),
    (ValueError, torch.zeros(M, N, dtype=torch.bfloat16, device="meta"), None)])
def test_a_refused_gradient_leaves_everything_as_it_was(error, dy, dh):
    block = layer()
    kept = block.kept
    with pytest.raises(error):
        block.backward(dy, dh, zero_first=False)
    assert block.nsml.made == [] and block.kept is kept
    block.backward(bf16(M, N), bf16(M, K))  # the corrected call
    assert len(block.nsml.made) == 3 and block.kept is None


@pytest.mark.parametrize("fail_at", ["nsml_q8_matmul_grad_weight", "nsml_q8_matmul_grad_input", "nsml_q8_rms_norm_backward"])
def test_what_was_kept_outlives_a_call_that_fails(fail_at):
    block = layer(fail_at)
    with pytest.raises(RuntimeError, match="refused"):
        block.backward(bf16(M, N))
    block.nsml = Calls()
    block.backward(bf16(M, N))
    assert block.kept is None


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n,pad,lead", [(16, 0, 0), (16, 8, 0), (13, 0, 0), (16, 4, 0), (16, 0, 3), (1, 0, 1)])
def test_the_products_are_given_rows_on_16_byte_boundaries(n, pad, lead, dtype):
    buf = torch.randn(lead + 5 * (n + pad), generator=torch.Generator().manual_seed(1)).to(dtype)
    dy = buf[lead:].view(5, n + pad)[:, :n]
    got = dp.NormLinear._for_products(dy)
    assert got.dtype is torch.bfloat16 and torch.equal(got, dy.bfloat16()) and got.data_ptr() % 16 == 0 and got.stride(0) % 8 == 0
    assert (got is dy) == (dtype is torch.bfloat16 and dy.data_ptr() % 16 == 0 and dy.stride(0) % 8 == 0)
    with_graph = dy.float().requires_grad_()
    assert not dp.NormLinear._for_products(with_graph).requires_grad
