"""8-bit products without tokens: the workspace's status is that of this call, whatever was there."""
import pytest
import torch

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    import paper_2506_16235_b200 as nsml
    from paper_2506_16235_b200 import dp

N, K = 24, 40


def empty():
    codes, scales = nsml.nsml_q8_pack(torch.randn(N, K, generator=torch.Generator().manual_seed(1)).cuda())
    return codes, scales, torch.empty(0, N, dtype=torch.bfloat16, device="cuda")


@pytest.mark.parametrize("zero_first", [True, False])
def test_status_of_products_without_tokens(zero_first):
    codes, scales, dy = empty()
    dw = torch.full((N, K), 2.0, device="cuda")
    for call in (lambda ws: nsml.nsml_q8_matmul(codes[:0], scales[:0], codes, scales, workspace=ws),
                 lambda ws: nsml.nsml_q8_matmul_grad_input(dy, codes, scales, workspace=ws),
                 lambda ws: nsml.nsml_q8_matmul_grad_weight(dy, codes[:0], scales[:0], dw=dw, zero_first=zero_first, workspace=ws)):
        ws = nsml.alloc_bytes(nsml.NSML_Q8_MATMUL_WORKSPACE_BYTES, "cuda").fill_(0x55)
        call(ws)
        assert nsml.nsml_last_status(ws) == nsml.NSML_OK
    assert bool((dw == (0.0 if zero_first else 2.0)).all())


def test_a_layers_status_after_an_empty_batch():
    bucket = torch.full((dp.NormLinear.size(N, K),), 3.0, device="cuda")
    block = dp.NormLinear(torch.randn(N, K, generator=torch.Generator().manual_seed(1)).cuda(), torch.ones(K, device="cuda"), bucket)
    for ws in (*block.workspaces, block.norm_workspace):
        ws.fill_(0x55)
    x = torch.empty(0, K, dtype=torch.bfloat16, device="cuda")
    y, h = block.forward(x)
    dx = block.backward(torch.empty(0, N, dtype=torch.bfloat16, device="cuda"))
    assert y.shape == (0, N) and dx.shape == (0, K) and bool((bucket == 0.0).all())
    assert [nsml.nsml_last_status(ws) for ws in (*block.workspaces, block.norm_workspace)] == [nsml.NSML_OK] * 4


def test_a_call_without_tokens_is_captured():
    codes, scales, dy = empty()
    ws, graph = nsml.alloc_bytes(nsml.NSML_Q8_MATMUL_WORKSPACE_BYTES, "cuda"), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        nsml.nsml_q8_matmul(codes[:0], scales[:0], codes, scales, workspace=ws)
    ws.fill_(0x55)
    graph.replay()
    assert nsml.nsml_last_status(ws) == nsml.NSML_OK
