"""The bounded waits inside the 8-bit products: a warp that waits as a whole gives up as a whole, and products that follow are right."""
import pytest
import torch

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    import paper_2506_16235_b200 as nsml


@pytest.mark.parametrize("lanes", [0, 1, 2, 17, 31, 32])
def test_lanes_whose_waits_end_differently_give_up_together(lanes):
    ws = nsml.alloc_bytes(nsml.NSML_Q8_MATMUL_WORKSPACE_BYTES, "cuda").fill_(0x55)
    stream = torch.cuda.current_stream().cuda_stream
    for _ in range(3):
        assert nsml.lib.nsml_selftest_q8_bounded_wait(ws.data_ptr(), ws.numel(), lanes, stream) == 0
        assert nsml.nsml_last_status(ws) == (nsml.NSML_ERR_TIMEOUT if lanes else nsml.NSML_OK)


def test_a_product_after_a_wait_that_ran_out():
    ws = nsml.alloc_bytes(nsml.NSML_Q8_MATMUL_WORKSPACE_BYTES, "cuda")
    assert nsml.lib.nsml_selftest_q8_bounded_wait(ws.data_ptr(), ws.numel(), 5, torch.cuda.current_stream().cuda_stream) == 0
    codes, scales = nsml.nsml_q8_pack(torch.randn(300, 400, generator=torch.Generator().manual_seed(1)).cuda())
    out = nsml.nsml_q8_matmul(codes, scales, codes, scales, dtype=torch.float32, workspace=ws)
    assert nsml.nsml_last_status(ws) == nsml.NSML_OK
    x = codes.double() * scales.double()[:, None]
    # the integer sum converted to float32, then two multiplies by powers of two: one rounding
    assert torch.equal(out, (x @ x.T).float())
