"""More refusals of the 8-bit operators' entry points, decided before anything is launched (no GPU)."""
import ctypes

import paper_2506_16235_b200 as nsml

lib, ARG, CAPACITY = nsml.lib, nsml.NSML_ERR_ARG, nsml.NSML_ERR_CAPACITY
BUFFER = (ctypes.c_char * 8192)()
AT = (ctypes.addressof(BUFFER) + 255) // 256 * 256  # an aligned address that stands in for device memory


def test_selftest_of_the_waits_refuses():
    wait = lib.nsml_selftest_q8_bounded_wait
    assert wait(None, 256, 1, None) == wait(AT + 16, 256, 1, None) == wait(AT, 256, -1, None) == wait(AT, 256, 33, None) == ARG
    assert wait(AT, 255, 1, None) == CAPACITY


def test_products_without_tokens_refuse_a_workspace_that_cannot_hold_a_status():
    def forward(ws, size):
        return lib.nsml_q8_matmul(None, 0, None, AT, 32, AT, 0, 9, 20, None, 0, 0, ws, size, None)

    def grad_input(ws, size):
        return lib.nsml_q8_matmul_grad_input(None, 0, AT, 32, AT, 0, 9, 20, None, 0, 0, ws, size, None)

    for call in (forward, grad_input):
        assert call(None, 256) == call(AT + 16, 256) == ARG and call(AT, 255) == CAPACITY
