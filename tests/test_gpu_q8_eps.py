"""The norm's eps is held in 64 bits."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    import paper_2506_16235_b200 as nsml


def rstd_of(x, eps):
    return nsml.nsml_q8_rms_norm(x, torch.ones(x.shape[1], device="cuda"), eps)[2].cpu().numpy()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("eps", [1e-3, 1e-5, 1e-6, 1e-8, 1e-12, 0.1, 0.3, 7.0])
def test_eps_is_held_in_64_bits(eps, dtype):
    # rows of zeros: rstd = 1 / sqrt(eps), rounded once
    for cols in (1, 8, 1000, 5000):
        assert np.array_equal(rstd_of(torch.zeros(3, cols, dtype=dtype, device="cuda"), eps), np.full(3, np.float32(1.0 / math.sqrt(eps))))
