"""The norm's reciprocal root is worked out in 64 bits and rounded to float32 once."""
import math
from decimal import Decimal, localcontext

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    import paper_2506_16235_b200 as nsml


def rstd_of(x, eps):
    return nsml.nsml_q8_rms_norm(x, torch.ones(x.shape[1], device="cuda"), eps)[2].cpu().numpy()


# float32 values whose 1 / sqrt(x^2 + eps) lies within 2^-46.5 of a border between two float32 (and no nearer than 2^-51)
BORDERS = {-20: (0x400E4F05, 0x3FD86961, 0x40800000, 0x3FBC0615, 0x3F7FFFED, 0x3FFFFFFB, 0x4116A135, 0x40D5BF2A, 0x3F84ADE0, 0x3EADF0E8, 0x3F11989F,
                 0x3FF220A0, 0x404F15B8, 0x40E2E8AC),
           -10: (0x40E19078, 0x3F1CD24D, 0x3F6D02C2, 0x401A5C6E, 0x402BB31A, 0x3EC7D04C, 0x3EAADE79, 0x3FBDC78F, 0x3FEEEB12, 0x412DF0E8, 0x40690619,
                 0x3EE16FC2, 0x3FC518B0),
           -5: (0x40FFF000, 0x40AD78F6, 0x3F33FBEC, 0x3F4EE258, 0x3EAFF877, 0x3E88214D, 0x417676AC, 0x3E889633, 0x40E68F19, 0x41515DB6, 0x3ECF7BA3)}


def nearest(root):
    """The float32 nearest to a decimal."""
    f = np.float32(float(root))
    return min((np.nextafter(f, np.float32(0)), f, np.nextafter(f, np.float32(math.inf))), key=lambda c: abs(Decimal(float(c)) - root))


@pytest.mark.parametrize("power", BORDERS)
def test_the_root_is_rounded_once(power):
    # the square and the sum are exact in 64 bits here; the root's error there is at most a few units of 2^-53
    x = np.array(BORDERS[power], dtype=np.uint32).view(np.float32)
    with localcontext() as ctx:
        ctx.prec = 60
        want = np.array([nearest(1 / (Decimal(float(v)) ** 2 + Decimal(2.0 ** power)).sqrt()) for v in x], dtype=np.float32)
    assert np.array_equal(rstd_of(torch.from_numpy(x).cuda()[:, None], 2.0 ** power), want)
