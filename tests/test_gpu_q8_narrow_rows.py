"""Gradient of the norm, rows that a warp takes by itself: aligned bfloat16 of 513 to 1024 columns, others of 129 to 256, with several
turns of a block.  u = 2^-24 is half a step of float32, relative; bfloat16's is 2^-8."""
import numpy as np
import pytest
import torch

from oracle import q8 as plain

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    import paper_2506_16235_b200 as nsml

U = 2.0 ** -24
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


def f64(t):
    return t.detach().cpu().double().numpy()


def rand(rows, cols, dtype, seed, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(rows, cols, generator=g) * scale * torch.exp2(torch.randint(-3, 4, (rows, 1), generator=g).float())).to(dtype).cuda()


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("weight_dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("cols,dtype", [(c, torch.bfloat16) for c in (129, 200, 249, 255, 512, 520, 640, 768, 1000, 1016, 1024)]
                         + [(c, torch.float32) for c in (129, 199, 255, 256, 512)])
def test_several_turns(cols, dtype, weight_dtype, packed):
    rows = 5003  # eight rows at a time in 296 blocks: three turns, the last one short
    weight = (1.0 + 0.1 * torch.randn(cols, generator=torch.Generator().manual_seed(1))).to(weight_dtype).cuda()
    h, dy, dh = rand(rows, cols, dtype, 1), rand(rows, cols, dtype, 2, 1e-3), rand(rows, cols, dtype, 3, 1e-3)
    h[4999] = 0.0
    rstd = nsml.nsml_q8_rms_norm(h, weight)[2]
    codes, scales = nsml.nsml_q8_pack(h)
    kept = f64(h) if not packed else plain.unpack(codes.cpu().numpy(), f64(scales))
    rows_kept = dict(codes=codes, scales=scales) if packed else dict(h=h)
    r, w, d = f64(rstd), f64(weight), f64(dy)
    for extra in (None, dh):
        dx, dweight = nsml.nsml_q8_rms_norm_backward(dy, weight, rstd, dh=extra, **rows_kept)
        want_dx, want_dw = plain.rms_norm_backward(d, kept, r, w, None if extra is None else f64(extra))
        n, g = np.abs(kept * r[:, None]), np.abs(d * w)
        c = np.mean(n * g, axis=1, keepdims=True)
        # n, g, n c, the difference, the product, the sum with dh: a rounding each; c: sums of up to 32 terms in float32
        tol = U * (6 * r[:, None] * (g + n * c) + 40 * r[:, None] * n * c + (0 if extra is None else np.abs(f64(extra))) + np.abs(want_dx))
        assert np.all(np.abs(f64(dx) - want_dx) <= 1.01 * (tol + HALF[dtype] * np.abs(want_dx)))
        # a rounding per row of a block's part, and per part
        assert np.all(np.abs(f64(dweight) - want_dw) <= (rows + 64) * U * np.sum(np.abs(d) * n, axis=0))
        again = nsml.nsml_q8_rms_norm_backward(dy, weight, rstd, dh=extra, **rows_kept)
        assert torch.equal(again[0], dx) and torch.equal(again[1], dweight)
