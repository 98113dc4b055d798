"""Training in 8 bits, what needs no GPU: the plain restatement against hand-worked values and differences, and every refusal
of the C entry points and of the binding."""
import ctypes
import math

import numpy as np
import pytest
import torch

import paper_2506_16235_b200 as nsml
from oracle import q8 as plain

lib, ARG, CAPACITY = nsml.lib, nsml.NSML_ERR_ARG, nsml.NSML_ERR_CAPACITY


# ---- the restatement -----------------------------------------------------------------------------------------------------
def test_scales_by_hand():
    assert plain.scale_of(127.0) == 1.0 and plain.scale_of(127.5) == 2.0 and plain.scale_of(128.0) == 2.0
    assert plain.scale_of(63.5) == 0.5 and plain.scale_of(1.0) == 2.0 ** -6 and plain.scale_of(0.0) == 0.0
    assert plain.scale_of(2.0 ** -149) == 2.0 ** -126 and plain.scale_of(3.4028234e38) == 2.0 ** 121
    assert math.isnan(plain.scale_of(math.inf)) and math.isnan(plain.scale_of(math.nan))


def test_codes_by_hand():
    codes, scales = plain.pack([[127.0, 126.5, -0.5, 0.5, 1.5], [0.0, 0.0, 0.0, 0.0, 0.0], [1.0, math.nan, 0.0, 0.0, 0.0]])
    assert codes.tolist() == [[127, 126, 0, 0, 2], [0] * 5, [0] * 5]
    assert scales[0] == 1.0 and scales[1] == 0.0 and math.isnan(scales[2])
    # a row's error is at most half a step, the step at most amax / 63.5
    x = np.random.default_rng(0).standard_normal((50, 40))
    codes, scales = plain.pack(x)
    assert np.all(np.abs(plain.unpack(codes, scales) - x) <= scales[:, None] / 2)
    assert np.all(scales * 63.5 <= np.abs(x).max(axis=1)) and np.abs(codes).max() <= 127


def test_round_bf16_is_torchs():
    x = np.random.default_rng(1).standard_normal(5000) * np.exp2(np.random.default_rng(2).integers(-140, 127, 5000))
    x = x.astype(np.float32)
    assert np.array_equal(plain.round_bf16(x), torch.from_numpy(x).bfloat16().double().numpy())


def test_norm_gradient_against_differences():
    rng = np.random.default_rng(3)
    h, w, c = rng.standard_normal((4, 9)), rng.standard_normal(9), rng.standard_normal((4, 9))
    rstd, _ = plain.rms_norm(h, w, 1e-3)
    dx, dw = plain.rms_norm_backward(c, h, rstd, w)
    loss = lambda hh, ww: np.sum(c * plain.rms_norm(hh, ww, 1e-3)[1])  # noqa: E731
    for i in np.ndindex(4, 9):
        d = np.zeros((4, 9))
        d[i] = 1e-6
        assert abs((loss(h + d, w) - loss(h - d, w)) / 2e-6 - dx[i]) < 1e-7
    for i in range(9):
        d = np.zeros(9)
        d[i] = 1e-6
        assert abs((loss(h, w + d) - loss(h, w - d)) / 2e-6 - dw[i]) < 1e-7


def test_product_gradients_against_differences():
    rng = np.random.default_rng(4)
    a, b = rng.integers(-127, 128, (5, 7)).astype(np.int8), rng.integers(-127, 128, (6, 7)).astype(np.int8)
    sa, sb, dy = np.exp2(rng.integers(-8, 0, 5)), np.exp2(rng.integers(-8, 0, 6)), rng.standard_normal((5, 6))
    x, w = plain.unpack(a, sa), plain.unpack(b, sb)
    assert np.allclose(plain.matmul(a, sa, b, sb), x @ w.T, rtol=1e-14)
    dx, dw = plain.matmul_grad_input(dy, b, sb), plain.matmul_grad_weight(dy, a, sa)
    step = 1e-5
    for i in ((0, 0), (4, 6), (2, 3)):
        d = np.zeros_like(x)
        d[i] = step
        assert abs(np.sum(dy * ((x + d) @ w.T - (x - d) @ w.T)) / (2 * step) - dx[i]) < 1e-6
    for i in ((0, 0), (5, 6), (2, 3)):
        d = np.zeros_like(w)
        d[i] = step
        assert abs(np.sum(dy * (x @ (w + d).T - x @ (w - d).T)) / (2 * step) - dw[i]) < 1e-6


# ---- refusals: decided before anything is launched ----------------------------------------------------------------------
@pytest.fixture(scope="module")
def at():
    """An aligned address that stands in for device memory; nothing reads it."""
    at.buf = (ctypes.c_char * 8192)()
    return (ctypes.addressof(at.buf) + 255) // 256 * 256


def test_row_bytes():
    assert [nsml.nsml_q8_row_bytes(c) for c in (0, -1, 1, 16, 17, 2147483632, 2147483633)] == [0, 0, 16, 16, 32, 2147483632, 0]


def test_the_norms_workspace_never_shrinks_with_the_width():
    sizes = [int(lib.nsml_q8_rms_norm_backward_workspace_bytes(c)) for c in range(1, 32769)]
    assert sizes == sorted(sizes) and sizes[0] >= 256


def test_pack_and_unpack_refuse(at):
    good = dict(x=at, rows=4, cols=20, ldx=20, dtype=0, codes=at, ldq=32, scales=at)

    def pack(**kw):
        a = {**good, **kw}
        return lib.nsml_q8_pack(a["x"], a["rows"], a["cols"], a["ldx"], a["dtype"], a["codes"], a["ldq"], a["scales"], None)

    def unpack(**kw):
        a = {**good, **kw}
        return lib.nsml_q8_unpack(a["codes"], a["ldq"], a["scales"], a["rows"], a["cols"], a["x"], a["ldx"], a["dtype"], None)

    for call in (pack, unpack):
        for bad in (dict(x=None), dict(codes=None), dict(scales=None), dict(rows=-1), dict(rows=1 << 31), dict(cols=0), dict(cols=1 << 31), dict(dtype=2),
                    dict(dtype=-1), dict(ldx=19), dict(ldq=31), dict(ldq=16), dict(codes=at + 8), dict(x=at + 2), dict(scales=at + 2)):
            assert call(**bad) == ARG, bad
        assert call(rows=0, x=None, codes=None, scales=None) == nsml.NSML_OK


def test_norm_refuses(at):
    good = dict(x=at, ldx=20, res=None, ldr=0, rows=4, cols=20, dtype=0, w=at, wd=0, eps=1e-5, h=None, ldh=0, codes=at, ldq=32, scales=at, rstd=None)

    def norm(**kw):
        a = {**good, **kw}
        return lib.nsml_q8_rms_norm(a["x"], a["ldx"], a["res"], a["ldr"], a["rows"], a["cols"], a["dtype"], a["w"], a["wd"], a["eps"], a["h"], a["ldh"],
                                    a["codes"], a["ldq"], a["scales"], a["rstd"], None)

    for bad in (dict(x=None), dict(w=None), dict(codes=None), dict(scales=None), dict(rows=-1), dict(cols=0), dict(cols=32769), dict(dtype=2), dict(wd=2),
                dict(eps=0.0), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(ldx=19), dict(res=at, ldr=3), dict(h=at, ldh=3),
                dict(ldq=24), dict(rstd=at + 1), dict(w=at + 2), dict(res=at + 2, ldr=20)):
        assert norm(**bad) == ARG, bad
    assert norm(rows=0) == nsml.NSML_OK


def test_norm_backward_refuses(at):
    need = int(lib.nsml_q8_rms_norm_backward_workspace_bytes(20))
    assert need > 0 and lib.nsml_q8_rms_norm_backward_workspace_bytes(0) == 0 == lib.nsml_q8_rms_norm_backward_workspace_bytes(32769)
    good = dict(dy=at, ldy=20, dh=None, lddh=0, h=at, ldh=20, codes=None, ldq=0, scales=None, rstd=at, rows=4, cols=20, dtype=0, w=at, wd=0, dx=at,
                lddx=20, dw=at, dwd=0, zero=1, ws=at, wsb=need)

    def back(**kw):
        a = {**good, **kw}
        return lib.nsml_q8_rms_norm_backward(a["dy"], a["ldy"], a["dh"], a["lddh"], a["h"], a["ldh"], a["codes"], a["ldq"], a["scales"], a["rstd"], a["rows"],
                                             a["cols"], a["dtype"], a["w"], a["wd"], a["dx"], a["lddx"], a["dw"], a["dwd"], a["zero"], a["ws"], a["wsb"], None)

    for bad in (dict(dy=None), dict(h=None), dict(codes=at, scales=at, ldq=32), dict(h=None, codes=at, ldq=32), dict(rstd=None), dict(w=None), dict(dx=None),
                dict(ws=None), dict(ws=at + 16), dict(rows=-1), dict(cols=0), dict(cols=32769), dict(dtype=2), dict(wd=3), dict(dwd=2), dict(ldy=1),
                dict(lddx=1), dict(ldh=1), dict(dh=at, lddh=1), dict(h=None, codes=at + 8, ldq=32, scales=at), dict(dw=at + 2)):
        assert back(**bad) == ARG, bad
    assert back(wsb=need - 1) == CAPACITY


def test_products_refuse(at):
    good = dict(a=at, lda=32, sa=at, b=at, ldb=32, sb=at, dy=at, ldy=16, m=4, n=9, k=20, out=at, ldo=20, dtype=0, ws=at, wsb=256)

    def forward(**kw):
        a = {**good, **kw}
        return lib.nsml_q8_matmul(a["a"], a["lda"], a["sa"], a["b"], a["ldb"], a["sb"], a["m"], a["n"], a["k"], a["out"], a["ldo"], a["dtype"], a["ws"], a["wsb"], None)

    def grad_input(**kw):
        a = {**good, **kw}
        return lib.nsml_q8_matmul_grad_input(a["dy"], a["ldy"], a["b"], a["ldb"], a["sb"], a["m"], a["n"], a["k"], a["out"], a["ldo"], a["dtype"], a["ws"], a["wsb"], None)

    def grad_weight(**kw):
        a = {**good, **kw}
        return lib.nsml_q8_matmul_grad_weight(a["dy"], a["ldy"], a["a"], a["lda"], a["sa"], a["m"], a["n"], a["k"], a["out"], a["ldo"], a["dtype"], 1, a["ws"], a["wsb"], None)

    for call in (forward, grad_input, grad_weight):
        for bad in (dict(m=-1), dict(m=1 << 31), dict(n=0), dict(n=1 << 31), dict(k=0), dict(k=1 << 31), dict(out=None), dict(out=at + 2), dict(dtype=2),
                    dict(ws=None), dict(ws=at + 16), dict(ldo=3)):
            assert call(**bad) == ARG, (call.__name__, bad)
        assert call(wsb=255) == CAPACITY
    for call in (forward, grad_weight):
        for bad in (dict(a=None), dict(sa=None), dict(a=at + 8), dict(lda=16), dict(lda=40), dict(sa=at + 2)):
            assert call(**bad) == ARG, (call.__name__, bad)
    for call in (forward, grad_input):
        for bad in (dict(b=None), dict(sb=None), dict(b=at + 8), dict(ldb=16), dict(ldb=40), dict(sb=at + 2)):
            assert call(**bad) == ARG, (call.__name__, bad)
    for call in (grad_input, grad_weight):
        for bad in (dict(dy=None), dict(dy=at + 8), dict(ldy=8), dict(ldy=12)):
            assert call(**bad) == ARG, (call.__name__, bad)
    assert forward(k=131072, lda=131072, ldb=131072) == ARG  # 128 * 128 * 131072 = 2^31
    assert grad_input(n=4194305, ldy=4194312, ldb=32) == ARG == grad_weight(m=4194305)  # longest sums of the gradients
    assert forward(m=0, a=None, out=None) == nsml.NSML_OK == grad_input(m=0, dy=None, out=None)


def test_the_binding_refuses_tensors_of_another_device_shape_or_type():
    x, codes, scales = torch.zeros(3, 20), torch.zeros(3, 32, dtype=torch.int8)[:, :20], torch.zeros(3)
    dy = torch.zeros(3, 8, dtype=torch.bfloat16)
    for call in (lambda: nsml.nsml_q8_pack(x), lambda: nsml.nsml_q8_unpack(codes, scales), lambda: nsml.nsml_q8_rms_norm(x, torch.ones(20)),
                 lambda: nsml.nsml_q8_rms_norm_backward(x, torch.ones(20), scales, h=x), lambda: nsml.nsml_q8_matmul(codes, scales, codes, scales),
                 lambda: nsml.nsml_q8_matmul_grad_input(dy, codes, scales), lambda: nsml.nsml_q8_matmul_grad_weight(dy, codes, scales)):
        with pytest.raises(ValueError, match="current CUDA device"):
            call()
    with pytest.raises(ValueError, match="2-D"):
        nsml.nsml_q8_pack(torch.zeros(4))
    with pytest.raises(ValueError, match="contiguous rows"):
        nsml.nsml_q8_pack(torch.zeros(4, 6).t())
    with pytest.raises(TypeError, match="int8"):
        nsml.nsml_q8_unpack(torch.zeros(3, 4), scales)
    with pytest.raises(TypeError, match="bfloat16"):
        nsml.nsml_q8_matmul_grad_input(x, codes, scales)
