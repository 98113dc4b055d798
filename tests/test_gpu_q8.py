"""Training in 8 bits on the GPU against plain 64-bit NumPy (oracle/q8.py): sizes from one to a few tiles, odd ones, strides,
rows of zeros, non-finite values, and the operators in a run as a training step makes them.

Tolerances.  u = 2^-24 is half a step of float32, relative; bfloat16's is 2^-8.  Sums of float32 products on the tensor cores
may round every addition by a whole step: depth * 2u * sum |terms|."""
import numpy as np
import pytest
import torch

from oracle import q8 as plain

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    import paper_2506_16235_b200 as nsml

U = 2.0 ** -24
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
TYPES = [torch.float32, torch.bfloat16]
WIDTHS = [1, 7, 8, 64, 255, 256, 257, 513, 1000, 1024, 2047, 2048, 2049, 4100, 8192, 8200, 16384, 16390, 32768]


def f64(t):
    return t.detach().cpu().double().numpy()


def rand(rows, cols, dtype, seed, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, cols, generator=g) * scale
    x *= torch.exp2(torch.randint(-3, 4, (rows, 1), generator=g).float())
    return x.to(dtype).cuda()


def strided(t, pad, lead=0):
    """The same values, rows `pad` elements further apart, starting `lead` elements into the buffer."""
    rows, cols = t.shape
    buf = torch.full((rows * (cols + pad) + lead,), 7.0, dtype=t.dtype, device=t.device)
    view = buf[lead:].view(rows, cols + pad)[:, :cols]
    view.copy_(t)
    return view


def codes_of(codes):
    return codes.cpu().numpy()


def check_pack(x, codes, scales):
    want_codes, want_scales = plain.pack(f64(x))
    assert np.array_equal(f64(scales), want_scales, equal_nan=True)
    assert np.array_equal(codes_of(codes), want_codes)


# ---- store and restore ---------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols", WIDTHS + [32776, 50257])
def test_pack_and_unpack(cols, dtype):
    x = rand(5, cols, dtype, cols)
    codes, scales = nsml.nsml_q8_pack(x)
    check_pack(x, codes, scales)
    for out in TYPES:
        back = nsml.nsml_q8_unpack(codes, scales, dtype=out)
        assert back.dtype == out
        assert np.array_equal(f64(back), plain.unpack(codes_of(codes), f64(scales)))  # exact in both types


@pytest.mark.parametrize("rows", [1, 2, 3, 4, 5, 127, 1000])
def test_pack_rows(rows):
    x = rand(rows, 96, torch.bfloat16, rows)
    check_pack(x, *nsml.nsml_q8_pack(x))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("pad,lead", [(8, 8), (3, 0), (0, 1), (1, 3)])
def test_pack_strides_and_alignment(pad, lead, dtype):
    x = strided(rand(9, 333, dtype, 3), pad, lead)
    codes, scales = nsml.nsml_q8_pack(x)
    check_pack(x, codes, scales)
    out = strided(torch.zeros(9, 333, dtype=dtype, device="cuda"), pad, lead)
    nsml.nsml_q8_unpack(codes, scales, out=out)
    assert np.array_equal(f64(out), plain.unpack(codes_of(codes), f64(scales)))


def test_pack_leaves_what_lies_between_and_behind_the_rows():
    x = rand(6, 77, torch.float32, 1)
    buf = torch.full((8, 96), 55, dtype=torch.int8, device="cuda")
    scales = torch.full((8,), 3.0, device="cuda")
    nsml.nsml_q8_pack(x, codes=buf[:6, :77], scales=scales[:6])
    check_pack(x, buf[:6, :77], scales[:6])
    assert bool((buf[:, 77:] == 55).all()) and bool((buf[6:] == 55).all()) and bool((scales[6:] == 3.0).all())
    out = torch.full((8, 80), 9.0, device="cuda")
    nsml.nsml_q8_unpack(buf[:6, :77], scales[:6], out=out[:6, :77])
    assert bool((out[6:] == 9.0).all()) and bool((out[:, 77:] == 9.0).all())


def test_pack_extreme_magnitudes():
    big, tiny = 3.4028234e38, 2.0 ** -149
    rows = [[0.0, -0.0, 0.0], [tiny, -tiny, 0.0], [2.0 ** -126, 2.0 ** -127, -(2.0 ** -128)], [big, -big, 1.0],
            [127.0, 126.5, -0.5], [127.0 * 2.0 ** 60, 63.5 * 2.0 ** 60, 1.0], [127.0000076, 1.0, 0.5], [1.0, 2.0 ** -20, -1.0],
            [127.0 * 2.0 ** -126, 2.0 ** -126, 2.0 ** -127], [63.5 * 2.0 ** -126, 1.5 * 2.0 ** -126, 2.5 * 2.0 ** -126]]
    x = torch.tensor(rows, dtype=torch.float32, device="cuda")
    codes, scales = nsml.nsml_q8_pack(x)
    check_pack(x, codes, scales)
    for out in TYPES:
        assert np.array_equal(f64(nsml.nsml_q8_unpack(codes, scales, dtype=out)), plain.unpack(codes_of(codes), f64(scales)))


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("cols", [5, 3000])
def test_a_row_that_is_not_finite_has_scale_nan_and_the_others_are_untouched(bad, cols):
    for dtype in TYPES:
        x = rand(4, cols, dtype, 2)
        x[1, cols - 1] = bad
        codes, scales = nsml.nsml_q8_pack(x)
        check_pack(x, codes, scales)
        assert bool(torch.isnan(scales[1])) and bool(torch.isnan(nsml.nsml_q8_unpack(codes, scales)[1]).all())


def test_no_rows():
    x = torch.empty(0, 64, device="cuda")
    codes, scales = nsml.nsml_q8_pack(x)
    assert codes.shape == (0, 64) and nsml.nsml_q8_unpack(codes, scales).shape == (0, 64)
    codes, scales, rstd, h = nsml.nsml_q8_rms_norm(x, torch.ones(64, device="cuda"))
    dweight = torch.full((64,), 4.0, device="cuda")
    nsml.nsml_q8_rms_norm_backward(x, torch.ones(64, device="cuda"), rstd, h=h, dweight=dweight, zero_first=False)
    assert bool((dweight == 4.0).all())
    dx, dweight = nsml.nsml_q8_rms_norm_backward(x, torch.ones(64, device="cuda"), rstd, h=h)
    assert dx.shape == (0, 64) and bool((dweight == 0).all())
    b, b_scales = nsml.nsml_q8_pack(rand(40, 64, torch.float32, 1))
    assert nsml.nsml_q8_matmul(codes, scales, b, b_scales).shape == (0, 40)
    dy = torch.empty(0, 40, dtype=torch.bfloat16, device="cuda")
    assert nsml.nsml_q8_matmul_grad_input(dy, b, b_scales).shape == (0, 64)
    assert bool((nsml.nsml_q8_matmul_grad_weight(dy, codes, scales) == 0).all())
    kept = torch.full((40, 64), 2.0, device="cuda")
    nsml.nsml_q8_matmul_grad_weight(dy, codes, scales, dw=kept, zero_first=False)
    assert bool((kept == 2.0).all())


# ---- norm ----------------------------------------------------------------------------------------------------------------
def check_norm(x, residual, weight, eps, codes, scales, rstd, h):
    kept = f64(x) if residual is None else f64((x.float() + residual.float()).to(x.dtype))
    assert np.array_equal(f64(h), kept)
    want_rstd, _ = plain.rms_norm(kept, f64(weight), np.float32(eps).astype(np.float64))
    # (the 64-bit sum may differ in its last bits: a thousandth of a step besides the rounding)
    assert np.all(np.abs(f64(rstd) - want_rstd) <= 1.001 * U * want_rstd)
    # with rstd as it is, two float32 multiplies and the format's own rounding: equal
    y = (kept.astype(np.float32) * rstd.cpu().numpy()[:, None]) * f64(weight).astype(np.float32)
    want_codes, want_scales = plain.pack(y)
    assert np.array_equal(f64(scales), want_scales) and np.array_equal(codes_of(codes), want_codes)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols", WIDTHS)
def test_norm(cols, dtype):
    weight = (1.0 + 0.1 * torch.randn(cols, generator=torch.Generator().manual_seed(1))).to(dtype).cuda()
    for residual in (None, rand(5, cols, dtype, cols + 1)):
        x = rand(5, cols, dtype, cols)
        x[3] = 0.0
        if residual is not None:
            residual[3] = 0.0
        codes, scales, rstd, h = nsml.nsml_q8_rms_norm(x, weight, 1e-5, residual=residual)
        check_norm(x, residual, weight, 1e-5, codes, scales, rstd, h)
        assert float(scales[3]) == 0.0


@pytest.mark.parametrize("weight_dtype", TYPES)
def test_norm_in_place_and_with_strides(weight_dtype):
    weight = (1.0 + 0.1 * torch.randn(331, generator=torch.Generator().manual_seed(1))).to(weight_dtype).cuda()
    for dtype in TYPES:
        for pad, lead in ((0, 0), (3, 1), (8, 0)):
            x, r = strided(rand(7, 331, dtype, 5), pad, lead), strided(rand(7, 331, dtype, 6), pad, lead)
            want = [t.clone() for t in nsml.nsml_q8_rms_norm(x, weight, 1e-3, residual=r)]
            check_norm(x, r, weight, 1e-3, *want)
            for into in (x, r):
                a, b = x.clone(), r.clone()
                target = a if into is x else b
                got = nsml.nsml_q8_rms_norm(a, weight, 1e-3, residual=b, h=target)
                assert got[3] is target
                assert all(torch.equal(p, q) for p, q in zip(got, want))


def test_norm_of_a_row_that_is_not_finite():
    x = rand(3, 100, torch.bfloat16, 1)
    x[0, 3], x[2, 99] = float("inf"), float("nan")
    codes, scales, rstd, h = nsml.nsml_q8_rms_norm(x, torch.ones(100, device="cuda"))
    assert torch.isnan(scales).tolist() == [True, False, True]
    assert bool((codes[0] == 0).all()) and bool((codes[2] == 0).all())
    check_norm(x[1:2], None, torch.ones(100), 1e-5, codes[1:2], scales[1:2], rstd[1:2], h[1:2])


def norm_grad_tolerance(dy, h, rstd, weight, dh, dx, dtype, rows):
    n, g = np.abs(h * rstd[:, None]), np.abs(dy * weight)
    c = np.mean(n * g, axis=1, keepdims=True)
    # n, g, n c, the difference, the product, the sum with dh: a rounding each; c: sums of up to 32 terms in float32
    tol = U * (6 * rstd[:, None] * (g + n * c) + 40 * rstd[:, None] * n * c + (0 if dh is None else np.abs(dh)) + np.abs(dx))
    return tol * 1.01 + HALF[dtype] * np.abs(dx) * 1.01, (rows + 64) * U * np.sum(np.abs(dy) * n, axis=0)


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols", WIDTHS)
def test_norm_backward(cols, dtype, packed):
    rows = 6
    weight = (1.0 + 0.1 * torch.randn(cols, generator=torch.Generator().manual_seed(1))).to(dtype).cuda()
    h, dy, dh = rand(rows, cols, dtype, 1), rand(rows, cols, dtype, 2, 1e-3), rand(rows, cols, dtype, 3, 1e-3)
    h[4] = 0.0
    rstd = nsml.nsml_q8_rms_norm(h, weight)[2]
    codes, scales = nsml.nsml_q8_pack(h)
    kept = f64(h) if not packed else plain.unpack(codes_of(codes), f64(scales))
    for extra in (None, dh):
        dx, dweight = nsml.nsml_q8_rms_norm_backward(dy, weight, rstd, dh=extra, **(dict(codes=codes, scales=scales) if packed else dict(h=h)))
        want_dx, want_dw = plain.rms_norm_backward(f64(dy), kept, f64(rstd), f64(weight), None if extra is None else f64(extra))
        tol, tol_w = norm_grad_tolerance(f64(dy), kept, f64(rstd), f64(weight), None if extra is None else f64(extra), want_dx, dtype, rows)
        assert np.all(np.abs(f64(dx) - want_dx) <= tol)
        assert np.all(np.abs(f64(dweight) - want_dw) <= tol_w)


@pytest.mark.parametrize("rows", [1, 2, 300, 5000])
def test_norm_backward_many_rows_into_a_bucket(rows):
    cols = 129
    weight = torch.ones(cols, device="cuda")
    h, dy = rand(rows, cols, torch.bfloat16, 1), rand(rows, cols, torch.bfloat16, 2, 1e-3)
    rstd = nsml.nsml_q8_rms_norm(h, weight)[2]
    want_dx, want_dw = plain.rms_norm_backward(f64(dy), f64(h), f64(rstd), f64(weight))
    _, tol_w = norm_grad_tolerance(f64(dy), f64(h), f64(rstd), f64(weight), None, want_dx, torch.bfloat16, rows)
    for dtype in TYPES:
        bucket = torch.full((cols + 9,), 0.5, dtype=dtype, device="cuda")
        for zero_first in (True, False):
            before = f64(bucket[5:5 + cols])
            nsml.nsml_q8_rms_norm_backward(dy, weight, rstd, h=h, dweight=bucket[5:5 + cols], zero_first=zero_first)
            want = want_dw if zero_first else before + want_dw
            assert np.all(np.abs(f64(bucket[5:5 + cols]) - want) <= tol_w + (U + HALF[dtype]) * 1.01 * (np.abs(want) + tol_w))
        assert bool((bucket[:5] == 0.5).all()) and bool((bucket[5 + cols:] == 0.5).all())
    # in place
    for into in ("dy", "dh"):
        a, b = dy.clone(), rand(rows, cols, torch.bfloat16, 9, 1e-3)
        want = nsml.nsml_q8_rms_norm_backward(a.clone(), weight, rstd, h=h, dh=b.clone())[0]
        assert torch.equal(nsml.nsml_q8_rms_norm_backward(a, weight, rstd, h=h, dh=b, dx=a if into == "dy" else b)[0], want)


def test_norm_backward_against_differences():
    # the loss sum(coeff * y) of rows in float64, differenced; y before its rounding to codes
    rng = np.random.default_rng(4)
    h, w, coeff = rng.standard_normal((3, 40)), 1.0 + 0.1 * rng.standard_normal(40), rng.standard_normal((3, 40))
    h, w, coeff = (v.astype(np.float32).astype(np.float64) for v in (h, w, coeff))
    loss = lambda hh, ww: float(np.sum(coeff * plain.rms_norm(hh, ww, 1e-5)[1]))  # noqa: E731
    cuda = lambda v: torch.from_numpy(v.astype(np.float32)).cuda()  # noqa: E731
    rstd = nsml.nsml_q8_rms_norm(cuda(h), cuda(w))[2]
    dx, dw = nsml.nsml_q8_rms_norm_backward(cuda(coeff), cuda(w), rstd, h=cuda(h))
    step = 1e-5
    for r, c in ((0, 0), (1, 17), (2, 39)):
        up, down = h.copy(), h.copy()
        up[r, c] += step
        down[r, c] -= step
        assert abs((loss(up, w) - loss(down, w)) / (2 * step) - float(dx[r, c])) < 1e-5  # (differences: step^2; float32: 1e-6)
    for c in (0, 20, 39):
        up, down = w.copy(), w.copy()
        up[c] += step
        down[c] -= step
        assert abs((loss(h, up) - loss(h, down)) / (2 * step) - float(dw[c])) < 1e-5


# ---- products --------------------------------------------------------------------------------------------------------------
SIZES = [(1, 1, 1), (1, 129, 16), (2, 64, 300), (7, 257, 1000), (8, 300, 64), (9, 40, 129), (15, 500, 2048), (16, 16, 4096),
         (17, 31, 33), (33, 1000, 128), (100, 77, 771), (128, 256, 128), (129, 257, 127), (130, 511, 513), (300, 300, 65),
         (257, 1030, 2000), (1000, 100, 3000)]


def codes_matrix(rows, cols, seed, extreme=False):
    """Random codes in a buffer whose padding holds rubbish, and scales: powers of two, a zero among them."""
    rng = np.random.default_rng(seed)
    buf = rng.integers(-127, 128, (rows, (cols + 15) // 16 * 16)).astype(np.int8)
    if extreme:
        buf[:, :cols] = -128
    scales = np.exp2(rng.integers(-9, 3, rows)).astype(np.float32)
    if rows > 2:
        scales[rows // 2] = 0.0
    return torch.from_numpy(buf).cuda()[:, :cols], torch.from_numpy(scales).cuda()


def gradient(rows, cols, seed):
    """bfloat16, rows a multiple of 16 bytes apart, rubbish (NaN) between them."""
    buf = torch.full((rows, (cols + 7) // 8 * 8), float("nan"), dtype=torch.bfloat16, device="cuda")
    buf[:, :cols] = rand(rows, cols, torch.bfloat16, seed, 1e-3)
    return buf[:, :cols]


def workspace():
    return torch.full((256,), 77, dtype=torch.uint8, device="cuda")


@pytest.mark.parametrize("m,n,k", SIZES + [(3, 20, 131071), (40, 130, 131071)])
def test_matmul(m, n, k):
    a, sa = codes_matrix(m, k, 1, extreme=k > 100000)
    b, sb = codes_matrix(n, k, 2, extreme=k > 100000)
    sums = codes_of(a).astype(np.int64) @ codes_of(b).astype(np.int64).T
    want = (sums.astype(np.float32) * sa.cpu().numpy()[:, None]) * sb.cpu().numpy()
    for dtype in TYPES:
        ws = workspace()
        out = nsml.nsml_q8_matmul(a, sa, b, sb, dtype=dtype, workspace=ws)
        assert nsml.nsml_last_status(ws) == 0
        assert torch.equal(out.cpu(), torch.from_numpy(want).to(dtype))  # the sum is exact, the roundings are the definition's


def check_gradient(got, want, terms, depth, dtype, before=None):
    tol = depth * 2 * U * terms
    if before is not None:
        want, tol = want + before, tol + U * (np.abs(want + before) + tol)
    assert np.all(np.abs(f64(got) - want) <= (tol + HALF[dtype] * (np.abs(want) + tol)) * 1.01)


@pytest.mark.parametrize("m,n,k", SIZES)
def test_grad_input(m, n, k):
    dy, (b, sb) = gradient(m, n, 3), codes_matrix(n, k, 2)
    want = plain.matmul_grad_input(f64(dy), codes_of(b), f64(sb))
    terms = np.abs(f64(dy)) @ np.abs(plain.unpack(codes_of(b), f64(sb)))
    for dtype in TYPES:
        ws = workspace()
        dx = nsml.nsml_q8_matmul_grad_input(dy, b, sb, dtype=dtype, workspace=ws)
        assert nsml.nsml_last_status(ws) == 0
        check_gradient(dx, want, terms, n, dtype)


@pytest.mark.parametrize("m,n,k", SIZES)
def test_grad_weight_into_a_bucket(m, n, k):
    dy, (a, sa) = gradient(m, n, 3), codes_matrix(m, k, 2)
    want = plain.matmul_grad_weight(f64(dy), codes_of(a), f64(sa))
    terms = np.abs(f64(dy)).T @ np.abs(plain.unpack(codes_of(a), f64(sa)))
    for dtype in TYPES:
        bucket = torch.full((n * k + 8,), 0.25, dtype=dtype, device="cuda")
        for lead in (4, 3):  # rows on even and on odd elements
            dw = bucket[lead:lead + n * k].view(n, k)
            for zero_first in (True, False):
                ws, before = workspace(), None if zero_first else f64(dw)
                nsml.nsml_q8_matmul_grad_weight(dy, a, sa, dw=dw, zero_first=zero_first, workspace=ws)
                assert nsml.nsml_last_status(ws) == 0
                check_gradient(dw, want, terms, m, dtype, before)
        assert bool((bucket[:3] == 0.25).all()) and bool((bucket[4 + n * k:] == 0.25).all())


@pytest.mark.parametrize("dtype", TYPES)
def test_products_leave_what_lies_between_and_behind_the_rows(dtype):
    m, n, k = 130, 70, 90
    a, sa = codes_matrix(m, k, 1)
    b, sb = codes_matrix(n, k, 2)
    dy = gradient(m, n, 3)
    for rows, cols, call in ((m, n, lambda o: nsml.nsml_q8_matmul(a, sa, b, sb, out=o)), (m, k, lambda o: nsml.nsml_q8_matmul_grad_input(dy, b, sb, dx=o)),
                             (n, k, lambda o: nsml.nsml_q8_matmul_grad_weight(dy, a, sa, dw=o)), (4, n, lambda o: nsml.nsml_q8_matmul(a[:4], sa[:4], b, sb, out=o))):
        for pad in (3, 8):
            buf = torch.full((rows + 2, cols + pad), 5.0, dtype=dtype, device="cuda")
            call(buf[:rows, :cols])
            assert bool((buf[rows:] == 5.0).all()) and bool((buf[:, cols:] == 5.0).all())
            assert torch.equal(buf[:rows, :cols], call(torch.empty(rows, cols, dtype=dtype, device="cuda")))


def test_scales_that_are_no_powers_of_two_and_ones_that_are_not_finite():
    m, n, k = 70, 90, 130
    a, _ = codes_matrix(m, k, 1)
    b, _ = codes_matrix(n, k, 2)
    dy = gradient(m, n, 3)
    rng = np.random.default_rng(5)
    sa, sb = (torch.from_numpy(rng.uniform(1e-3, 2.0, s).astype(np.float32)).cuda() for s in (m, n))
    sa[3], sb[4], sa[5] = 2.0 ** -140, 2.0 ** 121, -0.5
    sums = codes_of(a).astype(np.int64) @ codes_of(b).astype(np.int64).T
    with np.errstate(over="ignore"):
        want = (sums.astype(np.float32) * sa.cpu().numpy()[:, None]) * sb.cpu().numpy()
    assert torch.equal(nsml.nsml_q8_matmul(a, sa, b, sb, dtype=torch.float32).cpu(), torch.from_numpy(want))
    assert torch.equal(nsml.nsml_q8_matmul(a[:6], sa[:6], b, sb, dtype=torch.float32).cpu(), torch.from_numpy(want[:6]))
    sb[4] = 0.75
    want = plain.matmul_grad_input(f64(dy), codes_of(b), f64(sb))
    check_gradient(nsml.nsml_q8_matmul_grad_input(dy, b, sb, dtype=torch.float32), want, np.abs(f64(dy)) @ np.abs(plain.unpack(codes_of(b), f64(sb))), n, torch.float32)
    want = plain.matmul_grad_weight(f64(dy), codes_of(a), f64(sa))
    check_gradient(nsml.nsml_q8_matmul_grad_weight(dy, a, sa), want, np.abs(f64(dy)).T @ np.abs(plain.unpack(codes_of(a), f64(sa))), m, torch.float32)
    sa[7] = float("nan")
    out = nsml.nsml_q8_matmul(a, sa, b, sb)
    assert bool(torch.isnan(out[7]).all()) and not bool(torch.isnan(out[:7]).any()) and not bool(torch.isnan(out[8:]).any())
    assert bool(torch.isnan(nsml.nsml_q8_matmul_grad_weight(dy, a, sa)).all())


def test_calls_on_several_streams_and_repeated_calls_agree_bit_for_bit():
    m, n, k = 500, 700, 900
    a, sa = codes_matrix(m, k, 1)
    b, sb = codes_matrix(n, k, 2)
    dy = gradient(m, n, 3)
    calls = [lambda: nsml.nsml_q8_matmul(a, sa, b, sb), lambda: nsml.nsml_q8_matmul(a[:5], sa[:5], b, sb), lambda: nsml.nsml_q8_matmul_grad_input(dy, b, sb),
             lambda: nsml.nsml_q8_matmul_grad_weight(dy, a, sa)]
    want = [c() for c in calls]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(4)]
    got = []
    for _ in range(5):
        for s, c in zip(streams, calls):
            with torch.cuda.stream(s):
                got.append(c())
    torch.cuda.synchronize()
    for i, g in enumerate(got):
        assert torch.equal(g, want[i % 4])


# ---- a run of them, as a training step makes it ------------------------------------------------------------------------------
def layer_step(x, residual, wn, w, dy, bucket, ws):
    """Norm, product, and their gradients into one flat bucket: [norm weight | weight]."""
    n, k = w.shape
    codes, scales, rstd, h = nsml.nsml_q8_rms_norm(x, wn, residual=residual)
    wq, wscales = nsml.nsml_q8_pack(w)
    y = nsml.nsml_q8_matmul(codes, scales, wq, wscales, workspace=ws)
    hq, hscales = nsml.nsml_q8_pack(h)
    nsml.nsml_q8_matmul_grad_weight(dy, codes, scales, dw=bucket[k:].view(n, k), workspace=ws)
    dnormed = nsml.nsml_q8_matmul_grad_input(dy, wq, wscales, workspace=ws)
    dx, _ = nsml.nsml_q8_rms_norm_backward(dnormed, wn, rstd, codes=hq, scales=hscales, dweight=bucket[:k], workspace=ws)
    return y, dx


def test_a_layers_step_runs_and_is_captured_and_replayed():
    m, n, k = 333, 264, 520
    x, residual = rand(m, k, torch.bfloat16, 1), rand(m, k, torch.bfloat16, 2)
    wn, w = torch.ones(k, device="cuda") * 1.25, rand(n, k, torch.float32, 3, k ** -0.5)
    dy = rand(m, n, torch.bfloat16, 4, 1e-3)
    ws = nsml.alloc_bytes(nsml.lib.nsml_q8_rms_norm_backward_workspace_bytes(k), "cuda")
    bucket = torch.zeros(k + n * k, device="cuda")
    y, dx = layer_step(x, residual, wn, w, dy, bucket, ws)
    # plain: every stage from the one before as it was computed
    kept = f64((x.float() + residual.float()).bfloat16())
    rstd, normed = plain.rms_norm(kept, f64(wn), 1e-5)
    assert np.linalg.norm(f64(y) - normed @ f64(w).T) <= 0.03 * np.linalg.norm(f64(y))  # two 8-bit roundings of at most 2^-7 of a row's largest value
    codes, scales = nsml.nsml_q8_pack(w)
    dnormed = f64(dy) @ plain.unpack(codes_of(codes), f64(scales))
    want_dx, want_dwn = plain.rms_norm_backward(dnormed, kept, rstd, f64(wn))
    assert np.linalg.norm(f64(dx) - want_dx) <= 0.03 * np.linalg.norm(want_dx)
    assert np.linalg.norm(f64(bucket[:k]) - want_dwn) <= 0.03 * np.linalg.norm(want_dwn)
    want_dw = f64(dy).T @ normed
    assert np.linalg.norm(f64(bucket[k:].view(n, k)) - want_dw) <= 0.03 * np.linalg.norm(want_dw)
    # the bucket goes into the exchange as it is
    payload = nsml.nsml_compress(bucket, 0.1, 8)
    dense = torch.empty_like(bucket)
    nsml.nsml_decompress_accumulate([payload], dense)
    top = bucket.abs().topk(nsml.nsml_k_of(bucket.numel(), 0.1)).indices
    assert int((dense[top] != 0).sum()) > 0.9 * top.numel()
    # the same step captured once and replayed on new values in the same buffers
    static = dict(x=x.clone(), residual=residual.clone(), wn=wn, w=w, dy=dy.clone(), bucket=torch.zeros_like(bucket), ws=ws.clone())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        layer_step(**static)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = layer_step(**static)
    for seed in (11, 12):
        static["x"].copy_(rand(m, k, torch.bfloat16, seed))
        static["dy"].copy_(rand(m, n, torch.bfloat16, seed + 1, 1e-3))
        graph.replay()
        torch.cuda.synchronize()
        fresh = torch.zeros_like(bucket)
        y, dx = layer_step(static["x"].clone(), residual, wn, w, static["dy"].clone(), fresh, ws)
        assert torch.equal(y, out[0]) and torch.equal(dx, out[1]) and torch.equal(fresh, static["bucket"])


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols", [2047, 8200, 9681, 12288, 16390, 20480, 32768])
def test_norm_backward_several_wide_rows_per_block(cols, dtype, packed):
    rows = 310  # (three turns of a block that has an SM to itself)
    weight = (1.0 + 0.1 * torch.randn(cols, generator=torch.Generator().manual_seed(1))).to(dtype).cuda()
    h, dy, dh = rand(rows, cols, dtype, 1), rand(rows, cols, dtype, 2, 1e-3), rand(rows, cols, dtype, 3, 1e-3)
    rstd = nsml.nsml_q8_rms_norm(h, weight)[2]
    codes, scales = nsml.nsml_q8_pack(h)
    kept = f64(h) if not packed else plain.unpack(codes_of(codes), f64(scales))
    rows_kept = dict(codes=codes, scales=scales) if packed else dict(h=h)
    dx, dweight = nsml.nsml_q8_rms_norm_backward(dy, weight, rstd, dh=dh, **rows_kept)
    want_dx, want_dw = plain.rms_norm_backward(f64(dy), kept, f64(rstd), f64(weight), f64(dh))
    tol, tol_w = norm_grad_tolerance(f64(dy), kept, f64(rstd), f64(weight), f64(dh), want_dx, dtype, rows)
    assert np.all(np.abs(f64(dx) - want_dx) <= tol)
    assert np.all(np.abs(f64(dweight) - want_dw) <= tol_w)
    for into in (dy.clone(), dh.clone()):  # in place
        args = (into, dh) if torch.equal(into, dy) else (dy, into)
        assert torch.equal(nsml.nsml_q8_rms_norm_backward(args[0], weight, rstd, dh=args[1], dx=into, **rows_kept)[0], dx)
