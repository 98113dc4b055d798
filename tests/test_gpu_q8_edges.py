"""Training in 8 bits on the GPU where it goes wrong first: both forms of the products, sums in several pieces, scales off 16-byte
boundaries, offsets past 32 bits, streams, threads and captured graphs.  Tolerances as in test_gpu_q8.py: u = 2^-24; sums on the
tensor cores are off by at most a step of every addition, depth * 2u * sum |terms|."""
import subprocess
import sys
import threading

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


def f64(t):
    return t.detach().cpu().double().numpy()


def codes_matrix(rows, cols, seed, shift=0):
    """Codes with -128 among them, rubbish behind the rows; scales that start `shift` elements into their buffer."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    codes = torch.randint(-128, 128, (rows, (cols + 15) // 16 * 16), generator=g, device="cuda", dtype=torch.int8)[:, :cols]
    scales = torch.exp2(torch.randint(-9, 3, (rows + shift,), generator=g, device="cuda").float())[shift:]
    return codes, scales


def gradient(rows, cols, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    buf = torch.full((rows, (cols + 7) // 8 * 8), float("nan"), dtype=torch.bfloat16, device="cuda")
    buf[:, :cols] = torch.randn(rows, cols, generator=g, device="cuda") * 1e-3
    return buf[:, :cols]


def check(got, want, terms, depth, dtype):
    tol = depth * 2 * U * terms
    assert np.all(np.abs(f64(got) - want) <= (tol + HALF[dtype] * (np.abs(want) + tol)) * 1.01)


def restored(codes, scales):
    return plain.unpack(codes.cpu().numpy(), f64(scales))




# many tiles of 256 x 256 (pairs of blocks); few tiles and a long sum (clusters of blocks); both with ragged edges
@pytest.mark.parametrize("rows,depth,cols", [(2500, 200, 2600), (2573, 129, 2311), (2500, 130, 2602), (300, 9000, 140), (5, 60000, 300), (1030, 4096, 1030)])
def test_forward_in_both_forms(rows, depth, cols):
    a, sa = codes_matrix(rows, depth, 1, shift=3)
    b, sb = codes_matrix(cols, depth, 2, shift=1)
    sums = (a.cpu().numpy().astype(np.float64) @ b.cpu().numpy().astype(np.float64).T).astype(np.int64)  # exact: below 2^53
    want = (sums.astype(np.float32) * sa.cpu().numpy()[:, None]) * sb.cpu().numpy()
    for dtype in TYPES:
        assert torch.equal(nsml.nsml_q8_matmul(a, sa, b, sb, dtype=dtype).cpu(), torch.from_numpy(want).to(dtype))


@pytest.mark.parametrize("rows,depth,cols", [(2500, 200, 2600), (2573, 129, 2311), (2500, 130, 2602), (2600, 2500, 2400), (300, 5000, 140), (257, 9001, 300), (40, 20000, 64)])
@pytest.mark.parametrize("shift", [0, 1, 3])
def test_gradients_in_both_forms_with_sums_in_pieces(rows, depth, cols, shift):
    if shift and depth == 2500:
        return
    codes, scales = codes_matrix(depth, cols, 2, shift)
    values = restored(codes, scales)
    for dy, call in ((gradient(rows, depth, 3), lambda dy, t: nsml.nsml_q8_matmul_grad_input(dy, codes, scales, dtype=t)),
                     (gradient(depth, rows, 3), lambda dy, t: nsml.nsml_q8_matmul_grad_weight(dy, codes, scales, dtype=t))):
        d = f64(dy) if dy.shape[0] == rows else f64(dy).T
        want, terms = d @ values, np.abs(d) @ np.abs(values)
        for dtype in TYPES:
            check(call(dy, dtype), want, terms, depth, dtype)


def test_float32_sums_stay_exact_over_a_long_batch():
    # terms of one sign: what the tensor cores cut off would add up.  2048 products at a time: at most 2048 / 16 additions of 16
    # products, each short of at most a step, and one rounding per piece
    depth = 65536
    codes, scales = torch.ones(depth, 64, dtype=torch.int8, device="cuda"), torch.ones(depth, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(1)
    dy = (1.0 + torch.rand(depth, 64, generator=g, device="cuda")).bfloat16()
    got = f64(nsml.nsml_q8_matmul_grad_weight(dy, codes, scales))
    want = np.repeat(f64(dy).sum(axis=0)[:, None], 64, axis=1)
    assert np.all(np.abs(got - want) <= want * (2048 / 16 * 2 + depth / 2048 + 8) * U)


def test_accumulating_in_both_forms():
    for rows, depth, cols in ((2500, 2300, 2400), (300, 5000, 140)):
        codes, scales = codes_matrix(depth, cols, 2)
        dy = gradient(depth, rows, 3)
        want, terms = f64(dy).T @ restored(codes, scales), np.abs(f64(dy).T) @ np.abs(restored(codes, scales))
        for dtype in TYPES:
            dw = torch.full((rows, cols), 0.5, dtype=dtype, device="cuda")
            nsml.nsml_q8_matmul_grad_weight(dy, codes, scales, dw=dw, zero_first=False)
            # (float32 over several pairs' pieces: an addition per piece, each rounded)
            tol = depth * 2 * U * (terms + 0.5)
            assert np.all(np.abs(f64(dw) - (want + 0.5)) <= (tol + HALF[dtype] * (np.abs(want + 0.5) + tol)) * 1.01)


def test_offsets_past_32_bits():
    rows, cols = 66_000, 32_768  # 2.16e9 elements
    x = torch.zeros(rows, cols, dtype=torch.bfloat16, device="cuda")
    last = torch.randn(3, cols, generator=torch.Generator().manual_seed(1)).bfloat16()
    x[-3:] = last.cuda()
    codes, scales = nsml.nsml_q8_pack(x)
    want_codes, want_scales = plain.pack(f64(last))
    assert np.array_equal(codes[-3:].cpu().numpy(), want_codes) and np.array_equal(f64(scales[-3:]), want_scales)
    assert not bool(codes[-4].any()) and float(scales[-4]) == 0.0
    out = nsml.nsml_q8_unpack(codes, scales, out=x)
    assert np.array_equal(f64(out[-3:]), plain.unpack(want_codes, want_scales))
    weight = torch.ones(cols, dtype=torch.bfloat16, device="cuda")
    normed, nscales, rstd, _ = nsml.nsml_q8_rms_norm(x, weight)
    small = nsml.nsml_q8_rms_norm(x[-3:].clone(), weight)
    assert torch.equal(normed[-3:], small[0]) and torch.equal(nscales[-3:], small[1]) and torch.equal(rstd[-3:], small[2])
    dx, _ = nsml.nsml_q8_rms_norm_backward(x, weight, rstd, codes=codes, scales=scales, dx=x)
    want, _ = nsml.nsml_q8_rms_norm_backward(torch.from_numpy(plain.unpack(want_codes, want_scales)).bfloat16().cuda(), weight, small[2],
                                             codes=codes[-3:], scales=scales[-3:])
    assert torch.equal(dx[-3:], want)
    del x, out, dx, codes, normed
    # a result of more than 2^31 elements, from a short sum
    a, sa = codes_matrix(70_000, 64, 1)
    b, sb = codes_matrix(32_768, 64, 2)
    y = nsml.nsml_q8_matmul(a, sa, b, sb)
    assert torch.equal(y[-5:], nsml.nsml_q8_matmul(a[-5:], sa[-5:], b, sb))
    assert torch.equal(y[-2:, -300:], nsml.nsml_q8_matmul(a[-2:], sa[-2:], b[-300:], sb[-300:]))


def test_codes_far_apart():
    # a column block of a wide matrix of codes: rows 2^27 bytes apart, the last one past 2^32
    buf = torch.zeros(34, 1 << 27, dtype=torch.int8, device="cuda")
    codes, scales = codes_matrix(34, 100, 1)
    far = buf[:, 1 << 20:(1 << 20) + 100]
    far.copy_(codes)
    b, sb = codes_matrix(70, 100, 2)
    dy = gradient(34, 24, 3)
    assert torch.equal(nsml.nsml_q8_matmul(far, scales, b, sb), nsml.nsml_q8_matmul(codes, scales, b, sb))
    assert torch.equal(nsml.nsml_q8_matmul(far[-3:], scales[-3:], b, sb), nsml.nsml_q8_matmul(codes[-3:], scales[-3:], b, sb))
    assert torch.equal(nsml.nsml_q8_matmul_grad_weight(dy, far, scales), nsml.nsml_q8_matmul_grad_weight(dy, codes, scales))
    assert torch.equal(nsml.nsml_q8_unpack(far, scales), nsml.nsml_q8_unpack(codes, scales))


def test_stream_argument_and_threads():
    a, sa = codes_matrix(300, 400, 1)
    b, sb = codes_matrix(500, 400, 2)
    dy = gradient(300, 500, 3)
    want = (nsml.nsml_q8_matmul(a, sa, b, sb), nsml.nsml_q8_matmul_grad_input(dy, b, sb), nsml.nsml_q8_matmul_grad_weight(dy, a, sa))
    torch.cuda.synchronize()
    wrong = []

    def work():
        torch.cuda.set_device(0)
        stream = torch.cuda.Stream()
        for _ in range(20):
            with torch.cuda.stream(stream):  # (the results' memory belongs to this stream)
                got = (nsml.nsml_q8_matmul(a, sa, b, sb, stream=stream), nsml.nsml_q8_matmul_grad_input(dy, b, sb, stream=stream),
                       nsml.nsml_q8_matmul_grad_weight(dy, a, sa, stream=stream))
            stream.synchronize()
            wrong.extend(not torch.equal(g, w) for g, w in zip(got, want))

    threads = [threading.Thread(target=work) for _ in range(3)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert len(wrong) == 180 and not any(wrong)


def test_two_graphs_share_a_workspace_one_after_the_other():
    cols = 520
    weight = torch.ones(cols, device="cuda")
    ws = nsml.alloc_bytes(int(nsml.lib.nsml_q8_rms_norm_backward_workspace_bytes(cols)), "cuda")
    sets = []
    for seed in (1, 2):
        h = torch.randn(300 * seed, cols, generator=torch.Generator().manual_seed(seed)).cuda()
        dy = torch.randn(300 * seed, cols, generator=torch.Generator().manual_seed(seed + 10)).cuda()
        rstd = nsml.nsml_q8_rms_norm(h, weight)[2]
        want = nsml.nsml_q8_rms_norm_backward(dy, weight, rstd, h=h)
        dx, dw = torch.zeros_like(h), torch.zeros(cols, device="cuda")
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph):
            nsml.nsml_q8_rms_norm_backward(dy, weight, rstd, h=h, dx=dx, dweight=dw, workspace=ws)
        sets.append((graph, dx, dw, want))
    for _ in range(3):
        for graph, dx, dw, _ in sets:
            dx.zero_()
            dw.zero_()
            graph.replay()
        torch.cuda.synchronize()
        for _, dx, dw, want in sets:
            assert torch.equal(dx, want[0]) and torch.equal(dw, want[1])


def test_narrow_and_empty_products():
    for m, n, k in ((700, 1, 1), (1, 1, 131071), (1, 700, 1), (5, 1, 70), (700, 3, 5)):
        a, sa = codes_matrix(m, k, 1)
        b, sb = codes_matrix(n, k, 2)
        sums = a.cpu().numpy().astype(np.int64) @ b.cpu().numpy().astype(np.int64).T
        want = (sums.astype(np.float32) * sa.cpu().numpy()[:, None]) * sb.cpu().numpy()
        assert torch.equal(nsml.nsml_q8_matmul(a, sa, b, sb, dtype=torch.float32).cpu(), torch.from_numpy(want))
        dy = gradient(m, n, 3)
        check(nsml.nsml_q8_matmul_grad_input(dy, b, sb, dtype=torch.float32), f64(dy) @ restored(b, sb), np.abs(f64(dy)) @ np.abs(restored(b, sb)), n, torch.float32)
        check(nsml.nsml_q8_matmul_grad_weight(dy, a, sa), f64(dy).T @ restored(a, sa), np.abs(f64(dy).T) @ np.abs(restored(a, sa)), m, torch.float32)


def test_the_norms_gradient_leaves_a_status():
    cols = 40
    h, weight = torch.randn(5, cols, generator=torch.Generator().manual_seed(1)).cuda(), torch.ones(cols, device="cuda")
    rstd = nsml.nsml_q8_rms_norm(h, weight)[2]
    for rows in (5, 0):
        ws = nsml.alloc_bytes(int(nsml.lib.nsml_q8_rms_norm_backward_workspace_bytes(cols)), "cuda").fill_(0x55)
        nsml.nsml_q8_rms_norm_backward(h[:rows], weight, rstd[:rows], h=h[:rows], workspace=ws)
        assert nsml.nsml_last_status(ws) == 0


def test_what_a_call_allocates_belongs_to_its_stream():
    # the call waits on its stream; memory that the current stream is given meanwhile is not the call's
    h = torch.randn(600, 2048, generator=torch.Generator().manual_seed(1)).cuda()
    weight, stream = torch.ones(2048, device="cuda"), torch.cuda.Stream()
    rstd = nsml.nsml_q8_rms_norm(h, weight)[2]
    want, need = nsml.nsml_q8_rms_norm_backward(h, weight, rstd, h=h), int(nsml.lib.nsml_q8_rms_norm_backward_workspace_bytes(2048))
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        torch.cuda._sleep(100_000_000)
    got = nsml.nsml_q8_rms_norm_backward(h, weight, rstd, h=h, stream=stream)
    other = [torch.full((need,), 0x55, dtype=torch.uint8, device="cuda") for _ in range(4)]
    torch.cuda.synchronize()
    assert all(bool((o == 0x55).all()) for o in other)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_a_thread_that_has_made_no_call_before():
    a, sa = codes_matrix(300, 400, 1)
    b, sb = codes_matrix(504, 400, 2)
    dy = gradient(300, 504, 3)
    want = (nsml.nsml_q8_matmul(a, sa, b, sb), nsml.nsml_q8_matmul_grad_input(dy, b, sb), nsml.nsml_q8_matmul_grad_weight(dy, a, sa))
    outs, ws, got = [torch.zeros_like(w) for w in want], nsml.alloc_bytes(256, "cuda"), []
    torch.cuda.synchronize()

    def ptr(t):
        return t.data_ptr(), t.stride(0)

    calls = (lambda: nsml.lib.nsml_q8_matmul(*ptr(a), sa.data_ptr(), *ptr(b), sb.data_ptr(), 300, 504, 400, *ptr(outs[0]), nsml.NSML_BF16, ws.data_ptr(), 256, 0),
             lambda: nsml.lib.nsml_q8_matmul_grad_input(*ptr(dy), *ptr(b), sb.data_ptr(), 300, 504, 400, *ptr(outs[1]), nsml.NSML_BF16, ws.data_ptr(), 256, 0),
             lambda: nsml.lib.nsml_q8_matmul_grad_weight(*ptr(dy), *ptr(a), sa.data_ptr(), 300, 504, 400, *ptr(outs[2]), nsml.NSML_F32, 1, ws.data_ptr(), 256, 0))
    for call in calls:  # (a thread of its own for each)
        thread = threading.Thread(target=lambda: got.append(call()))
        thread.start()
        thread.join()
    torch.cuda.synchronize()
    assert got == [0, 0, 0] and all(torch.equal(o, w) for o, w in zip(outs, want))


FIRST_CALLS_IN_A_CAPTURE = """
import torch
import paper_2506_16235_b200 as nsml
m, n, k = 260, 264, 2048
x, w, dy = torch.randn(m, k, device="cuda"), torch.randn(n, k, device="cuda"), torch.randn(m, n, device="cuda").bfloat16()
weight, ws = torch.ones(k, device="cuda"), nsml.alloc_bytes(int(nsml.lib.nsml_q8_rms_norm_backward_workspace_bytes(k)), "cuda")
def step():
    codes, scales, rstd, h = nsml.nsml_q8_rms_norm(x, weight)
    b, sb = nsml.nsml_q8_pack(w)
    y = nsml.nsml_q8_matmul(codes, scales, b, sb)
    token = nsml.nsml_q8_matmul(codes[:1], scales[:1], b, sb)
    dw = nsml.nsml_q8_matmul_grad_weight(dy, codes, scales)
    dx = nsml.nsml_q8_matmul_grad_input(dy, b, sb, dtype=torch.float32)
    return y, token, dw, *nsml.nsml_q8_rms_norm_backward(dx, weight, rstd, h=h, workspace=ws), nsml.nsml_q8_unpack(codes, scales)
graph = torch.cuda.CUDAGraph()
torch.cuda.synchronize()
with torch.cuda.graph(graph):
    got = step()
for _ in range(2):
    graph.replay()
want = step()
torch.cuda.synchronize()
assert all(torch.equal(g, w) for g, w in zip(got, want))
print("equal")
"""


def test_a_programs_first_calls_are_captured():
    done = subprocess.run([sys.executable, "-c", FIRST_CALLS_IN_A_CAPTURE], capture_output=True, text=True, timeout=120)
    assert done.returncode == 0 and done.stdout.strip() == "equal", done.stderr[-2000:]
