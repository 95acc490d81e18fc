"""The product of operands in microscaled 4-bit floating point against the exact product in 64 bits, and its gradient."""
import numpy as np
import pytest
import torch

import _operators as ref

pytestmark = pytest.mark.gpu
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24}


@pytest.fixture(scope="module")
def mx():
    from paper_2502_18554_b200 import build, mx
    build.build()
    return mx


def operand(rows, cols, seed, spread=4):
    """Random codes and scales of every size, made without the package; (bytes on the GPU, values in 64 bits on the GPU)."""
    rng = np.random.default_rng(seed)
    blocks = -(-cols // 32)
    v = ref.NIBBLES[rng.integers(0, 16, (rows, blocks, 32))]
    v.reshape(rows, -1)[:, cols:] = 0
    s = rng.integers(127 - spread, 128 + spread, (rows, blocks))
    codes, scales = ref.pack(v, s)
    return torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda(), torch.from_numpy(ref.values(v, s, cols)).cuda()


def close(got, a, b):
    """Products are exact; a sum of k of them in binary32, in any order, is off by at most (k - 1) 2^-24 of the sum of magnitudes (rounded to
    nearest; twice that if an addition truncates); then one rounding to the output's type."""
    want, size = a @ b.t(), a.abs() @ b.abs().t()
    off = max(a.shape[1] - 1, 0) * 2.0 ** -23 * size
    half = HALF[got.dtype]
    top = float(torch.finfo(got.dtype).max)
    error = (got.double() - want).abs()
    bound = off + (want.abs() + off) * half + TINY[got.dtype]
    assert bool(((error <= bound) | (want.abs() + off > top)).all()), float((error / bound).max())


def product(mx, m, n, k, dtype, seed=0):
    ac, as_, a = operand(m, k, seed)
    bc, bs, b = operand(n, k, seed + 1)
    got = mx.matmul(mx.Mx4(ac, as_, m, k), mx.Mx4(bc, bs, n, k), dtype)
    assert got.shape == (m, n) and got.dtype == dtype
    close(got, a, b)
    assert mx.status() == 0
    return got


def test_one_tile(mx):
    product(mx, 128, 128, 256, torch.float32)


@pytest.mark.parametrize("k", [1, 31, 32, 33, 64, 65, 96, 97, 128, 129, 160, 192, 224, 255, 256, 257, 288, 385, 512, 1000, 4161])
def test_depths(mx, k):
    """Every way in which the last block, group of blocks and stage can end."""
    product(mx, 40, 130, k, torch.float32, k)
    product(mx, 300, 200, k, torch.float32, k)


@pytest.mark.parametrize("m", [1, 2, 15, 16, 17, 32, 33, 63, 64, 65, 100, 127, 128, 129])
@pytest.mark.parametrize("n", [1, 8, 127, 129, 1000])
def test_few_rows(mx, m, n):
    product(mx, m, n, 700, torch.bfloat16, m)
    product(mx, n, m, 700, torch.float16, m)


@pytest.mark.parametrize("m,n,k", [(1, 16384, 8192), (3, 5000, 20000), (2, 200, 300_000), (13, 10007, 4161), (128, 257, 9000), (130, 140, 16384), (500, 600, 300), (777, 1531, 1000), (2049, 3001, 520), (4097, 2500, 321), (12800, 400, 512), (6000, 6001, 100)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_shapes(mx, m, n, k, dtype):
    product(mx, m, n, k, dtype, 5)


def test_large(mx):
    product(mx, 4096, 8192, 8192, torch.bfloat16, 9)


def test_an_output_beyond_32_bits(mx):
    a, b = operand(70_001, 32, 1), operand(65_536, 32, 2)
    y = mx.matmul(mx.Mx4(a[0], a[1], 70_001, 32), mx.Mx4(b[0], b[1], 65_536, 32), torch.bfloat16)
    for rows in (slice(0, 130), slice(65_400, 65_700), slice(69_900, 70_001)):
        close(y[rows], a[2][rows], b[2])


def test_scales_of_every_size(mx):
    """Magnitudes from the smallest to what still sums in binary32."""
    for spread in (20, 60):
        ac, as_, a = operand(50, 640, 1, spread)
        bc, bs, b = operand(300, 640, 2, spread)
        close(mx.matmul(mx.Mx4(ac, as_, 50, 640), mx.Mx4(bc, bs, 300, 640), torch.float32), a, b)


def test_a_block_that_is_not_a_number_reaches_its_row_alone(mx):
    for m, n in ((5, 300), (300, 400)):
        x = torch.randn(m, 500)
        x[2, 70] = float("nan")
        x[4, 499] = float("inf")
        a, b = mx.quantize(x.cuda()), mx.quantize(torch.randn(n, 500).cuda())
        y = mx.matmul(a, b, torch.float32)
        assert bool(torch.isnan(y[[2, 4]]).all()) and bool(torch.isfinite(y[[0, 1, 3]]).all()) and bool(torch.isfinite(y[5:]).all())


def test_output_with_a_pitch_and_what_surrounds_it(mx):
    for m, n, k in ((20, 130, 300), (200, 170, 300), (300, 20, 300), (500, 5000, 64)):
        for dtype in (torch.float32, torch.bfloat16, torch.float16):
            ac, as_, a = operand(m, k, 3)
            bc, bs, b = operand(n, k, 4)
            for shift, pitch in ((0, n + 6), (1, n + 3), (8, n + 40)):
                whole = torch.full((m * pitch + 64,), 7.0, dtype=dtype, device="cuda")
                out = whole[shift:shift + m * pitch].view(m, pitch)[:, :n]
                mx.matmul(mx.Mx4(ac, as_, m, k), mx.Mx4(bc, bs, n, k), out=out)
                close(out, a, b)
                out.fill_(7.0)
                assert bool((whole == 7.0).all())


def test_nothing_to_sum_and_nothing_to_write(mx):
    e = lambda r, c: mx.empty(r, c, "cuda")  # noqa: E731
    assert not mx.matmul(e(5, 0), e(7, 0), out=torch.ones(5, 7, device="cuda")).any()
    assert mx.matmul(e(0, 64), e(7, 64)).shape == (0, 7) and mx.matmul(e(5, 64), e(0, 64)).shape == (5, 0)


def test_the_same_call_gives_the_same_bits(mx):
    for m, n, k in ((1, 4000, 8192), (100, 4000, 8192), (1000, 1000, 4096)):
        a, b = operand(m, k, 1), operand(n, k, 2)
        one = mx.matmul(mx.Mx4(a[0], a[1], m, k), mx.Mx4(b[0], b[1], n, k), torch.float32)
        for _ in range(3):
            assert torch.equal(one, mx.matmul(mx.Mx4(a[0], a[1], m, k), mx.Mx4(b[0], b[1], n, k), torch.float32))


def test_several_products_at_once_on_several_streams(mx):
    """Kernels of every form side by side: they share the SMs' tensor memory."""
    shapes = [(1, 4096, 4096), (64, 4096, 4096), (128, 3000, 5000), (1500, 1500, 2048), (4096, 4096, 512), (200, 200, 8192)]
    work = []
    for i, (m, n, k) in enumerate(shapes):
        a, b = operand(m, k, i), operand(n, k, i + 50)
        work.append((mx.Mx4(a[0], a[1], m, k), mx.Mx4(b[0], b[1], n, k)))
    want = [mx.matmul(a, b, torch.float32) for a, b in work]
    streams = [torch.cuda.Stream() for _ in work]
    torch.cuda.synchronize()
    got = []
    for _ in range(20):
        got = [mx.matmul(a, b, torch.float32, stream=s) for (a, b), s in zip(work, streams)]
    torch.cuda.synchronize()
    assert mx.status() == 0
    assert all(torch.equal(x, y) for x, y in zip(want, got))


def test_captured(mx):
    x, w = torch.randn(9, 1000, device="cuda", dtype=torch.bfloat16), mx.quantize(torch.randn(700, 1000, device="cuda"))
    mx.linear(x, w)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = mx.linear(x, w)
    x.copy_(torch.randn(9, 1000))
    graph.replay()
    assert torch.equal(y, mx.linear(x, w))


# ---- linear and its gradient

def rounded(x):
    v, s = ref.quantize(x.float().cpu().numpy().astype(np.float64))
    return torch.from_numpy(ref.values(v, s, x.shape[1])).cuda()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("m,k,n", [(1, 32, 32), (5, 70, 33), (200, 300, 140), (777, 1000, 531)])
def test_linear_and_its_gradient_against_the_formula(mx, m, k, n, dtype):
    gen = torch.Generator().manual_seed(m)
    rand = lambda *s: torch.randn(*s, generator=gen).to(dtype).cuda()  # noqa: E731
    x, w, dy = rand(m, k).requires_grad_(), rand(n, k).requires_grad_(), rand(m, n)
    y = mx.linear(x, w)
    y.backward(dy)
    close(y.detach(), rounded(x.detach()), rounded(w.detach()))
    close(x.grad, rounded(dy), rounded(w.detach().t()))
    close(w.grad, rounded(dy.t()), rounded(x.detach().t()))
    dx, dw = mx.linear_backward(dy, x.detach(), w.detach())
    assert torch.equal(dx, x.grad) and torch.equal(dw, w.grad)
    assert torch.equal(mx.linear(x.detach(), mx.quantize(w.detach())), y)


def test_gradient_against_differences(mx):
    """On values that the form holds exactly along both axes (one magnitude of scale, elements of the grid) quantisation is the identity, so
    the output moves by exactly the gradient times the step: every partial derivative of a weighted sum of outputs."""
    gen = torch.Generator().manual_seed(0)
    grid = torch.tensor([0.5, 1.0, 1.5, 2.0, 3.0])
    pick = lambda *s: grid[torch.randint(0, 5, s, generator=gen)] * (torch.randint(0, 2, s, generator=gen) * 2 - 1)  # noqa: E731
    pin = lambda t: t.index_fill(0, torch.arange(0, t.shape[0], 32), 4.0).index_fill(1, torch.arange(0, t.shape[1], 32), 4.0)  # noqa: E731
    x, w, dy = (pin(pick(40, 64)).cuda(), pin(pick(36, 64)).cuda(), pin(pick(40, 36)).cuda())
    x.requires_grad_()
    w.requires_grad_()
    mx.linear(x, w).backward(dy)
    loss = lambda a, b: float((mx.linear(a, b).double() * dy.double()).sum())  # noqa: E731
    with torch.no_grad():
        for t, grad, f in ((x, x.grad, lambda q: loss(q, w)), (w, w.grad, lambda q: loss(x, q))):
            for r, c in ((1, 1), (5, 40), (33, 63), (20, 33)):
                up, down = t.detach().clone(), t.detach().clone()
                up[r, c], down[r, c] = 2.0, -2.0
                assert f(up) - f(down) == 4.0 * float(grad[r, c])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("m", [1, 2, 3, 5, 8, 9, 13, 16, 17, 40, 64, 65, 129])
def test_a_layer_with_held_weights_is_quantising_and_multiplying(mx, m, dtype):
    """Few rows are quantised inside the product: the same bits, at every way in which the depth can end and for rows that begin anywhere."""
    for k, n in ((1, 20), (31, 200), (64, 129), (127, 300), (129, 1000), (257, 300), (1000, 500), (2049, 700), (4161, 3000), (8192, 4096), (20000, 300)):
        gen = torch.Generator().manual_seed(m * 31 + k)
        w = mx.quantize(torch.randn(n, k, generator=gen).cuda())
        for shift, pitch in ((0, k + (-k) % 8), (1, k + 3)):
            flat = (torch.randn(m * pitch + 16, generator=gen) * torch.exp2(torch.randint(-5, 6, (m * pitch + 16,), generator=gen).float())).to(dtype).cuda()
            x = flat[shift:shift + m * pitch].view(m, pitch)[:, :k]
            assert torch.equal(mx.linear(x, w), mx.matmul(mx.quantize(x), w, dtype)), (k, n, shift)
    assert mx.status() == 0


def test_a_token_that_is_not_a_number_stays_alone(mx):
    x = torch.randn(3, 600, device="cuda")
    x[1, 5] = float("inf")
    y = mx.linear(x, mx.quantize(torch.randn(500, 600, device="cuda")))
    assert bool(torch.isnan(y[1]).all()) and bool(torch.isfinite(y[[0, 2]]).all())


def test_layers_of_a_few_tokens_on_several_streams(mx):
    x = [torch.randn(m, 4096, device="cuda", dtype=torch.bfloat16) for m in (1, 2, 4, 1, 3, 64)]
    w = [mx.quantize(torch.randn(n, 4096, device="cuda")) for n in (4096, 3000, 500, 9000, 4096, 4096)]
    want = [mx.linear(a, b) for a, b in zip(x, w)]
    streams = [torch.cuda.Stream() for _ in x]
    torch.cuda.synchronize()
    for _ in range(20):
        got = []
        for a, b, s in zip(x, w, streams):
            with torch.cuda.stream(s):
                got.append(mx.linear(a, b))
    torch.cuda.synchronize()
    assert mx.status() == 0 and all(torch.equal(p, q) for p, q in zip(want, got))


def test_leading_dimensions_and_refusals(mx):
    x, w = torch.randn(2, 3, 64, device="cuda"), torch.randn(40, 64, device="cuda")
    y = mx.linear(x, w)
    assert y.shape == (2, 3, 40) and torch.equal(y.view(6, 40), mx.linear(x.view(6, 64), w))
    q, p = mx.quantize(w), mx.quantize(torch.randn(5, 96, device="cuda"))
    with pytest.raises(ValueError):
        mx.matmul(q, p)
    with pytest.raises(ValueError):
        mx.matmul(q, q, torch.float64)
    with pytest.raises(ValueError):
        mx.matmul(q, q, out=torch.empty(40, 41, device="cuda"))
    with pytest.raises(ValueError):
        mx.matmul(mx.Mx4(q.codes, q.scales, 40, 96), mx.Mx4(q.codes, q.scales, 40, 96))     # too few bytes
    with pytest.raises(ValueError):
        mx.matmul(q, mx.Mx4(q.codes.cpu(), q.scales, 40, 64))
    with pytest.raises(ValueError):
        mx.linear(x, w.bfloat16())
    with pytest.raises(ValueError):
        mx.linear(x.clone().requires_grad_(), q)
    with pytest.raises(RuntimeError):
        big = torch.zeros(q.codes.numel() + 8, dtype=torch.uint8, device="cuda")
        mx.matmul(mx.Mx4(big[8:], q.scales, 40, 64), q)


def test_pairs_of_ctas_that_follow_each_other(mx):
    """Short products of many tiles on several streams, so that one's CTAs take the places (shared and tensor memory, barriers) that another's have just left; every
    round's outputs are compared."""
    shapes = [(4096, 4096, 64), (4097, 3900, 300), (2600, 2600, 1300), (128, 20000, 256), (6000, 6001, 32)]
    work = []
    for i, (m, n, k) in enumerate(shapes):
        a, b = operand(m, k, i), operand(n, k, i + 50)
        work.append((mx.Mx4(a[0], a[1], m, k), mx.Mx4(b[0], b[1], n, k)))
    want = [mx.matmul(a, b) for a, b in work]
    streams = [torch.cuda.Stream() for _ in work]
    torch.cuda.synchronize()
    for _ in range(8):
        got = [[mx.matmul(a, b, stream=s) for _ in range(3)] for (a, b), s in zip(work, streams)]
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, ys in zip(want, got) for y in ys)
    assert mx.status() == 0


def test_every_round_of_products_on_several_streams(mx):
    """Kernels of every form side by side, each round's outputs compared."""
    shapes = [(1, 4096, 4096), (64, 4096, 4096), (128, 3000, 5000), (1500, 1500, 2048), (4096, 4096, 512), (200, 200, 8192)]
    work = []
    for i, (m, n, k) in enumerate(shapes):
        a, b = operand(m, k, i), operand(n, k, i + 50)
        work.append((mx.Mx4(a[0], a[1], m, k), mx.Mx4(b[0], b[1], n, k)))
    want = [mx.matmul(a, b, torch.float32) for a, b in work]
    streams = [torch.cuda.Stream() for _ in work]
    torch.cuda.synchronize()
    rounds = [[mx.matmul(a, b, torch.float32, stream=s) for (a, b), s in zip(work, streams)] for _ in range(20)]
    torch.cuda.synchronize()
    assert mx.status() == 0
    assert all(torch.equal(x, y) for got in rounds for x, y in zip(want, got))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_calls_that_read_what_the_call_in_front_writes(mx, dtype):
    """Products, forms along rows and columns, the way back and layers one behind the other without a synchronisation, each reading what the kernel in front has
    just written; inputs change from round to round, so that what is left from the last round would show."""
    gen = torch.Generator().manual_seed(11)
    for m, k, n in ((5, 300, 260), (300, 260, 512), (1500, 1100, 900)):
        w = mx.quantize((torch.randn(k, n, generator=gen) * 0.1).to(dtype).cuda(), transpose=True)      # [n, k]
        back = mx.quantize((torch.randn(k, n, generator=gen) * 0.1).to(dtype).cuda())                   # [k, n]
        xs = [torch.randn(m, k, generator=gen).to(dtype).cuda() for _ in range(6)]

        def chain(x, settle):
            out = []
            for _ in range(3):
                steps = [lambda a: mx.quantize(a), lambda a: mx.matmul(a, w, dtype), lambda a: mx.quantize(a, transpose=True), lambda a: mx.dequantize(a, dtype).t().contiguous(),
                         lambda a: mx.linear(a, back)]
                for step in steps:
                    x = step(x)
                    if settle:
                        torch.cuda.synchronize()
                    out += [x.codes, x.scales] if isinstance(x, mx.Mx4) else [x]
            return out

        want = [chain(x, True) for x in xs]
        got = [chain(x, False) for x in xs]
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for p, q in zip(want, got) for a, b in zip(p, q))
    assert mx.status() == 0


def test_forward_mode_tangents_are_refused(mx):
    """There is no forward-mode derivative: a dual tensor raises instead of losing its tangent."""
    import torch.autograd.forward_ad as fwd
    x, w = torch.randn(4, 64, device="cuda"), torch.randn(40, 64, device="cuda")
    q = mx.quantize(w)
    with fwd.dual_level():
        dual, dual_w = fwd.make_dual(x, torch.ones_like(x)), fwd.make_dual(w, torch.ones_like(w))
        for call in (lambda: mx.linear(dual, w), lambda: mx.linear(x, dual_w), lambda: mx.linear(dual, q), lambda: mx.linear(dual[None], q), lambda: mx.quantize(dual),
                     lambda: mx.quantize_all([x, dual]), lambda: mx.linear_backward(torch.randn(4, 40, device="cuda"), dual, w)):
            with pytest.raises(ValueError, match="tangent"):
                call()
        with pytest.raises((ValueError, RuntimeError, NotImplementedError)):
            mx.linear(dual, w.clone().requires_grad_())
        mx.linear(x, w)                                         # others are none the worse for it
    with torch.no_grad(), pytest.raises(Exception):
        torch.func.jvp(lambda t: mx.linear(t, w), (x,), (torch.ones_like(x),))


@pytest.mark.filterwarnings("ignore")
def test_a_trace_is_refused(mx):
    """A trace would hold the output for the first input as a constant."""
    x, w = torch.randn(4, 64, device="cuda"), torch.randn(40, 64, device="cuda")
    q = mx.quantize(w)
    for call in (lambda t: mx.linear(t, w), lambda t: mx.linear(t, q), lambda t: mx.dequantize(mx.quantize(t)), lambda t: t + mx.matmul(q, q).sum()):
        with pytest.raises(ValueError, match="trace"):
            torch.jit.trace(call, (x,))
    mx.linear(x, q)


@pytest.mark.parametrize("lead", [(), (3,), (2, 3), (0,), (2, 0, 3)])
@pytest.mark.parametrize("k", [0, 1, 64])
def test_layers_of_any_leading_dimensions(mx, lead, k):
    """Empty ones and rows without elements included: nothing to sum is zeros."""
    x, w = torch.randn(*lead, k, device="cuda"), torch.randn(5, k, device="cuda")
    for weights in (w, mx.quantize(w)):
        y = mx.linear(x, weights)
        assert y.shape == (*lead, 5)
        if x.numel() == 0:
            assert not y.any()
        else:
            close(y.reshape(-1, 5), rounded(x.reshape(-1, k)), rounded(w))
    x.requires_grad_()
    w.requires_grad_()
    mx.linear(x, w).sum().backward()
    assert x.grad.shape == x.shape and w.grad.shape == w.shape


def test_a_wait_that_ran_out_is_told_by_the_next_call(mx):
    """Recorded by a thread that waits for nothing: products and layers are refused until the record has been read, and go on afterwards; other calls run."""
    from paper_2502_18554_b200 import zccl as z
    x, w = torch.randn(4, 64, device="cuda"), torch.randn(40, 64, device="cuda")
    q = mx.quantize(w)
    want = mx.matmul(q, q), mx.linear(x, q), mx.linear(x, w)
    assert mx.status() == z.OK
    start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    start.record()
    mx.debug_wait()
    end.record()
    torch.cuda.synchronize()
    assert start.elapsed_time(end) < 10_000
    for call in (lambda: mx.matmul(q, q), lambda: mx.linear(x, q), lambda: mx.linear(x, w), lambda: mx.linear_backward(torch.zeros(4, 40, device="cuda"), x, w)):
        with pytest.raises(z.ZcclError) as e:
            call()
        assert e.value.code == z.E_TIMEOUT
    assert torch.equal(mx.quantize(w).codes, q.codes)
    assert mx.status() == z.E_TIMEOUT and mx.status() == z.OK
    assert all(torch.equal(a, b) for a, b in zip(want, (mx.matmul(q, q), mx.linear(x, q), mx.linear(x, w))))


def test_the_first_product_of_a_process_may_be_a_captured_one():
    """What a device is prepared with is prepared then, too."""
    import subprocess
    import sys
    from pathlib import Path
    program = """
import torch
from paper_2502_18554_b200 import mx
x, w = torch.randn(300, 128, device="cuda"), torch.randn(400, 128, device="cuda")
graph = torch.cuda.CUDAGraph()
torch.cuda.synchronize()
with torch.cuda.graph(graph):
    y = mx.linear(x, w)
graph.replay()
assert torch.equal(y, mx.linear(x, w)) and mx.status() == 0
print("captured")
"""
    r = subprocess.run([sys.executable, "-c", program], cwd=Path(__file__).resolve().parent.parent, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "captured" in r.stdout, r.stderr[-2000:]


@pytest.mark.parametrize("m", [1, 20, 300])
def test_weights_that_were_written_just_before(mx, m):
    """Weights quantised anew into the same memory, and a layer right behind: the product asks for them before x is through."""
    gen = torch.Generator().manual_seed(m)
    ws = [torch.randn(900, 2000, generator=gen).cuda() for _ in range(4)]
    x = torch.randn(m, 2000, generator=gen).cuda()
    want = [mx.linear(x, mx.quantize(w)) for w in ws]
    q = mx.empty(900, 2000, "cuda")
    torch.cuda.synchronize()
    got = []
    for _ in range(10):
        for w in ws:
            mx.quantize(w, out=q)
            got.append(mx.linear(x, q))
    torch.cuda.synchronize()
    assert all(torch.equal(want[i % 4], y) for i, y in enumerate(got)) and mx.status() == 0
