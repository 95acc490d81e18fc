"""Microscaled 4-bit floating point on the GPU against the 64-bit reference: codes and scales byte for byte, values bit for bit."""
import numpy as np
import pytest
import torch

import _operators as ref

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.bfloat16, torch.float16]


@pytest.fixture(scope="module")
def mx():
    from paper_2502_18554_b200 import build, mx
    build.build()
    return mx


def data(rows, cols, dtype, seed, spread=8):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, cols, generator=g) * torch.exp2(torch.randint(-spread, spread + 1, (rows, cols), generator=g).float())
    x[torch.rand(rows, cols, generator=g) < 0.1] = 0
    if rows > 2:
        x[1] = 0                                    # whole blocks of zeros
    return x.to(dtype)


def wide(x):
    return x.float().numpy().astype(np.float64)


def check(mx, x, transpose, q):
    want, s = ref.quantize(wide(x).T if transpose else wide(x))
    codes, scales = ref.pack(want, s)
    # a block that reads as NaN has zeros for codes
    assert np.array_equal(q.codes.cpu().numpy().reshape(-1), codes)
    assert np.array_equal(q.scales.cpu().numpy().reshape(-1), scales)
    return ref.values(want, s, q.cols)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("transpose", [False, True])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 32), (1, 4096), (2, 31), (33, 65), (31, 128), (128, 127), (129, 384), (257, 130), (300, 4161), (1000, 8)])
def test_codes_scales_and_values(mx, rows, cols, dtype, transpose):
    x = data(rows, cols, dtype, rows * 7 + cols)
    q = mx.quantize(x.cuda(), transpose=transpose)
    assert (q.rows, q.cols) == ((cols, rows) if transpose else (rows, cols))
    want = check(mx, x, transpose, q)
    for out in TYPES:
        y = mx.dequantize(q, out)
        assert y.dtype == out and torch.equal(y.cpu(), torch.from_numpy(want).to(out))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("transpose", [False, True])
def test_pitch_and_alignment(mx, dtype, transpose):
    """Rows that lie apart, and that begin on no 16-byte boundary."""
    for shift, pitch in ((0, 136), (1, 131), (2, 132), (8, 136), (3, 160)):
        base = data(50, pitch, dtype, shift)
        flat = torch.zeros(50 * pitch + 16, dtype=dtype)
        flat[shift:shift + 50 * pitch] = base.reshape(-1)
        x = flat.cuda()[shift:shift + 50 * pitch].view(50, pitch)[:, :130]
        q = mx.quantize(x, transpose=transpose)
        want = check(mx, x.cpu(), transpose, q)
        if not transpose:
            out = torch.full((50 * pitch + 16,), 7.0, dtype=dtype, device="cuda")
            y = out[shift:shift + 50 * pitch].view(50, pitch)[:, :130]
            mx.dequantize(q, out=y)
            assert torch.equal(y.cpu(), torch.from_numpy(want).to(dtype))
            y.fill_(7.0)
            assert bool((out == 7.0).all())          # nothing around it was written


def test_ties_extremes_and_what_is_not_finite(mx):
    top = torch.finfo(torch.float32).max
    rows = [[0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 7.0, 4.0], [-0.25, -0.75, -1.25, -5.0, -7.99, 4.0], [top, -top, 1.0, 2.0 ** 125], [2.0 ** -149, -2.0 ** -130, 2.0 ** -127],
            [2.0 ** -149], [2.0 ** -126, 2.0 ** -125, 3 * 2.0 ** -128], [float("inf"), 1.0], [1.0, float("nan"), float("inf")], [-0.0, 0.0], [2.0 ** -123, 2.0 ** -124 * 1.5]]
    x = torch.zeros(len(rows), 96)
    for i, r in enumerate(rows):
        x[i, 32:32 + len(r)] = torch.tensor(r)
    for transpose in (False, True):
        y = x.t().contiguous() if transpose else x
        q = mx.quantize(y.cuda(), transpose=transpose)
        want = check(mx, y, transpose, q)
        got = mx.dequantize(q).cpu().numpy()
        assert np.array_equal(got, want.astype(np.float32), equal_nan=True)
        assert np.isnan(got[6, 32:64]).all() and np.isnan(got[7, 32:64]).all() and np.isfinite(got[6, :32]).all()


def test_every_half_value_lands_where_the_formula_says(mx):
    """All finite 16-bit floats, each as the smaller one in a block whose largest is a power of two."""
    bits = torch.arange(0, 1 << 16, dtype=torch.int32).to(torch.int16).view(torch.float16)
    bits = bits[torch.isfinite(bits)]
    x = torch.zeros(bits.numel(), 32, dtype=torch.float16)
    x[:, 0], x[:, 5] = bits, bits * 0.37
    x[:, 31] = 4.0
    check(mx, x, False, mx.quantize(x.cuda()))


@pytest.mark.parametrize("transpose", [False, True])
@pytest.mark.parametrize("top", [0.0, 2.0 ** -133, 2.0 ** -126, 1.0, 1.5 * 2.0 ** 127])
def test_every_bfloat16_lands_where_the_formula_says(mx, top, transpose):
    """Every pattern of 16 bits, infinities and NaN among them, next to numbers from the smallest to the largest binade."""
    bits = torch.arange(0, 1 << 16, dtype=torch.int32).to(torch.int16).view(torch.bfloat16)
    x = torch.zeros(bits.numel(), 32, dtype=torch.bfloat16)
    x[:, 0], x[:, 30] = bits, top
    x = x.t().contiguous() if transpose else x
    check(mx, x, transpose, mx.quantize(x.cuda(), transpose=transpose))


@pytest.mark.parametrize("transpose", [False, True])
def test_a_large_matrix(mx, transpose):
    """Sizes at which warps go round several times, against the same formula on the GPU in 64 bits (torch)."""
    x = torch.randn(16385, 4097, device="cuda", dtype=torch.bfloat16)
    q = mx.quantize(x, transpose=transpose)
    got = mx.dequantize(q, torch.bfloat16)
    t = (x.t() if transpose else x).double()
    rows, cols = t.shape
    b = torch.nn.functional.pad(t, (0, -cols % 32)).view(rows, -1, 32)
    unit = torch.exp2(torch.floor(torch.log2(b.abs().amax(-1, keepdim=True).clamp(min=2.0 ** -120))) - 2)
    a = b.abs() / unit
    grid = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    want = (torch.copysign((torch.round(a / grid) * grid).clamp(max=6), b) * unit).view(rows, -1)[:, :cols]
    assert torch.equal(got, want.to(torch.bfloat16))


def test_offsets_beyond_32_bits(mx):
    """A matrix of more than 2^32 elements, along its rows and along its columns, at its last rows and columns."""
    rows, cols = 70_001, 65_536
    x = torch.zeros(rows, cols, device="cuda", dtype=torch.bfloat16)
    end = data(33, cols, torch.bfloat16, 5)
    x[-33:] = end.cuda()
    q = mx.quantize(x)
    y = mx.dequantize(q, torch.bfloat16)
    want, s = ref.quantize(wide(end))
    assert torch.equal(y[-33:].cpu(), torch.from_numpy(ref.values(want, s, cols)).bfloat16()) and not y[: 1 << 12].any()
    del q, y
    q = mx.quantize(x, transpose=True)                  # [65536, 70001]
    y = mx.dequantize(q, torch.bfloat16)
    part = torch.zeros(64, 96, dtype=torch.bfloat16)    # the last 64 columns' last 81 elements, from a block's begin on
    part[:, :81] = x[rows - 81:, cols - 64:].t().cpu()
    want, s = ref.quantize(wide(part))
    assert (rows - 81) % 32 == 0 and torch.equal(y[-64:, rows - 81:].cpu(), torch.from_numpy(ref.values(want, s, 96)[:, :81]).bfloat16())


def test_streams_graphs_and_buffers_that_are_given(mx):
    x = data(70, 200, torch.float32, 1).cuda()
    want = mx.quantize(x)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = mx.quantize(x, stream=side)
    y = mx.dequantize(got, stream=side)
    side.synchronize()
    assert torch.equal(got.codes, want.codes) and torch.equal(got.scales, want.scales) and torch.equal(y, mx.dequantize(want))
    out = mx.empty(70, 200, x.device)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        mx.quantize(x, out=out)
        y = mx.dequantize(out)
    x.copy_(data(70, 200, torch.float32, 2))
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out.codes, mx.quantize(x).codes) and torch.equal(y, mx.dequantize(mx.quantize(x)))


@pytest.mark.parametrize("dtype", TYPES)
def test_several_matrices_in_one_call(mx, dtype):
    """Of every kind (rows in strips, rows, rows and columns on no boundary, columns), more than one launch takes, empty ones between them."""
    shapes = [(300, 520, False), (1, 32, False), (70, 131, False), (65, 96, True), (33, 77, True), (0, 64, False), (5, 0, True), (513, 1024, False), (1000, 8, True), (2, 4096, False), (129, 130, True)]
    xs = [data(r, c, dtype, i) for i, (r, c, _) in enumerate(shapes)]
    xs[7] = data(513, 8192, dtype, 7)                       # enough groups for strips of four
    forms = mx.quantize_all([x.cuda() for x in xs], [t for _, _, t in shapes])
    assert len(forms) == len(xs)
    for x, (_, _, t), q in zip(xs, shapes, forms):
        assert (q.rows, q.cols) == (tuple(reversed(x.shape)) if t else tuple(x.shape))
        if x.numel():
            check(mx, x, t, q)
    assert mx.quantize_all([]) == []
    with pytest.raises(ValueError):
        mx.quantize_all([xs[0].cuda(), xs[1].cuda().double()])
    with pytest.raises(ValueError):
        mx.quantize_all([xs[0].cuda()], [True, False])


def test_refusals(mx):
    x = torch.zeros(4, 64, device="cuda")
    q = mx.quantize(x)
    with pytest.raises(ValueError):
        mx.quantize(x.double())
    with pytest.raises(ValueError):
        mx.quantize(x.t())                                         # rows that are not contiguous
    with pytest.raises(ValueError):
        mx.quantize(x[0].expand(4, 64))                            # rows that overlap
    with pytest.raises(ValueError):
        mx.quantize(x, out=mx.empty(4, 96, x.device))
    with pytest.raises(ValueError):
        mx.quantize(x, out=mx.Mx4(q.codes[:-16], q.scales, 4, 64))
    with pytest.raises(ValueError):
        mx.quantize(x, out=mx.Mx4(q.codes, q.scales.float(), 4, 64))
    with pytest.raises(ValueError):
        mx.quantize(x, out=mx.Mx4(q.codes, q.scales.cpu(), 4, 64))
    with pytest.raises(ValueError):
        mx.dequantize(q, torch.float64)
    with pytest.raises(ValueError):
        mx.dequantize(q, out=torch.empty(4, 32, device="cuda"))
    with pytest.raises(ValueError):
        mx.quantize(x.to_sparse())
    with pytest.raises(ValueError):
        mx.quantize(torch._neg_view(x))
    with pytest.raises(RuntimeError):                              # codes that begin on no 16-byte boundary
        buffer = torch.zeros(q.codes.numel() + 1, dtype=torch.uint8, device="cuda")
        mx.dequantize(mx.Mx4(buffer[1:], q.scales, 4, 64))


def test_nothing_to_do(mx):
    for rows, cols in ((0, 64), (64, 0), (0, 0)):
        q = mx.quantize(torch.zeros(rows, cols, device="cuda"))
        assert mx.dequantize(q).shape == (rows, cols)
        q = mx.quantize(torch.zeros(rows, cols, device="cuda"), transpose=True)
        assert mx.dequantize(q).shape == (cols, rows)


def test_autograd_is_told_that_an_output_was_written(mx):
    """A tensor that was saved for a backward pass and then handed in as an output."""
    x = torch.randn(8, 64, device="cuda")
    q = mx.quantize(x)
    weights = torch.ones(8, 64, device="cuda", requires_grad=True)

    def saved(shape):
        t = torch.randn(shape, device="cuda")
        return t, (t * weights[:shape[0], :shape[1]]).sum()

    for shape, write in (((8, 64), lambda t: mx.dequantize(q, out=t)), ((8, 8), lambda t: mx.matmul(q, q, out=t))):
        t, loss = saved(shape)
        write(t)
        with pytest.raises(RuntimeError, match="modified by an inplace"):
            loss.backward()
    versions = q.codes._version, q.scales._version
    mx.quantize(x, out=q)
    assert q.codes._version > versions[0] and q.scales._version > versions[1]
    with torch.inference_mode():
        t = torch.empty(8, 64, device="cuda")
        mx.dequantize(q, out=t)                  # has no version
    assert torch.equal(t, mx.dequantize(q))


def test_autograd_is_told_that_a_norm_was_written(mx):
    from paper_2502_18554_b200 import optim
    g = [torch.randn(100, device="cuda")]
    scale = torch.ones(1, device="cuda", requires_grad=True)
    norm = optim.grad_norm(g)
    loss = (norm * scale).sum()
    optim.grad_norm(g, out=norm)
    with pytest.raises(RuntimeError, match="modified by an inplace"):
        loss.backward()


def test_an_option_that_is_neither_true_nor_false(mx):
    """What its truth value raises is what the call raises."""
    x = torch.randn(4, 64, device="cuda")
    many = np.array([1, 2])
    for call in (lambda: mx.quantize(x, transpose=many), lambda: mx.quantize_all([x], [many]), lambda: mx.linear_backward(x, x, torch.randn(64, 64, device="cuda"), (many, True))):
        with pytest.raises(ValueError):
            call()
