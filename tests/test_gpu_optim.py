"""The AdamW step over many tensors and the gradients' norm on the GPU against 64-bit references."""
import numpy as np
import pytest
import torch

import _operators as ref

pytestmark = pytest.mark.gpu
U = 2.0 ** -24      # half a step of binary32, relative
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
HYPER = dict(lr=3e-3, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.1, step=7)


@pytest.fixture(scope="module")
def optim():
    from paper_2502_18554_b200 import build, optim
    build.build()
    return optim


def wide(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def tensors(sizes, param, grad, bits, seed=0, shift=0):
    """Lists p, g, m, v (and scales) of CUDA tensors; `shift` elements into their memory."""
    gen = torch.Generator().manual_seed(seed)
    rand = lambda n, dtype, scale: (torch.randn(n + shift, generator=gen) * scale).to(dtype).cuda()[shift:]  # noqa: E731
    s = {"p": [rand(n, param, 0.05) for n in sizes], "g": [rand(n, grad, 1e-2) for n in sizes]}
    for g in s["g"]:
        g[torch.rand(g.shape, generator=gen).cuda() < 0.1] = 0
    if bits == 32:
        s["m"] = [rand(n, torch.float32, 3e-3) for n in sizes]
        s["v"] = [rand(n, torch.float32, 1e-2).square() for n in sizes]
    else:
        byte = lambda n, top: torch.randint(0, top, (n + shift,), generator=gen, dtype=torch.uint8).cuda()[shift:]  # noqa: E731
        sign = lambda n: torch.randint(0, 2, (n + shift,), generator=gen, dtype=torch.uint8).cuda()[shift:] * 128  # noqa: E731
        s["m"] = [(byte(n, 0x7F) | sign(n)).view(torch.float8_e4m3fn) for n in sizes]
        s["v"] = [byte(n, 0x7F).view(torch.float8_e4m3fn) for n in sizes]
        exponent = lambda n, lo, hi: torch.randint(lo, hi, (-(-n // 32) + shift,), generator=gen, dtype=torch.uint8).cuda()[shift:]  # noqa: E731
        s["ms"] = [exponent(n, 108, 112) for n in sizes]
        s["vs"] = [exponent(n, 110, 114) for n in sizes]
    return s


def states(s, i, bits):
    """(m, v) of tensor i in 64 bits."""
    m, v = wide(s["m"][i]), wide(s["v"][i])
    if bits == 8:
        scale = lambda k: np.repeat(np.ldexp(1.0, s[k][i].cpu().numpy().astype(int) - 127), 32)[:m.size]  # noqa: E731
        m, v = m * scale("ms"), (v * scale("vs")) ** 2
    return m, v


def run(optim, s, **more):
    optim.adamw(s["p"], s["g"], s["m"], s["v"], s.get("ms"), s.get("vs"), **{**HYPER, **more})


def bounds(p, g, m, v, hyper, norm=None):
    """What binary32 may be off by in p, m and v (before p's rounding to its type).
    m: b1, 1 - b1 and b1 m are rounded, then one fused sum: at most 4 roundings of |b1 m| + |(1 - b1) g|; clipping adds the norm's own
    rounding, a sum, a division and a product: 4 more of the second term.  v: the same with g twice.  The quotient: v's error halved, the root (2^-22 at
    most), two roundings of the sum, __fdividef's 2 ulp, the products with the rounded constants: below 24 roundings together."""
    b1, b2 = hyper["betas"]
    lr, wd, t = hyper["lr"], hyper["weight_decay"], hyper["step"]
    more = 4 if norm is not None else 0
    if norm is not None:
        g = g * min(1.0, hyper.get("max_norm", 1.0) / (norm + 1e-6))
    dm = U * (4 * b1 * np.abs(m) + (4 + more) * (1 - b1) * np.abs(g))
    dv = U * (4 * b2 * v + (6 + 2 * more) * (1 - b2) * g * g)
    new_v = b2 * v + (1 - b2) * g * g
    new_m = b1 * m + (1 - b1) * g
    denominator = np.sqrt(new_v) / np.sqrt(1 - b2 ** t) + hyper["eps"]
    rate = lr / (1 - b1 ** t)
    relative = np.where(new_v > 0, dv / np.where(new_v > 0, new_v, 1), 0)
    dp = 3 * U * np.abs(p) * (1 + lr * wd) + rate / denominator * (dm + np.abs(new_m) * (relative + 24 * U))
    return dp + 1e-45, dm + 1e-45, dv + 1e-45


def check(s, before, optim_hyper, bits, norm=None, seed=0, copies=None):
    place = 0
    for i, (p, g, m, v) in enumerate(before):
        want_p, want_m, want_v = ref.step_of(p, g, m, v, norm=norm, max_norm=optim_hyper.get("max_norm", 1.0), **{k: optim_hyper[k] for k in HYPER})
        dp, dm, dv = bounds(p, g, m, v, optim_hyper, norm)
        dtype = s["p"][i].dtype
        tiny = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24}
        assert (np.abs(wide(s["p"][i]) - want_p) <= dp + (np.abs(want_p) + dp) * (HALF[dtype] if dtype != torch.float32 else 0) + tiny[dtype]).all(), (i, "p")
        if copies:
            half = HALF[copies[i].dtype]
            assert (np.abs(wide(copies[i]) - want_p) <= dp + (np.abs(want_p) + dp) * half + tiny[copies[i].dtype]).all(), (i, "copy")
        if bits == 32:
            got_m, got_v = states(s, i, 32)
            assert (np.abs(got_m - want_m) <= dm).all() and (np.abs(got_v - want_v) <= dv).all(), i
        elif p.size:
            random = ref.random_bits(seed, optim_hyper["step"], np.arange(p.size, dtype=np.uint64) + np.uint64(place))
            off = 0
            for key, x, part, root in (("m", want_m, random >> np.uint64(16), False), ("v", np.sqrt(want_v), random & np.uint64(0xFFFF), True)):
                want, scale, grid = ref.encode8(x, part.astype(np.float64), root)
                got = wide(s[key][i])
                got_scale = s[key + "s"][i].cpu().numpy().astype(int)
                value = got * np.repeat(np.ldexp(1.0, got_scale - 127), 32)[:x.size]
                # one of the two neighbours on the grid, or the smallest element where the root would be zero
                assert (np.abs(value - x) < grid * (1 + 2.0 ** -10)).all(), (i, key)
                off += np.count_nonzero(value != want * np.repeat(np.ldexp(1.0, scale - 127), 32)[:x.size])
            # binary32 carries over where 64 bits do not only where the fraction is within its own error of the border: below 32 U of the value, 16
            # steps at most to a value, a chance of 2^-15 per element and state; five standard deviations and one block around the expectation
            mean = 2 * p.size * 2.0 ** -15
            assert off <= mean + 5 * np.sqrt(mean) + 1, (i, off)
        place += -(-p.size // 32) * 32


def snapshot(s, bits):
    return [(wide(p), wide(g), *states(s, i, bits)) for i, (p, g) in enumerate(zip(s["p"], s["g"]))]


SIZES = [1, 0, 7, 8, 31, 32, 33, 2048, 8191, 8192, 8193, 100_003]


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("param,grad", [(torch.float32, torch.float32), (torch.float32, torch.bfloat16), (torch.float32, torch.float16), (torch.bfloat16, torch.bfloat16),
                                        (torch.bfloat16, torch.float32), (torch.bfloat16, torch.float16), (torch.float16, torch.float16), (torch.float16, torch.bfloat16), (torch.float16, torch.float32)])
def test_one_step(optim, param, grad, bits):
    s = tensors(SIZES, param, grad, bits)
    before = snapshot(s, bits)
    run(optim, s, seed=12345678901234567)
    check(s, before, HYPER, bits, seed=12345678901234567)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("shift", [1, 2, 3])
def test_tensors_that_begin_anywhere(optim, bits, shift):
    s = tensors([5, 100, 9000], torch.bfloat16, torch.float32, bits, shift=shift)
    before = snapshot(s, bits)
    run(optim, s, seed=3)
    check(s, before, HYPER, bits, seed=3)


@pytest.mark.parametrize("count", [40, 41, 42, 129, 130, 132, 133, 364, 365, 380, 381, 1000])
def test_many_tensors(optim, count):
    """The numbers of tensors around which the list's form and the number of launches change."""
    sizes = [(7 * i) % 97 for i in range(count - 1)] + [20_000]
    for bits in (32, 8):
        s = tensors(sizes, torch.float32, torch.float32, bits, seed=count)
        before = snapshot(s, bits)
        run(optim, s, seed=9)
        check(s, before, HYPER, bits, seed=9)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("copy", [torch.bfloat16, torch.float16])
def test_clipping_and_copies(optim, bits, copy):
    for max_norm in (0.5, 1e6):
        s = tensors(SIZES, torch.float32, torch.bfloat16, bits)
        copies = [torch.zeros(p.shape, dtype=copy, device="cuda") for p in s["p"]]
        before = snapshot(s, bits)
        want = np.sqrt(sum((g ** 2).sum() for _, g, _, _ in before))
        norm = optim.grad_norm(s["g"])
        assert abs(float(norm) - want) <= 4 * U * want
        run(optim, s, norm=norm, max_norm=max_norm, copies=copies)
        check(s, before, {**HYPER, "max_norm": max_norm}, bits, norm=want, copies=copies)


def flat_bytes(s):
    return [t.view(torch.uint8).clone() if t.dtype != torch.float32 else t.view(torch.int32).clone() for k in ("p", "m", "v", "ms", "vs") if k in s for t in s[k]]


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("norm", [float("inf"), float("nan"), float("-inf")])
def test_a_norm_that_is_not_finite_leaves_everything(optim, bits, norm):
    s = tensors(SIZES, torch.float32, torch.float32, bits)
    copies = [torch.full(p.shape, 5.0, dtype=torch.bfloat16, device="cuda") for p in s["p"]]
    before = flat_bytes(s)
    run(optim, s, norm=torch.tensor([norm], device="cuda"), copies=copies)
    assert all(torch.equal(a, b) for a, b in zip(before, flat_bytes(s))) and all(bool((c == 5.0).all()) for c in copies)


@pytest.mark.parametrize("scale", [1e15, 1e-13])
def test_large_and_small_gradients(optim, scale):
    """Blocks whose powers of two are far from 1 (at 1e15 the scale's reciprocal is applied in two steps)."""
    for bits in (32, 8):
        s = tensors([5000, 77], torch.float32, torch.float32, bits)
        for k in ("g", "m", "v"):
            for x in s[k]:
                if bits == 32 or k == "g":
                    x.mul_(scale * scale if k == "v" else scale)
        if bits == 8:
            for k in ("ms", "vs"):
                for x in s[k]:
                    x.add_(int(np.round(np.log2(scale))))
        before = snapshot(s, bits)
        run(optim, s, seed=21)
        check(s, before, HYPER, bits, seed=21)


def test_offsets_beyond_32_bits(optim):
    """A tensor of 2^32 elements and some behind another one, states in 8 bits: its end against the reference, random bits by their place included."""
    n, first = (1 << 32) + 77, 45
    make = lambda k, dtype: torch.zeros(k, dtype=dtype, device="cuda")  # noqa: E731
    s = {key: [make(first, dtype), make(n, dtype)] for key, dtype in (("p", torch.bfloat16), ("g", torch.bfloat16), ("m", torch.float8_e4m3fn), ("v", torch.float8_e4m3fn))}
    s |= {key: [make(2, torch.uint8), make(-(-n // 32), torch.uint8)] for key in ("ms", "vs")}
    tail = 4096 + 77
    g = (torch.randn(tail, generator=torch.Generator().manual_seed(3)) * 1e-2).bfloat16().cuda()
    s["g"][1][n - tail:] = g
    s["p"][1][n - tail:] = 1.0
    norm = optim.grad_norm(s["g"])
    want_norm = np.sqrt((wide(g) ** 2).sum())
    assert abs(float(norm) - want_norm) <= 6 * U * want_norm
    run(optim, s, seed=8)
    want_p, want_m, want_v = ref.step_of(np.ones(tail), wide(g), np.zeros(tail), np.zeros(tail), **HYPER)
    dp, _, _ = bounds(np.ones(tail), wide(g), np.zeros(tail), np.zeros(tail), HYPER)
    assert (np.abs(wide(s["p"][1][n - tail:]) - want_p) <= dp + (np.abs(want_p) + dp) * HALF[torch.bfloat16]).all()
    random = ref.random_bits(8, HYPER["step"], np.arange(n - tail, n, dtype=np.uint64) + np.uint64(64))
    for key, x, part, root in (("m", want_m, random >> np.uint64(16), False), ("v", np.sqrt(want_v), random & np.uint64(0xFFFF), True)):
        want, scale, _ = ref.encode8(x, part.astype(np.float64), root)
        got = wide(s[key][1][n - tail:]) * np.repeat(np.ldexp(1.0, s[key + "s"][1][(n - tail) // 32:].cpu().numpy().astype(int) - 127), 32)[:tail]
        off = np.count_nonzero(got != want * np.repeat(np.ldexp(1.0, scale - 127), 32)[:tail])
        assert off <= 2      # see check(): a chance of 2^-15 per element
    assert not s["p"][1][:1 << 20].any() and not s["m"][1][1 << 31:(1 << 31) + (1 << 20)].view(torch.uint8).any()


def test_a_step_of_many_elements_is_that_of_few(optim):
    """How elements are divided among CTAs depends on how many there are in all; what becomes of a tensor does not."""
    n, more = 9_000_011, (1 << 26) - 9_000_011
    make = lambda: tensors([n], torch.bfloat16, torch.bfloat16, 8, seed=5)  # noqa: E731
    s, twin = make(), make()
    run(optim, s, seed=2)
    other = {key: torch.zeros(more, dtype=x[0].dtype, device="cuda") for key, x in twin.items() if key in ("p", "g", "m", "v")}
    other |= {key: torch.zeros(-(-more // 32), dtype=torch.uint8, device="cuda") for key in ("ms", "vs")}
    run(optim, {key: x + [other[key]] for key, x in twin.items() if key in other}, seed=2)
    for key in other:
        assert torch.equal(s[key][0].view(torch.uint8), twin[key][0].view(torch.uint8)), key


def test_a_gradient_that_is_not_finite_stays_in_its_block(optim):
    for bits in (32, 8):
        s = tensors([200], torch.float32, torch.float32, bits)
        s["g"][0][70] = float("nan")
        s["g"][0][130] = float("inf")
        before = snapshot(s, bits)
        run(optim, s)
        p = wide(s["p"][0])
        assert np.isnan(p[[70, 130]]).all() and np.isfinite(np.delete(p, [70, 130])).all()
        if bits == 8:
            assert s["ms"][0].tolist()[2] == 255 and s["ms"][0].tolist()[4] == 255 and s["vs"][0].tolist()[2] == 255
            assert 255 not in s["ms"][0].tolist()[:2] + [s["ms"][0].tolist()[3]]
            run(optim, s)                          # and reads as NaN from then on, the others go on
            p = wide(s["p"][0])
            assert np.isnan(p[64:96]).all() and np.isnan(p[128:160]).all() and np.isfinite(p[:64]).all() and np.isfinite(p[96:128]).all()
        assert len(before)


def test_zeros_and_the_smallest_numbers(optim):
    """Nothing to learn from: no division of 0 by 0; roots above zero stay above zero."""
    z = lambda dtype: [torch.zeros(64, dtype=dtype, device="cuda")]  # noqa: E731
    p = [torch.ones(64, device="cuda")]
    m, v, ms, vs = z(torch.float8_e4m3fn), z(torch.float8_e4m3fn), [torch.zeros(2, dtype=torch.uint8, device="cuda")], [torch.zeros(2, dtype=torch.uint8, device="cuda")]
    optim.adamw(p, z(torch.float32), m, v, ms, vs, **HYPER)
    assert torch.allclose(p[0], torch.full_like(p[0], 1 - HYPER["lr"] * HYPER["weight_decay"]), rtol=2 * U, atol=0) and not m[0].view(torch.uint8).any() and not vs[0].any()
    g = torch.full((64,), 1e-9, device="cuda")
    g[0] = 1.0
    optim.adamw(p, [g], m, v, ms, vs, **HYPER)
    assert bool((v[0].float()[:32] > 0).all())      # 1e-9 is far below the first block's smallest element
    optim.adamw(p, z(torch.float32), m, v, ms, vs, **HYPER)
    assert bool(torch.isfinite(p[0]).all())


def test_rounding_is_unbiased(optim):
    """The mean over 400 seeds is the value, within five standard deviations of a rounding between two neighbours (half a step at most); roots
    below the block's smallest element are that element, never 0."""
    n, seeds = 256, 400
    gen = torch.Generator().manual_seed(0)
    g = (torch.randn(n, generator=gen) * torch.exp2(torch.randint(-6, 1, (n,), generator=gen).float())).cuda()
    g[3], g[100] = 1e-12, -1e-7
    total_m, total_r = np.zeros(n), np.zeros(n)
    for seed in range(seeds):
        s = {"p": [torch.zeros(n, device="cuda")], "g": [g], "m": [torch.zeros(n, device="cuda").to(torch.float8_e4m3fn)], "v": [torch.zeros(n, device="cuda").to(torch.float8_e4m3fn)],
             "ms": [torch.zeros(8, dtype=torch.uint8, device="cuda")], "vs": [torch.zeros(8, dtype=torch.uint8, device="cuda")]}
        run(optim, s, seed=seed * 7919)
        m, v = states(s, 0, 8)
        total_m += m
        total_r += np.sqrt(v)
    x = wide(g)
    for total, want in ((total_m, 0.1 * x), (total_r, np.sqrt(0.001) * np.abs(x))):
        _, scale, grid = ref.encode8(want, np.zeros(n), False)
        if total is total_r:
            want = np.maximum(want, np.repeat(np.ldexp(2.0 ** -9, scale - 127), 32))
        assert (np.abs(total / seeds - want) <= 5 * 0.5 * grid / np.sqrt(seeds) + 2.0 ** -16 * grid).all()


def test_the_same_call_gives_the_same_bits(optim):
    got = []
    for _ in range(2):
        s = tensors(SIZES, torch.bfloat16, torch.bfloat16, 8, seed=4)
        norm = optim.grad_norm(s["g"])
        run(optim, s, norm=norm, max_norm=0.1, seed=77)
        got.append([norm.clone()] + flat_bytes(s))
    assert all(torch.equal(a, b) for a, b in zip(*got))


@pytest.mark.parametrize("bits", [32, 8])
def test_captured_steps_read_step_rate_and_norm_when_they_run(optim, bits):
    s, twin = tensors(SIZES, torch.float32, torch.float32, bits, seed=6), tensors(SIZES, torch.float32, torch.float32, bits, seed=6)
    step = torch.zeros(1, dtype=torch.int64, device="cuda")
    lr = torch.zeros(1, device="cuda")
    hyper = {k: HYPER[k] for k in ("betas", "eps", "weight_decay")}
    graph = torch.cuda.CUDAGraph()
    optim.grad_norm(s["g"])                       # loads the kernels
    with torch.cuda.graph(graph):
        step.add_(1)
        norm = optim.grad_norm(s["g"])
        optim.adamw(s["p"], s["g"], s["m"], s["v"], s.get("ms"), s.get("vs"), step=step, lr=lr, norm=norm, max_norm=0.3, seed=5, **hyper)
    for t in (1, 2, 3):
        rate = 1e-3 * t
        lr.fill_(rate)
        for a, b in zip(s["g"], twin["g"]):
            a.mul_(1.5)
            b.mul_(1.5)
        graph.replay()
        n2 = optim.grad_norm(twin["g"])
        before = snapshot(twin, bits)
        optim.adamw(twin["p"], twin["g"], twin["m"], twin["v"], twin.get("ms"), twin.get("vs"), step=t, lr=float(lr), norm=n2, max_norm=0.3, seed=5, **hyper)
        torch.cuda.synchronize()
        assert torch.equal(norm, n2)
        assert all(torch.equal(a, b) for a, b in zip(flat_bytes(s)[len(SIZES):], flat_bytes(twin)[len(SIZES):]))    # states do not depend on the rate
        for a, b, (p, g, m, v) in zip(s["p"], twin["p"], before):
            # the constants are computed on the device in binary64 and rounded to binary32: each may end one step away
            dp, _, _ = bounds(p, g, m, v, {**HYPER, "lr": rate, "step": t, "max_norm": 0.3}, float(n2))
            assert (np.abs(wide(a) - wide(b)) <= 2 * dp).all()
    assert int(step) == 3


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_norm(optim, dtype):
    for sizes, scale in (([1], 1.0), ([0, 3], 1.0), (SIZES, 1e-3), ([9] * 900 + [300_001], 1.0), ([8192 * 1025 + 17], 1e-2)):
        g = [(torch.randn(n, device="cuda") * scale).to(dtype) for n in sizes]
        want = np.sqrt(sum((wide(x) ** 2).sum() for x in g))
        # eight squares are added in binary32 (8 roundings at most of a sum of positive numbers), the rest in binary64; the root halves that, and the result is rounded
        assert abs(float(optim.grad_norm(g)) - want) <= 6 * U * want
    g = [torch.zeros(100, dtype=dtype, device="cuda")]
    assert float(optim.grad_norm(g)) == 0.0
    for bad in (float("inf"), float("nan")):
        g[0][50] = bad
        assert not np.isfinite(float(optim.grad_norm(g)))
    out = torch.full((1,), 9.0, device="cuda")
    assert float(optim.grad_norm([], out=out)) == 0.0


def test_norm_of_numbers_whose_squares_leave_binary32(optim):
    for value in (1e-30, 2.0 ** -140, 1e25, 3e38):
        g = [torch.full((1000,), value, device="cuda")]
        want = float(torch.tensor(value)) * np.sqrt(1000.0)
        got = float(optim.grad_norm(g))
        if want > 3.4028235e38:
            assert got == float("inf")
        else:
            assert abs(got - want) <= max(4 * U * want, 2.0 ** -149)


def test_on_another_stream(optim):
    s, twin = tensors(SIZES, torch.float32, torch.float32, 8, seed=8), tensors(SIZES, torch.float32, torch.float32, 8, seed=8)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    norm = optim.grad_norm(s["g"], stream=side)
    run(optim, s, norm=norm, stream=side)
    side.synchronize()
    run(optim, twin, norm=optim.grad_norm(twin["g"]))
    assert all(torch.equal(a, b) for a, b in zip(flat_bytes(s), flat_bytes(twin)))


def test_autograd_is_told_that_parameters_changed(optim):
    s = tensors([64], torch.float32, torch.float32, 32)
    p = s["p"][0].requires_grad_()
    y = (p * p).sum()
    run(optim, s)
    with pytest.raises(RuntimeError):
        y.backward()


def test_refusals(optim):
    def fresh(**changes):
        s = tensors([64, 32], torch.float32, torch.float32, 32)
        s.update(changes)
        return s

    t = lambda n, **k: torch.zeros(n, device="cuda", **k)  # noqa: E731
    with pytest.raises(ValueError):
        run(optim, fresh(g=[t(64)]))                                       # lists of different lengths
    with pytest.raises(ValueError):
        run(optim, fresh(g=[t(64), t(31)]))
    with pytest.raises(ValueError):
        run(optim, fresh(p=[t(64), t(32, dtype=torch.bfloat16)]))          # two types in a list
    with pytest.raises(ValueError):
        run(optim, fresh(p=[t(64), t(32, dtype=torch.float64)]))
    with pytest.raises(ValueError):
        run(optim, fresh(m=[t(64), t(64)[::2]]))                           # not contiguous
    with pytest.raises(ValueError):
        run(optim, fresh(v=[t(64), torch.zeros(32)]))                      # not on the GPU
    with pytest.raises(ValueError):
        run(optim, fresh(m=[t(64, dtype=torch.bfloat16), t(32, dtype=torch.bfloat16)]))
    both = t(80)
    with pytest.raises(ValueError):
        run(optim, fresh(p=[both[:64], both[48:]]))                        # overlapping parameters
    one = t(64)
    with pytest.raises(ValueError):
        run(optim, fresh(m=[one, one[:32]]))
    with pytest.raises(ValueError):
        run(optim, fresh(), copies=[t(64), t(32)])                         # float32 copies
    with pytest.raises(ValueError):
        run(optim, fresh(ms=[t(2, dtype=torch.uint8), t(1, dtype=torch.uint8)]))
    with pytest.raises(ValueError):
        run(optim, fresh(), norm=t(2))
    with pytest.raises(ValueError):
        run(optim, fresh(), lr=torch.zeros(1))
    with pytest.raises(ValueError):
        run(optim, fresh(), step=t(1))
    with pytest.raises(RuntimeError):
        run(optim, fresh(), step=0)
    with pytest.raises(RuntimeError):
        run(optim, fresh(), betas=(0.9, 1.0))
    for other in (t(64).to_sparse(), torch.zeros(64, device="meta")):
        with pytest.raises((ValueError, RuntimeError)):
            run(optim, fresh(g=[other, t(32)]))
        with pytest.raises((ValueError, RuntimeError)):
            optim.grad_norm([other])
    s = tensors([64, 32], torch.float32, torch.float32, 8)
    s["vs"][0] = s["vs"][0][:1]
    with pytest.raises(ValueError):
        run(optim, s)
    with pytest.raises(ValueError):
        optim.grad_norm([t(5), t(5, dtype=torch.bfloat16)])
    with pytest.raises(ValueError):
        optim.grad_norm([t(6)[::2]])
    run(optim, {"p": [], "g": [], "m": [], "v": []})                       # nothing to do


@pytest.mark.parametrize("bits", [32, 8])
def test_the_smallest_eps(optim, bits):
    """Nothing learnt and nothing to learn: 0 / eps is 0 down to the smallest normal number; what is below it is refused."""
    make = lambda: tensors([64, 5000], torch.float32, torch.float32, bits)  # noqa: E731
    for eps in (2.0 ** -126, 1e-30, 1e-8):
        s = make()
        for key in ("g", "m", "v"):
            for x in s[key]:
                x.view(torch.uint8).zero_()
        before = [p.clone() for p in s["p"]]
        run(optim, s, eps=eps)
        for p, q in zip(s["p"], before):
            assert torch.allclose(p, q * (1 - HYPER["lr"] * HYPER["weight_decay"]), rtol=4 * U, atol=0)
    for eps in (1e-40, 1e-60):
        s = make()
        before = flat_bytes(s)
        with pytest.raises(RuntimeError):
            run(optim, s, eps=eps)
        assert all(torch.equal(a, b) for a, b in zip(before, flat_bytes(s)))


@pytest.mark.parametrize("bits", [32, 8])
def test_tensors_that_are_in_two_lists_are_refused(optim, bits):
    """A parameter's gradient, states, scales and copy share no memory, wherever in the list it stands."""
    for i in (0, 1, 2):
        s = tensors([64, 7, 4096], torch.float32, torch.float32, bits)
        before = flat_bytes(s)
        other = lambda key, x: {**s, key: [x if j == i else t for j, t in enumerate(s[key])]}  # noqa: E731
        cases = [other("v", s["m"][i]), {**s, "v": s["m"]}]
        if bits == 32:
            cases += [other("g", s["p"][i]), other("m", s["p"][i]), other("v", s["g"][i])]
        else:
            cases += [other("vs", s["ms"][i]), other("ms", s["p"][i].view(torch.uint8)[:s["ms"][i].numel()])]
        for case in cases:
            with pytest.raises(ValueError, match="overlap"):
                run(optim, case)
        copies = [torch.zeros(t.numel(), dtype=torch.bfloat16, device="cuda") for t in s["p"]]
        copies[i] = s["p"][i].view(torch.bfloat16)[:s["p"][i].numel()]
        with pytest.raises(ValueError, match="overlap"):
            run(optim, s, copies=copies)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(before, flat_bytes(s)))


@pytest.mark.parametrize("param", [torch.float32, torch.float16])
def test_a_step_of_many_elements_is_that_of_few_in_every_type(optim, param):
    """As test_a_step_of_many_elements_is_that_of_few: elements are divided among CTAs in another way from 64 Mi of 16 bits on, and not of binary32."""
    n, more = 5_000_011, (1 << 26) - 5_000_011
    make = lambda: tensors([n], param, torch.bfloat16, 8, seed=5)  # noqa: E731
    s, twin = make(), make()
    run(optim, s, seed=2)
    other = {key: torch.zeros(more, dtype=x[0].dtype, device="cuda") for key, x in twin.items() if key in ("p", "g", "m", "v")}
    other |= {key: torch.zeros(-(-more // 32), dtype=torch.uint8, device="cuda") for key in ("ms", "vs")}
    run(optim, {key: x + [other[key]] for key, x in twin.items() if key in other}, seed=2)
    for key in other:
        assert torch.equal(s[key][0].view(torch.uint8), twin[key][0].view(torch.uint8)), key
