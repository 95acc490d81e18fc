"""What the time of the operators around a gradient exchange is measured on: quantisation to microscaled 4-bit floating
point and back, the product of operands in that form with its gradient, and the AdamW step over many tensors with states in
32 or 8 bits, as programs call them (`mx`, `optim`).

The plain forms compute the same from elementary torch operations in 32 bits.  Both take the same buffers:

* a matrix [rows, cols] in microscaled form is `codes` uint8 [rows, 16 * blocks] (blocks of 32 along the row, the last one
  filled up with zeros; element 2j in the low half of byte j: sign, two exponent bits, one mantissa bit) and `scales` uint8
  (per block the exponent + 127), in tiles of 128 rows x 4 blocks of 512 bytes, rows r, r + 32, r + 64, r + 96 of a tile side by side;
* parameters, gradients and states are views of flat arrays, every tensor beginning at a multiple of 32 elements.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
LR, BETA1, BETA2, EPS, DECAY, MAX_NORM, SEED = 1e-3, 0.9, 0.999, 1e-8, 0.1, 1.0, 0x5DEECE66D


def listed():
    return [
        # one token's activations on their way into a product
        {"name": "quantise 1x4096", "op": "quantize", "rows": 1, "cols": 4096, "type": "bf16", "transpose": False},
        # the activations of a large batch
        {"name": "quantise 16384x4096", "op": "quantize", "rows": 16384, "cols": 4096, "type": "bf16", "transpose": False},
        # a gradient of no round size, along the other axis, as the weights' gradient needs it
        {"name": "quantise columns 5003x2055", "op": "quantize", "rows": 5003, "cols": 2055, "type": "f32", "transpose": True},
        # one token through a large layer whose weights are kept in 4 bits: latency and the weights' bytes
        {"name": "linear 1x8192x16384", "op": "linear", "m": 1, "k": 8192, "n": 16384, "type": "bf16"},
        # a few sequences' next tokens, sizes that fill no tile
        {"name": "linear 13x4161x10007", "op": "linear", "m": 13, "k": 4161, "n": 10007, "type": "bf16"},
        # a prompt
        {"name": "linear 4096x8192x8192", "op": "linear", "m": 4096, "k": 8192, "n": 8192, "type": "f16"},
        # training: output, gradient of the input and of the weights; small and ragged, then large
        {"name": "train 777x1000x1531", "op": "train", "m": 777, "k": 1000, "n": 1531, "type": "bf16"},
        {"name": "train 4096x4096x4096", "op": "train", "m": 4096, "k": 4096, "n": 4096, "type": "bf16"},
        # the step of a small model: latency
        {"name": "adamw 20000", "op": "adamw", "bits": 32, "tensors": 6, "total": 20_000, "param": "f32", "grad": "f32", "clip": False, "copy": False},
        # 32-bit weights with a 16-bit copy for the forward pass, gradients clipped by their norm
        {"name": "adamw 64Mi", "op": "adamw", "bits": 32, "tensors": 150, "total": 1 << 26, "param": "f32", "grad": "bf16", "clip": True, "copy": True},
        # 16-bit weights, states in 8 bits, no clipping
        {"name": "adamw8 128Mi", "op": "adamw", "bits": 8, "tensors": 290, "total": 1 << 27, "param": "bf16", "grad": "bf16", "clip": False, "copy": False},
        # tensors of odd sizes, states in 8 bits, clipped
        {"name": "adamw8 1000003", "op": "adamw", "bits": 8, "tensors": 37, "total": 1_000_003, "param": "f32", "grad": "f32", "clip": True, "copy": False},
    ]


def _size(rng, lo, hi):
    """Log-uniform over [lo, hi]; one out of two is odd, the others a multiple of 32 where that leaves any."""
    n = int(math.exp(rng.uniform(math.log(lo), math.log(hi))))
    return max(lo, n & ~31) if rng.random() < 0.5 else max(lo, min(hi, n | 1))


def draw(rng: random.Random):
    op = rng.choice(["quantize", "linear", "linear", "train", "adamw", "adamw"])
    if op == "quantize":
        rows = _size(rng, 1, 16384)
        return {"op": op, "rows": rows, "cols": _size(rng, 8, min(16384, (1 << 26) // rows)), "type": rng.choice(list(DTYPES)), "transpose": rng.random() < 0.5}
    if op == "linear":
        return {"op": op, "m": _size(rng, 1, 4096), "k": _size(rng, 32, 8192), "n": _size(rng, 32, 8192), "type": rng.choice(["bf16", "f16"])}
    if op == "train":
        return {"op": op, "m": _size(rng, 32, 4096), "k": _size(rng, 32, 4096), "n": _size(rng, 32, 4096), "type": rng.choice(["bf16", "f16"])}
    bits = rng.choice([8, 32])
    param = rng.choice(["f32", "bf16"])
    return {"op": op, "bits": bits, "tensors": rng.randint(1, 300), "total": _size(rng, 4000, 1 << 26), "param": param, "grad": rng.choice([param, "bf16"]),
            "clip": rng.random() < 0.5, "copy": param == "f32" and rng.random() < 0.5}


# ---- inputs

def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _activations(rows, cols, dtype, g):
    """Normal values whose columns differ in size, a few columns twenty times the others."""
    channel = torch.exp(0.5 * torch.randn(cols, device="cuda", generator=g))
    channel = torch.where(torch.rand(cols, device="cuda", generator=g) < 0.005, 20 * channel, channel)
    return (torch.randn(rows, cols, device="cuda", generator=g) * channel).to(dtype)


def _gradients(shape, dtype, g):
    """Laplace-distributed with scale 1e-3, a tenth of them exact zeros."""
    u = torch.rand(shape, device="cuda", generator=g) - 0.5
    x = -1e-3 * torch.sign(u) * torch.log1p(-2 * u.abs().clamp(max=0.4999999))
    return torch.where(torch.rand(shape, device="cuda", generator=g) < 0.1, 0.0, x).to(dtype)


def _sizes(case):
    """Elements of the case's tensors: a few large ones among many small ones, together `total`."""
    rng = random.Random(case["total"] * 1009 + case["tensors"])
    count = min(case["tensors"], case["total"])
    share = [math.exp(rng.uniform(0, 6)) for _ in range(count)]
    left = case["total"] - count
    sizes = [1 + int(left * s / sum(share)) for s in share]
    sizes[-1] += case["total"] - sum(sizes)
    return sizes


def _layout(sizes):
    """Where each tensor begins, and the length of the flat array."""
    at, offsets = 0, []
    for n in sizes:
        offsets.append(at)
        at += -(-n // 32) * 32
    return offsets, at


def prepare(case, seed):
    g = _generator(seed)
    op = case["op"]
    if op == "quantize":
        make = _gradients if case["transpose"] else lambda s, t, q: _activations(*s, t, q)
        return dict(case, x=make((case["rows"], case["cols"]), DTYPES[case["type"]], g))
    if op in ("linear", "train"):
        m, k, n, dtype = case["m"], case["k"], case["n"], DTYPES[case["type"]]
        s = dict(case, x=_activations(m, k, dtype, g))
        w = (torch.randn(n, k, device="cuda", generator=g) * (0.5 / math.sqrt(k))).to(dtype)
        if op == "linear":
            codes, exponents = _quantize(w)
            s |= {"codes": _pack(codes), "scales": _tile_scales(exponents)}   # the weights, laid out once
        else:
            s |= {"w": w, "dy": _gradients((m, n), dtype, g)}
        return s
    sizes = _sizes(case)
    offsets, total = _layout(sizes)
    inside = torch.zeros(total, dtype=torch.bool, device="cuda")
    for o, n in zip(offsets, sizes):
        inside[o:o + n] = True
    flat = lambda x, dtype: torch.where(inside, x, 0).to(dtype)  # noqa: E731
    s = dict(case, step=100)
    s["p"] = flat(0.02 * torch.randn(total, device="cuda", generator=g), DTYPES[case["param"]])
    s["g"] = flat(_gradients((total,), torch.float32, g), DTYPES[case["grad"]])
    m = flat(4e-4 * torch.randn(total, device="cuda", generator=g), torch.float32)
    v = flat(1e-6 * torch.exp(torch.randn(total, device="cuda", generator=g)), torch.float32)
    if case["bits"] == 8:
        half = torch.full((total,), 1 << 15, dtype=torch.int32, device="cuda")
        s["m"], s["m_scale"] = _pack8(m, half, False)
        s["v"], s["v_scale"] = _pack8(v.sqrt(), half, True)
    else:
        s["m"], s["v"] = m, v
    if case["copy"]:
        s["copy"] = torch.zeros(total, dtype=torch.bfloat16, device="cuda")
    # what a training program holds: lists of tensors
    per = {"p": 1, "g": 1, "m": 1, "v": 1, "copy": 1, "m_scale": 32, "v_scale": 32}
    s["lists"] = {key: [s[key][o // d:o // d + -(-n // d)] for o, n in zip(offsets, sizes)] for key, d in per.items() if torch.is_tensor(s.get(key))}
    return s


# ---- plain forms

def _tile_scales(exponents):
    """Biased exponents [rows, blocks] in tiles of 128 rows x 4 blocks."""
    rows, blocks = exponents.shape
    full = torch.nn.functional.pad(exponents, (0, -blocks % 4, 0, -rows % 128))
    return full.view(full.shape[0] // 128, 4, 32, full.shape[1] // 4, 4).permute(0, 3, 2, 1, 4).reshape(-1).to(torch.uint8)


def _untile_scales(scales, rows, blocks):
    across, down = -(-blocks // 4), -(-rows // 128)
    return scales.view(down, across, 32, 4, 4).permute(0, 3, 2, 1, 4).reshape(down * 128, across * 4)[:rows, :blocks].int()


def _power(biased):
    """2 ** (biased - 127) in 32 bits, for biased exponents 0 ... 254."""
    return torch.where(biased > 0, biased << 23, 1 << 22).int().view(torch.float32)


def _quantize(x):
    """Codes [rows, 32 * blocks] and biased exponents [rows, blocks] of x [rows, cols]."""
    rows, cols = x.shape
    x = torch.nn.functional.pad(x.float(), (0, -cols % 32)).view(rows, -1, 32)
    biased = ((x.abs().amax(-1).view(torch.int32) >> 23) - 2).clamp(min=0)
    y = x * _power(254 - biased)[..., None]
    a = y.abs()
    code = (a > 0.25).int() + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5)
    return (code + 8 * torch.signbit(y)).view(rows, -1), biased


def _pack(codes):
    return (codes[:, 0::2] + 16 * codes[:, 1::2]).to(torch.uint8)


def _unpack(packed):
    return torch.stack((packed & 15, packed >> 4), -1).view(packed.shape[0], -1).int()


def _values(codes, biased, cols):
    """What codes and exponents stand for, in 32 bits, [rows, cols]."""
    table = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6], device=codes.device)
    return (table[codes].view(codes.shape[0], -1, 32) * _power(biased)[..., None]).view(codes.shape[0], -1)[:, :cols]


def _rounded(x):
    """x as its microscaled form has it."""
    return _values(*_quantize(x), x.shape[1])


def _random16(total, seed, step):
    """Two 16-bit random numbers for each element: a mix of its place, the seed and the step's number."""
    key = (seed + step * 0x9E3779B97F4A7C15) & 0xFFFFFFFFFFFFFFFF
    at = torch.arange(total, dtype=torch.int64, device="cuda")
    h = ((at ^ (key & 0xFFFFFFFF)) & 0xFFFFFFFF) * 0x7FEB352D & 0xFFFFFFFF
    h = ((h ^ (h >> 15)) ^ (key >> 32) ^ (at >> 32)) * 0x846CA68B & 0xFFFFFFFF
    h = (h ^ (h >> 13)) * 0x6C8E9CF5 & 0xFFFFFFFF
    h = h ^ (h >> 16)
    return (h >> 16).int(), (h & 0xFFFF).int()


def _pack8(x, noise, floor):
    """Blocks of 32 with one power of two each: (float8 values, biased exponents).  An element goes to the next value of the grid
    further from zero where its 16 random bits, in units of 1 / 65536 of a step, carry over.  `floor`: nothing above 0 becomes 0."""
    blocks = x.view(-1, 32)
    bits = blocks.abs().amax(-1).view(torch.int32)
    biased = ((bits >> 23) - 8 + ((bits & 0x7FFFFF) > 0x600000)).clamp(min=0)
    y = (blocks * _power(254 - biased)[:, None]).view(-1)
    a = y.abs()
    noise = noise << 4
    normal = ((a.view(torch.int32) + noise) >> 20) - (120 << 3)
    small = ((a * 2.0 ** 29).int() + noise) >> 20
    code = torch.where(a >= 2.0 ** -6, normal, small)
    if floor:
        code = torch.where(x > 0, code.clamp(min=1), code)
    return (code + 128 * (x < 0)).to(torch.uint8).view(torch.float8_e4m3fn), biased.to(torch.uint8)


def _unpack8(codes, biased):
    return (codes.float().view(-1, 32) * _power(biased.int())[:, None]).view(-1)


def _adamw(s):
    s["step"] += 1
    t, out = s["step"], {}
    g = s["g"].float()
    if s["clip"]:
        norm = g.double().square().sum().sqrt().float()
        g = g * torch.clamp(MAX_NORM / (norm + 1e-6), max=1.0)
        out["norm"] = norm.view(1)
    eight = s["bits"] == 8
    m, v = (_unpack8(s["m"], s["m_scale"]), _unpack8(s["v"], s["v_scale"]).square()) if eight else (s["m"], s["v"])
    m = BETA1 * m + (1 - BETA1) * g
    v = BETA2 * v + (1 - BETA2) * g * g
    root = v.sqrt()
    p = s["p"].float() * (1 - LR * DECAY) - LR / (1 - BETA1 ** t) * (m / (root / math.sqrt(1 - BETA2 ** t) + EPS))
    s["p"].copy_(p)
    if torch.is_tensor(s["copy"]):
        s["copy"].copy_(p)
    if eight:
        first, second = _random16(m.numel(), SEED, t)
        for key, (codes, biased) in (("m", _pack8(m, first, False)), ("v", _pack8(root, second, True))):
            s[key].view(torch.uint8).copy_(codes.view(torch.uint8))
            s[key + "_scale"].copy_(biased)
    else:
        s["m"].copy_(m)
        s["v"].copy_(v)
    return _updated(s, out)


def _updated(s, out):
    out |= {key: s[key] for key in ("p", "m", "v", "copy") if torch.is_tensor(s.get(key))}
    return out | {key: s[key].view(torch.float8_e8m0fnu) for key in ("m_scale", "v_scale") if key in s}


def _plain(s):
    op = s["op"]
    if op == "quantize":
        return _rounded(s["x"].t() if s["transpose"] else s["x"]).to(s["x"].dtype)
    if op == "linear":
        x = _rounded(s["x"])
        w = _values(_unpack(s["codes"]), _untile_scales(s["scales"], s["n"], -(-s["k"] // 32)), s["k"])
        return (x @ w.t()).to(s["x"].dtype)
    if op == "train":
        x, w, dy, dtype = s["x"], s["w"], s["dy"], s["x"].dtype
        y = _rounded(x) @ _rounded(w).t()
        dx = _rounded(dy) @ _rounded(w.t()).t()
        dw = _rounded(dy.t()) @ _rounded(x.t()).t()
        return {"y": y.to(dtype), "dx": dx.to(dtype), "dw": dw.to(dtype)}
    return _adamw(s)


def run(s):
    if own:
        return _own(s)
    return _plain(s)


# ---- the framework's calls

def _own(s):
    from paper_2502_18554_b200 import mx, optim
    op = s["op"]
    if op == "quantize":
        return mx.dequantize(mx.quantize(s["x"], transpose=s["transpose"]), s["x"].dtype)
    if op == "linear":
        return mx.linear(s["x"], mx.Mx4(s["codes"], s["scales"], s["n"], s["k"]))
    if op == "train":
        y = mx.linear(s["x"], s["w"])
        dx, dw = mx.linear_backward(s["dy"], s["x"], s["w"])
        return {"y": y, "dx": dx, "dw": dw}
    s["step"] += 1
    t, out = s["lists"], {}
    if s["clip"]:
        out["norm"] = optim.grad_norm(t["g"])
    optim.adamw(t["p"], t["g"], t["m"], t["v"], t.get("m_scale"), t.get("v_scale"), copies=t.get("copy"), step=s["step"], lr=LR, betas=(BETA1, BETA2),
                eps=EPS, weight_decay=DECAY, norm=out.get("norm"), max_norm=MAX_NORM, seed=SEED)
    return _updated(s, out)


# ---- what a pass cannot do without

def work(case):
    size = lambda key: DTYPES[case[key]].itemsize  # noqa: E731
    if case["op"] == "quantize":
        return {"bytes": 2 * case["rows"] * case["cols"] * size("type"), "flops": 0}
    if case["op"] == "adamw":
        per = 2 * size("param") + size("grad") + (4 * (1 + 1 / 32) if case["bits"] == 8 else 16) + 2 * case["copy"]
        return {"bytes": case["total"] * per, "flops": 16 * case["total"]}
    m, k, n, b = case["m"], case["k"], case["n"], size("type")
    if case["op"] == "linear":
        return {"bytes": (m * k + m * n) * b + n * k * 17 / 32, "flops": 2 * m * k * n}
    return {"bytes": 2 * (m * k + n * k + m * n) * b, "flops": 6 * m * k * n}


# ---- the definition in 64 bits

def _exact_rounded(x):
    """Nearest multiple of the element's step, ties to the even one, by division instead of comparisons."""
    rows, cols = x.shape
    x = torch.nn.functional.pad(x.double(), (0, -cols % 32)).view(rows, -1, 32)
    _, e = torch.frexp(x.abs().amax(-1, keepdim=True))
    unit = torch.exp2((e - 3).clamp(min=-127).double())
    unit = torch.where(x.abs().amax(-1, keepdim=True) > 0, unit, torch.exp2(torch.tensor(-127.0, dtype=torch.float64, device=x.device)))
    a = x.abs() / unit
    grid = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    return (torch.copysign((torch.round(a / grid) * grid).clamp(max=6), x) * unit).view(rows, -1)[:, :cols]


def _exact_pack8(x, noise, floor):
    x = x.view(-1, 32)
    top = x.abs().amax(-1, keepdim=True)
    fraction, e = torch.frexp(top)
    e = (e - 9 + (fraction > 0.875)).clamp(min=-127)
    e = torch.where(top > 0, e, -127)
    unit = torch.exp2(e.double())
    a = x.abs() / unit
    _, at = torch.frexp(a)
    grid = torch.exp2((at - 4).clamp(min=-9).double())
    q = torch.floor(a / grid + noise.view(-1, 32).double() / 65536) * grid
    if floor:
        q = torch.where(a > 0, q.clamp(min=2.0 ** -9), q)
    return torch.copysign(q, x).view(-1), unit.view(-1)


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "quantize":
        return _exact_rounded(s["x"].t() if case["transpose"] else s["x"])
    if op == "linear":
        unit = torch.exp2(_untile_scales(s["scales"], case["n"], -(-case["k"] // 32)).double() - 127)
        c = _unpack(s["codes"]).long()
        e, f = (c >> 1) & 3, (c & 1).double()
        w = torch.where(e > 0, (1 + f / 2) * torch.exp2(e.double() - 1), f / 2) * (1 - 2 * (c >> 3))
        w = (w.view(case["n"], -1, 32) * unit[..., None]).view(case["n"], -1)[:, :case["k"]]
        return _exact_rounded(s["x"]) @ w.t()
    if op == "train":
        x, w, dy = s["x"], s["w"], s["dy"]
        q = _exact_rounded
        return {"y": q(x) @ q(w).t(), "dx": q(dy) @ q(w.t()).t(), "dw": q(dy.t()) @ q(x.t()).t()}
    t, g, out = s["step"] + 1, s["g"].double(), {}
    if case["clip"]:
        out["norm"] = torch.linalg.vector_norm(g).view(1)
        g = g * min(1.0, MAX_NORM / (float(out["norm"]) + 1e-6))
    m, v = s["m"].double(), s["v"].double()
    if case["bits"] == 8:
        scale = lambda key: torch.exp2(s[key].double() - 127).repeat_interleave(32)  # noqa: E731
        m, v = m * scale("m_scale"), (v * scale("v_scale")) ** 2
    m = torch.lerp(g, m, BETA1)
    v = torch.lerp(g * g, v, BETA2)
    step = m / (1 - BETA1 ** t) / (torch.sqrt(v / (1 - BETA2 ** t)) + EPS)
    out["p"] = s["p"].double() - LR * (DECAY * s["p"].double() + step)
    if case["copy"]:
        out["copy"] = out["p"]
    if case["bits"] == 8:
        first, second = _random16(m.numel(), SEED, t)
        out["m"], out["m_scale"] = _exact_pack8(m, first, False)
        out["v"], out["v_scale"] = _exact_pack8(v.sqrt(), second, True)
    else:
        out["m"], out["v"] = m, v
    return out
