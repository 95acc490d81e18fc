"""Microscaled 4-bit floating point and the AdamW step without a GPU: the reference that the GPU tests go by, sizes, and what the
boundary and the binding refuse."""
import ctypes as C

import numpy as np
import pytest
import torch

import _operators as ref


@pytest.fixture(scope="module")
def lib():
    from paper_2502_18554_b200 import build, zccl
    build.build()
    return zccl.lib()


def test_reference_rounds_to_the_nearest_element_and_ties_to_even():
    x = np.array([[0.0, 0.25, 0.26, 0.75, 0.74, 1.25, 1.75, 2.5, 3.5, 5.0, 5.01, 6.0, 7.0, 4.0, -0.25, -0.75, -7.9] + [0.0] * 15])
    v, s = ref.quantize(x)
    assert s[0, 0] == 127     # the largest magnitude, 7.9, has exponent 2
    assert v[0, 0, :17].tolist() == [0, 0, 0.5, 1, 0.5, 1, 2, 2, 4, 4, 6, 6, 6, 4, 0, -1, -6]


def test_reference_against_brute_force():
    rng = np.random.default_rng(3)
    x = (rng.standard_normal((7, 70)) * 10.0 ** rng.integers(-30, 30, (7, 70))).astype(np.float32)
    v, s = ref.quantize(x)
    got = ref.values(v, s, 70)
    for r in range(7):
        for b in range(3):
            block = x[r, 32 * b:32 * b + 32].astype(np.float64)
            e = int(np.floor(np.log2(np.abs(block).max()))) - 2
            for i, value in enumerate(block):
                every = ref.NIBBLES * 2.0 ** e
                assert abs(got[r, 32 * b + i] - value) == np.abs(every - value).min()


def test_layout_goes_there_and_back():
    rng = np.random.default_rng(4)
    for rows, cols in ((1, 1), (3, 33), (130, 128), (257, 300)):
        v, s = ref.quantize(rng.standard_normal((rows, cols)))
        codes, scales = ref.pack(v, s)
        v2, s2 = ref.unpack(codes, scales, rows, cols)
        assert np.array_equal(v, v2) and np.array_equal(s, s2)


def test_sizes(lib):
    for rows, cols in ((0, 5), (5, 0), (1, 1), (1, 32), (1, 33), (128, 128), (129, 129), (5000, 4161)):
        blocks = -(-cols // 32)
        assert lib.zccl_mx4_code_bytes(rows, cols) == rows * blocks * 16
        assert lib.zccl_mx4_scale_bytes(rows, cols) == -(-rows // 128) * -(-cols // 128) * 512


def test_the_boundary_refuses_bad_arguments_without_cuda(lib):
    from paper_2502_18554_b200 import zccl
    p, odd = C.c_void_p(4096), C.c_void_p(4097)
    q = lib.zccl_mx4_quantize
    q.argtypes = [C.c_void_p, C.c_int, C.c_size_t, C.c_size_t, C.c_size_t, C.c_int, C.c_void_p, C.c_void_p, C.c_void_p]
    ok = [p, 0, 4, 32, 32, 0, p, p, None]
    for i, bad in ((0, None), (0, odd), (1, 3), (1, -1), (4, 31), (6, None), (6, odd), (7, None), (7, C.c_void_p(4104)), (2, 1 << 40), (3, 1 << 40)):
        args = list(ok)
        args[i] = bad
        assert q(*args) == zccl.E_ARG, (i, bad)
    assert q(None, 0, 0, 32, 32, 0, None, None, None) == zccl.OK      # nothing to do
    d = lib.zccl_mx4_dequantize
    d.argtypes = [C.c_void_p, C.c_void_p, C.c_size_t, C.c_size_t, C.c_void_p, C.c_int, C.c_size_t, C.c_void_p]
    assert d(None, p, 4, 32, p, 0, 32, None) == zccl.E_ARG
    assert d(p, p, 4, 32, p, 7, 32, None) == zccl.E_ARG
    assert d(p, p, 4, 32, p, 0, 8, None) == zccl.E_ARG
    assert d(p, p, 4, 0, None, 0, 0, None) == zccl.OK


class Tensor(C.Structure):
    _fields_ = [(k, C.c_void_p) for k in ("p", "g", "m", "v", "m_scale", "v_scale", "copy")] + [("n", C.c_size_t)]


class Config(C.Structure):
    _fields_ = [(k, C.c_int) for k in ("param_type", "grad_type", "copy_type", "state_bits")] + \
               [(k, C.c_double) for k in ("lr", "beta1", "beta2", "eps", "weight_decay")] + \
               [("step", C.c_longlong), ("step_device", C.c_void_p), ("lr_device", C.c_void_p), ("seed", C.c_ulonglong), ("norm", C.c_void_p), ("max_norm", C.c_double)]


def test_the_step_refuses_bad_arguments_without_cuda(lib):
    from paper_2502_18554_b200 import zccl
    step = lib.zccl_adamw
    step.argtypes = [C.POINTER(Tensor), C.c_size_t, C.POINTER(Config), C.c_void_p]

    def call(tensor=None, count=1, **changes):
        t = Tensor(4096, 4096, 4096, 4096, 4096, 4096, None, 5)
        for key, value in (tensor or {}).items():
            setattr(t, key, value)
        k = Config(0, 0, 1, 32, 1e-3, 0.9, 0.999, 1e-8, 0.0, 1, None, None, 0, None, 1.0)
        for key, value in changes.items():
            setattr(k, key, value)
        return step(C.byref(t), count, C.byref(k), None)

    for tensor in ({"p": None}, {"p": 4098}, {"g": None}, {"m": None}, {"m": 4097}, {"v": 4098}, {"n": 1 << 50}, {"copy": 4097}):
        assert call(tensor) == zccl.E_ARG, tensor
    assert call({"m_scale": None}, state_bits=8) == zccl.E_ARG
    assert call({"copy": 4096}, param_type=1) == zccl.E_ARG and call({"copy": 4096}, copy_type=0) == zccl.E_ARG
    nan, inf = float("nan"), float("inf")
    for changes in ({"param_type": 3}, {"grad_type": -1}, {"state_bits": 16}, {"beta1": 1.0}, {"beta1": -0.1}, {"beta2": nan}, {"eps": -1.0}, {"eps": inf},
                    {"lr": nan}, {"weight_decay": inf}, {"step": 0}, {"norm": 4096, "max_norm": 0.0}, {"norm": 4098}, {"lr_device": 4097}, {"step_device": 4100}):
        assert call(**changes) == zccl.E_ARG, changes
    assert call({"n": 0, "p": None}) == zccl.OK and step(None, 0, C.byref(Config(0, 0, 1, 32, 1e-3, 0.9, 0.999, 1e-8, 0.0, 1, None, None, 0, None, 1.0)), None) == zccl.OK
    assert step(None, 1, C.byref(Config()), None) == zccl.E_ARG
    norm = lib.zccl_grad_norm
    norm.argtypes = [C.c_void_p, C.c_void_p, C.c_size_t, C.c_int, C.c_void_p, C.c_void_p, C.c_void_p]
    assert norm(None, None, 1, 0, 4096, 4096, None) == zccl.E_ARG
    assert norm(None, None, 0, 5, 4096, 4096, None) == zccl.E_ARG
    assert norm(None, None, 0, 0, None, 4096, None) == zccl.E_ARG
    assert norm(None, None, 0, 0, 4096, 4100, None) == zccl.E_ARG


def test_the_binding_refuses_tensors_that_are_not_on_a_gpu(lib):
    from paper_2502_18554_b200 import mx, optim
    x = torch.zeros(4, 64)
    with pytest.raises(ValueError):
        mx.quantize(x)
    with pytest.raises(ValueError):
        mx.quantize(torch.zeros(64))
    with pytest.raises(ValueError):
        mx.dequantize(mx.empty(4, 64, "cpu"))
    with pytest.raises(ValueError):
        optim.adamw([x], [x], [x], [x], step=1, lr=1e-3)
    with pytest.raises(ValueError):
        optim.grad_norm([])
    with pytest.raises(ValueError):
        optim.grad_norm([x])


def test_random_bits_of_the_reference_are_spread():
    bits = ref.random_bits(7, 1, np.arange(1 << 16, dtype=np.uint64))
    for half in (bits >> np.uint64(16), bits & np.uint64(0xFFFF)):
        u = half.astype(np.float64) / 65536
        assert abs(u.mean() - 0.5) < 5 * np.sqrt(1 / 12 / u.size)
        assert abs(np.corrcoef(u[:-1], u[1:])[0, 1]) < 5 / np.sqrt(u.size)


def test_the_step_refuses_an_eps_that_binary32_holds_as_a_subnormal_number(lib):
    """By such a one nothing can be divided (its reciprocal is no number of binary32); 0 and from 2^-126 on is what the formula is kept for."""
    from paper_2502_18554_b200 import zccl
    step = lib.zccl_adamw
    step.argtypes = [C.POINTER(Tensor), C.c_size_t, C.POINTER(Config), C.c_void_p]
    nothing = Tensor(None, None, None, None, None, None, None, 0)
    for eps, want in ((1e-40, zccl.E_ARG), (1e-60, zccl.E_ARG), (2.0 ** -127, zccl.E_ARG), (5e-324, zccl.E_ARG), (2.0 ** -126, zccl.OK), (1e-30, zccl.OK), (0.0, zccl.OK)):
        k = Config(0, 0, 1, 32, 1e-3, 0.9, 0.999, eps, 0.0, 1, None, None, 0, None, 1.0)
        assert step(C.byref(nothing), 1, C.byref(k), None) == want, eps


class Job(C.Structure):
    _fields_ = [("x", C.c_void_p), ("rows", C.c_size_t), ("cols", C.c_size_t), ("pitch", C.c_size_t), ("transpose", C.c_int), ("codes", C.c_void_p), ("scales", C.c_void_p)]


@pytest.mark.skipif(torch.cuda.is_available(), reason="the pointers are none")
@pytest.mark.parametrize("transpose", [0, 1])
def test_a_matrix_too_large_is_refused_before_anything_runs(lib, transpose):
    """Behind as many as one launch takes: nothing has been launched, which here, without a GPU, would be another error."""
    from paper_2502_18554_b200 import zccl
    call = lib.zccl_mx4_quantize_all
    call.argtypes = [C.POINTER(Job), C.c_int, C.c_int, C.c_void_p]
    small, large = Job(4096, 4, 32, 32, 0, 4096, 4096), Job(4096, 1 << 30, 1 << 20, 1 << 20, transpose, 4096, 4096)
    for before in (0, 1, 8, 9, 16):
        jobs = (Job * (before + 1))(*[small] * before, large)
        assert call(jobs, before + 1, 1, None) == zccl.E_ARG, before
    assert call((Job * 1)(small), 1, 1, None) == zccl.E_CUDA
