"""The operators together, as a data-parallel training step uses them: a layer in microscaled 4 bits and its gradient, the gradients' compressed
exchange, their norm and the AdamW step."""
import os
import sys
from pathlib import Path

import numpy as np
import pytest
import torch
import torch.distributed as dist
import torch.multiprocessing as mp

import _operators as ref
from test_gpu_optim import bounds, wide

ROOT = Path(__file__).resolve().parent.parent
pytestmark = pytest.mark.gpu
HYPER = dict(lr=1e-2, betas=(0.9, 0.99), eps=1e-8, weight_decay=0.05)
SHAPES = [(96, 70), (40, 96), (130,)]


@pytest.mark.parametrize("bits", [32, 8])
def test_two_emulated_ranks_train_a_small_network(bits):
    """Two layers, two emulated ranks with data of their own, gradients exchanged by the emulated ring, three steps.  Each step's gradients are the
    formula's, and its update the formula's from the reduced gradients."""
    from paper_2502_18554_b200 import build, mx, optim, zccl as z
    build.build()
    gen = torch.Generator().manual_seed(1)
    rand = lambda *s: torch.randn(*s, generator=gen).cuda()  # noqa: E731
    w = [(rand(96, 64) * 0.1).requires_grad_(), (rand(40, 96) * 0.1).requires_grad_()]
    opt = optim.AdamW(w, state_bits=bits, **HYPER)
    ctx = z.Context(1 << 16, 2)
    total = sum(p.numel() for p in w)
    for step in range(1, 4):
        flats = []
        for rank in range(2):
            x, target = rand(50, 64), rand(50, 40)
            h = mx.linear(x, w[0])
            y = mx.linear(torch.relu(h), w[1])
            dy = (y - target).detach() / 50
            grads = torch.autograd.grad(y, w, dy)
            # the last layer's gradient against the formula, in 64 bits
            q = lambda t: torch.from_numpy(ref.values(*ref.quantize(wide(t)), t.shape[1])).cuda()  # noqa: E731
            a, b = q(dy.t()), q(torch.relu(h).detach().t())
            # 50 products: their sum in binary32, and one rounding
            assert bool(((grads[1].double() - a @ b.t()).abs() <= 51 * 2.0 ** -23 * (a.abs() @ b.abs().t()) + 1e-45).all())
            flats.append(torch.cat([g.reshape(-1) for g in grads]))
        reduced = [torch.empty_like(f) for f in flats]
        ctx.sim_allreduce(flats, reduced, z.EB_ABS, 1e-4, flags=z.OP_AVG | z.CONSISTENT_OWNER)
        ctx.check()
        assert torch.equal(reduced[0], reduced[1])
        mean = (flats[0].double() + flats[1].double()) / 2
        assert bool(((reduced[0].double() - mean).abs() <= 1e-4 + 1e-7 * mean.abs()).all())     # two compressions of a sum, halved
        grads = [g.view(p.shape) for g, p in zip(torch.split(reduced[0], [p.numel() for p in w]), w)]
        before = [wide(p) for p in w]
        m0, v0 = [t.clone() for t in opt.exp_avg], [t.clone() for t in opt.exp_avg_sq]
        scales = [None if bits == 32 else [t.clone() for t in s] for s in (opt.exp_avg_scale, opt.exp_avg_sq_scale)]
        norm = opt.step(grads, max_norm=0.5)
        want = float(reduced[0].double().norm())
        assert abs(float(norm) - want) <= 6 * 2.0 ** -24 * want
        for i, p in enumerate(w):
            m, v = wide(m0[i]).reshape(-1), wide(v0[i]).reshape(-1)
            if bits == 8:
                scale = [np.repeat(np.ldexp(1.0, s[i].cpu().numpy().astype(int) - 127), 32)[:m.size] for s in scales]
                m, v = m * scale[0], (v * scale[1]) ** 2
            hyper = {**HYPER, "step": step, "max_norm": 0.5}
            g = wide(grads[i]).reshape(-1)
            new, _, _ = ref.step_of(before[i].reshape(-1), g, m, v, norm=want, **hyper)
            dp, _, _ = bounds(before[i].reshape(-1), g, m, v, hyper, want)
            assert (np.abs(wide(p).reshape(-1) - new) <= dp + np.abs(new) * 2.0 ** -24).all()
    assert opt.steps == 3 and total == sum(p.numel() for p in w)
    ctx.close()


def test_states_are_saved_and_loaded():
    from paper_2502_18554_b200 import optim
    make = lambda: [torch.ones(100, device="cuda"), torch.ones(7, 9, device="cuda")]  # noqa: E731
    g = [torch.randn(100, device="cuda"), torch.randn(7, 9, device="cuda")]
    for bits in (32, 8):
        a, b = optim.AdamW(make(), state_bits=bits, seed=3), optim.AdamW(make(), state_bits=bits, seed=3)
        a.step(g)
        b.load_state_dict(a.state_dict())
        for p, q in zip(a.params, b.params):
            q.copy_(p)
        a.step(g)
        b.step(g)
        assert b.steps == 2 and all(torch.equal(p, q) for p, q in zip(a.params, b.params))


def _gradients(rank):
    g = torch.Generator().manual_seed(70 + rank)
    return [(torch.randn(s, generator=g) * 1e-2) for s in SHAPES]


def _params():
    g = torch.Generator().manual_seed(7)
    return [torch.randn(s, generator=g) * 0.1 for s in SHAPES]


def _worker(rank, world, port, q):
    os.environ.update(MASTER_ADDR="127.0.0.1", MASTER_PORT=str(port), RANK=str(rank), WORLD_SIZE=str(world))
    sys.path.insert(0, str(ROOT))
    try:
        from paper_2502_18554_b200 import optim, ring, zccl as z
        torch.cuda.set_device(0)
        dist.init_process_group("gloo", rank=rank, world_size=world)
        R = ring.Ring(1 << 15)
        params = [p.cuda() for p in _params()]
        for p, g in zip(params, _gradients(rank)):
            p.requires_grad_()
            p.grad = g.cuda()
        opt = optim.AdamW(params, state_bits=8, seed=5, **HYPER)
        norm = opt.step(max_norm=0.1, ring=R, eb_mode=z.EB_REL, eb=1e-3)
        q.put((rank, [p.detach().cpu().numpy() for p in params] + [norm.cpu().numpy()], None))
        dist.barrier()
        dist.destroy_process_group()
    except Exception as e:
        import traceback
        q.put((rank, None, traceback.format_exc()))
        raise e


def test_real_ranks_end_with_the_parameters_of_the_emulated_exchange():
    """Two processes on the one GPU exchange their gradients through host memory; both end, bit for bit, with what the oracle's emulated ring and one
    AdamW step here give."""
    import oracle
    from paper_2502_18554_b200 import build, optim
    build.build()
    world = 2
    ctx = mp.get_context("spawn")
    q = ctx.Queue()
    port = 28100 + os.getpid() % 500
    procs = [ctx.Process(target=_worker, args=(r, world, port, q)) for r in range(world)]
    for p in procs:
        p.start()
    got = {}
    for _ in range(world):
        rank, res, err = q.get(timeout=300)
        assert err is None, err
        got[rank] = res
    for p in procs:
        p.join(120)
        assert p.exitcode == 0
    flats = [np.concatenate([np.concatenate([g.reshape(-1).numpy(), np.zeros(-g.numel() % 32, np.float32)]) for g in _gradients(r)]) for r in range(world)]
    want, _ = oracle.sim_allreduce(flats, oracle.EB_REL, 1e-3, flags=oracle.OP_AVG | oracle.FLAG_CONSISTENT_OWNER)
    params, grads, at = [p.cuda() for p in _params()], [], 0
    for p in params:
        grads.append(torch.from_numpy(want[0][at:at + p.numel()].copy()).cuda().view(p.shape))
        at += -(-p.numel() // 32) * 32
    norm = optim.AdamW(params, state_bits=8, seed=5, **HYPER).step(grads, max_norm=0.1)
    for r in range(world):
        for a, b in zip(got[r], params + [norm]):
            np.testing.assert_array_equal(a, b.cpu().numpy())


def _refusing_worker(rank, world, port, q):
    os.environ.update(MASTER_ADDR="127.0.0.1", MASTER_PORT=str(port), RANK=str(rank), WORLD_SIZE=str(world))
    sys.path.insert(0, str(ROOT))
    try:
        from paper_2502_18554_b200 import optim, ring, zccl as z
        torch.cuda.set_device(0)
        dist.init_process_group("gloo", rank=rank, world_size=world)
        res = {}
        for name in ("nan", "inf", "zeros", "out of range", "sum out of range"):
            params = [p.cuda() for p in _params()]
            grads = [g.cuda() for g in _gradients(rank)]
            R = ring.Ring(optim.exchange_elems(params))
            mode, eb = z.EB_REL, 1e-3
            if name == "zeros":
                grads = [torch.zeros_like(g) for g in grads]
            elif name in ("nan", "inf") and rank == 1:
                grads[1][3, 4] = float(name)
            elif name == "out of range":
                mode, eb = z.EB_ABS, 1e-3
                if rank == 1:
                    grads[1][3, 4] = 3e6            # 2^30 steps of this bound are 2.1e6
            elif name == "sum out of range":
                mode, eb = z.EB_ABS, 1e-3
                grads[1][3, 4] = 1.5e6
            opt = optim.AdamW(params, state_bits=8, seed=5, **HYPER)
            try:
                norm = opt.step(grads, max_norm=0.1, ring=R, eb_mode=mode, eb=eb)
                outcome = "finite" if bool(torch.isfinite(norm)) else "left out"
            except z.ZcclError as exc:
                outcome = exc.code
            res[name] = (outcome, opt.steps, [p.cpu().numpy() for p in params])
            assert R.codec.ctx.status() == 0
        q.put((rank, res, None))
        dist.barrier()
        dist.destroy_process_group()
    except Exception as e:
        import traceback
        q.put((rank, None, traceback.format_exc()))
        raise e


def test_real_ranks_end_alike_whatever_the_gradients_hold():
    """Two processes on the one GPU: gradients that are not finite on one rank leave the step out on both, zeros are a step, and what the codec refuses on one rank
    (as it is, or summed up on the way) is refused by both; parameters stay what they were, and the codec is usable afterwards."""
    from paper_2502_18554_b200 import build, zccl as z
    build.build()
    ctx = mp.get_context("spawn")
    q = ctx.Queue()
    port = 28600 + os.getpid() % 500
    procs = [ctx.Process(target=_refusing_worker, args=(r, 2, port, q)) for r in range(2)]
    for p in procs:
        p.start()
    got = {}
    for _ in range(2):
        rank, res, err = q.get(timeout=300)
        assert err is None, err
        got[rank] = res
    for p in procs:
        p.join(120)
        assert p.exitcode == 0
    before = [p.numpy() for p in _params()]
    for r in range(2):
        for name, outcome, steps in (("nan", "left out", 1), ("inf", "left out", 1), ("zeros", "finite", 1), ("out of range", z.E_RANGE, 0), ("sum out of range", z.E_RANGE, 0)):
            assert got[r][name][:2] == (outcome, steps), (name, r, got[r][name][:2])
            for a, b in zip(got[r][name][2], before):
                if name == "zeros":     # decayed alone: 1 - lr weight_decay and the product are rounded
                    np.testing.assert_allclose(a, b.astype(np.float64) * (1 - HYPER["lr"] * HYPER["weight_decay"]), rtol=3 * 2.0 ** -24, atol=0)
                else:
                    np.testing.assert_array_equal(a, b)


@pytest.mark.parametrize("bits", [32, 8])
def test_a_refused_step_leaves_no_trace(bits):
    """A step with a gradient of the wrong size is refused; the next one is that of an optimizer that was never given it."""
    from paper_2502_18554_b200 import optim
    g = [torch.randn(100, device="cuda"), torch.randn(7, 9, device="cuda")]
    a, b = (optim.AdamW([torch.ones(100, device="cuda"), torch.ones(7, 9, device="cuda")], state_bits=bits, seed=3) for _ in range(2))
    for bad in ([g[0]], [g[0], g[1].double()], [g[0][:50], g[1]]):
        with pytest.raises(ValueError):
            a.step(bad, max_norm=1.0 if len(bad) == 1 else None)
    a.step(g, max_norm=1.0)
    b.step(g, max_norm=1.0)
    assert a.steps == b.steps == 1 and all(torch.equal(p, q) for p, q in zip(a.params, b.params))
    assert all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(a.exp_avg + a.exp_avg_sq, b.exp_avg + b.exp_avg_sq))


def test_a_run_goes_on_in_an_optimizer_that_was_made_with_another_seed():
    from paper_2502_18554_b200 import optim
    gen = torch.Generator().manual_seed(2)
    grads = [[torch.randn(3000, generator=gen).cuda()] for _ in range(4)]
    a, b = optim.AdamW([torch.ones(3000, device="cuda")], state_bits=8, seed=3), optim.AdamW([torch.ones(3000, device="cuda")], state_bits=8)
    for g in grads[:2]:
        a.step(g)
    b.load_state_dict(a.state_dict())
    b.params[0].copy_(a.params[0])
    for g in grads[2:]:
        a.step(g)
        b.step(g)
        for x, y in zip(a.params + a.exp_avg + a.exp_avg_sq + a.exp_avg_scale, b.params + b.exp_avg + b.exp_avg_sq + b.exp_avg_scale):
            assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))


def test_other_threads_go_on_while_a_launch_waits():
    """With the GPU's queue full (it spins for a while) launches wait, and the interpreter lock is not held meanwhile."""
    import threading
    import time
    from paper_2502_18554_b200 import build, mx, optim
    build.build()
    x, w = torch.randn(4, 64, device="cuda"), torch.randn(40, 64, device="cuda")
    q, y = mx.quantize(w), torch.empty(40, 40, device="cuda")
    state = lambda: [torch.zeros(64, device="cuda")]  # noqa: E731
    p, m, v, g, norm = state(), state(), state(), state(), torch.zeros(1, device="cuda")
    calls = [lambda: mx.matmul(q, q, out=y), lambda: mx.quantize(w, out=q), lambda: mx.dequantize(q, out=w), lambda: optim.grad_norm(g, out=norm),
             lambda: optim.adamw(p, g, m, v, step=1, lr=1e-3), lambda: mx.linear(x, q), lambda: mx.linear(x, w), lambda: mx.linear_backward(torch.zeros(4, 40, device="cuda"), x, w),
             lambda: mx.quantize_all([x, w])]
    for call in calls:
        call()
    torch.cuda.synchronize()
    for call in calls:
        done = threading.Event()

        def work():
            torch.cuda._sleep(2_500_000_000)         # 1.3 s
            for _ in range(2500):                    # more than the queue holds
                call()
            done.set()

        thread = threading.Thread(target=work)
        thread.start()
        last, gap = time.perf_counter(), 0.0
        while not done.is_set():
            time.sleep(0.002)
            now = time.perf_counter()
            last, gap = now, max(gap, now - last)
        thread.join()
        torch.cuda.synchronize()
        assert gap < 0.8, gap


def test_a_list_that_another_thread_changes():
    """The tensors of a call are its own, whatever becomes of the lists they came in."""
    import threading
    from paper_2502_18554_b200 import build, optim
    build.build()
    lists = [[torch.zeros(50, device="cuda") for _ in range(200)] for _ in range(4)]
    whole = [list(x) for x in lists]
    stop = threading.Event()

    def change():
        while not stop.is_set():
            for x, all_ in zip(lists, whole):
                del x[100:]
                x.extend(all_[100:])

    thread = threading.Thread(target=change)
    thread.start()
    done = 0
    try:
        for _ in range(300):
            try:
                optim.adamw(*lists, step=1, lr=1e-3)
                done += 1
            except ValueError:                       # lists of different lengths just then
                pass
    finally:
        stop.set()
        thread.join()
    torch.cuda.synchronize()
    assert not any(bool(t.any()) for x in whole for t in x)
