"""The exchange of gradients in front of the AdamW step (optim.exchange) as gloo processes on CPU, the codec's steps taken by the oracle: every rank
ends with the emulated ring's average, tensor by tensor."""
import os
import sys
from pathlib import Path

import numpy as np
import pytest
import torch
import torch.distributed as dist
import torch.multiprocessing as mp

from test_ring_ranks_cpu import HostCodec

ROOT = Path(__file__).resolve().parent.parent
SHAPES = [(3, 50), (1,), (0,), (7000,), (64, 33)]


def gradients(rank):
    g = torch.Generator().manual_seed(50 + rank)
    return [(torch.randn(s, generator=g) * 1e-2).to(torch.bfloat16 if i == 3 else torch.float32) for i, s in enumerate(SHAPES)]


def flat_of(grads):
    out = []
    for g in grads:
        n = g.numel()
        out.append(np.concatenate([g.float().reshape(-1).numpy(), np.zeros(-n % 32, np.float32)]))
    return np.concatenate(out)


def _worker(rank, world, port, q):
    os.environ.update(MASTER_ADDR="127.0.0.1", MASTER_PORT=str(port), RANK=str(rank), WORLD_SIZE=str(world))
    sys.path[:0] = [str(ROOT), str(ROOT / "tests")]
    try:
        from paper_2502_18554_b200 import optim, ring, zccl as z
        dist.init_process_group("gloo", rank=rank, world_size=world)
        R = ring.Ring(20000, codec=HostCodec())
        res = [optim.exchange(R, gradients(rank), mode, eb) for mode, eb in ((z.EB_REL, 1e-3), (z.EB_ABS, 1e-4))]
        q.put((rank, [[t.numpy() for t in r] for r in res], None))
        dist.barrier()
        dist.destroy_process_group()
    except Exception as e:
        import traceback
        q.put((rank, None, traceback.format_exc()))
        raise e


@pytest.mark.parametrize("world", [1, 2, 3])
def test_every_rank_ends_with_the_same_average(world):
    import oracle
    ctx = mp.get_context("spawn")
    q = ctx.Queue()
    port = 28700 + (os.getpid() * 5 + world * 11) % 900
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
    flats = [flat_of(gradients(r)) for r in range(world)]
    for i, (mode, eb) in enumerate(((oracle.EB_REL, 1e-3), (oracle.EB_ABS, 1e-4))):
        if world == 1:
            want = flats
        else:
            want, _ = oracle.sim_allreduce(flats, mode, eb, flags=oracle.OP_AVG | oracle.FLAG_CONSISTENT_OWNER)
        for r in range(world):
            at = 0
            for shape, t in zip(SHAPES, got[r][i]):
                n = int(np.prod(shape))
                assert t.shape == shape
                np.testing.assert_array_equal(t.reshape(-1), want[r][at:at + n])
                np.testing.assert_array_equal(t, got[0][i][SHAPES.index(shape)])
                at += -(-n // 32) * 32


def test_refusals():
    from paper_2502_18554_b200 import optim
    p = [torch.zeros(5)]
    with pytest.raises(ValueError):
        optim.AdamW(p, state_bits=16)
    o = optim.AdamW(p)
    with pytest.raises(ValueError):
        o.step()                                # no gradient
    with pytest.raises(ValueError):
        o.step([torch.zeros(5)])                # not on a GPU
    with pytest.raises(ValueError):
        o.load_state_dict(optim.AdamW(p, state_bits=8).state_dict())
    with pytest.raises(ValueError):
        o.load_state_dict(optim.AdamW([torch.zeros(6)]).state_dict())


# ---- gradients that the codec cannot take

class LateCodec(HostCodec):
    """As a codec on a GPU: what is wrong with the values that this rank compresses is told when the first collective ends."""

    def __init__(self, code):
        super().__init__()
        self.code = code

    def finish(self):
        from paper_2502_18554_b200 import zccl as z
        code, self.code = self.code, 0
        if code:
            raise z.ZcclError(code, "device status")
        return 0


def _case(name, rank, world):
    """(gradients, eb_mode, eb, code that this rank's codec ends with)"""
    from paper_2502_18554_b200 import zccl as z
    g, mode, eb, code = gradients(rank), z.EB_REL, 1e-3, 0
    last = rank == world - 1
    if name in ("nan", "inf", "-inf") and last:
        g[3][77] = float(name)
    elif name == "nan everywhere":
        g = [torch.full_like(t, float("nan")) for t in g]
    elif name == "inf, absolute bound":
        mode, eb = z.EB_ABS, 1e-4
        if last:
            g[0][2, 5] = float("inf")
    elif name == "zeros":
        g = [torch.zeros_like(t) for t in g]
    elif name == "zeros, absolute bound":
        g, mode, eb = [torch.zeros_like(t) for t in g], z.EB_ABS, 1e-4
    elif name == "one value":
        g = [torch.full((64,), 0.375)]
    elif name == "no elements":
        g = [torch.zeros(0), torch.zeros(0, 3)]
    elif name == "out of range":
        mode, eb = z.EB_ABS, 1e-12
        if last:
            g[4][1, 1] = 5.0
    elif name == "range overflows" and last:
        g[4][1, 1], g[4][1, 2] = 3e38, -3e38
    elif name == "one rank's codec fails" and last:
        code = z.E_RANGE
    return g, mode, eb, code


FILLED = ["nan", "inf", "-inf", "nan everywhere", "inf, absolute bound"]
EXACT = ["zeros", "zeros, absolute bound", "one value", "no elements"]
REFUSED = ["out of range", "range overflows", "one rank's codec fails"]


def _bad_worker(rank, world, port, q):
    os.environ.update(MASTER_ADDR="127.0.0.1", MASTER_PORT=str(port), RANK=str(rank), WORLD_SIZE=str(world))
    sys.path[:0] = [str(ROOT), str(ROOT / "tests")]
    try:
        from datetime import timedelta
        from paper_2502_18554_b200 import optim, ring, zccl as z
        dist.init_process_group("gloo", rank=rank, world_size=world, timeout=timedelta(seconds=60))
        stepped = []
        optim.adamw = lambda *a, **k: stepped.append(k["step"])          # the step itself needs a GPU
        res = {}
        for name in FILLED + EXACT + REFUSED:
            grads, mode, eb, code = _case(name, rank, world)
            R = ring.Ring(20000, codec=LateCodec(code))
            opt = optim.AdamW([torch.zeros(t.shape) for t in grads])
            del stepped[:]
            try:
                out = opt.step(grads, ring=R, eb_mode=mode, eb=eb)
                assert out is None
                outcome = "stepped" if stepped else "left out"
            except (z.ZcclError, ValueError) as exc:
                outcome = type(exc).__name__
            steps = opt.steps
            norm = opt.step(grads, ring=R, eb_mode=mode, eb=eb, max_norm=1.0) if name in FILLED else None
            averaged = [t.numpy() for t in optim.exchange(R, grads, mode, eb)] if name not in REFUSED else None
            res[name] = (outcome, steps, None if norm is None else float(norm), averaged)
        q.put((rank, res, None))
        dist.barrier()
        dist.destroy_process_group()
    except Exception as e:
        import traceback
        q.put((rank, None, traceback.format_exc()))
        raise e


@pytest.mark.parametrize("world", [2, 3])
def test_gradients_that_the_codec_cannot_take(world):
    """Whatever one rank's gradients hold, all ranks end alike: not finite on one leaves the step out on all, what is refused is refused by all, zeros are zeros."""
    ctx = mp.get_context("spawn")
    q = ctx.Queue()
    port = 29700 + (os.getpid() * 5 + world * 11) % 900
    procs = [ctx.Process(target=_bad_worker, args=(r, world, port, q)) for r in range(world)]
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
    for r in range(world):
        for name in FILLED:
            outcome, steps, norm, averaged = got[r][name]
            assert (outcome, steps) == ("left out", 1) and not np.isfinite(norm), (name, r)
            assert [a.shape for a in averaged] == SHAPES and all(np.isnan(a).all() for a in averaged), (name, r)
        for name in EXACT:
            outcome, steps, _, averaged = got[r][name]
            assert (outcome, steps) == ("stepped", 1), (name, r)
            want = [t.float().numpy() for t in _case(name, r, world)[0]]
            assert len(want) == len(averaged) and all(np.array_equal(a, b) for a, b in zip(want, averaged)), (name, r)
        for name in REFUSED:
            outcome, steps, _, _ = got[r][name]
            assert outcome in ("ZcclError", "DegenerateRange") and steps == 0, (name, r, outcome)


def test_the_bound_is_the_codecs():
    """Bounds and refusals of the exchange against the oracle's, on both sides of its limit of 2^30 steps."""
    import oracle
    from paper_2502_18554_b200 import optim, ring, zccl as z
    rng = np.random.default_rng(5)
    for _ in range(300):
        low, high = sorted(float(np.float32(x)) for x in rng.standard_normal(2) * 10.0 ** rng.integers(-30, 30))
        eb = float(10.0 ** rng.uniform(-12, 3))
        for mode, name in ((z.EB_ABS, oracle.EB_ABS), (z.EB_REL, oracle.EB_REL)):
            try:
                ea, _, r = oracle.resolve(name, eb, mn=low, mx=high)
            except oracle.OracleError:
                if mode == z.EB_REL:
                    with pytest.raises(ring.DegenerateRange):
                        optim._bound(low, high, mode, eb, 2)
                continue
            x = np.array([low, high], np.float32)
            try:
                oracle.quantise(x, r)
            except oracle.OracleError:
                with pytest.raises(z.ZcclError):
                    optim._bound(low, high, mode, eb, 2)
                assert optim._bound(low, high, mode, eb, 1) == float(ea)      # nothing is compressed on one rank
            else:
                assert optim._bound(low, high, mode, eb, 2) == float(ea)
    assert optim._bound(2.0, 2.0, z.EB_REL, 1e-3, 2) is None
    for eb in (0.0, -1.0, float("nan"), float("inf")):
        with pytest.raises(ValueError):
            optim._bound(0.0, 1.0, z.EB_ABS, eb, 2)
    with pytest.raises(ValueError):
        optim._bound(0.0, 1.0, z.EB_RESOLVED, 1.0, 2)


def test_a_refused_step_is_not_counted(monkeypatch):
    from paper_2502_18554_b200 import optim
    p = [torch.zeros(5)]
    o = optim.AdamW(p)
    with pytest.raises(ValueError):
        o.step([torch.zeros(5)])                # not on a GPU
    assert o.steps == 0
    seen = []
    monkeypatch.setattr(optim, "adamw", lambda *a, **k: seen.append(k["step"]))
    o.step([torch.zeros(5)])
    o.step([torch.zeros(5)])
    assert seen == [1, 2] and o.steps == 2


def test_the_seed_is_saved_and_loaded():
    from paper_2502_18554_b200 import optim
    a, b = optim.AdamW([torch.zeros(40)], state_bits=8, seed=11), optim.AdamW([torch.zeros(40)], state_bits=8, seed=4)
    a.steps = 6
    state = a.state_dict()
    b.load_state_dict(state)
    assert (b.steps, b.seed) == (6, 11)
    del state["seed"]                           # as saved before seeds were
    c = optim.AdamW([torch.zeros(40)], state_bits=8, seed=4)
    c.load_state_dict(state)
    assert (c.steps, c.seed) == (6, 4)
    with pytest.raises(KeyError):
        c.load_state_dict({k: v for k, v in state.items() if k != "steps"})


def test_exchanged_gradients_are_no_part_of_a_graph():
    """Gradients that require gradients themselves: their values are exchanged."""
    from types import SimpleNamespace
    from paper_2502_18554_b200 import optim, zccl as z
    alone = SimpleNamespace(N=1, codec=SimpleNamespace(device=torch.device("cpu")), allreduce=lambda x, out, mode, eb, flags: out.copy_(x))
    for g in (torch.arange(40.0), torch.full((32,), 3.0), torch.tensor([1.0, float("nan")])):
        (out,) = optim.exchange(alone, [g.clone().requires_grad_() * 1], z.EB_REL, 1e-3)
        assert not out.requires_grad
        assert torch.equal(out, g) or not bool(torch.isfinite(g).all())
