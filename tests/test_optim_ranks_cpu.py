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
