"""Clipping over ranks: streams, refusals and what comes back, on the host with a context made of torch operations."""
import contextlib
import math
import os
import socket

import numpy as np
import pytest
import torch
import torch.distributed as dist
import torch.multiprocessing as mp
from torch.utils._python_dispatch import TorchDispatchMode

from paper_2510_23938_b200 import binding, sharded


class HostSetOps:
    """grad_norm and grad_scale of a context, for float32 tensors on the host; `seen` receives what was called."""

    def __init__(self, seen=None):
        self.seen = seen if seen is not None else []

    @staticmethod
    def _parts(base, offsets, lengths):
        return [base[o // 4:(o + n) // 4] for o, n in zip(offsets.tolist(), lengths.tolist())]

    @classmethod
    def _squares(cls, base, offsets, lengths):
        return [p.double().square().sum() for p in cls._parts(base, offsets, lengths)]

    def grad_norm(self, base, offsets, lengths, result, norms=None, dtype=None, types=None, stream=None):
        self.seen.append(("grad_norm", stream))
        parts = self._parts(base, offsets, lengths)
        each = torch.stack(self._squares(base, offsets, lengths))
        result.view(torch.float64)[2] = each.sum()
        result.view(torch.int32)[1] = sum(int(not torch.isfinite(p).all()) for p in parts)
        result.view(torch.int64)[3] = sum(p.numel() for p in parts)
        if norms is not None:
            norms.copy_(each.sqrt())

    def grad_scale(self, base, offsets, lengths, scale, out=None, out_offsets=None, dtype=None, types=None, out_dtype=None,
                   stream=None):
        self.seen.append(("grad_scale", stream))
        for p in self._parts(base, offsets, lengths):
            p.mul_(scale)


def _two_halves(flat):
    half = flat.numel() // 2 * 4
    return torch.tensor([0, half]), torch.tensor([half, flat.numel() * 4 - half])


def _free_port():
    with socket.socket() as s:
        s.bind(("127.0.0.1", 0))
        return s.getsockname()[1]


def test_everything_runs_on_the_given_stream(monkeypatch):
    """The two calls and every torch operation between them are issued with the caller's stream as the current one; nothing
    is handed a stream of its own beside operations on another."""
    seen, inside = [], []

    @contextlib.contextmanager
    def entered(stream):
        inside.append(stream)
        yield
        inside.pop()

    class Operations(TorchDispatchMode):
        def __torch_dispatch__(self, func, types, args=(), kwargs=None):
            outside_of.append(str(func)) if not inside else None
            return func(*args, **(kwargs or {}))

    class Ops(HostSetOps):
        def grad_norm(self, *args, **kw):
            seen.append(("grad_norm", kw.get("stream") or (inside and inside[-1])))
            super().grad_norm(*args, **kw)

        def grad_scale(self, *args, **kw):
            seen.append(("grad_scale", kw.get("stream") or (inside and inside[-1])))
            super().grad_scale(*args, **kw)

    outside_of = []
    monkeypatch.setattr(torch.cuda, "stream", entered)
    flat = torch.tensor([3.0, 4.0, 0.0, 0.0])
    offsets, lengths = _two_halves(flat)
    with Operations():
        norm, scale, bad = sharded.sharded_grad_clip(Ops(), flat, offsets, lengths, 1.0, stream="side")
    assert seen == [("grad_norm", "side"), ("grad_scale", "side")] and outside_of == [] and inside == []
    assert float(norm) == 5.0 and flat.tolist()[:2] == [pytest.approx(0.6), pytest.approx(0.8)]


@pytest.mark.parametrize("limit", [-1.0, -1e-30, math.nan, -math.inf])
def test_a_limit_that_is_none_is_refused_before_anything_runs(limit):
    """As grad_clip refuses it; every rank has the same limit, so none is left waiting in the exchange."""
    ops, flat = HostSetOps(), torch.tensor([3.0, 4.0])
    offsets, lengths = _two_halves(flat)
    with pytest.raises(binding.IvError) as err:
        sharded.sharded_grad_clip(ops, flat, offsets, lengths, limit)
    assert err.value.code == binding.IV_ERR_INVALID_ARG and ops.seen == [] and flat.tolist() == [3.0, 4.0]


@pytest.mark.parametrize("limit", [0.0, -0.0, math.inf])
def test_limits_at_the_ends_are_taken(limit):
    flat = torch.tensor([3.0, 4.0])
    norm, scale, bad = sharded.sharded_grad_clip(HostSetOps(), flat, *_two_halves(flat), limit)
    assert float(norm) == 5.0 and float(scale) == (1.0 if limit else 0.0) and flat.tolist() == [3.0 * float(scale), 4.0 * float(scale)]


def test_the_limit_is_rounded_as_grad_clip_takes_it():
    """grad_clip takes a 32-bit limit: scale = round(limit32 / norm), the quotient in 64 bits."""
    limit, seen = float(np.float32(0.1)), set()
    for seed in range(200):
        flat = torch.randn(64, generator=torch.Generator().manual_seed(seed))
        want = np.float32(limit / math.sqrt(sum(HostSetOps._squares(flat, *_two_halves(flat)))))
        norm, scale, bad = sharded.sharded_grad_clip(HostSetOps(), flat, *_two_halves(flat), 0.1)
        assert float(scale) == want, seed
        seen.add(float(scale))
    assert len(seen) > 100


def test_norms_of_this_ranks_tensors():
    flat, norms = torch.tensor([3.0, 4.0, 6.0, 8.0]), torch.zeros(2)
    norm, scale, bad = sharded.sharded_grad_clip(HostSetOps(), flat, *_two_halves(flat), 100.0, norms=norms)
    assert norms.tolist() == [5.0, 10.0] and float(norm) == pytest.approx(math.sqrt(125))


class IllFormedOnOneRank(HostSetOps):
    """Rank 1 has left a tensor out (status 2), as the kernels do with an offset that no element starts at."""

    def grad_norm(self, base, offsets, lengths, result, **kw):
        super().grad_norm(base, offsets, lengths, result, **kw)
        result.view(torch.int32)[0] = 2 if dist.get_rank() == 1 else 0


def _rank(rank, world, port, out):
    os.environ.update(MASTER_ADDR="127.0.0.1", MASTER_PORT=str(port), RANK=str(rank), WORLD_SIZE=str(world))
    dist.init_process_group("gloo", rank=rank, world_size=world)
    flat = torch.arange(1.0, 5.0 + rank)
    result = torch.zeros(32, dtype=torch.uint8)
    norm, scale, bad = sharded.sharded_grad_clip(IllFormedOnOneRank(), flat, *_two_halves(flat), 1.0, result=result)
    torch.save((float(norm), float(scale), binding.read_norm_result(result)), f"{out}/{rank}.pt")
    dist.destroy_process_group()


def test_every_rank_gets_the_record_of_all_ranks(tmp_path):
    mp.spawn(_rank, args=(2, _free_port(), str(tmp_path)), nprocs=2)
    got = [torch.load(tmp_path / f"{r}.pt") for r in range(2)]
    assert got[0] == got[1]
    norm, scale, record = got[0]
    assert record == {"status": 2, "n_nonfinite": 0, "norm": norm, "scale": scale, "sum_squares": 30.0 + 55.0, "n_elements": 9}
    assert norm == np.float32(math.sqrt(85.0)) and scale == np.float32(1.0 / math.sqrt(85.0))


def test_the_record_of_one_rank():
    flat, result = torch.tensor([3.0, 4.0, math.inf]), torch.full((32,), 255, dtype=torch.uint8)
    sharded.sharded_grad_clip(HostSetOps(), flat, torch.tensor([0, 8]), torch.tensor([8, 4]), 1.0, result=result)
    assert binding.read_norm_result(result) == {"status": 0, "n_nonfinite": 1, "norm": math.inf, "scale": 0.0,
                                                "sum_squares": math.inf, "n_elements": 3}
