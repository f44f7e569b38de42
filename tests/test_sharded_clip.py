"""Clipping by the common norm of gradients on several ranks: the host logic over gloo, with a context made of torch operations."""
import os
import socket

import pytest
import torch
import torch.distributed as dist
import torch.multiprocessing as mp

from paper_2510_23938_b200 import sharded


class PlainSetOps:
    """grad_norm and grad_scale of a context, for float32 tensors on the host."""

    @staticmethod
    def _parts(base, offsets, lengths):
        return [base[o // 4:(o + n) // 4] for o, n in zip(offsets.tolist(), lengths.tolist())]

    def grad_norm(self, base, offsets, lengths, result):
        parts = self._parts(base, offsets, lengths)
        result.view(torch.float64)[2] = sum((p.double().square().sum() for p in parts), torch.zeros((), dtype=torch.float64))
        result.view(torch.int32)[1] = sum(int(not torch.isfinite(p).all()) for p in parts)

    def grad_scale(self, base, offsets, lengths, scale):
        for p in self._parts(base, offsets, lengths):
            p.mul_(scale)


def _shares(world):
    g = torch.Generator().manual_seed(7)
    return [torch.randn(100 + 31 * r, generator=g) for r in range(world)]


def _rank(rank, world, port, max_norm, out):
    os.environ.update(MASTER_ADDR="127.0.0.1", MASTER_PORT=str(port), RANK=str(rank), WORLD_SIZE=str(world))
    dist.init_process_group("gloo", rank=rank, world_size=world)
    flat = _shares(world)[rank].clone()
    half = flat.numel() // 2 * 4
    offsets, lengths = torch.tensor([0, half]), torch.tensor([half, flat.numel() * 4 - half])
    norm, scale, bad = sharded.sharded_grad_clip(PlainSetOps(), flat, offsets, lengths, max_norm)
    torch.save((flat, float(norm), float(scale), int(bad)), f"{out}/{rank}.pt")
    dist.destroy_process_group()


def _free_port():
    with socket.socket() as s:
        s.bind(("127.0.0.1", 0))
        return s.getsockname()[1]


@pytest.mark.parametrize("world", [2, 3])
@pytest.mark.parametrize("max_norm", [1.0, 1e6])
def test_ranks_clip_by_the_common_norm(tmp_path, world, max_norm):
    mp.spawn(_rank, args=(world, _free_port(), max_norm, str(tmp_path)), nprocs=world)
    shares = _shares(world)
    norm = torch.cat(shares).double().norm()
    got = [torch.load(tmp_path / f"{r}.pt") for r in range(world)]
    assert len({g[1:] for g in got}) == 1                       # the same norm, scale and count on every rank
    assert abs(got[0][1] - float(norm)) <= 2.0 ** -23 * float(norm) and got[0][3] == 0
    scale = min(1.0, max_norm / float(norm))
    assert abs(got[0][2] - scale) <= 2.0 ** -23 * scale
    for share, g in zip(shares, got):
        assert torch.equal(g[0], share * torch.tensor(got[0][2]))


def test_one_rank_without_a_process_group_and_a_bad_tensor():
    flat = torch.tensor([3.0, 4.0, float("inf"), 1.0])
    offsets, lengths = torch.tensor([0, 8]), torch.tensor([8, 8])
    norm, scale, bad = sharded.sharded_grad_clip(PlainSetOps(), flat, offsets, lengths, 1.0)
    assert float(norm) == float("inf") and float(scale) == 0.0 and int(bad) == 1
