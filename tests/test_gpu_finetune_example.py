"""The example that runs the training-step operators together with verification, and the sharded clipping on one rank."""
import importlib.util
import math
import os

import pytest
import torch

from paper_2510_23938_b200 import binding, inputs, sharded

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _example():
    spec = importlib.util.spec_from_file_location("verified_finetune_step", os.path.join(ROOT, "examples", "verified_finetune_step.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_steps_change_what_they_say_and_the_retained_tree_follows():
    example = _example()
    runs = []
    for _ in range(2):
        with binding.Context(0) as ctx:
            runs.append(example.run(ctx, inputs.tiny_tensors(layers=4, v=3001), "embed.weight", "layers.0.up.weight",
                                    chunk_bytes=2048, steps=4, n_tokens=40))
            assert ctx.device_status() == 0
    r = runs[0]
    assert r["root"] == r["fresh_root"] and not r["root_ok"]
    assert set(r["changed"]) <= set(r["dirty"]) and 0 < len(r["dirty"]) < r["chunks"]
    assert all(math.isfinite(x) for x in r["losses"] + r["norms"]) and r["losses"][-1] < r["losses"][0]
    assert runs[1] == r                                   # the same steps, the same bits


def test_chunks_of_a_row():
    example = _example()
    starts = torch.tensor([0, 4095, 4096, 10_000])
    assert example.chunks_of(starts, 2, 4096).tolist() == [0, 1, 2]
    assert example.chunks_of(starts[:1], 4096, 4096).tolist() == [0]
    assert example.chunks_of(starts[1:2], 8193, 4096).tolist() == [0, 1, 2]


def test_sharded_clipping_on_one_rank_is_the_plain_one():
    flat = torch.randn(5000, device="cuda")
    offsets, lengths = torch.tensor([0, 8000], device="cuda"), torch.tensor([8000, 12_000], device="cuda")
    with binding.Context(0) as ctx:
        one, two, result = flat.clone(), flat.clone(), binding.new_norm_result("cuda")
        ctx.grad_clip(one, offsets, lengths, 0.5, result)
        norm, scale, bad = sharded.sharded_grad_clip(ctx, two, offsets, lengths, 0.5)
        r = binding.read_norm_result(result)
        assert torch.equal(one, two) and float(norm) == r["norm"] and float(scale) == r["scale"] and int(bad) == 0
