"""The example with a norm and the AdamW step: the retained tree follows what the steps changed, and the gradients are those of the formula."""
import importlib.util
import math
import os

import pytest
import torch

from paper_2510_23938_b200 import binding, inputs

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("verified_finetune_step", os.path.join(ROOT, "examples", "verified_finetune_step.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("optimizer", ["sgd", "adamw", "adamw8"])
@pytest.mark.parametrize("norm", [None, "layers.0.norm.weight"], ids=["plain", "norm"])
def test_steps_change_what_they_say_and_the_retained_tree_follows(example, optimizer, norm):
    runs = []
    for _ in range(2):
        with binding.Context(0) as ctx:
            runs.append(example.run(ctx, inputs.tiny_tensors(layers=4, v=3001), "embed.weight", "layers.0.up.weight", chunk_bytes=2048,
                                    steps=4, n_tokens=40, norm_weight=norm, optimizer=optimizer))
            assert ctx.device_status() == 0
    r = runs[0]
    assert r["root"] == r["fresh_root"] and not r["root_ok"]
    assert 0 < len(r["changed"]) and set(r["changed"]) <= set(r["dirty"]) and len(r["dirty"]) < r["chunks"]
    assert all(math.isfinite(x) for x in r["losses"] + r["norms"])
    assert runs[1] == r                                   # the same steps, the same bits


def test_gradients_are_those_of_the_formula(example):
    """Against 64-bit automatic differentiation.  Lookup, norm, product, its error, the two products back and the norm's gradient are
    rounded to 8 digits: seven roundings of at most 2^-9 of a value's norm each (the products' sums in 32 bits add far less), and
    each can pass through the six that follow it with a factor of about one: 7 * 2^-9 of the gradient's norm, taken twice."""
    generator = torch.Generator(device="cuda")
    generator.manual_seed(3)
    randn = lambda *shape: torch.randn(shape, generator=generator, device="cuda")  # noqa: E731
    rows, h, f, n = 50, 96, 160, 33
    table, up, norm = (x.to(torch.bfloat16) for x in (0.1 * randn(rows, h), 0.1 * randn(f, h), 1 + 0.1 * randn(h)))
    tokens, target = torch.randint(0, rows, (n,), generator=generator, device="cuda"), randn(n, f)
    with binding.Context(0) as ctx:
        s = example.forward(ctx, table, up, norm, tokens, target)
        d_up, d_hidden, d_norm = example.backward(ctx, s, up, norm)
        d_table = ctx.embedding_grad(d_hidden, tokens, rows, scale=math.sqrt(h))
    leaves = [x.double().requires_grad_() for x in (table, up, norm)]
    hidden = math.sqrt(h) * leaves[0][tokens]
    inner = hidden / (hidden.square().mean(1, keepdim=True) + 1e-5).sqrt() * leaves[2]
    (inner @ leaves[1].t() - target.double()).square().mean().backward()
    for got, leaf in zip((d_table, d_up, d_norm), leaves):
        off = float((got.double() - leaf.grad).norm() / leaf.grad.norm())
        assert off <= 2 * 7 * 2.0 ** -9, off
