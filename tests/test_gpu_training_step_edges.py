"""Edges of the training-step operators: what their first tests leave out."""
import math

import numpy as np
import pytest
import torch

from paper_2510_23938_b200 import binding

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    assert torch.cuda.is_available(), "the gpu-marked tests need a CUDA device"
    c = binding.Context(0)
    yield c
    assert c.device_status() == 0
    c.close()


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


# ------------------------------------------------------------------------------------------------- the sort's cluster

@pytest.mark.parametrize("n", [513, 1025, 2049, 4097, 4100, 8192 + 1, 2 * 8192 + 1, 8 * 8192 + 1])
def test_sort_of_a_cluster_whose_blocks_have_very_different_shares(ctx, n):
    """Sizes just above a power of two leave the cluster's last blocks with few keys or none: they are the first to write
    into the others' shared memory.  Over and over beside work that keeps the other multiprocessors busy, the rows and
    their sums (small whole numbers: exact in any order) are right every time."""
    rows, dim = 3000, 8
    tokens = torch.randint(0, rows, (n,), generator=_gen(n), device="cuda", dtype=torch.int32)
    grad = torch.randint(-8, 9, (n, dim), generator=_gen(n + 1), device="cuda").float()
    distinct = torch.unique(tokens.long())
    want = torch.zeros(rows, dim, dtype=torch.float64, device="cuda").index_add_(0, tokens.long(), grad.double())[distinct]
    busy, side = torch.randn(1 << 22, device="cuda"), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    wrong = torch.zeros((), dtype=torch.int64, device="cuda")
    for _ in range(100):
        with torch.cuda.stream(side):
            busy.mul_(1.0)
        r, g, c = ctx.embedding_grad_rows(grad, tokens, rows)
        wrong += (c[0] != distinct.numel()) | (r[:distinct.numel()] != distinct).any() | (g[:distinct.numel()] != want).any()
    torch.cuda.current_stream().wait_stream(side)
    assert int(wrong) == 0
