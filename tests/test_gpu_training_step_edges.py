"""Edges of the training-step operators: what their first tests leave out."""
import math

import numpy as np
import pytest
import torch

from paper_2510_23938_b200 import binding, sharded

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


# ------------------------------------------------------------------------------------------------- tokens outside the table

@pytest.mark.parametrize("dtype", [torch.int32, torch.int64], ids=str)
@pytest.mark.parametrize("padding", [None, 3])
@pytest.mark.parametrize("form", ["table", "added", "rows"])
def test_gradient_reports_token_minus_one(ctx, form, padding, dtype):
    """-1 stands for "no padding row"; as a token it is a row that is not there, in the gradient as in the lookup."""
    tokens = torch.tensor([2, -1, 0, 2], dtype=dtype, device="cuda")
    grad = torch.ones(4, 5, device="cuda")
    if form == "rows":
        rows, got, count = ctx.embedding_grad_rows(grad, tokens, 6, padding_row=padding)
        assert rows.tolist() == [0, 2, -1, -1] and int(count) == 2 and got[:, 0].tolist() == [1, 2, 0, 0]
    else:
        out = torch.full((6, 5), 10.0, device="cuda")
        got = ctx.embedding_grad(grad, tokens, 6, padding_row=padding, out=out, accumulate=form == "added")
        old = 10 if form == "added" else 0
        assert got[:, 0].tolist() == [old + 1, old, old + 2, old, old, old]
    assert ctx.device_status() == 2 and ctx.device_status() == 0


def test_gradient_does_not_report_padding(ctx):
    """A padding row inside the table or behind it gives no gradient and no complaint."""
    grad = torch.ones(3, 5, device="cuda")
    for padding in (0, 4, 2 ** 31):
        tokens = torch.tensor([1, padding, 1], device="cuda")
        assert ctx.embedding_grad(grad, tokens, 4, padding_row=padding)[:, 0].tolist() == [0, 2, 0, 0]
        assert ctx.device_status() == 0


# ------------------------------------------------------------------------------------------------- tensors of their own

def _own(*shapes):
    return [torch.randn(*s, generator=_gen(50 + i), device="cuda") for i, s in enumerate(shapes)]


@pytest.mark.parametrize("shapes", [[(0, 8), (300,), (7,)], [(300,), (0,), (7,)], [(300,), (7,), (0, 8)],
                                    [(0,), (0, 4), (5,)]], ids=str)
def test_empty_tensors_anywhere_in_a_set(ctx, shapes):
    """A step without tokens hands over a gradient of no rows."""
    tensors = _own(*shapes)
    before = [t.clone() for t in tensors]
    base, offsets, lengths, types = binding.tensor_ranges(tensors)
    result, norms = binding.new_norm_result("cuda"), torch.full((len(tensors),), 9.0, device="cuda")
    ctx.grad_clip(base, offsets, lengths, 0.5, result, norms=norms, types=types)
    r = binding.read_norm_result(result)
    whole = torch.cat([b.reshape(-1) for b in before]).double()
    assert r["status"] == 0 and r["n_elements"] == whole.numel()
    assert abs(r["norm"] - float(whole.norm())) <= 34 * 2.0 ** -24 * float(whole.norm())     # 65 u / 2 + u
    for t, b, norm in zip(tensors, before, norms.tolist()):
        assert torch.equal(t, b * r["scale"]) and (norm == 0) == (t.numel() == 0)


@pytest.mark.parametrize("tensors", [[], [(0,)], [(0, 3), (0,)]], ids=str)
def test_sets_of_nothing(ctx, tensors):
    base, offsets, lengths, types = binding.tensor_ranges(_own(*tensors))
    assert offsets.numel() == lengths.numel() == types.numel() == len(tensors)
    result, factor = binding.new_norm_result("cuda"), torch.ones(1, device="cuda")
    nothing = {"status": 0, "n_nonfinite": 0, "norm": 0.0, "scale": 1.0, "sum_squares": 0.0, "n_elements": 0}
    ctx.grad_norm(base, offsets, lengths, result, types=types)
    assert binding.read_norm_result(result) == nothing
    ctx.grad_clip(base, offsets, lengths, 1.0, result, types=types)
    assert binding.read_norm_result(result) == nothing
    ctx.grad_scale(base, offsets, lengths, factor, types=types)
    assert ctx.device_status() == 0


# ------------------------------------------------------------------------------------------------- clipping over ranks

def test_sharded_clipping_on_another_stream_with_work_in_front(ctx):
    """The gradients are still being written on that stream when the call returns to the host."""
    flat = torch.randn(70_001, generator=_gen(1), device="cuda")
    offsets, lengths = torch.tensor([0, 40_000], device="cuda"), torch.tensor([40_000, 240_004], device="cuda")
    side, front = torch.cuda.Stream(), torch.ones(8192, 8192, device="cuda")
    want, result = flat.clone(), binding.new_norm_result("cuda")
    ctx.grad_clip(want, offsets, lengths, 0.5, result)
    r = binding.read_norm_result(result)
    for _ in range(5):
        late = torch.zeros_like(flat)
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            front @ front
            late.copy_(flat)
        norm, scale, bad = sharded.sharded_grad_clip(ctx, late, offsets, lengths, 0.5, stream=side)
        side.synchronize()
        assert (float(norm), float(scale), int(bad)) == (r["norm"], r["scale"], 0) and torch.equal(late, want)


@pytest.mark.parametrize("limit", [0.1, 0.3, 1e-3])
def test_sharded_clipping_on_one_rank_is_grad_clip_bit_for_bit(ctx, limit):
    """Limits that 32 bits do not hold exactly, over several gradients."""
    offsets, lengths = torch.tensor([0, 8000], device="cuda"), torch.tensor([8000, 12_000], device="cuda")
    for seed in range(40):
        flat = torch.randn(5000, generator=_gen(seed), device="cuda")
        other, result = flat.clone(), binding.new_norm_result("cuda")
        ctx.grad_clip(flat, offsets, lengths, limit, result)
        norm, scale, bad = sharded.sharded_grad_clip(ctx, other, offsets, lengths, limit)
        r = binding.read_norm_result(result)
        assert (float(norm), float(scale), int(bad)) == (r["norm"], r["scale"], r["n_nonfinite"]), seed
        assert torch.equal(flat, other), seed


def test_sharded_clipping_tells_of_an_ill_formed_tensor(ctx):
    flat = torch.ones(100, device="cuda")
    offsets, lengths = torch.tensor([0, 42], device="cuda"), torch.tensor([40, 40], device="cuda")
    result, norms = binding.new_norm_result("cuda"), torch.full((2,), 9.0, device="cuda")
    sharded.sharded_grad_clip(ctx, flat, offsets, lengths, 1.0, norms=norms, result=result)
    got = result.clone()
    assert ctx.device_status() == 2 and binding.read_norm_result(got)["status"] == 2
    other = torch.ones(100, device="cuda")
    ctx.grad_clip(other, offsets, lengths, 1.0, result)
    assert ctx.device_status() == 2 and torch.equal(got, result) and torch.equal(flat, other) and float(norms[1]) == 0


# ------------------------------------------------------------------------------------------------- two descriptions of a set

@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32], ids=str)
@pytest.mark.parametrize("lengths", [[100_003, 7, 0, 40_000], [8193], [20_000] * 1100 + [300_000], [5_000_000, 3]],
                         ids=lambda s: f"{len(s)}x{sum(s)}")
def test_bits_do_not_depend_on_how_the_set_is_described(ctx, dtype, lengths):
    """One type for all tensors, or the same type tensor by tensor, with a tensor of another type and no elements too."""
    size = torch.empty(0, dtype=dtype).element_size()
    flat = (torch.randn(sum(lengths), generator=_gen(4), device="cuda") * torch.rand(sum(lengths), generator=_gen(5), device="cuda")).to(dtype)
    nbytes = torch.tensor(lengths, dtype=torch.int64, device="cuda") * size
    offsets = torch.cumsum(nbytes, 0) - nbytes
    code, n = binding.DTYPES[dtype], len(lengths)
    types = torch.full((n,), code, dtype=torch.uint8, device="cuda")
    zero = torch.zeros(1, dtype=torch.int64, device="cuda")
    sets = [(offsets, nbytes, None), (offsets, nbytes, types)]
    sets += [(torch.cat([zero, offsets]), torch.cat([zero, nbytes]), torch.cat([torch.full_like(types[:1], other), types]))
             for other in (0, 1)]
    got = []
    for where, sizes, kinds in sets:
        clipped, result, norms = flat.clone(), binding.new_norm_result("cuda"), torch.empty(where.numel(), device="cuda")
        ctx.grad_clip(clipped, where, sizes, 1.0, result, norms=norms, types=kinds)
        r = binding.read_norm_result(result)
        got.append((r, norms[-n:].tolist(), clipped))
    for r, norms, clipped in got[1:]:
        assert r == got[0][0] and norms == got[0][1] and torch.equal(clipped, got[0][2])


# ------------------------------------------------------------------------------------------------- captured calls and scratch

def _step(ctx, n, rows, dim, tensors):
    """Inputs and outputs of a gradient of either form, a clip and a scale, and the calls."""
    tokens = torch.randint(0, rows, (n,), generator=_gen(n), device="cuda")
    grad = torch.randn(n, dim, generator=_gen(n + 1), device="cuda")
    flat = torch.randn(tensors * 100, generator=_gen(tensors), device="cuda")
    lengths = torch.full((tensors,), 400, dtype=torch.int64, device="cuda")
    offsets = torch.cumsum(lengths, 0) - lengths
    result, factor = binding.new_norm_result("cuda"), torch.full((1,), 0.5, device="cuda")
    cap = min(n, rows)
    out = [torch.zeros(rows, dim, device="cuda"), torch.zeros(cap, dtype=torch.int64, device="cuda"), torch.zeros(cap, dim, device="cuda"),
           torch.zeros(1, dtype=torch.int64, device="cuda"), torch.zeros_like(flat), torch.zeros_like(flat), result]
    calls = {
        "embedding_grad": lambda: ctx.embedding_grad(grad, tokens, rows, out=out[0]),
        "embedding_grad_rows": lambda: ctx.embedding_grad_rows(grad, tokens, rows, rows=out[1], out=out[2], count=out[3]),
        "grad_clip": lambda: ctx.grad_clip(flat, offsets, lengths, 1.0, result, out=out[4], out_offsets=offsets),
        "grad_norm": lambda: ctx.grad_norm(flat, offsets, lengths, result),
        "grad_scale": lambda: ctx.grad_scale(flat, offsets, lengths, factor, out=out[5], out_offsets=offsets),
    }
    return out, calls


def test_a_graph_outlives_the_growth_of_its_context():
    """Captured on small inputs, replayed after larger calls have enlarged the scratch, and between them."""
    with binding.Context(0) as ctx:
        out, calls = _step(ctx, 3000, 40, 264, 1100)
        for call in calls.values():
            call()
        torch.cuda.synchronize()
        want = [t.clone() for t in out]
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            for call in calls.values():
                call()
        for size in (2, 7, 20):
            large, larger_calls = _step(ctx, 3000 * size, 50, 264 + 8 * size, 1100 * size)
            for call in larger_calls.values():
                call()
            kept = [t.clone() for t in large]
            for t in out:
                t.zero_()
            graph.replay()
            filler = torch.full((1 << 24,), 7, dtype=torch.int32, device="cuda")      # takes freed memory, if there is any
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(out, want))
            for call in larger_calls.values():
                call()
            assert all(torch.equal(a, b) for a, b in zip(large, kept))
            del filler
        assert ctx.device_status() == 0
        del graph


@pytest.mark.parametrize("name", ["embedding_grad", "embedding_grad_rows", "grad_clip", "grad_norm", "grad_scale"])
@pytest.mark.parametrize("mode", ["global", "thread_local", "relaxed"])
def test_growth_under_capture_is_refused(name, mode):
    """With an error and nothing else: the capture goes on, and the call works afterwards."""
    with binding.Context(0) as ctx:
        out, calls = _step(ctx, 2000, 300, 40, 50)
        launched, mark = ctx.kernel_launches, torch.zeros(1, device="cuda")
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, capture_error_mode=mode):
            mark.add_(1)
            with pytest.raises(binding.IvError) as err:
                calls[name]()
        assert err.value.code == binding.IV_ERR_CUDA and err.value.cuda_error == 900 and ctx.kernel_launches == launched
        graph.replay()
        calls[name]()
        torch.cuda.synchronize()
        assert float(mark) == 1 and ctx.device_status() == 0
        first, again = [t.clone() for t in out], torch.cuda.CUDAGraph()
        with torch.cuda.graph(again, capture_error_mode=mode):
            calls[name]()
        for t in out:
            t.zero_()
        again.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, first)) and any(bool(t.any()) for t in out)
        del graph, again
