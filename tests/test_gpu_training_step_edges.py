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


# ------------------------------------------------------------------------------------------------- types the first tests leave out

U = 2.0 ** -24
ROUND = {t: torch.finfo(t).eps / 2 for t in (torch.float32, torch.float16, torch.bfloat16)}      # unit roundoff
TINY = {torch.float32: 2.0 ** -150, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134}      # half the smallest number


@pytest.mark.parametrize("pair", [(torch.bfloat16, torch.float32), (torch.float16, torch.float16), (torch.float32, torch.float16)],
                         ids=lambda p: f"{p[0]}-{p[1]}".replace("torch.", ""))
@pytest.mark.parametrize("shape", [(1, 3, 1, 0, 0), (129, 300, 257, 3, 1), (511, 700, 2048, 0, 0), (2049, 2, 40, 1, 2), (9000, 4, 515, 0, 0),
                                   (20_001, 5000, 129, 1, 0)], ids=str)
def test_gradient_of_the_other_type_pairs(ctx, shape, pair):
    """n, rows, dim, elements before the first and between the rows.  m terms: (m - 1) u of their magnitudes, one u each for the
    scale's own rounding, the product and (added) the sum with the old value, one rounding to the output's type."""
    n, rows, dim, skew, gap = shape
    kind, out_kind = pair
    def strided(r, values, dtype):
        flat = torch.zeros(skew + r * (dim + gap), dtype=dtype, device="cuda")
        view = flat[skew:].view(r, dim + gap)[:, :dim]
        return view.copy_(values) if values is not None else view
    grad = strided(n, torch.randn(n, dim, generator=_gen(n), device="cuda") * 0.05, kind)
    tokens = torch.randint(0, rows, (n,), generator=_gen(n + 1), device="cuda")
    old = (torch.randn(rows, dim, generator=_gen(2), device="cuda") * 0.05).to(out_kind)
    scale = 1.5
    true = torch.zeros(rows, dim, dtype=torch.float64, device="cuda").index_add_(0, tokens, grad.double()) * scale
    size = torch.zeros_like(true).index_add_(0, tokens, grad.double().abs()) * scale
    terms = torch.bincount(tokens, minlength=rows)[:, None].double()

    def close(got, want, extra):
        limit = ((terms + 3.0) * U * size + extra) * (1 + 1e-6)
        limit = limit + ROUND[out_kind] * (want.abs() + limit) + TINY[out_kind]
        return bool(((got.double() - want).abs() <= limit).all())

    dense = ctx.embedding_grad(grad, tokens, rows, scale=scale, out=strided(rows, None, out_kind))
    assert close(dense, true, 0.0)
    cap = min(n, rows)
    touched, packed, count = ctx.embedding_grad_rows(grad, tokens, rows, scale=scale, out=strided(cap, None, out_kind))
    distinct = torch.unique(tokens)
    assert int(count) == distinct.numel() and torch.equal(touched[:int(count)], distinct)
    assert torch.equal(packed[:int(count)], dense[distinct]) and not bool(packed[int(count):].any())
    added = ctx.embedding_grad(grad, tokens, rows, scale=scale, out=strided(rows, old, out_kind), accumulate=True)
    assert close(added, true + old.double(), U * (old.double().abs() + size))


@pytest.mark.parametrize("cap", [5, 6, 40, 1000])
def test_compact_gradient_with_more_room_than_tokens(ctx, cap):
    tokens = torch.tensor([7, 2, 7, 9, 2], device="cuda")
    grad = torch.arange(1, 6, device="cuda").float()[:, None].expand(5, 300).contiguous()
    rows = torch.full((cap,), 55, device="cuda")
    r, g, c = ctx.embedding_grad_rows(grad, tokens, 10, rows=rows, out=torch.full((cap, 300), 7.0, device="cuda"))
    assert r.tolist() == [2, 7, 9] + [-1] * (cap - 3) and int(c) == 3
    assert bool((g == torch.tensor([7.0, 4.0, 4.0] + [0.0] * (cap - 3), device="cuda")[:, None]).all())


def test_outputs_of_more_than_32_bits_of_bytes(ctx):
    """Lookup and table gradient whose last rows lie behind 2^32 bytes."""
    n, dim, rows = 530_000, 4096, 1000                       # 4.3 GB of 16-bit rows
    table = torch.randn(rows, dim, generator=_gen(1), device="cuda").to(torch.bfloat16)
    tokens = torch.randint(0, rows, (n,), generator=_gen(2), device="cuda")
    got = ctx.embedding(table, tokens)
    for at in range(0, n, 53_000):
        assert torch.equal(got[at:at + 53_000], table[tokens[at:at + 53_000]])
    del got
    torch.cuda.empty_cache()
    few = torch.tensor([0, n - 1, 524_287, 524_288, n - 1], device="cuda")
    grad = torch.arange(1, 6, device="cuda").to(torch.bfloat16)[:, None].expand(5, dim).contiguous()
    out = torch.full((n, dim), 3.0, dtype=torch.bfloat16, device="cuda")
    ctx.embedding_grad(grad, few, n, out=out)
    want = {0: 1.0, n - 1: 7.0, 524_287: 3.0, 524_288: 4.0}
    for row, value in want.items():
        assert bool((out[row] == value).all()), row
        out[row] = 0
    assert not bool(out.view(torch.int64).any())


# ------------------------------------------------------------------------------------------------- sets of several types

def _mixed(seed=0):
    """Tensors of three types in one byte buffer, some at odd multiples of their element, one of several blocks' pieces."""
    kinds = [torch.float32, torch.bfloat16, torch.float16, torch.bfloat16, torch.float32, torch.float16]
    counts = [1_000_003, 2_500_001, 7, 0, 12_345, 700_000]
    places, at = [], 4
    for kind, count in zip(kinds, counts):
        size = torch.empty(0, dtype=kind).element_size()
        at = -(-at // size) * size
        places.append(at)
        at += count * size + 2
    raw = torch.zeros(at + 16, dtype=torch.uint8, device="cuda")
    views = [raw[p:p + c * torch.empty(0, dtype=k).element_size()].view(k) for k, c, p in zip(kinds, counts, places)]
    for i, v in enumerate(views):
        v.copy_(torch.randn(v.numel(), generator=_gen(seed + i), device="cuda") * 0.01)
    offsets = torch.tensor(places, dtype=torch.int64, device="cuda")
    lengths = torch.tensor([v.numel() * v.element_size() for v in views], dtype=torch.int64, device="cuda")
    types = torch.tensor([binding.DTYPES[k] for k in kinds], dtype=torch.uint8, device="cuda")
    return raw, views, offsets, lengths, types


def test_mixed_set_norm_and_clip_in_place(ctx):
    raw, views, offsets, lengths, types = _mixed()
    before, untouched = [v.clone() for v in views], raw.clone()
    want = torch.stack([v.double().square().sum() for v in views])
    result, norms = binding.new_norm_result("cuda"), torch.empty(len(views), device="cuda")
    ctx.grad_clip(raw, offsets, lengths, 0.25, result, norms=norms, types=types)
    r = binding.read_norm_result(result)
    tolerance = 65 * U / 2 + U
    assert r["status"] == 0 and r["n_elements"] == sum(v.numel() for v in views)
    assert abs(r["norm"] - float(want.sum().sqrt())) <= tolerance * r["norm"]
    assert bool(((norms.double() - want.sqrt()).abs() <= tolerance * want.sqrt()).all())
    for v, b in zip(views, before):
        assert torch.equal(v, (b.float() * r["scale"]).to(b.dtype))
        v.copy_(b)
    assert r["scale"] < 1 and torch.equal(raw, untouched)            # and nothing between the tensors


@pytest.mark.parametrize("out_dtype", [None, torch.float32], ids=str)
@pytest.mark.parametrize("call", ["grad_clip", "grad_scale"])
def test_mixed_set_into_another_buffer(ctx, call, out_dtype):
    raw, views, offsets, lengths, types = _mixed(10)
    kept = raw.clone()
    kinds = [out_dtype or v.dtype for v in views]
    places, at = [], 8
    for v, k in zip(views, kinds):
        size = torch.empty(0, dtype=k).element_size()
        at = -(-at // size) * size
        places.append(at)
        at += v.numel() * size + 6
    out = torch.full((at + 16,), 0xA5, dtype=torch.uint8, device="cuda")
    where = torch.tensor(places, dtype=torch.int64, device="cuda")
    result, factor = binding.new_norm_result("cuda"), torch.full((1,), 0.3, device="cuda")
    if call == "grad_clip":
        ctx.grad_clip(raw, offsets, lengths, 0.25, result, out=out, out_offsets=where, types=types, out_dtype=out_dtype)
        scale = binding.read_norm_result(result)["scale"]
    else:
        ctx.grad_scale(raw, offsets, lengths, factor, out=out, out_offsets=where, types=types, out_dtype=out_dtype)
        scale = float(factor)
    want = torch.full_like(out, 0xA5)
    for v, k, p in zip(views, kinds, places):
        values = (v.float() * scale).to(k)
        want[p:p + values.numel() * values.element_size()] = values.view(torch.uint8)
    assert torch.equal(out, want) and torch.equal(raw, kept) and ctx.device_status() == 0


def test_mixed_set_with_outputs_that_cannot_be(ctx):
    """An output type that a tensor's type is not rounded to, and an output that no element starts at: status 2, and that
    tensor's output stays as it was; the others are written."""
    tensors = [torch.full((300,), 2.0, device="cuda"), torch.full((300,), 2.0, device="cuda").half(),
               torch.full((300,), 2.0, device="cuda").bfloat16()]
    base, offsets, lengths, types = binding.tensor_ranges(tensors)
    factor, where = torch.full((1,), 0.5, device="cuda"), torch.tensor([0, 600, 1200], device="cuda")
    out = torch.full((900,), 7.0, dtype=torch.bfloat16, device="cuda")
    ctx.grad_scale(base, offsets, lengths, factor, out=out, out_offsets=where, types=types, out_dtype=torch.bfloat16)
    assert ctx.device_status() == 2
    assert out.view(3, 300).float().tolist() == [[1.0] * 300, [7.0] * 300, [1.0] * 300]
    out = torch.full((1204,), 7.0, device="cuda")
    ctx.grad_scale(base, offsets, lengths, factor, out=out, out_offsets=torch.tensor([0, 1202, 2404], device="cuda"), types=types,
                   out_dtype=torch.float32)
    assert ctx.device_status() == 2
    assert bool((out[:300] == 1).all()) and bool((out[300:601] == 7).all()) and bool((out[601:901] == 1).all()) and bool((out[901:] == 7).all())


def test_more_pieces_of_one_tensor_in_a_block_than_it_keeps(ctx):
    """160,000 small tensors beside a large one: the set is cut into pieces of 8,192 elements, of which one block has over 256
    of the large tensor in a row."""
    small, large = 160_000, 40_000_000
    flat = torch.randn(small * 3 + large, generator=_gen(1), device="cuda")
    lengths = torch.cat([torch.full((small // 2,), 12, device="cuda"), torch.tensor([large * 4], device="cuda"),
                         torch.full((small // 2,), 12, device="cuda")])
    offsets = torch.cumsum(lengths, 0) - lengths
    result, norms = binding.new_norm_result("cuda"), torch.empty(small + 1, device="cuda")
    ctx.grad_norm(flat, offsets, lengths, result, norms=norms)
    r = binding.read_norm_result(result)
    first = small // 2 * 3
    want = torch.cat([flat[:first].view(-1, 3).double().square().sum(1), flat[first:first + large].double().square().sum()[None],
                      flat[first + large:].view(-1, 3).double().square().sum(1)])
    assert r["status"] == 0 and r["n_elements"] == flat.numel()
    assert abs(r["sum_squares"] - float(want.sum())) <= 65 * U * r["sum_squares"]
    assert bool(((norms.double() - want.sqrt()).abs() <= (65 * U / 2 + U) * want.sqrt()).all())
    again = binding.new_norm_result("cuda")
    ctx.grad_norm(flat, offsets, lengths, again)
    assert torch.equal(again, result)
