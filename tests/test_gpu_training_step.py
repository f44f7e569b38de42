"""Embedding lookup, its gradient, the global gradient norm and clipping against plain 64-bit forms.

Tolerances are derived, not tuned.  u = 2^-24 is the unit roundoff of 32-bit floats; an output of type T adds one
rounding of at most ROUND[T] relative (or half the type's smallest number).  A lookup is one 32-bit product, so it must
equal the same product bit for bit.  A 32-bit sum of m terms in any order is within (m - 1) u sum|terms| of the true
one; scaling and adding to what is there are two more roundings.  In a norm a square goes through
at most 64 roundings of 32 bits (its own, and the additions of its share of a piece) and everything above is in 64 bits, the
root halves the relative error, and the result is rounded once to 32 bits: 65 u / 2 + u.
"""
import ctypes
import math

import numpy as np
import pytest
import torch

from paper_2510_23938_b200 import binding

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
ROUND = {t: torch.finfo(t).eps / 2 for t in (torch.float32, torch.float16, torch.bfloat16)}      # unit roundoff
TINY = {torch.float32: 2.0 ** -150, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134}
PAIRS = [(torch.bfloat16, torch.bfloat16), (torch.float32, torch.float32), (torch.float16, torch.float32),
         (torch.float32, torch.bfloat16), (torch.bfloat16, torch.float32), (torch.float16, torch.float16),
         (torch.float32, torch.float16)]
NORM_TOLERANCE = 65 * U / 2 + U

SENTINEL = 0xA5
MARGIN = 512


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


class Guarded:
    """rows x cols elements, rows `stride` apart, `skew` elements past a 512-byte boundary, inside sentinel bytes."""

    def __init__(self, rows, cols, dtype, skew=0, stride=None, fill=None):
        self.stride = cols if stride is None else stride
        size = torch.empty(0, dtype=dtype).element_size()
        room = max(1, (max(rows - 1, 0) * self.stride + cols)) * size
        self.raw = torch.full((2 * MARGIN + skew * size + (room + 15) // 16 * 16,), SENTINEL, dtype=torch.uint8, device="cuda")
        lo = MARGIN + skew * size
        self.view = self.raw[lo:lo + room].view(dtype)[:max(0, (rows - 1) * self.stride + cols)].as_strided(
            (rows, cols), (self.stride, 1)) if rows else torch.empty(0, cols, dtype=dtype, device="cuda")
        if fill is not None and rows:
            self.view.copy_(fill)
        mask = torch.zeros_like(self.raw, dtype=torch.bool)
        if rows and cols:
            at = (torch.arange(rows, device="cuda")[:, None] * self.stride * size
                  + torch.arange(cols * size, device="cuda")[None, :]).reshape(-1) + lo
            mask[at] = True
        self.outside = ~mask

    def check(self):
        torch.cuda.synchronize()
        assert bool((self.raw[self.outside] == SENTINEL).all()), "bytes outside the output were written"


def _tokens(n, rows, seed, kind="zipf", dtype=torch.int64):
    g = _gen(seed)
    if kind == "same":
        t = torch.full((n,), rows // 2, device="cuda")
    elif kind == "distinct":
        t = torch.randperm(rows, generator=g, device="cuda")[:n]
    elif kind == "descending":
        t = (rows - 1) - torch.arange(n, device="cuda") % rows
    else:
        u = torch.rand(n, generator=g, device="cuda", dtype=torch.float64)
        t = (torch.exp(u * math.log(rows + 1)).floor() - 1).clamp(0, rows - 1)
    return t.to(dtype)


# ------------------------------------------------------------------------------------------------- lookup

LOOKUPS = [  # n, rows, dim, table skew (elements), row padding, out skew, out padding
    (1, 1, 1, 0, 0, 0, 0), (1, 7, 4096, 4, 0, 0, 0), (5, 11, 3, 1, 2, 1, 3), (33, 100, 1023, 3, 1, 5, 0),
    (64, 50, 2048, 4, 0, 0, 0), (17, 29, 1025, 0, 0, 7, 1), (300, 40, 129, 2, 7, 0, 0), (9, 1000, 5000, 6, 3, 2, 4),
]


@pytest.mark.parametrize("shape", LOOKUPS)
@pytest.mark.parametrize("pair", PAIRS, ids=lambda p: f"{p[0]}-{p[1]}".replace("torch.", ""))
def test_lookup_is_one_rounded_product(ctx, shape, pair):
    n, rows, dim, skew, pad, oskew, opad = shape
    kind, out_kind = pair
    table = Guarded(rows, dim, kind, skew, dim + pad, torch.randn(rows, dim, generator=_gen(1), device="cuda"))
    tokens = _tokens(n, rows, 2, dtype=torch.int32 if n % 2 else torch.int64)
    scale = math.sqrt(dim)
    out = Guarded(n, dim, out_kind, oskew, dim + opad)
    got = ctx.embedding(table.view, tokens, scale=scale, out=out.view)
    out.check()
    table.check()
    want = table.view.float()[tokens.long()] * torch.tensor(scale, dtype=torch.float32, device="cuda")
    assert torch.equal(got, want.to(out_kind))
    true = table.view.double()[tokens.long()] * scale
    limit = (U + U + ROUND[out_kind]) * true.abs() * (1 + 1e-6) + TINY[out_kind]     # the factor, the product, the output
    assert bool(((got.double() - true).abs() <= limit).all())


def test_lookup_shapes_of_tokens_and_defaults(ctx):
    table = torch.randn(50, 24, device="cuda", dtype=torch.bfloat16)
    tokens = _tokens(24, 50, 3).view(2, 3, 4)
    got = ctx.embedding(table, tokens)
    assert got.shape == (2, 3, 4, 24) and torch.equal(got, table[tokens])
    assert torch.equal(ctx.embedding(table, tokens, out_dtype=torch.float32), table.float()[tokens])
    assert ctx.embedding(table, tokens[:0]).shape == (0, 3, 4, 24)
    assert ctx.embedding(table[:, :0], tokens).shape == (2, 3, 4, 0)


def test_lookup_keeps_infinities_and_nan(ctx):
    table = torch.tensor([[math.inf, -math.inf, math.nan, 0.0, -0.0, 3.4e38, 1e-45, 1.0]], device="cuda")
    got = ctx.embedding(table, torch.zeros(3, dtype=torch.int64, device="cuda"), scale=2.0, out_dtype=torch.bfloat16)
    want = (table * 2.0).to(torch.bfloat16).expand(3, 8)
    assert torch.equal(torch.nan_to_num(got.float(), nan=7.0), torch.nan_to_num(want.float(), nan=7.0))
    assert torch.equal(torch.isnan(got), torch.isnan(want))


@pytest.mark.parametrize("dtype", [torch.int32, torch.int64])
@pytest.mark.parametrize("bad", [-1, 40, -(2 ** 31), 2 ** 31 - 1])
def test_lookup_of_a_row_that_is_not_there(ctx, dtype, bad):
    table = torch.randn(40, 1030, device="cuda", dtype=torch.float16)
    tokens = torch.tensor([3, bad, 39, 0], dtype=dtype, device="cuda")
    got = ctx.embedding(table, tokens)
    assert ctx.device_status() == 2 and ctx.device_status() == 0
    want = table[tokens.long().clamp(0, 39)]
    want[1] = 0
    assert torch.equal(got, want)


def test_lookup_past_32_bit_offsets(ctx):
    """A table of more than 2^32 bytes and 2^31 elements: its last rows."""
    rows, dim = 600_000, 4096
    table = torch.empty(rows, dim, dtype=torch.bfloat16, device="cuda")
    tokens = torch.tensor([0, 299_999, 524_288, rows - 1], device="cuda")
    for i, t in enumerate(tokens.tolist()):
        table[t] = i + 1
    got = ctx.embedding(table, tokens)
    assert torch.equal(got.float(), torch.arange(1, 5, device="cuda").float()[:, None].expand(4, dim))


def test_lookup_on_another_stream(ctx):
    side = torch.cuda.Stream()
    table = torch.randn(1000, 512, device="cuda")
    tokens = _tokens(4000, 1000, 5)
    side.wait_stream(torch.cuda.current_stream())
    got = ctx.embedding(table, tokens, scale=3.0, stream=side)
    side.synchronize()
    assert torch.equal(got, table[tokens] * 3.0)


# ------------------------------------------------------------------------------------------------- gradient

def _true_gradient(grad, tokens, rows, scale, padding=None):
    """(gradient, sum of magnitudes, number of terms) per row and column in 64 bits."""
    t = tokens.reshape(-1).long()
    g = grad.reshape(t.numel(), -1).double()
    keep = (t >= 0) & (t < rows)
    if padding is not None:
        keep &= t != padding
    t, g = t[keep], g[keep]
    total = torch.zeros(rows, g.shape[1], dtype=torch.float64, device="cuda").index_add_(0, t, g) * scale
    size = torch.zeros_like(total).index_add_(0, t, g.abs()) * abs(scale)
    return total, size, torch.bincount(t, minlength=rows)


def _close(got, true, size, terms, old=None):
    """Within (m - 1) u of the sum, one u for the product with the scale (itself rounded once), one for the addition."""
    kind = got.dtype
    extra = 0.0 if old is None else U * (old.double().abs() + size)
    limit = ((terms[:, None].double() + 3.0) * U * size + extra) * (1 + 1e-6)
    limit = limit + ROUND[kind] * (true.abs() + limit) + TINY[kind]
    return bool(((got.double() - true).abs() <= limit).all())


GRADS = [  # n, rows, dim, kind, grad skew, grad padding, out skew, out padding
    (1, 1, 1, "zipf", 0, 0, 0, 0), (1, 50257, 64, "zipf", 0, 0, 0, 0), (7, 5, 3, "zipf", 1, 2, 1, 1),
    (64, 9, 130, "same", 0, 0, 0, 0), (65, 9, 130, "same", 3, 1, 1, 0), (129, 300, 257, "zipf", 0, 0, 5, 2),
    (511, 700, 2048, "distinct", 4, 0, 0, 0), (2047, 3, 72, "zipf", 0, 0, 0, 0), (2048, 1, 40, "same", 0, 0, 0, 0),
    (2049, 2, 40, "same", 0, 0, 0, 0), (4500, 1000, 96, "descending", 0, 5, 0, 3), (10_000, 128_256, 33, "zipf", 2, 0, 0, 0),
    (20_001, 262_200, 16, "zipf", 0, 0, 0, 0), (70_000, 300_000, 8, "zipf", 0, 0, 0, 0), (70_001, 2, 24, "same", 0, 0, 0, 0),
    (3, 2_000_000_000, 8, "huge", 0, 0, 0, 0), (8_192, 50_257, 12, "zipf", 0, 0, 0, 0), (8_193, 513, 12, "zipf", 0, 0, 0, 0),
    (33_000, 511, 9, "zipf", 0, 0, 0, 0), (131_072, 128_256, 8, "zipf", 0, 0, 0, 0), (131_073, 262_144, 8, "zipf", 0, 0, 0, 0),
    (300_000, 140_000, 4, "descending", 0, 0, 0, 0), (257, 100_000, 515, "distinct", 1, 3, 2, 1),
]


@pytest.mark.parametrize("shape", GRADS, ids=str)
@pytest.mark.parametrize("pair", PAIRS[:4], ids=lambda p: f"{p[0]}-{p[1]}".replace("torch.", ""))
def test_gradient_against_64_bits(ctx, shape, pair):
    n, rows, dim, how, skew, pad, oskew, opad = shape
    kind, out_kind = pair
    scale = math.sqrt(dim)
    grad = Guarded(n, dim, kind, skew, dim + pad, torch.randn(n, dim, generator=_gen(n), device="cuda"))
    if how == "huge":                                  # a table too long to hold: the compact form only
        tokens = torch.tensor([rows - 1, 5, rows - 1], device="cuda")
        r, g, c = ctx.embedding_grad_rows(grad.view, tokens, rows, scale=scale, out_dtype=out_kind)
        assert r.tolist() == [5, rows - 1, -1] and int(c) == 2
        small = torch.tensor([1, 0, 1], device="cuda")
        assert _close(g, *_true_gradient(grad.view, small, 3, scale))
        return
    tokens = _tokens(n, rows, n + 1, how, torch.int32 if n % 2 else torch.int64)
    true, size, terms = _true_gradient(grad.view, tokens, rows, scale)

    out = Guarded(rows, dim, out_kind, oskew, dim + opad)
    got = ctx.embedding_grad(grad.view, tokens, rows, scale=scale, out=out.view)
    out.check()
    assert _close(got, true, size, terms)
    assert not bool(got[terms == 0].float().abs().any())

    cap = min(n, rows)
    packed = Guarded(cap, dim, out_kind, oskew, dim + opad)
    r, g, c = ctx.embedding_grad_rows(grad.view, tokens, rows, scale=scale, out=packed.view)
    packed.check()
    grad.check()
    distinct = torch.unique(tokens.long())
    assert int(c) == distinct.numel()
    assert torch.equal(r, torch.cat([distinct, torch.full((cap - distinct.numel(),), -1, device="cuda")]))
    assert torch.equal(g[:distinct.numel()], got[distinct]) and not bool(g[distinct.numel():].float().abs().any())

    old = torch.randn(rows, dim, generator=_gen(3), device="cuda").to(out_kind)
    added = Guarded(rows, dim, out_kind, oskew, dim + opad, old)
    ctx.embedding_grad(grad.view, tokens, rows, scale=scale, out=added.view, accumulate=True)
    added.check()
    assert torch.equal(added.view[terms == 0], old[terms == 0])
    assert _close(added.view, true + old.double(), size, terms, old)


def test_gradient_sum_order_is_the_stated_one(ctx):
    """32 terms a piece, 32 pieces a group, first to last, in 32 bits: bit for bit, for one row among others."""
    n, hot = 6000, 4321
    g = _gen(9)
    tokens = torch.randint(0, 50, (n,), generator=g, device="cuda")
    at = torch.randperm(n, generator=g, device="cuda")[:hot].sort().values
    tokens[at] = 77
    grad = torch.randn(n, 12, generator=g, device="cuda") * torch.exp(4 * torch.randn(n, 12, generator=g, device="cuda"))
    got = ctx.embedding_grad(grad, tokens, 100, scale=3.0)
    terms = grad[at].cpu().numpy()

    def in_order(parts):
        s = np.zeros(12, dtype=np.float32)
        for p in parts:
            s = s + p
        return s

    pieces = [in_order(terms[i:i + 32]) for i in range(0, hot, 32)]
    groups = [in_order(pieces[i:i + 32]) for i in range(0, len(pieces), 32)]
    want = in_order(groups) * np.float32(3.0)
    assert np.array_equal(got[77].cpu().numpy(), want)


def test_gradient_bits_do_not_depend_on_the_other_rows(ctx):
    """A row's gradient depends on its own terms only: the same terms among other tokens give the same bits."""
    g = _gen(11)
    grad = torch.randn(3000, 40, generator=g, device="cuda")
    mine = torch.full((700,), 5, device="cuda")
    alone = ctx.embedding_grad(grad[:700], mine, 10)[5].clone()
    others = torch.randint(6, 10, (2300,), generator=g, device="cuda")
    tokens = torch.cat([others, mine])
    among = ctx.embedding_grad(torch.cat([grad[700:], grad[:700]]), tokens, 10)[5]
    assert torch.equal(alone, among)
    assert torch.equal(ctx.embedding_grad(torch.cat([grad[700:], grad[:700]]), tokens, 10)[5], among)


def test_gradient_with_padding_and_rows_that_are_not_there(ctx):
    tokens = torch.tensor([4, 9, 4, -1, 10, 0, 9, 4], device="cuda")
    grad = torch.randn(8, 20, device="cuda")
    got = ctx.embedding_grad(grad, tokens, 10, padding_row=9)
    assert ctx.device_status() == 2
    true, size, terms = _true_gradient(grad, tokens, 10, 1.0, padding=9)
    assert _close(got, true, size, terms)
    rows, g, count = ctx.embedding_grad_rows(grad, tokens, 10, padding_row=9)
    assert ctx.device_status() == 2
    assert rows.tolist() == [0, 4] + [-1] * 6 and int(count) == 2
    assert torch.equal(g[:2], got[torch.tensor([0, 4], device="cuda")]) and not bool(g[2:].any())
    assert ctx.device_status() == 0
    # nothing but padding: no row at all
    rows, g, count = ctx.embedding_grad_rows(grad, torch.full((8,), 9, device="cuda"), 10, padding_row=9)
    assert int(count) == 0 and bool((rows == -1).all()) and not bool(g.any())
    assert not bool(ctx.embedding_grad(grad, torch.full((8,), 9, device="cuda"), 10, padding_row=9).any())
    old = torch.randn(10, 20, device="cuda")
    kept = old.clone()
    ctx.embedding_grad(grad, torch.full((8,), 9, device="cuda"), 10, padding_row=9, out=kept, accumulate=True)
    assert torch.equal(kept, old) and ctx.device_status() == 0


def test_gradient_of_no_tokens(ctx):
    grad, none = torch.zeros(0, 16, device="cuda"), torch.zeros(0, dtype=torch.int64, device="cuda")
    out = torch.ones(5, 16, device="cuda")
    assert not bool(ctx.embedding_grad(grad, none, 5, out=out).any())
    out = torch.ones(5, 16, device="cuda")
    assert bool((ctx.embedding_grad(grad, none, 5, out=out, accumulate=True) == 1).all())
    rows, g, count = ctx.embedding_grad_rows(grad, none, 5)
    assert rows.numel() == 0 and g.shape == (0, 16) and int(count) == 0
    # a compact form with more room than tokens is filled all the same
    rows, g, count = ctx.embedding_grad_rows(grad, none, 5, rows=torch.zeros(4, dtype=torch.int64, device="cuda"),
                                             out=torch.ones(4, 16, device="cuda"))
    assert rows.tolist() == [-1] * 4 and not bool(g.any()) and int(count) == 0


def test_gradient_without_columns_or_without_rows(ctx):
    tokens = torch.tensor([3, 1, 3], device="cuda")
    rows, g, count = ctx.embedding_grad_rows(torch.empty(3, 0, device="cuda"), tokens, 5)
    assert rows.tolist() == [1, 3, -1] and g.shape == (3, 0) and int(count) == 2
    odd = torch.zeros(8, dtype=torch.uint8, device="cuda")[2:6].view(torch.float16)[:0].view(3, 0)   # no columns at an odd place
    rows, g, count = ctx.embedding_grad_rows(odd, tokens, 5)
    assert rows.tolist() == [1, 3, -1] and int(count) == 2
    assert ctx.embedding_grad(torch.empty(3, 0, device="cuda"), tokens, 5).shape == (5, 0) and ctx.device_status() == 0
    # a table without rows: no token is in it
    rows, g, count = ctx.embedding_grad_rows(torch.ones(3, 4, device="cuda"), tokens, 0)
    assert rows.numel() == 0 and int(count) == 0 and ctx.device_status() == 2
    assert ctx.embedding_grad(torch.ones(3, 4, device="cuda"), tokens, 0).shape == (0, 4) and ctx.device_status() == 2
    assert not bool(ctx.embedding(torch.ones(0, 4, device="cuda"), tokens).any()) and ctx.device_status() == 2


def test_gradient_passes_infinities_and_nan_to_their_rows_only(ctx):
    tokens = torch.tensor([0, 1, 2, 1], device="cuda")
    grad = torch.ones(4, 9, device="cuda")
    grad[0, 3], grad[1, 4], grad[3, 4], grad[2, 5] = math.inf, math.inf, -math.inf, math.nan
    got = ctx.embedding_grad(grad, tokens, 4)
    assert got[0, 3] == math.inf and bool(torch.isnan(got[1, 4])) and bool(torch.isnan(got[2, 5]))
    assert int((~torch.isfinite(got)).sum()) == 3 and not bool(got[3].any())


def test_gradient_against_differences_of_the_lookup(ctx):
    """The loss sum(w * lookup) is linear in the table: a central difference with a step that is a power of two is the
    derivative up to the rounding of the lookups (2 u |scale * table| a term) over twice the step."""
    rows, dim, n, scale, step = 6, 10, 40, 3.0, 0.25
    g = _gen(21)
    table = torch.randn(rows, dim, generator=g, device="cuda")
    w = torch.randn(n, dim, generator=g, device="cuda")
    tokens = torch.randint(0, rows - 1, (n,), generator=g, device="cuda")     # the last row has no token
    grad = ctx.embedding_grad(w, tokens, rows, scale=scale).double()
    for r in range(rows):
        for c in (0, 4, 9):
            loss = []
            for sign in (1, -1):
                moved = table.clone()
                moved[r, c] += sign * step
                loss.append(float((ctx.embedding(moved, tokens, scale=scale).double() * w.double()).sum()))
            difference = (loss[0] - loss[1]) / (2 * step)
            mine = w[tokens == r, c].double().abs().sum().item()
            limit = mine * scale * (4 * U * (4 + step) / (2 * step) + 45 * U) + 1e-12 * n * dim * 12 / (2 * step)
            assert abs(difference - float(grad[r, c])) <= limit


def test_two_gradients_in_a_row_leave_no_trace(ctx):
    """The scratch of one call (arrival counters, partial sums, another size) does not reach the next."""
    for n, rows, dim in ((9000, 4, 300), (100, 3, 520), (9000, 4, 300), (5000, 2, 20)):
        grad = torch.randn(n, dim, generator=_gen(n), device="cuda")
        tokens = torch.randint(0, rows, (n,), generator=_gen(dim), device="cuda")
        true, size, terms = _true_gradient(grad, tokens, rows, 1.0)
        assert _close(ctx.embedding_grad(grad, tokens, rows), true, size, terms)


# ------------------------------------------------------------------------------------------------- norm and clipping

def _packed(lengths, dtype, seed, skew=0, gap=0):
    """Tensors of the given numbers of elements in one buffer: (buffer, starts, byte offsets, byte lengths)."""
    size = torch.empty(0, dtype=dtype).element_size()
    starts, at = [], skew
    for m in lengths:
        starts.append(at)
        at += m + gap
    flat = (torch.randn(max(at, 1), generator=_gen(seed), device="cuda") * 0.01).to(dtype)
    offsets = torch.tensor(starts, dtype=torch.int64, device="cuda") * size
    return flat, starts, offsets, torch.tensor(list(lengths), dtype=torch.int64, device="cuda") * size


def _true_norms(flat, starts, lengths):
    return torch.stack([flat[a:a + m].double().square().sum().sqrt() for a, m in zip(starts, lengths)])


def _near(got, want, tolerance):
    return abs(float(got) - float(want)) <= tolerance * abs(float(want))


SETS = [[1], [0], [0, 0, 3], [7, 0, 1, 4096, 4097, 4095, 2, 8191], [100_003], [1] * 1500, [3, 300_001, 65_536, 17],
        [64] * 33 + [0] + [1000] * 3, [1 << 20, 5, 1 << 18]]


@pytest.mark.parametrize("lengths", SETS, ids=lambda s: f"{len(s)}x{sum(s)}")
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16], ids=str)
@pytest.mark.parametrize("skew", [0, 1, 3])
def test_norm_and_clipping_against_64_bits(ctx, lengths, dtype, skew):
    flat, starts, offsets, nbytes = _packed(lengths, dtype, len(lengths), skew)
    want = _true_norms(flat, starts, lengths)
    norm = float(want.square().sum().sqrt())
    result, norms = binding.new_norm_result("cuda"), torch.full((len(lengths),), 7.0, device="cuda")
    ctx.grad_norm(flat, offsets, nbytes, result, norms=norms)
    r = binding.read_norm_result(result)
    assert r["status"] == 0 and r["n_nonfinite"] == 0 and r["n_elements"] == sum(lengths) and r["scale"] == 1.0
    assert _near(r["norm"], norm, NORM_TOLERANCE) and _near(r["sum_squares"], norm ** 2, 65 * U)
    assert bool(((norms.double() - want).abs() <= NORM_TOLERANCE * want).all())

    for max_norm in (0.5 * norm, 2.0 * norm + 1.0, 0.0):
        max_norm = float(np.float32(max_norm))
        before = flat.clone()
        ctx.grad_clip(flat, offsets, nbytes, max_norm, result, norms=norms)
        c = binding.read_norm_result(result)
        assert c["norm"] == r["norm"] and c["sum_squares"] == r["sum_squares"]
        scale = np.float32(1.0 if math.sqrt(c["sum_squares"]) <= max_norm else max_norm / math.sqrt(c["sum_squares"]))
        assert c["scale"] == scale
        after = before.clone()
        for a, m in zip(starts, lengths):
            after[a:a + m] = (before[a:a + m].float() * float(scale)).to(dtype)
        assert torch.equal(flat, after)                  # and nothing beside the tensors has changed
        flat = before


@pytest.mark.parametrize("pair", PAIRS, ids=lambda p: f"{p[0]}-{p[1]}".replace("torch.", ""))
@pytest.mark.parametrize("skews", [(0, 0), (1, 0), (0, 3), (5, 2)], ids=str)
def test_clipping_into_another_buffer(ctx, pair, skews):
    kind, out_kind = pair
    lengths = [5, 4096, 0, 10_001, 1, 70_000, 8]
    flat, starts, offsets, nbytes = _packed(lengths, kind, 4, skews[0], gap=2)
    out = Guarded(1, sum(lengths) + 3 * len(lengths), out_kind, skews[1])
    out.view.fill_(3.0)
    places, at = [], 0
    for m in lengths:
        places.append(at)
        at += m + 3
    size = out.view.element_size()
    result = binding.new_norm_result("cuda")
    keep = flat.clone()
    ctx.grad_clip(flat, offsets, nbytes, 0.25, result, out=out.view.view(-1),
                  out_offsets=torch.tensor(places, dtype=torch.int64, device="cuda") * size)
    out.check()
    assert torch.equal(flat, keep)
    r = binding.read_norm_result(result)
    want = torch.full_like(out.view.view(-1), 3.0)
    for a, b, m in zip(starts, places, lengths):
        want[b:b + m] = (flat[a:a + m].float() * r["scale"]).to(out_kind)
    assert r["scale"] < 1 and torch.equal(out.view.view(-1), want)
    # a factor of one still fills the other buffer
    ctx.grad_clip(flat, offsets, nbytes, math.inf, result, out=out.view.view(-1),
                  out_offsets=torch.tensor(places, dtype=torch.int64, device="cuda") * size)
    for a, b, m in zip(starts, places, lengths):
        want[b:b + m] = flat[a:a + m].to(out_kind)
    assert binding.read_norm_result(result)["scale"] == 1.0 and torch.equal(out.view.view(-1), want)


def test_tensors_of_their_own_and_of_different_types(ctx):
    tensors = [torch.randn(1000, device="cuda"), torch.randn(37, 11, device="cuda").to(torch.bfloat16),
               torch.randn(1, device="cuda").half(), torch.randn(256, 256, device="cuda")]
    base, offsets, lengths, types = binding.tensor_ranges(tensors)
    want = torch.stack([t.double().square().sum().sqrt() for t in tensors])
    result, norms = binding.new_norm_result("cuda"), torch.empty(4, device="cuda")
    before = [t.clone() for t in tensors]
    ctx.grad_clip(base, offsets, lengths, 1.0, result, norms=norms, types=types)
    r = binding.read_norm_result(result)
    assert bool(((norms.double() - want).abs() <= NORM_TOLERANCE * want).all())
    assert _near(r["norm"], want.square().sum().sqrt(), NORM_TOLERANCE)
    for t, b in zip(tensors, before):
        assert torch.equal(t, (b.float() * r["scale"]).to(b.dtype))
    assert ctx.device_status() == 0


def test_norm_bits_do_not_depend_on_the_alignment(ctx):
    lengths = [1, 5000, 123_457, 9, 40_000]
    for dtype in (torch.float32, torch.bfloat16):
        results = []
        values = _packed(lengths, dtype, 8)[0]
        for skew in range(9):
            flat = torch.zeros(skew + values.numel(), dtype=dtype, device="cuda")
            flat[skew:] = values
            size = flat.element_size()
            starts = np.cumsum([0] + lengths[:-1]) + skew
            result, norms = binding.new_norm_result("cuda"), torch.empty(5, device="cuda")
            ctx.grad_norm(flat, torch.tensor(starts * size, dtype=torch.int64, device="cuda"),
                          torch.tensor(lengths, dtype=torch.int64, device="cuda") * size, result, norms=norms)
            results.append((result.tolist(), norms.tolist()))
        assert all(r == results[0] for r in results)


@pytest.mark.parametrize("size", [1e30, 3e38, 1e-30, 1e-38, 1e-42])
def test_norm_of_gradients_whose_squares_leave_the_range_of_32_bits(ctx, size):
    flat = torch.full((10_000,), size, device="cuda")
    flat[::3] = 0
    offsets, lengths = torch.tensor([0, 20_000], device="cuda"), torch.tensor([20_000, 20_000], device="cuda")
    result, norms = binding.new_norm_result("cuda"), torch.empty(2, device="cuda")
    ctx.grad_norm(flat, offsets, lengths, result, norms=norms)
    r = binding.read_norm_result(result)
    want = float(flat.double().square().sum())
    assert r["n_nonfinite"] == 0 and _near(r["sum_squares"], want, 1e-12)
    expected = math.sqrt(want)
    if expected < 3.4e38:
        assert abs(r["norm"] - expected) <= U * expected + 2.0 ** -150
        assert abs(float(norms[0]) - float(flat[:5000].double().norm())) <= U * expected + 2.0 ** -150
    else:
        assert r["norm"] == math.inf
    ctx.grad_clip(flat, offsets, lengths, 1.0, result)       # the scale comes from the 64-bit norm
    r = binding.read_norm_result(result)
    assert r["scale"] == np.float32(1.0 if expected <= 1.0 else 1.0 / math.sqrt(r["sum_squares"]))


def test_infinities_and_nan_are_counted_and_passed_on(ctx):
    lengths = [10, 5000, 300, 20_000]
    flat, starts, offsets, nbytes = _packed(lengths, torch.float32, 6)
    flat[starts[1] + 4999] = math.inf
    flat[starts[3] + 12_345] = -math.inf
    result, norms = binding.new_norm_result("cuda"), torch.empty(4, device="cuda")
    ctx.grad_norm(flat, offsets, nbytes, result, norms=norms)
    r = binding.read_norm_result(result)
    assert r["n_nonfinite"] == 2 and r["norm"] == math.inf and torch.isfinite(norms).tolist() == [True, False, True, False]
    clipped = flat.clone()
    ctx.grad_clip(clipped, offsets, nbytes, 1.0, result)
    assert binding.read_norm_result(result)["scale"] == 0.0
    assert bool(torch.isnan(clipped[starts[1] + 4999])) and float(clipped[0]) == 0.0
    flat[starts[2]] = math.nan
    ctx.grad_clip(flat, offsets, nbytes, 1.0, result, norms=norms)
    r = binding.read_norm_result(result)
    assert r["n_nonfinite"] == 3 and math.isnan(r["norm"]) and math.isnan(r["scale"]) and bool(torch.isnan(flat).all())


def test_tensors_that_are_ill_formed_are_left_out(ctx):
    flat = torch.ones(100, device="cuda")
    offsets, lengths = torch.tensor([0, 6, 80, 200], device="cuda"), torch.tensor([40, 40, 42, 80], device="cuda")
    result, norms = binding.new_norm_result("cuda"), torch.full((4,), 9.0, device="cuda")
    ctx.grad_clip(flat, offsets, lengths, 1.0, result, norms=norms)
    r = binding.read_norm_result(result)
    assert r["status"] == 2 and r["n_elements"] == 30 and ctx.device_status() == 2
    assert norms.tolist() == [np.float32(math.sqrt(10)), 0.0, 0.0, np.float32(math.sqrt(20))]
    assert bool((flat[10:50] == 1).all()) and bool((flat[:10] < 1).all())
    types = torch.tensor([0, 3, 255, 0], dtype=torch.uint8, device="cuda")
    ctx.grad_norm(flat, torch.tensor([0, 40, 80, 200], device="cuda"), torch.full((4,), 40, device="cuda"), result, types=types)
    assert binding.read_norm_result(result)["n_elements"] == 20 and ctx.device_status() == 2


def test_norm_of_no_tensors(ctx):
    none = torch.zeros(0, dtype=torch.int64, device="cuda")
    result = binding.new_norm_result("cuda")
    ctx.grad_clip(torch.ones(4, device="cuda"), none, none, 1.0, result)
    assert binding.read_norm_result(result) == {"status": 0, "n_nonfinite": 0, "norm": 0.0, "scale": 1.0,
                                                "sum_squares": 0.0, "n_elements": 0}


def test_scaling_by_a_factor_on_the_device(ctx):
    lengths = [3, 7000, 1]
    flat, starts, offsets, nbytes = _packed(lengths, torch.bfloat16, 12, 1)
    before, factor = flat.clone(), torch.tensor([0.3], device="cuda")
    ctx.grad_scale(flat, offsets, nbytes, factor)
    assert torch.equal(flat[1:], (before[1:].float() * factor).to(torch.bfloat16)) and flat[0] == before[0]
    ctx.grad_scale(flat, offsets, nbytes, torch.ones(1, device="cuda"))
    assert torch.equal(flat[1:], (before[1:].float() * factor).to(torch.bfloat16))
    out = torch.zeros(7010, device="cuda")
    ctx.grad_scale(before, offsets, nbytes, factor, out=out, out_offsets=offsets * 2)
    assert torch.equal(out[1:7005], before[1:].float() * factor)


def test_norm_on_another_stream(ctx):
    side = torch.cuda.Stream()
    flat, starts, offsets, nbytes = _packed([100_000, 33], torch.float32, 2)
    result = binding.new_norm_result("cuda")
    side.wait_stream(torch.cuda.current_stream())
    ctx.grad_clip(flat, offsets, nbytes, 0.5, result, stream=side)
    side.synchronize()
    assert 0 < binding.read_norm_result(result)["scale"] < 1 and _near(flat.double().norm(), 0.5, 1e-6)


def test_large_sets(ctx):
    """More tensors than one block of the plan holds, and a tensor of more than 2^31 bytes."""
    lengths = [int(x) for x in np.random.RandomState(1).randint(0, 300, 12_000)]
    flat, starts, offsets, nbytes = _packed(lengths, torch.bfloat16, 3, 1)
    result, norms = binding.new_norm_result("cuda"), torch.empty(len(lengths), device="cuda")
    ctx.grad_norm(flat, offsets, nbytes, result, norms=norms)
    segment = torch.repeat_interleave(torch.arange(len(lengths), device="cuda"), torch.tensor(lengths, device="cuda"))
    squares = torch.zeros(len(lengths), dtype=torch.float64, device="cuda").index_add_(0, segment, flat[1:].double().square())
    assert bool(((norms.double() - squares.sqrt()).abs() <= NORM_TOLERANCE * squares.sqrt()).all())
    assert _near(binding.read_norm_result(result)["norm"], squares.sum().sqrt(), NORM_TOLERANCE)
    big = torch.full((600_000_001,), 0.5, device="cuda")
    one, size = torch.zeros(1, dtype=torch.int64, device="cuda"), torch.tensor([4 * big.numel()], device="cuda")
    ctx.grad_clip(big, one, size, 1.0, result)
    r = binding.read_norm_result(result)
    assert _near(r["norm"], 0.5 * math.sqrt(big.numel()), NORM_TOLERANCE) and r["n_elements"] == big.numel()
    assert bool((big == big[0]).all()) and big[0] == np.float32(0.5) * np.float32(r["scale"])


# ------------------------------------------------------------------------------------------------- streams and graphs

def test_two_contexts_side_by_side():
    """Two contexts on two streams, gradients and clipping under way at the same time, three times without waiting."""
    work, results = [], []
    for k in range(2):
        g = _gen(100 + k)
        grad = torch.randn(20_000, 512, generator=g, device="cuda")
        tokens = _tokens(20_000, 30_000, 200 + k)
        flat, starts, offsets, nbytes = _packed([300_000, 17, 70_000], torch.float32, 300 + k)
        work.append((binding.Context(0), torch.cuda.Stream(), grad, tokens, flat, offsets, nbytes))
        with binding.Context(0) as alone:
            clipped, result = flat.clone(), binding.new_norm_result("cuda")
            alone.grad_clip(clipped, offsets, nbytes, 0.5, result)
            results.append((alone.embedding_grad(grad, tokens, 30_000), alone.embedding_grad_rows(grad, tokens, 30_000)[1], clipped))
    torch.cuda.synchronize()
    for _ in range(3):
        got = []
        for ctx, stream, grad, tokens, flat, offsets, nbytes in work:
            with torch.cuda.stream(stream):
                clipped, result = flat.clone(), binding.new_norm_result("cuda")
                dense = ctx.embedding_grad(grad, tokens, 30_000)
                rows = ctx.embedding_grad_rows(grad, tokens, 30_000)[1]
                ctx.grad_clip(clipped, offsets, nbytes, 0.5, result)
                got.append((dense, rows, clipped))
        torch.cuda.synchronize()
        for a, b in zip(got, results):
            assert all(torch.equal(x, y) for x, y in zip(a, b))
    for w in work:
        assert w[0].device_status() == 0
        w[0].close()


def test_calls_in_a_graph(ctx):
    """A step captured once and replayed on new inputs (after a first call has sized the scratch)."""
    n, rows, dim = 3000, 5000, 264
    tokens, grad = _tokens(n, rows, 1), torch.randn(n, dim, generator=_gen(2), device="cuda")
    table = torch.randn(rows, dim, generator=_gen(3), device="cuda")
    out, dense = torch.empty(n, dim, device="cuda"), torch.empty(rows, dim, device="cuda")
    touched, d_rows, count = (torch.empty(n, dtype=torch.int64, device="cuda"), torch.empty(n, dim, device="cuda"),
                              torch.empty(1, dtype=torch.int64, device="cuda"))
    result = binding.new_norm_result("cuda")
    zero, size = torch.zeros(1, dtype=torch.int64, device="cuda"), torch.tensor([4 * n * dim], device="cuda")

    def step():
        ctx.embedding(table, tokens, scale=2.0, out=out)
        ctx.embedding_grad(grad, tokens, rows, out=dense)
        ctx.embedding_grad_rows(grad, tokens, rows, rows=touched, out=d_rows, count=count)
        ctx.grad_clip(d_rows, zero, size, 1.0, result)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed in (10, 20):
        tokens.copy_(_tokens(n, rows, seed))
        grad.copy_(torch.randn(n, dim, generator=_gen(seed), device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (out, dense, touched, d_rows, count, result)]
        step()
        assert all(torch.equal(a, b) for a, b in zip(got, (out, dense, touched, d_rows, count, result)))
        assert torch.equal(out, table[tokens] * 2.0)


# ------------------------------------------------------------------------------------------------- refusals

def test_refusals_of_the_binding(ctx):
    table, tokens = torch.zeros(4, 8, device="cuda"), torch.zeros(3, dtype=torch.int64, device="cuda")
    for call in (lambda: ctx.embedding(table.t(), tokens), lambda: ctx.embedding(table, tokens.float()),
                 lambda: ctx.embedding(table, tokens, out=torch.zeros(2, 8, device="cuda")),
                 lambda: ctx.embedding(table.cpu(), tokens), lambda: ctx.embedding_grad(table, tokens, 9),
                 lambda: ctx.embedding_grad(table[:3], tokens, 9, out=torch.zeros(8, 8, device="cuda")),
                 lambda: ctx.embedding_grad(table[:3], tokens, 9, accumulate=True)):
        with pytest.raises(AssertionError):
            call()
    for call in (lambda: ctx.embedding(table.half(), tokens, out_dtype=torch.bfloat16),
                 lambda: ctx.embedding_grad(table[:3], tokens, 9, padding_row=-2),
                 lambda: ctx.embedding_grad_rows(table[:3], tokens, 9, out=torch.zeros(2, 8, device="cuda"))):
        with pytest.raises(binding.IvError) as err:
            call()
        assert err.value.code == binding.IV_ERR_INVALID_ARG
    with pytest.raises(KeyError):
        ctx.embedding(table.double(), tokens)
    one = torch.zeros(1, dtype=torch.int64, device="cuda")
    result = binding.new_norm_result("cuda")
    for bad in (math.nan, -1.0):
        with pytest.raises(binding.IvError) as err:
            ctx.grad_clip(table, one, one, bad, result)
        assert err.value.code == binding.IV_ERR_INVALID_ARG


def test_refusals_of_the_c_entry_points(ctx):
    lib, h = ctx._lib, ctx._h
    a = torch.zeros(4096, dtype=torch.uint8, device="cuda").data_ptr()
    launched = ctx.kernel_launches
    invalid, large = binding.IV_ERR_INVALID_ARG, binding.IV_ERR_TOO_LARGE
    f32, f16, bf16 = 0, 1, 2

    def look(table=a, tt=f32, rows=4, dim=8, stride=8, tokens=a, tb=8, n=2, out=a, ot=f32, ostride=8, c=h):
        return lib.iv_embedding(c, table, tt, rows, dim, stride, tokens, tb, n, 1.0, out, ot, ostride, None)

    assert look(n=0) == look(dim=0) == 0
    for kw in (dict(c=None), dict(table=None), dict(tokens=None), dict(out=None), dict(tt=3), dict(ot=-1), dict(tb=2),
               dict(tt=f16, ot=bf16), dict(stride=7), dict(ostride=7), dict(table=a + 2), dict(out=a + 1), dict(tokens=a + 4)):
        assert look(**kw) == invalid, kw
    assert look(n=(1 << 30) + 1) == large and look(dim=(1 << 24) + 1, stride=1 << 32, ostride=1 << 32) == large

    def grad(g=a, gt=f32, gs=8, dim=8, tokens=a, tb=8, n=2, rows=4, pad=-1, out=a, ot=f32, os=8, c=h):
        return lib.iv_embedding_grad(c, g, gt, gs, dim, tokens, tb, n, rows, pad, 1.0, 0, out, ot, os, None)

    for kw in (dict(c=None), dict(g=None), dict(tokens=None), dict(out=None), dict(gt=7), dict(ot=9), dict(tb=1),
               dict(gt=bf16, ot=f16), dict(gs=7), dict(os=7), dict(g=a + 2), dict(out=a + 2), dict(tokens=a + 2), dict(pad=-2)):
        assert grad(**kw) == invalid, kw
    assert grad(n=(1 << 30) + 1) == grad(rows=(1 << 31) + 1) == grad(dim=(1 << 24) + 1, gs=1 << 25, os=1 << 25) == large

    def rows_(rows=a, count=a, cap=2, out=a, c=h):
        return lib.iv_embedding_grad_rows(c, a, f32, 8, 8, a, 8, 2, 4, -1, 1.0, rows, out, f32, 8, cap, count, None)

    for kw in (dict(c=None), dict(rows=None), dict(count=None), dict(cap=1), dict(out=None), dict(rows=a + 4), dict(count=a + 4)):
        assert rows_(**kw) == invalid, kw

    def norm(base=a, off=a, length=a, types=None, t=f32, n=2, norms=a, result=a, c=h):
        return lib.iv_grad_norm(c, base, off, length, types, t, n, norms, result, None)

    for kw in (dict(c=None), dict(base=None), dict(off=None), dict(length=None), dict(t=3), dict(result=None),
               dict(off=a + 4), dict(length=a + 1), dict(result=a + 4), dict(norms=a + 2)):
        assert norm(**kw) == invalid, kw
    assert norm(n=(1 << 30) + 1) == large

    def clip(out=a, ooff=a, ot=f32, t=f32, limit=1.0, scale_only=False):
        return lib.iv_grad_clip(h, a, a, a, None, t, 2, limit, out, ooff, ot, None, a, None)

    for kw in (dict(ooff=None), dict(ot=5), dict(t=f16, ot=bf16), dict(out=None, ot=bf16), dict(limit=-0.5),
               dict(limit=math.nan), dict(ooff=a + 2)):
        assert clip(**kw) == invalid, kw
    assert lib.iv_grad_scale(h, a, a, a, None, f32, 2, None, None, None, -1, None) == invalid
    assert lib.iv_grad_scale(h, a, a, a, None, f32, 2, a + 2, None, None, -1, None) == invalid
    assert ctx.kernel_launches == launched                    # nothing ran


def test_result_record_layout():
    assert ctypes.sizeof(binding.NormResult) == 32 and binding.NormResult.sum_squares.offset == 16
