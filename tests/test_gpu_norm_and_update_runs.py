"""Long runs of the norm kernels and the AdamW step: rings of copies that are filled again and again, tensors that give a warp many blocks.

Small sets end before a ring's first place is used twice; the sizes here are counted from a B200's 148 SMs so that every
form of the kernels goes round its ring at least once.  Bounds are those of test_gpu_norm_and_update.py.
"""
import pytest
import torch

from test_gpu_norm_and_update import BF16, F16, F32, KINDS, TOP, U, Set, _gen, _id, _randn, _true_grad, _true_norm, _within, _words, ctx  # noqa: F401

pytestmark = pytest.mark.gpu

SMS = 148


# ------------------------------------------------------------------------------------------------- AdamW

# A warp takes runs of blocks / (2 CTAs of 8 warps per SM) blocks, so this is one of nine, in steps of two in 8 bits: an odd one out.
BLOCKS = 9 * 2 * 8 * SMS + 700
PLACES = {  # skews in elements of weights and gradients: every class of places that the kernels tell apart
    "16 bytes": lambda w, g: (0, 0),
    "8 bytes": lambda w, g: (8 // w, 0),
    "odd": lambda w, g: (3, 5),
}


@pytest.mark.parametrize("place", list(PLACES))
@pytest.mark.parametrize("kind", KINDS, ids=_id)
@pytest.mark.parametrize("bits", [32, 8])
def test_many_blocks_a_warp(ctx, place, kind, bits):  # noqa: F811
    weight, grad, master = kind
    size = lambda t: torch.empty(0, dtype=t).element_size()  # noqa: E731
    skew, grad_skew = PLACES[place](size(weight), size(grad))
    # whole vectors, so that every tensor lies as the first does; all but one end inside a block, and runs go over their ends
    counts = [256 * 9000 + 8, 256 * 11 + 240, 256 * 5, 256 * (BLOCKS - 9000 - 19) + 16]
    s = Set(counts, weight, grad, bits, master, skew, grad_skew)
    ctx.adamw_step(*s.args(), **s.state)
    s.check()
    s.back()
    ctx.adamw_step(*s.args(), **s.state, lr=1e-2, betas=(0.8, 0.95), eps=1e-4, weight_decay=0.5, stochastic=True, seed=(7 << 40) + 5)
    s.check(lr=1e-2, betas=(0.8, 0.95), eps=1e-4, decay=0.5, stochastic=True, seed=(7 << 40) + 5)


@pytest.mark.parametrize("kind", [KINDS[0], KINDS[5]], ids=_id)
@pytest.mark.parametrize("bits", [32, 8])
def test_the_longest_runs(ctx, kind, bits):  # noqa: F811
    """Runs of 16 blocks (32 in 8 bits), more than one to a warp."""
    weight, grad, master = kind
    s = Set([256 * (33 * 2 * 8 * SMS) + 100], weight, grad, bits, master, 4, 0)
    ctx.adamw_step(*s.args(), **s.state, seed=3)
    s.check(seed=3)


def _codes(x, words, name):
    """Codes (as bytes) and scales of blocks of 256 numbers by elementary operations in 32 bits."""
    rows = x.view(-1, 256)
    safe = rows.abs().amax(1).clamp(min=2.0 ** -110)
    scaled = rows.abs() * (safe.reciprocal() * TOP)[:, None] * 2.0 ** -120      # a code is the upper bits of such a float
    code = (scaled.view(torch.int32).view(-1) + (words >> 12).int()) >> 20
    if name == "v":
        code = torch.maximum(code, (x > 0).int())
    return torch.where(x < 0, code | 128, code).to(torch.uint8), safe * (1.0 / TOP)


@pytest.mark.parametrize("seed", [1, 2, 3])
def test_codes_are_those_of_elementary_operations(ctx, seed):  # noqa: F811
    """Bit for bit.  A root that is off in its last place has another code with a probability of 2^-20 and less, hence so many."""
    n = 1 << 24
    s = Set([n], F32, F32, 8, seed=10 * seed)
    want = {}
    t, places = int(s.state["step"]) + 1, torch.arange(n, device="cuda")
    old = {name: (s.state[name].float().view(-1, 256) * s.state[name + "_scales"][:, None]).view(-1) for name in ("m", "v")}
    g = s.g[:n]
    m, v = old["m"] * 0.9 + g * (1 - 0.9), old["v"] * old["v"] * 0.999 + g * g * (1 - 0.999)
    for name, x, first in (("m", m, 0), ("v", v.sqrt(), 8)):
        want[name] = _codes(x, _words(seed, t, places, first), name)
    ctx.adamw_step(*s.args(), **s.state, seed=seed)
    for name, (code, scale) in want.items():
        assert torch.equal(s.state[name + "_scales"], scale)
        assert torch.equal(s.state[name].view(torch.uint8), code)


@pytest.mark.parametrize("lr", [1e-3, 0.7, 3e-5])
def test_update_from_32_bit_moments_is_right_to_the_last_place(ctx, lr):  # noqa: F811
    """Weights of 0, betas of 0 and gradients of 12 digits, whose squares are exact: the update is lr g / |g|, so the weight is the product
    -lr g, rounded, over |g|, rounded: within 2^-24 of that quotient, and 2^-40 for what a step of correction leaves."""
    g = torch.cat([torch.arange(2048, 4096, device="cuda").float() * 2.0 ** e for e in (-40, -19, -12, 3)])
    s = Set([len(g)], F32, F32, 32, step=0)
    s.w.zero_()
    s.g[:len(g)] = g
    s.keep()
    ctx.adamw_step(*s.args(), **s.state, lr=lr, betas=(0.0, 0.0), eps=0.0, weight_decay=0.0)
    assert torch.equal(s.state["m"][:len(g)], g) and torch.equal(s.state["v"][:len(g)], g * g)
    true = (g * -lr).double() / g.double()
    assert bool(((s.w[:len(g)].double() - true).abs() <= (U + 2.0 ** -40) * true.abs()).all())


# ------------------------------------------------------------------------------------------------- rows

# For every number of threads to a row (8 to 512) and of vectors a thread: the full width, fewer whole vectors, an odd width.
WIDTHS = [64, 40, 61, 128, 104, 101, 256, 200, 255, 512, 400, 511, 1024, 1000, 1023, 2048, 1600, 2047, 4096, 2560, 4095, 8192, 7168,
          8191, 16384, 13000, 16383]
TYPES = [(BF16, BF16), (F32, F32), (F16, F32), (F32, BF16)]


def _groups(dim, threads=512):
    """Rows that the threads of a CTA take side by side."""
    t = 8
    while t < threads and 8 * t < dim:
        t *= 2
    return threads // t


def _steps(dim, size, most):
    """Steps that a ring of 192 KiB holds at `most` rows a group, and one more turn of its places."""
    row = _groups(dim) * max(dim, 64) * size
    return -(-(192 << 10) // (row * most)) + 2


@pytest.mark.parametrize("pair", TYPES, ids=_id)
@pytest.mark.parametrize("dim", WIDTHS)
def test_norm_of_many_rows_a_cta(ctx, dim, pair):  # noqa: F811
    kind, out_kind = pair
    rows = 4 if dim <= 8192 else 2
    n = SMS * rows * _groups(dim) * min(_steps(dim, kind.itemsize, rows), 10) + 5
    n = n * (2 if 2048 < dim <= 4096 else 1)                       # two CTAs an SM there
    x = (_randn((n, dim), 1, 2.0) + 0.5).to(kind)
    w, b = _randn((dim,), 2).to(out_kind), _randn((dim,), 3).to(out_kind)
    mean, rstd = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    for rms in (False, True):
        y = ctx.layer_norm(x, weight=w, bias=b, eps=1e-3, rms=rms, out_dtype=out_kind, mean=mean, rstd=rstd)
        true_y, true_mean, true_rstd = _true_norm(x, w, b, 1e-3, rms)
        _within(y, *true_y)
        _within(mean, *true_mean)
        _within(rstd, *true_rstd)


def _many_rows(dim, kinds):
    """So many that every ring of the gradient is filled again: x and dy of a row side by side, up to 4 rows a group."""
    rows = 4 if dim <= 4096 else 1
    return SMS * rows * _groups(dim) * min(_steps(dim, sum(k.itemsize for k in kinds), rows), 10) + 5


@pytest.mark.parametrize("pair", TYPES, ids=_id)
@pytest.mark.parametrize("dim", WIDTHS[:-3])
def test_gradient_of_many_rows_a_cta(ctx, dim, pair):  # noqa: F811
    kind, y_kind = pair
    n = _many_rows(dim, pair)
    x, dy, w = (_randn((n, dim), 1, 2.0) + 0.5).to(kind), _randn((n, dim), 2).to(y_kind), _randn((dim,), 3).to(y_kind)
    mean, rstd = x.float().mean(1), 1 / (x.float().var(1, unbiased=False) + 1e-3).sqrt()
    dw, db = torch.empty(dim, device="cuda"), torch.empty(dim, device="cuda")
    # a thread adds up its group's rows of a CTA's run, then come the groups, and 5 + 32 sums of runs
    depth = -(-n // (SMS * _groups(dim))) + 1 + _groups(dim) + 5 + 32
    for rms in (False, True):
        dx = ctx.layer_norm_grad(dy, x, None if rms else mean, rstd, weight=w, rms=rms, weight_grad=dw, bias_grad=db)
        true_dx, (true_dw, _), (true_db, _) = _true_grad(dy, x, mean, rstd, w, rms)
        _within(dx, *true_dx)
        h = ((x.double() if rms else x.double() - mean.double()[:, None]) * rstd.double()[:, None]).abs_()
        magnitude = dy.double().abs()
        _within(db, true_db, depth * U * magnitude.sum(0))
        _within(dw, true_dw, (depth + 3) * U * (magnitude * h).sum(0))              # h is rounded twice


@pytest.mark.parametrize("pair", TYPES, ids=_id)
@pytest.mark.parametrize("dim", WIDTHS[:-3])
def test_sums_over_many_rows_are_exact_where_they_can_be(ctx, dim, pair):  # noqa: F811
    """Small whole numbers: every row counts once, or a sum is off by a whole number."""
    kind, y_kind = pair
    n = _many_rows(dim, pair)
    x = torch.randint(-4, 5, (n, dim), generator=_gen(1), device="cuda").to(kind)
    dy = torch.randint(-2, 3, (n, dim), generator=_gen(2), device="cuda").to(y_kind)
    dw, db = torch.empty(dim, device="cuda"), torch.empty(dim, device="cuda")
    ctx.layer_norm_grad(dy, x, None, torch.ones(n, device="cuda"), rms=True, weight_grad=dw, bias_grad=db)
    assert torch.equal(dw, (dy.double() * x.double()).sum(0).float()) and torch.equal(db, dy.double().sum(0).float())
