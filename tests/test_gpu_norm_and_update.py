"""Layer norm, its gradient and the AdamW step against plain 64-bit forms.

Tolerances are derived, not tuned.  u = 2^-24 is the unit roundoff of 32-bit floats; an output of type T adds one rounding of at
most ROUND[T] relative (or half the type's smallest number).  A sum along at most D additions of 32 bits is within D u of the sum
of its terms' magnitudes; D is counted from the kernels' order of additions (a thread's own elements, then a tree).
"""
import math

import pytest
import torch

from paper_2510_23938_b200 import binding

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
ROUND = {t: torch.finfo(t).eps / 2 for t in (F32, F16, BF16)}
TINY = {F32: 2.0 ** -150, F16: 2.0 ** -25, BF16: 2.0 ** -134}
PAIRS = [(BF16, BF16), (F32, F32), (F16, F32), (F32, BF16), (BF16, F32), (F16, F16), (F32, F16)]
SENTINEL, MARGIN = 0xA5, 512
MORE = 1 + 1e-3                                      # products of two roundings


def _id(p):
    return "-".join(str(t).replace("torch.", "") for t in p) if isinstance(p, tuple) and p and isinstance(p[0], torch.dtype) else str(p)


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


def _randn(shape, seed, std=1.0):
    return torch.randn(shape, generator=_gen(seed), device="cuda") * std


class Guarded:
    """rows x cols elements, rows `stride` apart, `skew` elements past a 512-byte boundary, between sentinel bytes."""

    def __init__(self, rows, cols, dtype, skew=0, stride=None, fill=None):
        stride = cols if stride is None else stride
        size = torch.empty(0, dtype=dtype).element_size()
        room = max(1, max(rows - 1, 0) * stride + cols) * size
        self.raw = torch.full((2 * MARGIN + skew * size + (room + 15) // 16 * 16,), SENTINEL, dtype=torch.uint8, device="cuda")
        lo = MARGIN + skew * size
        self.view = self.raw[lo:lo + room].view(dtype).as_strided((rows, cols), (stride, 1)) if rows and cols else \
            torch.empty(rows, cols, dtype=dtype, device="cuda")
        if fill is not None:
            self.view.copy_(fill)
        mask = torch.zeros_like(self.raw, dtype=torch.bool)
        if rows and cols:
            mask[(torch.arange(rows, device="cuda")[:, None] * stride * size
                  + torch.arange(cols * size, device="cuda")[None, :]).reshape(-1) + lo] = True
        self.outside = ~mask

    def check(self):
        torch.cuda.synchronize()
        assert bool((self.raw[self.outside] == SENTINEL).all()), "bytes outside the tensor were written"


def _within(got, true, limit):
    limit = limit * MORE + ROUND[got.dtype] * (true.abs() + limit) * MORE + TINY[got.dtype]
    bad = ~((got.double() - true).abs() <= limit)
    assert not bool(bad.any()), f"{int(bad.sum())} of {bad.numel()} out of bounds, worst {float(((got.double() - true).abs() / limit).max())}"


# ------------------------------------------------------------------------------------------------- layer norm

def _true_norm(x, w, b, eps, rms):
    """y, mean, rstd in 64 bits and how far each may be off before it is rounded to its type."""
    x, dim = x.double(), x.shape[1]
    depth = 24 + dim // 8192
    mu = torch.zeros(x.shape[0], 1, dtype=torch.float64, device="cuda") if rms else x.mean(1, keepdim=True)
    e_mu = 0 * mu if rms else (depth + 3) * U * x.abs().mean(1, keepdim=True)
    d = x - mu
    var = d.square().mean(1, keepdim=True)
    e_var = 2 * e_mu * d.abs().mean(1, keepdim=True) + e_mu ** 2 + (depth + 5) * U * var
    r = 1 / (var + eps).sqrt()
    rel_r = (0.5 * e_var / (var + eps) + 4 * U) * MORE
    h = d * r
    w = torch.ones(dim, dtype=torch.float64, device="cuda") if w is None else w.double()
    y = h * w + (0 if b is None else b.double())
    e_y = (r * w.abs()) * (e_mu + U * d.abs()) + (h * w).abs() * (rel_r + 2 * U) + U * y.abs()
    return (y, e_y), (mu[:, 0], e_mu[:, 0]), (r[:, 0], (r * rel_r)[:, 0])


NORMS = [  # n, dim, x skew, x padding, y skew, y padding
    (1, 1, 0, 0, 0, 0), (3, 2, 1, 0, 0, 0), (1, 4096, 0, 0, 0, 0), (5, 7, 1, 2, 1, 1), (33, 64, 0, 0, 0, 0), (70, 65, 0, 0, 0, 0),
    (9, 128, 4, 8, 4, 8), (40, 255, 0, 0, 3, 0), (17, 512, 0, 0, 0, 0), (6, 1000, 8, 0, 8, 0), (300, 1023, 0, 0, 0, 0),
    (257, 2048, 0, 0, 0, 0), (2, 2049, 5, 3, 1, 2), (1200, 4096, 0, 0, 0, 0), (3, 5001, 1, 0, 1, 0), (7, 8192, 0, 0, 0, 0),
    (4, 16384, 0, 8, 0, 0), (3, 16385, 1, 1, 0, 0), (2, 40_000, 0, 0, 0, 0),
]


@pytest.mark.parametrize("shape", NORMS, ids=str)
@pytest.mark.parametrize("pair", PAIRS, ids=_id)
@pytest.mark.parametrize("rms", [False, True], ids=["layer", "rms"])
def test_norm_against_64_bits(ctx, shape, pair, rms):
    n, dim, skew, pad, y_skew, y_pad = shape
    kind, out_kind = pair
    param = (BF16, F32, F16)[(n + dim) % 3]
    x = Guarded(n, dim, kind, skew, dim + pad, _randn((n, dim), 1, 2.0) + 0.5)
    params = [Guarded(1, dim, param, n % 4, fill=_randn((1, dim), 2 + i)) for i in range(2)]
    w, b = (params[0].view[0] if n % 5 else None), (params[1].view[0] if n % 2 else None)
    y = Guarded(n, dim, out_kind, y_skew, dim + y_pad)
    mean, rstd = (Guarded(1, n, F32) for _ in range(2))
    got = ctx.layer_norm(x.view, weight=w, bias=b, eps=1e-3, rms=rms, out=y.view, mean=mean.view[0], rstd=rstd.view[0])
    for part in (x, y, mean, rstd, *params):
        part.check()
    true_y, true_mean, true_rstd = _true_norm(x.view, w, b, 1e-3, rms)
    _within(got, *true_y)
    _within(mean.view[0], *true_mean)
    _within(rstd.view[0], *true_rstd)


def test_norm_defaults_and_empty_inputs(ctx):
    x = _randn((2, 3, 96), 1)
    plain = ctx.layer_norm(x)
    assert plain.shape == x.shape and torch.equal(plain.view(6, 96), ctx.layer_norm(x.view(6, 96)))
    assert ctx.layer_norm(x, out_dtype=BF16).dtype == BF16
    assert ctx.layer_norm(x[:0]).shape == (0, 3, 96) and ctx.layer_norm(x[..., :0]).shape == (2, 3, 0)
    assert ctx.layer_norm(torch.empty(5, 0, device="cuda")).shape == (5, 0) and ctx.layer_norm(torch.empty(0, 5, device="cuda")).shape == (0, 5)
    assert torch.equal(ctx.layer_norm(x[0, 0]), plain[0, 0])
    wide = _randn((7, 200), 2)
    assert torch.equal(ctx.layer_norm(wide[:, 8:104]), ctx.layer_norm(wide[:, 8:104].contiguous()))
    empty = torch.empty(5, 0, device="cuda")
    assert ctx.layer_norm_grad(empty, empty, torch.empty(5, device="cuda"), torch.empty(5, device="cuda")).shape == (5, 0)


def test_moments_are_those_of_elementary_operations(ctx):
    """Products and sums rounded one by one: bit for bit what torch's operations give."""
    s = Set([70_000], F32, BF16, 32)
    m, v, g = s.state["m"].clone(), s.state["v"].clone(), s.g[:70_000].float()
    ctx.adamw_step(*s.args(), **s.state)
    assert torch.equal(s.state["m"][:70_000], m[:70_000] * 0.9 + g * (1 - 0.9))
    assert torch.equal(s.state["v"][:70_000], v[:70_000] * 0.999 + g * g * (1 - 0.999))


@pytest.mark.parametrize("dim", [40, 96, 640, 4096, 20_000])
def test_rows_do_not_depend_on_one_another_nor_on_where_they_lie(ctx, dim):
    x, w = _randn((700, dim), 3).to(BF16), _randn((dim,), 4)
    whole = ctx.layer_norm(x, weight=w)
    for a, b in ((0, 1), (5, 9), (650, 700)):
        assert torch.equal(ctx.layer_norm(x[a:b], weight=w), whole[a:b])
    for skew in (1, 2, 4):
        moved, out = Guarded(700, dim, BF16, skew, dim + 1, x), Guarded(700, dim, BF16, 3, dim + 5)
        assert torch.equal(ctx.layer_norm(moved.view, weight=w, out=out.view), whole)
        out.check()


@pytest.mark.parametrize("rms", [False, True])
def test_bad_values_stay_in_their_row(ctx, rms):
    x = _randn((40, 500), 5)
    clean = ctx.layer_norm(x, rms=rms)
    x[3, 7], x[20, 499], x[21, 0] = math.inf, math.nan, -math.inf
    got = ctx.layer_norm(x, rms=rms)
    rest = [i for i in range(40) if i not in (3, 20, 21)]
    assert torch.equal(got[rest], clean[rest])
    assert bool(torch.isnan(got[3, 7])) and bool(torch.isnan(got[20]).all()) and bool(torch.isnan(got[21, 0]))


def test_constant_rows_and_far_means(ctx):
    x = torch.full((4, 2048), 3.0, device="cuda")
    assert not bool(ctx.layer_norm(x).any())                             # 0 / sqrt(eps)
    x = _randn((8, 2048), 6) + 1e4                                       # the mean is 1e4 deviations away
    true_y, _, _ = _true_norm(x, None, None, 1e-5, False)
    _within(ctx.layer_norm(x), *true_y)


def test_norm_past_32_bit_offsets(ctx):
    n, dim = 1_050_000, 4096                                             # 4.3e9 elements
    x = torch.zeros(n, dim, dtype=BF16, device="cuda")
    x[-3:] = _randn((3, dim), 7).to(BF16)
    x[0] = 1
    y = ctx.layer_norm(x, rms=True)
    assert torch.equal(y[-3:], ctx.layer_norm(x[-3:].clone(), rms=True)) and not bool(y[1:-3].any())
    dw = torch.empty(dim, device="cuda")
    rstd = torch.ones(n, device="cuda")
    dx = ctx.layer_norm_grad(x, x, None, rstd, rms=True, out=y, weight_grad=dw)
    assert not bool(dx[1:-3].any())
    _within(dw, x[-3:].double().square().sum(0) + 1, 8 * U * (x[-3:].double().square().sum(0) + 1))


# ------------------------------------------------------------------------------------------------- its gradient

def _true_grad(dy, x, mean, rstd, w, rms):
    dy, x, dim = dy.double(), x.double(), x.shape[1]
    r = rstd.double()[:, None]
    h = (x if rms else x - mean.double()[:, None]) * r
    w = torch.ones(dim, dtype=torch.float64, device="cuda") if w is None else w.double()
    p = dy * w
    depth = 40 + 8 * (dim // 4096)
    mp = 0 * r if rms else p.mean(1, keepdim=True)
    e_mp = 0 * r if rms else (depth + 4) * U * p.abs().mean(1, keepdim=True)
    mh, e_mh = (p * h).mean(1, keepdim=True), (depth + 7) * U * (p * h).abs().mean(1, keepdim=True)
    dx = r * (p - mp - h * mh)
    e_dx = r * (3 * U * p.abs() + e_mp + h.abs() * e_mh + 4 * U * (h * mh).abs() + 2 * U * mp.abs()) + 2 * U * dx.abs()
    n = x.shape[0]
    sums = ((dy * h).sum(0), (n + 5) * U * (dy * h).abs().sum(0)), (dy.sum(0), (n + 2) * U * dy.abs().sum(0))
    return (dx, e_dx), *sums


GRADS = [  # n, dim, skews and padding of dy, x, dx
    (1, 1, 0, 0), (3, 5, 1, 1), (1, 4096, 0, 0), (2, 64, 0, 0), (500, 64, 0, 0), (301, 100, 1, 3), (77, 128, 0, 8), (1000, 256, 0, 0),
    (65, 257, 0, 0), (130, 1000, 8, 0), (600, 1023, 0, 0), (509, 2048, 0, 0), (4, 2049, 3, 1), (2500, 4096, 0, 0), (50, 4100, 0, 0),
    (90, 8192, 0, 0), (5, 8191, 1, 0), (40, 8200, 0, 0), (3, 20_001, 1, 2),
]


@pytest.mark.parametrize("shape", GRADS, ids=str)
@pytest.mark.parametrize("pair", PAIRS, ids=_id)
@pytest.mark.parametrize("rms", [False, True], ids=["layer", "rms"])
def test_gradient_against_64_bits(ctx, shape, pair, rms):
    n, dim, skew, pad = shape
    kind, y_kind = pair
    sum_kind, param = (F32, BF16, F16)[n % 3], (BF16, F16, F32)[dim % 3]
    x = Guarded(n, dim, kind, skew, dim + pad, _randn((n, dim), 1, 2.0) + 0.5)
    dy = Guarded(n, dim, y_kind, 2 * skew, dim + pad, _randn((n, dim), 2))
    w = _randn((dim,), 3).to(param) if n % 4 else None
    mean = None if rms else x.view.float().mean(1)
    rstd = 1 / (x.view.float().var(1, unbiased=False) + 1e-3).sqrt()
    true_dx, true_dw, true_db = _true_grad(dy.view, x.view, mean, rstd, w, rms)
    dx = Guarded(n, dim, kind, skew, dim + 2 * pad)
    dw, db = (Guarded(1, dim, sum_kind, 1) for _ in range(2))
    ctx.layer_norm_grad(dy.view, x.view, mean, rstd, weight=w, rms=rms, out=dx.view, weight_grad=dw.view[0], bias_grad=db.view[0])
    for part in (x, dy, dx, dw, db):
        part.check()
    _within(dx.view, *true_dx)
    _within(dw.view[0], *true_dw)
    _within(db.view[0], *true_db)
    old = _randn((dim,), 4).to(sum_kind)
    added = old.clone()
    ctx.layer_norm_grad(dy.view, x.view, mean, rstd, weight=w, rms=rms, out=dx.view, weight_grad=added, accumulate=True)
    _within(added, true_dw[0] + old.double(), true_dw[1] + U * (true_dw[0] + old.double()).abs())
    only = Guarded(1, dim, sum_kind)
    ctx.layer_norm_grad(dy.view, x.view, mean, rstd, weight=w, rms=rms, out=dx.view, bias_grad=only.view[0])
    only.check()
    assert torch.equal(only.view[0], db.view[0])


@pytest.mark.parametrize("rms", [False, True])
def test_gradient_against_differences(ctx, rms):
    """The directional derivative of sum(y c) along z, by central differences of a 64-bit forward form."""
    n, dim = 20, 300
    x, w, c, z, zw = (_randn(s, i) for i, s in enumerate(((n, dim), (dim,), (n, dim), (n, dim), (dim,)), 1))
    mean, rstd = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    ctx.layer_norm(x, weight=w, rms=rms, mean=mean, rstd=rstd)
    dw = torch.empty(dim, device="cuda")
    dx = ctx.layer_norm_grad(c, x, mean, rstd, weight=w, rms=rms, weight_grad=dw)

    def value(step):
        a, b = x.double() + step * z.double(), w.double() + step * zw.double()
        mu = 0 if rms else a.mean(1, keepdim=True)
        return float((((a - mu) / ((a - mu).square().mean(1, keepdim=True) + 1e-5).sqrt() * b) * c.double()).sum())

    slope = (value(1e-5) - value(-1e-5)) / 2e-5
    got = float((dx.double() * z.double()).sum() + (dw.double() * zw.double()).sum())
    # the gradients' own bounds along the direction, four times over for the rounded mean and rstd; the differences' are
    # 1e-10 / 6 times a third derivative of order 100 n dim, and 2^-53 |value| / 1e-5
    (_, e_dx), (_, e_dw), _ = _true_grad(c, x, mean, rstd, w, rms)
    limit = 4 * float((e_dx * z.abs()).sum() + (e_dw * zw.abs()).sum()) + 1e-4
    assert abs(got - slope) <= limit


def test_gradient_without_rows(ctx):
    x = torch.empty(0, 100, device="cuda")
    dw, db = torch.full((100,), 7.0, device="cuda"), torch.full((100,), 8.0, device="cuda")
    ctx.layer_norm_grad(x, x, x[:, 0], x[:, 0], weight_grad=dw, bias_grad=db, accumulate=True)
    assert bool((dw == 7).all()) and bool((db == 8).all())
    ctx.layer_norm_grad(x, x, x[:, 0], x[:, 0], weight_grad=dw, bias_grad=db)
    assert not bool(dw.any()) and not bool(db.any())


def test_gradient_is_the_same_bits_wherever_it_lies(ctx):
    for n, dim in ((333, 136), (91, 1500), (70, 4096), (9, 9000)):
        x, dy, w = _randn((n, dim), 1).to(BF16), _randn((n, dim), 2).to(BF16), _randn((dim,), 3)
        mean, rstd = _randn((n,), 4, 0.1), _randn((n,), 5).abs()
        dw, db = torch.empty(dim, device="cuda"), torch.empty(dim, device="cuda")
        dx = ctx.layer_norm_grad(dy, x, mean, rstd, weight=w, weight_grad=dw, bias_grad=db)
        for skew in (1, 4):
            moved = [Guarded(n, dim, BF16, skew + i, dim + 1 + i, t) for i, t in enumerate((x, dy))]
            out, dw2, db2 = Guarded(n, dim, BF16, 2, dim + 3), torch.empty_like(dw), torch.empty_like(db)
            ctx.layer_norm_grad(moved[1].view, moved[0].view, mean, rstd, weight=w, out=out.view, weight_grad=dw2, bias_grad=db2)
            out.check()
            assert torch.equal(out.view, dx) and torch.equal(dw, dw2) and torch.equal(db, db2)


# ------------------------------------------------------------------------------------------------- AdamW

TOP = 447.9995


def _mix(x):
    x = x ^ (x >> 16)
    x = (x * 0x6A09E667) & 0xffffffff
    x = x ^ (x >> 15)
    x = (x * 0xBB67AE85) & 0xffffffff
    return x ^ (x >> 16)


def _words(seed, t, places, first):
    """The word of each place, first + place % 8 of its group (int64 holding 32 bits)."""
    one = lambda x: int(_mix(torch.tensor(x & 0xffffffff)))  # noqa: E731
    k0 = one(one(one(seed + 0x9E3779B9) + (seed >> 32)) + t)
    k1 = one(k0 + (t >> 32) + 0x9E3779B9)
    b = _mix((places // 8) ^ k0)
    a = _mix((b + k1) & 0xffffffff)
    return (b + (first + places % 8 + 1) * a) & 0xffffffff


def _grid(x, digits, lowest, random):
    e = torch.floor(torch.log2(x.clamp(min=2.0 ** (lowest - 1)))).clamp(min=lowest)
    unit = torch.exp2(e - digits)
    return torch.floor(x / unit + random) * unit


class Set:
    """Tensors of a set, back to back from `skew` elements past a boundary, with their state; and what a step makes of them in 64 bits."""

    def __init__(self, counts, kind, grad_kind, bits, master=False, skew=0, grad_skew=0, seed=1, gap=0, step=41):
        self.counts, self.kind, self.grad_kind, self.bits = counts, kind, grad_kind, bits
        total = sum(counts) + gap * len(counts)
        size = lambda t: torch.empty(0, dtype=t).element_size()  # noqa: E731
        starts = [skew + sum(counts[:k]) + gap * k for k in range(len(counts))]
        grad_starts = [s - skew + grad_skew for s in starts]
        self.starts, self.grad_starts = starts, grad_starts
        self.w = _randn((skew + total + 64,), seed, 0.02).to(kind)
        self.g = _randn((grad_skew + total + 64,), seed + 1, 1e-3).to(grad_kind)
        i64 = lambda v: torch.tensor(v, dtype=torch.int64, device="cuda")  # noqa: E731
        self.offsets, self.lengths = i64([s * size(kind) for s in starts]), i64([c * size(kind) for c in counts])
        self.grad_offsets = i64([s * size(grad_kind) for s in grad_starts])
        self.state = binding.adamw_state(counts, "cuda", bits, master)
        self.places = self.state["state_offsets"].tolist()
        self.state["step"].fill_(step)
        n = self.state["m"].numel()
        m, root = _randn((n,), seed + 2, 3e-4), _randn((n,), seed + 3, 1e-3).abs()
        if bits == 32:
            self.state["m"].copy_(m)
            self.state["v"].copy_(root.square())
        else:
            for name, x in (("m", m), ("v", root)):
                scale = x.view(-1, 256).abs().amax(1) / 448
                self.state[name].copy_((x.view(-1, 256) / scale[:, None]).view(-1).to(torch.float8_e4m3fn))
                self.state[name + "_scales"].copy_(scale)
        if master:
            self.state["master"].copy_(_randn((n,), seed + 4, 0.02))
        self.keep()

    def keep(self):
        self.before = {k: v.clone() for k, v in {"w": self.w, "g": self.g, **self.state}.items()}

    def back(self):
        """Weights, gradients and state as they were made."""
        for k, v in {"w": self.w, "g": self.g, **self.state}.items():
            v.copy_(self.before[k])

    def args(self):
        return self.w, self.offsets, self.lengths, self.g, self.grad_offsets

    def moments(self, of, k):
        """m, and v or its root, of tensor k in 64 bits."""
        a = slice(self.places[k], self.places[k] + self.counts[k])
        if self.bits == 32:
            return of["m"][a].double(), of["v"][a].double()
        block = torch.arange(a.start, a.stop, device="cuda") // 256
        return (of["m"][a].double() * of["m_scales"].double()[block], of["v"][a].double() * of["v_scales"].double()[block])

    def check(self, lr=1e-3, betas=(0.9, 0.999), eps=1e-8, decay=1e-2, factor=1.0, stochastic=False, seed=0, skip=()):
        """Against 64 bits; everything outside the tensors, and the tensors in `skip`, as before."""
        torch.cuda.synchronize()
        old, t = self.before, int(self.before["step"]) + 1
        assert int(self.state["step"]) == t and torch.equal(self.g, old["g"])
        w_left, state_left = torch.ones_like(self.w, dtype=torch.bool), torch.ones_like(self.state["m"], dtype=torch.bool)
        for k, count in enumerate(self.counts):
            if k in skip or not count:
                continue
            a, s = slice(self.starts[k], self.starts[k] + count), slice(self.places[k], self.places[k] + count)
            w_left[a], state_left[s] = False, False
            g = old["g"][self.grad_starts[k]:self.grad_starts[k] + count].double() * factor
            m0, v0 = self.moments(old, k)
            v0 = v0 if self.bits == 32 else v0.square()
            m = betas[0] * m0 + (1 - betas[0]) * g
            v = betas[1] * v0 + (1 - betas[1]) * g.square()
            e_m = 8 * U * (betas[0] * m0.abs() + (1 - betas[0]) * g.abs())      # constants, factor, products, addition
            right = v.sqrt() / math.sqrt(1 - betas[1] ** t) + eps
            size = lr / (1 - betas[0] ** t)
            w0 = (old["master"][s] if "master" in old else old["w"][a]).double()
            update = size * m / right
            w = w0 * (1 - lr * decay) - update
            # v within 12 u, its root within 6 u + 4 u (2^-22, approximate root), quotient within 4 u, four more factors
            e_w = 3 * U * (w0.abs() + w.abs()) + size * e_m / right + 24 * U * update.abs()
            if "master" in old:
                _within(self.state["master"][s], w, e_w)
            places = torch.arange(s.start, s.stop, device="cuda")
            got = self.w[a]
            if stochastic and self.kind is not F32:
                bits, digits, lowest = (16, 7, -126) if self.kind is BF16 else (13, 10, -14)
                random = (_words(seed, t, places, 16) >> (32 - bits)).double() / 2 ** bits
                lo, hi = (_grid((w.abs() + d * e_w).clamp(min=0), digits, lowest, random) for d in (-1, 1))
                assert bool(((lo <= got.double().abs()) & (got.double().abs() <= hi)).all())
                assert float((lo == hi).double().mean()) > 0.9 or count < 1000
            else:
                _within(got, w, e_w)
            if self.bits == 32:
                _within(self.state["m"][s], m, e_m)
                _within(self.state["v"][s], v, 12 * U * v + 2.0 ** -149)
                continue
            root = v.sqrt()
            for name, x, e_x, first in (("m", m.abs(), e_m, 0), ("v", root, 12 * U * root, 8)):
                for b in range(0, count, 256):                                  # a block's scale
                    if b % 25600 and b + 256 < count:
                        continue
                    top, e_top = float(x[b:b + 256].max()), float(e_x[b:b + 256].max())
                    scale = float(self.state[name + "_scales"][(s.start + b) // 256])
                    assert abs(scale - top / TOP) <= (e_top + 4 * U * top) / TOP * MORE
                # codes, from the scales as they are
                scales = self.state[name + "_scales"].double()[places // 256]
                random = (_words(seed, t, places, first) >> 12).double() / 2 ** 20
                y, e_y = x / scales.clamp(min=1e-300), (e_x / scales.clamp(min=1e-300) + 4 * U * x / scales.clamp(min=1e-300)) * MORE
                lo, hi = (_grid((y + d * e_y).clamp(min=0), 3, -6, random) for d in (-1, 1))
                if name == "v":
                    lo, hi = (torch.where(x > 0, z.clamp(min=2.0 ** -9), z) for z in (lo, hi))
                code = self.state[name][s].double()
                live = scales > 0
                assert bool(((lo <= code.abs()) & (code.abs() <= hi))[live].all()) and not bool(code[~live].any())
                assert float((lo == hi)[live].double().mean()) > 0.99 or count < 1000
                if name == "m":
                    assert bool((code * m >= 0).all())
        assert torch.equal(self.w[w_left], old["w"][w_left])
        for name in ("m", "v", "master"):
            if name in old:
                x, y = self.state[name], old[name]
                if x.dtype == torch.float8_e4m3fn:
                    x, y = x.view(torch.uint8), y.view(torch.uint8)
                assert torch.equal(x[state_left], y[state_left])


KINDS = [(BF16, BF16, False), (BF16, BF16, True), (F16, F16, False), (F32, F32, False), (F32, BF16, False), (BF16, F32, True),
         (F16, F32, False), (F32, F16, False), (F16, F16, True)]
SETS = [  # counts, weights' skew, gradients' skew, gap between tensors (elements)
    ([1], 0, 0, 0), ([255, 0, 256, 257], 0, 0, 0), ([7, 300, 1000, 0, 0, 513, 1], 1, 0, 0), ([5000, 4096], 4, 0, 0), ([3000, 70_001], 3, 5, 2),
    ([0, 0], 0, 0, 0), ([100_000], 8, 8, 0), ([2049] * 40, 2, 0, 0),
]


@pytest.mark.parametrize("shape", SETS, ids=lambda s: f"{len(s[0])}x{max(s[0])}+{s[1]}")
@pytest.mark.parametrize("kind", KINDS, ids=_id)
@pytest.mark.parametrize("bits", [32, 8])
def test_step_against_64_bits(ctx, shape, kind, bits):
    counts, skew, grad_skew, gap = shape
    weight, grad, master = kind
    s = Set(counts, weight, grad, bits, master, skew, grad_skew, gap=gap)
    ctx.adamw_step(*s.args(), **s.state)
    s.check()
    s.back()
    ctx.adamw_step(*s.args(), **s.state, lr=1e-2, betas=(0.8, 0.95), eps=1e-4, weight_decay=0.5, stochastic=True, seed=(7 << 40) + 5)
    s.check(lr=1e-2, betas=(0.8, 0.95), eps=1e-4, decay=0.5, stochastic=True, seed=(7 << 40) + 5)


@pytest.mark.parametrize("bits", [32, 8])
def test_first_step_and_no_averages(ctx, bits):
    s = Set([1000, 300], F32, F32, bits, step=0)
    for name in ("m", "v", "m_scales", "v_scales"):
        if name in s.state:
            s.state[name].view(torch.uint8).zero_()
    s.keep()
    ctx.adamw_step(*s.args(), **s.state, betas=(0.0, 0.0), eps=0.0, weight_decay=0.0)
    s.check(betas=(0.0, 0.0), eps=0.0, decay=0.0)


@pytest.mark.parametrize("bits", [32, 8])
def test_clipping_by_the_record(ctx, bits):
    s = Set([5000, 301], BF16, BF16, bits, skew=1)
    grads = torch.tensor([2 * c for c in s.counts], dtype=torch.int64, device="cuda")
    record = binding.new_norm_result("cuda")
    ctx.grad_norm(s.g, s.grad_offsets, grads, record)
    norm = math.sqrt(sum(float(s.g[a:a + c].double().square().sum()) for a, c in zip(s.grad_starts, s.counts)))
    ctx.adamw_step(*s.args(), **s.state, norm=record, max_norm=norm / 3)
    s.check(factor=1 / 3)
    for limit in (None, 2 * norm):
        s.back()
        ctx.adamw_step(*s.args(), **s.state, norm=record, max_norm=limit)
        s.check()
    s.back()
    clipped = torch.empty_like(s.g)
    ctx.grad_clip(s.g, s.grad_offsets, grads, 0.0, record, out=clipped, out_offsets=s.grad_offsets)
    ctx.adamw_step(*s.args(), **s.state, norm=record, max_norm=0.0)
    s.check(factor=0.0)


@pytest.mark.parametrize("bits", [32, 8])
def test_a_step_with_a_bad_gradient_changes_nothing(ctx, bits):
    s = Set([5000, 301], BF16, F32, bits)
    s.g[17] = math.nan
    s.keep()
    record = binding.new_norm_result("cuda")
    ctx.grad_norm(s.g, s.grad_offsets, torch.tensor([4 * c for c in s.counts], device="cuda"), record)
    ctx.adamw_step(*s.args(), **s.state, norm=record, max_norm=1.0)
    torch.cuda.synchronize()
    for k, v in {"w": s.w, **s.state}.items():
        assert torch.equal(v.view(torch.uint8), s.before[k].view(torch.uint8)), k


def test_bad_moments_leave_their_block_alone(ctx):
    """Without a record an infinity or a NaN goes through: into its own element only."""
    s, clean = (Set([1024, 700], F32, F32, 8) for _ in range(2))
    s.g[5], s.g[300], s.g[1024 + 600] = math.inf, math.nan, 1e30          # 1e30: its square leaves the range
    clean.g[5], clean.g[300], clean.g[1024 + 600] = 0.0, 0.0, 0.0
    for x in (s, clean):
        x.state["m"].view(torch.uint8)[[5, 300, 1024 + 600]] = 0
        x.state["v"].view(torch.uint8)[[5, 300, 1024 + 600]] = 0
        ctx.adamw_step(*x.args(), **x.state)
    bad = torch.zeros(1792, dtype=torch.bool, device="cuda")
    bad[[5, 300]] = True
    m, v = s.state["m"].float(), s.state["v"].float()
    assert torch.equal(torch.isnan(m), bad)
    bad[1024 + 600] = True
    assert torch.equal(torch.isnan(v), bad)
    assert torch.equal(v[~bad], clean.state["v"].float()[~bad]) and torch.equal(s.state["v_scales"], clean.state["v_scales"])
    first = torch.arange(1792, device="cuda") < 1024                      # the last tensor's m holds a finite 1e29
    assert torch.equal(m[first & ~bad], clean.state["m"].float()[first & ~bad])
    w_bad = torch.zeros_like(s.w, dtype=torch.bool)
    w_bad[[5, 300, 1024 + 600]] = True
    assert torch.equal(s.w[~w_bad], clean.w[~w_bad])


@pytest.mark.parametrize("kind", [BF16, F16])
def test_bad_weights_stay_bad_however_they_are_rounded(ctx, kind):
    for stochastic in (False, True):
        s = Set([600], kind, F32, 32)
        s.w[3], s.w[300], s.w[599], s.g[40], s.g[50] = math.inf, math.nan, -math.inf, math.nan, -math.inf
        ctx.adamw_step(*s.args(), **s.state, stochastic=stochastic, seed=11)
        w = s.w[:600].float()
        assert float(w[3]) == math.inf and float(w[599]) == -math.inf
        bad = torch.zeros(600, dtype=torch.bool, device="cuda")
        bad[[300, 40, 50]] = True                                          # an infinite gradient: infinity / infinity
        assert torch.equal(torch.isnan(w), bad)


def test_averages_in_8_bits_do_not_stick(ctx):
    """Roots of 1 and gradients of 0, but for one element a block whose gradient of 1 holds the scale: rounding is unbiased, so
    the mean of the others follows 0.999^(t / 2).  A rounding goes to one of two codes at most 32 / 448 apart, so its
    deviation is at most half of that; 100 of them over the elements, rounded independently of one another, deviate by at
    most 10 * 16 / 448 / sqrt(n); six of those are allowed."""
    n, steps = 1 << 18, 100
    s = Set([n], F32, F32, 8)
    s.g.zero_()
    s.g[0:n:256] = 1.0
    s.state["m"].view(torch.uint8).zero_()
    s.state["v"].copy_(torch.full((n,), 448.0).to(torch.float8_e4m3fn))
    s.state["v_scales"].fill_(1 / 448)
    for i in range(steps):
        ctx.adamw_step(*s.args(), **s.state, seed=9)
    roots = s.state["v"].double().view(-1, 256) * s.state["v_scales"].double()[:, None]
    assert abs(float(roots[:, 1:].mean()) - 0.999 ** (steps / 2)) <= 6 * 10 * 16 / 448 / math.sqrt(n)
    # A block's top is scaled to 447.9995 and rounded to 448 with the probability 1 - 0.0005 / 32, to 416 otherwise: right on
    # average, and 448 / 447.9995 of itself, 1.2e-6 more, in nearly every step, so 1.2e-4 more after a hundred.
    top = (448 / TOP) ** steps * (1 + 8 * steps * U)
    assert bool((roots[:, 0] <= top).all()) and float(roots[:, 0].mean()) >= 1 - 6 * 10 * 16 / 448 / math.sqrt(n // 256)
    assert not bool(s.state["m"].view(-1, 256)[:, 1:].float().any())


def test_small_moments_and_large_ones(ctx):
    for std in (1e-30, 1e-19, 1e-12, 1e15):
        s = Set([3000], F32, F32, 8)
        s.g.mul_(std / 1e-3)
        s.state["m_scales"].mul_(std / 1e-3)
        s.state["v_scales"].mul_(std / 1e-3)
        s.keep()
        ctx.adamw_step(*s.args(), **s.state, eps=1e-35 if std < 1e-15 else 1e-8)
        assert bool(torch.isfinite(s.w).all()) and bool(torch.isfinite(s.state["m"].float()).all())
        if std > 1e-15:
            s.check()


def test_the_same_call_gives_the_same_bits_and_another_seed_others(ctx):
    got = []
    for seed in (3, 3, 4):
        s = Set([30_000, 77], BF16, BF16, 8, skew=1)
        for _ in range(3):
            ctx.adamw_step(*s.args(), **s.state, stochastic=True, seed=seed)
        got.append([s.w, s.state["m"].view(torch.uint8), s.state["v"].view(torch.uint8), s.state["m_scales"]])
    assert all(torch.equal(a, b) for a, b in zip(got[0], got[1]))
    assert not any(torch.equal(a, b) for a, b in zip(got[0][:3], got[2][:3]))


@pytest.mark.parametrize("bits", [32, 8])
def test_many_tensors(ctx, bits):
    s = Set([(i * 37) % 600 for i in range(1500)], BF16, BF16, bits, skew=1)
    ctx.adamw_step(*s.args(), **s.state)
    s.check()


@pytest.mark.parametrize("bits", [32, 8])
def test_ill_formed_tensors_are_left_out(ctx, bits):
    def bad(change, skip):
        s = Set([1000, 600, 300, 2000], BF16, F32, bits)
        change(s)
        s.keep()
        ctx.adamw_step(*s.args(), **s.state)
        assert ctx.device_status() == 2
        s.check(skip=skip)

    bad(lambda s: s.offsets[1:2].add_(1), {1})
    bad(lambda s: s.grad_offsets[1:2].add_(2), {1})
    bad(lambda s: s.lengths[2:3].add_(1), {2})
    bad(lambda s: s.state["state_offsets"][1:2].add_(8), {1})
    bad(lambda s: s.lengths[1:2].add_(2 * 800), {1})                       # beyond the next tensor's place
    bad(lambda s: s.lengths[3:4].add_(2 * 800), {3})                       # beyond the state's end


def test_learning_rate_on_the_device(ctx):
    s = Set([3000], BF16, BF16, 32)
    lr = torch.tensor([0.25], device="cuda")
    ctx.adamw_step(*s.args(), **s.state, lr=lr)
    s.check(lr=0.25)


def test_step_past_32_bit_offsets(ctx):
    """A state of 2^32 elements and more, one tensor: its last blocks against the same elements as a small tensor."""
    n = (1 << 32) + 5000
    w, g = torch.zeros(n, dtype=BF16, device="cuda"), torch.zeros(n, dtype=BF16, device="cuda")
    tail = 5000
    w[-tail:], g[-tail:] = _randn((tail,), 1).to(BF16), _randn((tail,), 2).to(BF16)
    state, small = binding.adamw_state([n], "cuda", 8), binding.adamw_state([tail], "cuda", 8)
    zero, i64 = torch.zeros(1, dtype=torch.int64, device="cuda"), lambda x: torch.tensor([x], dtype=torch.int64, device="cuda")
    w2, g2 = w[-tail:].clone(), g[-tail:].clone()
    ctx.adamw_step(w, zero, i64(2 * n), g, zero, **state)
    ctx.adamw_step(w2, zero, i64(2 * tail), g2, zero, **small)
    assert torch.equal(w[-tail:], w2) and not bool(w[:-tail].any())
    assert torch.equal(state["v_scales"][1 << 24:], small["v_scales"]) and torch.equal(state["m_scales"][1 << 24:], small["m_scales"])
    assert int(state["v"].view(torch.uint8)[n - 100:n].count_nonzero()) > 0


# ------------------------------------------------------------------------------------------------- streams, graphs, refusals

def test_on_another_stream(ctx):
    side = torch.cuda.Stream()
    x, w = _randn((500, 1024), 1), _randn((1024,), 2)
    s = Set([40_000], BF16, BF16, 8)
    side.wait_stream(torch.cuda.current_stream())
    y = ctx.layer_norm(x, weight=w, stream=side)
    ctx.adamw_step(*s.args(), **s.state, stream=side)
    side.synchronize()
    assert torch.equal(y, ctx.layer_norm(x, weight=w))
    s.check()


def test_a_captured_step_counts_on(ctx):
    """Norm, gradient, norm of the gradients and update as one graph, replayed: as the same calls one by one, with the
    learning rate changed between replays."""
    n, dim = 64, 512
    x, dy = _randn((n, dim), 1), _randn((n, dim), 2)
    i64 = lambda v: torch.tensor([v], dtype=torch.int64, device="cuda")  # noqa: E731

    def make():
        return {"w": torch.ones(dim, device="cuda"), "dw": torch.zeros(dim, device="cuda"), "mean": torch.empty(n, device="cuda"),
                "rstd": torch.empty(n, device="cuda"), "y": torch.empty(n, dim, device="cuda"), "dx": torch.empty(n, dim, device="cuda"),
                "record": binding.new_norm_result("cuda"), "lr": torch.tensor([0.1], device="cuda"),
                "state": binding.adamw_state([dim], "cuda", 8), "zero": i64(0), "bytes": i64(4 * dim)}

    def step(p):
        ctx.layer_norm(x, weight=p["w"], out=p["y"], mean=p["mean"], rstd=p["rstd"])
        ctx.layer_norm_grad(dy, x, p["mean"], p["rstd"], weight=p["w"], out=p["dx"], weight_grad=p["dw"])
        ctx.grad_norm(p["dw"], p["zero"], p["bytes"], p["record"])
        ctx.adamw_step(p["w"], p["zero"], p["bytes"], p["dw"], p["zero"], **p["state"], lr=p["lr"], norm=p["record"], max_norm=1.0, seed=1)

    eager, played = make(), make()
    step(make())                                         # scratch for the capture
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(played)
    for i in range(4):
        for p in (eager, played):
            p["lr"].fill_(0.1 / (i + 1))
        step(eager)
        graph.replay()
    torch.cuda.synchronize()
    assert int(played["state"]["step"]) == 4
    for key in ("w", "dw", "y", "dx"):
        assert torch.equal(eager[key], played[key])
    for key in ("m", "v", "m_scales", "v_scales"):
        assert torch.equal(eager["state"][key].view(torch.uint8), played["state"][key].view(torch.uint8))


def test_two_graphs_take_turns(ctx):
    """Two captured calls that share the context's scratch, replayed in turn and after calls of a larger size."""
    inputs = [(_randn((n, 640), i), _randn((n, 640), i + 9), torch.ones(n, device="cuda"), torch.zeros(640, device="cuda"), torch.empty(n, 640, device="cuda"))
              for i, n in enumerate((50, 900))]
    call = lambda p: ctx.layer_norm_grad(p[0], p[1], None, p[2], rms=True, out=p[4], weight_grad=p[3])  # noqa: E731
    want = []
    for p in inputs:
        call(p)
        want.append((p[3].clone(), p[4].clone()))
    graphs = []
    for p in inputs:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call(p)
        graphs.append(graph)
    big = _randn((5000, 8192), 3)
    for turn in range(3):
        for p, graph, (dw, dx) in zip(inputs, graphs, want):
            p[3].zero_()
            p[4].zero_()
            graph.replay()
            assert torch.equal(p[3], dw) and torch.equal(p[4], dx)
        ctx.layer_norm_grad(big, big, None, torch.ones(5000, device="cuda"), rms=True, weight_grad=torch.empty(8192, device="cuda"))


def test_two_contexts_at_once():
    streams = [torch.cuda.Stream() for _ in range(2)]
    contexts = [binding.Context(0) for _ in range(2)]
    sets = [Set([200_000, 31], BF16, BF16, 8, skew=k) for k in range(2)]
    xs = [_randn((3000, 1000), k) for k in range(2)]
    torch.cuda.synchronize()
    got = []
    for _ in range(3):
        for c, stream, s, x in zip(contexts, streams, sets, xs):
            c.adamw_step(*s.args(), **s.state, stream=stream)
            dw = torch.empty(1000, device="cuda")
            with torch.cuda.stream(stream):
                got.append((x, dw, c.layer_norm_grad(x, x, None, torch.ones(3000, device="cuda"), rms=True, weight_grad=dw, stream=stream)))
    torch.cuda.synchronize()
    for s in sets:
        assert int(s.state["step"]) == 44
        after = {k: v.clone() for k, v in {"w": s.w, **s.state}.items()}
        s.back()
        for _ in range(3):
            contexts[0].adamw_step(*s.args(), **s.state)
        assert all(torch.equal(after[k].view(torch.uint8), v.view(torch.uint8)) for k, v in {"w": s.w, **s.state}.items())
    for x, dw, dx in got:
        want = torch.empty_like(dw)
        assert torch.equal(contexts[0].layer_norm_grad(x, x, None, torch.ones(3000, device="cuda"), rms=True, weight_grad=want), dx)
        assert torch.equal(dw, want)
    for c in contexts:
        c.close()


def test_growth_under_capture_is_refused():
    with binding.Context(0) as c:
        x, rstd, dw = _randn((64, 512), 1), torch.ones(64, device="cuda"), torch.zeros(512, device="cuda")
        s = Set([100], F32, F32, 32)
        out = torch.empty_like(x)
        torch.cuda.synchronize()
        for call in (lambda: c.layer_norm_grad(x, x, None, rstd, rms=True, out=out, weight_grad=dw), lambda: c.adamw_step(*s.args(), **s.state)):
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                with pytest.raises(binding.IvError) as err:
                    call()
            assert err.value.code == binding.IV_ERR_CUDA
        assert int(s.state["step"]) == 41


def test_refusals(ctx):
    x, v, other = torch.zeros(4, 8, device="cuda"), torch.zeros(8, device="cuda"), torch.zeros(4, device="cuda")
    half = torch.zeros(8, dtype=F16, device="cuda")
    with pytest.raises(AssertionError):
        ctx.layer_norm(x, weight=other)
    with pytest.raises(AssertionError):
        ctx.layer_norm(x, weight=v, bias=half)
    with pytest.raises(AssertionError):
        ctx.layer_norm(x.t())
    with pytest.raises(AssertionError):
        ctx.layer_norm(x, rstd=v)
    for eps in (-1.0, math.nan):
        with pytest.raises(binding.IvError) as err:
            ctx.layer_norm(x, eps=eps)
        assert err.value.code == binding.IV_ERR_INVALID_ARG
    with pytest.raises(binding.IvError):
        ctx.layer_norm(x.to(F16), out_dtype=BF16)
    with pytest.raises(binding.IvError):
        ctx.layer_norm_grad(x, x, None, other)                             # no means
    with pytest.raises(AssertionError):
        ctx.layer_norm_grad(x, x, other, other, out=x.to(F16))
    with pytest.raises(AssertionError):
        ctx.layer_norm_grad(x, x, other, other, weight_grad=v, bias_grad=half)
    s = Set([1000], BF16, BF16, 8)
    for wrong in ({"lr": -1.0}, {"lr": math.nan}, {"lr": math.inf}, {"betas": (1.0, 0.5)}, {"betas": (0.5, -0.1)}, {"eps": -1e-8},
                  {"weight_decay": math.nan}, {"norm": binding.new_norm_result("cuda"), "max_norm": -1.0},
                  {"norm": binding.new_norm_result("cuda"), "max_norm": math.nan}, {"grad_dtype": F16}):
        with pytest.raises(binding.IvError) as err:
            ctx.adamw_step(*s.args(), **s.state, **wrong)
        assert err.value.code == binding.IV_ERR_INVALID_ARG
    for wrong in ({"max_norm": 1.0}, {"m": s.state["m"].float()}, {"m_scales": None}, {"v_scales": s.state["v_scales"][1:]}, {"step": s.state["step"].int()},
                  {"state_offsets": s.state["state_offsets"].int()}, {"m": s.state["m"].view(torch.uint8)}):
        with pytest.raises(AssertionError):
            ctx.adamw_step(*s.args(), **{**s.state, **wrong})
    whole = torch.zeros(1032, device="cuda")
    with pytest.raises(binding.IvError):                                   # moments off a 32-byte boundary
        ctx.adamw_step(*s.args(), **{**s.state, "m": whole[1:1025], "v": whole[:1024]})
    with pytest.raises(binding.IvError):                                   # not a whole number of blocks
        ctx.adamw_step(*s.args(), **{**s.state, "m": whole[:1000], "v": whole[:1000]})
    f = Set([1000], F32, F32, 32)
    with pytest.raises(binding.IvError):                                   # a 32-bit copy of 32-bit weights
        ctx.adamw_step(*f.args(), **{**f.state, "master": torch.zeros(1024, device="cuda")})
    torch.cuda.synchronize()
    assert int(s.state["step"]) == 41 and torch.equal(s.w, s.before["w"])
