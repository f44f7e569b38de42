"""Layer norm of rows whose elements are all the same, and its gradient there: y is the bias and h is 0, whatever the width."""
import pytest
import torch

from test_gpu_norm_and_update import BF16, F16, F32, U, Guarded, _randn, _true_grad, _within, ctx  # noqa: F401

pytestmark = pytest.mark.gpu

# widths whose reciprocal is rounded, beside those where it is not; wide enough for each form of the kernels
DIMS = [7, 40, 96, 100, 136, 1000, 1023, 1024, 2049, 5001, 7168, 8192, 13_000, 16_384, 20_001, 40_000]


@pytest.mark.parametrize("kind", [BF16, F32])
@pytest.mark.parametrize("dim", DIMS)
def test_gradient_of_large_constant_rows(ctx, dim, kind):  # noqa: F811
    """mean * rstd is beyond 32 bits, while x - mean is 0 in every column there is."""
    n = 9
    x = torch.full((n, dim), 2.0 ** 110, device="cuda").to(kind)
    dy, w = _randn((n, dim), 1).to(kind), _randn((dim,), 2)
    mean, rstd = torch.full((n,), 2.0 ** 110, device="cuda"), torch.full((n,), 1e6, device="cuda")
    assert bool(torch.isinf(mean * rstd).all())
    for skew in (0, 1):
        moved = [Guarded(n, dim, kind, skew, dim + skew, t) for t in (dy, x)]
        dw, db = torch.empty(dim, device="cuda"), torch.empty(dim, device="cuda")
        dx = ctx.layer_norm_grad(moved[0].view, moved[1].view, mean, rstd, weight=w, weight_grad=dw, bias_grad=db)
        true_dx, _, true_db = _true_grad(dy, x, mean, rstd, w, False)
        _within(dx, *true_dx)
        _within(db, *true_db)
        assert not bool(dw.any())


@pytest.mark.parametrize("kind", [BF16, F16, F32])
@pytest.mark.parametrize("dim", DIMS)
def test_constant_rows_of_16_bits_give_exact_zeros(ctx, dim, kind):  # noqa: F811
    """A sum of n equal numbers of 8 digits has at most 8 + log2(n) of them, of 11 digits 11 + log2(n): exact in 24 for every
    partial sum here (2^16 and 2^13 columns), so the mean is the number itself if the sum is divided by n."""
    values = torch.arange(128, 256, device="cuda").float()                # every mantissa of bf16
    if kind is not BF16 and dim <= 1 << 13:
        values = torch.arange(1024, 2048, 7, device="cuda").float()
    values = torch.cat([values * 2.0 ** -7, -values * 2.0 ** 5])
    x = values[:, None].expand(-1, dim).to(kind).contiguous()
    bias = _randn((dim,), 1)
    for eps in (1e-5, 1e-12):
        mean, rstd = (torch.empty(len(values), device="cuda") for _ in range(2))
        y = ctx.layer_norm(x, eps=eps, mean=mean, rstd=rstd)
        assert torch.equal(mean, values) and not bool(y.any())
        assert bool(((rstd * eps ** 0.5 - 1).abs() <= 5 * U).all())        # eps, root, quotient and, here, root and product
        y = ctx.layer_norm(x, weight=bias, bias=bias, eps=eps, out_dtype=F32)
        assert torch.equal(y, bias.expand_as(y))
    moved = Guarded(len(values), dim, kind, 1, dim + 1, x)
    assert not bool(ctx.layer_norm(moved.view).any())


@pytest.mark.parametrize("kind", [BF16, F32])
@pytest.mark.parametrize("dim", DIMS)
def test_gradient_that_is_the_same_for_a_row(ctx, dim, kind):  # noqa: F811
    """dx = rstd (p - mean(p) - h mean(p h)) with h = 0 and one p for all columns: exactly 0, however large rstd is."""
    values = torch.arange(128, 256, device="cuda").float() * 2.0 ** -9
    dy = values[:, None].expand(-1, dim).to(kind).contiguous()
    x = torch.full_like(dy, 3.0)
    mean, rstd = torch.full_like(values, 3.0), torch.full_like(values, 1e6)
    for skew in (0, 1):
        moved = [Guarded(len(values), dim, kind, skew, dim + skew, t) for t in (dy, x)]
        assert not bool(ctx.layer_norm_grad(moved[0].view, moved[1].view, mean, rstd).any())
