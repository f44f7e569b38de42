"""The gradient of layer norm at rows whose elements are all the same: h is 0 there, whatever the width."""
import pytest
import torch

from test_gpu_norm_and_update import BF16, F32, Guarded, _randn, _true_grad, _within, ctx  # noqa: F401

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
