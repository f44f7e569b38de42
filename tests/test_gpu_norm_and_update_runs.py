"""Long runs of the norm kernels and the AdamW step: rings of copies that are filled again and again, tensors that give a warp many blocks.

Small sets end before a ring's first place is used twice; the sizes here are counted from a B200's 148 SMs so that every
form of the kernels goes round its ring at least once.  Bounds are those of test_gpu_norm_and_update.py.
"""
import pytest
import torch

from test_gpu_norm_and_update import BF16, F16, F32, KINDS, Set, _id, ctx  # noqa: F401

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
