"""The state's 32-bit copies of the weights: made from the weights, or by the documented call into room for them."""
import pytest
import torch

from paper_2510_23938_b200 import binding

COUNTS = [300, 0, 256, 7, 1000]


def _weights(device):
    g = torch.Generator()
    g.manual_seed(1)
    shapes = [(30, 10), (0,), (256,), (7, 1), (10, 100)]
    return [torch.randn(s, generator=g).to(torch.bfloat16).to(device) for s in shapes]


def _check(state, weights):
    assert state["master"].dtype is torch.float32
    rest = torch.ones_like(state["master"], dtype=torch.bool)
    for place, w in zip(state["state_offsets"].tolist(), weights):
        assert torch.equal(state["master"][place:place + w.numel()], w.reshape(-1).float())
        rest[place:place + w.numel()] = False
    assert not bool(state["master"][rest].any())


@pytest.mark.parametrize("bits", [8, 32])
def test_copies_of_the_weights(bits):
    weights = _weights("cpu")
    weights[4] = weights[4].t()                          # any strides
    _check(binding.adamw_state(COUNTS, "cpu", bits, weights), weights)
    assert not bool(binding.adamw_state(COUNTS, "cpu", bits, True)["master"].any())
    assert "master" not in binding.adamw_state(COUNTS, "cpu", bits)
    assert binding.adamw_state([], "cpu", bits, [])["master"].numel() == 0


def test_weights_of_other_sizes_are_refused():
    for wrong in (_weights("cpu")[:-1], [torch.zeros(n + 1) for n in COUNTS]):
        with pytest.raises(AssertionError):
            binding.adamw_state(COUNTS, "cpu", 32, wrong)


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [8, 32])
def test_steps_from_both_ways_are_the_same(bits):
    with binding.Context(0) as ctx:
        got = []
        for copied in (True, False):
            weights = _weights("cuda")
            flat = torch.cat([w.reshape(-1) for w in weights])
            starts = torch.tensor([0, 300, 300, 556, 563], device="cuda")
            lengths = 2 * torch.tensor(COUNTS, device="cuda")
            state = binding.adamw_state(COUNTS, "cuda", bits, weights if copied else True)
            if not copied:
                ctx.grad_scale(flat, 2 * starts, lengths, torch.ones(1, device="cuda"), out=state["master"], out_offsets=4 * state["state_offsets"])
            _check(state, weights)
            grads = flat * 0.1
            ctx.adamw_step(flat, 2 * starts, lengths, grads, 2 * starts, **state, lr=1e-3)
            got.append([flat, *state.values()])
        assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(*got))
        near = torch.cat([w.reshape(-1) for w in _weights("cuda")])
        assert bool(((got[0][0] - near).abs() <= 2e-3 + near.abs() / 64).all())       # a step of 1e-3 from the weights, not from 0
