"""Host-side checks of layer norm and the AdamW step that need no GPU: record layout, the state's layout, refusals without a context."""
import ctypes
import os
import re

import pytest
import torch

from paper_2510_23938_b200 import binding

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_layouts_match_the_header():
    assert ctypes.sizeof(binding.AdamwOptions) == 56
    assert [getattr(binding.AdamwOptions, f).offset for f, _ in binding.AdamwOptions._fields_] == [0, 8, 16, 24, 32, 40, 44, 48]
    text = open(os.path.join(ROOT, "include", "iv.h")).read()
    assert int(re.search(r"#define IV_ADAMW_BLOCK (\d+)", text).group(1)) == binding.ADAMW_BLOCK


def test_every_call_refuses_a_missing_context():
    lib = binding.load_library()
    none, o = None, binding.AdamwOptions(1e-3, 0.9, 0.999, 1e-8, 0.0, 1.0, 0, 0)
    bad = binding.IV_ERR_INVALID_ARG
    assert lib.iv_layer_norm(none, 16, 0, 1, 1, 1, 16, 16, 0, 1e-5, 0, 16, 0, 1, 16, 16, none) == bad
    assert lib.iv_layer_norm_grad(none, 16, 0, 1, 16, 0, 1, 1, 1, 16, 0, 16, 16, 0, 16, 1, 16, 16, 0, 0, none) == bad
    assert lib.iv_adamw_step(none, 16, 16, 16, 0, 1, 16, 16, 0, 16, 256, 32, 32, 32, none, none, none, o, none, none, 16, none) == bad


@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("master", [False, True])
def test_state_layout(bits, master):
    state = binding.adamw_state([1, 0, 256, 257, 5], "cpu", bits, master)
    assert state["state_offsets"].tolist() == [0, 256, 256, 512, 1024]
    assert state["m"].numel() == state["v"].numel() == 1280 and int(state["step"]) == 0
    assert state["m"].dtype == (torch.float32 if bits == 32 else torch.float8_e4m3fn)
    assert ("m_scales" in state) == (bits == 8) and ("master" in state) == master
    if bits == 8:
        assert state["m_scales"].numel() == state["v_scales"].numel() == 5
    assert not any(bool(state[k].float().any()) for k in state if k != "state_offsets")


def test_state_of_nothing_and_of_other_widths():
    assert binding.adamw_state([], "cpu")["m"].numel() == 0
    with pytest.raises(AssertionError):
        binding.adamw_state([5], "cpu", bits=16)
