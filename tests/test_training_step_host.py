"""Host-side checks of the training-step operators that need no GPU: record layout, type codes, refusals without a context."""
import ctypes
import os
import re

import torch

from paper_2510_23938_b200 import binding

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_record_layout_matches_the_header():
    assert ctypes.sizeof(binding.NormResult) == 32
    assert [getattr(binding.NormResult, f).offset for f, _ in binding.NormResult._fields_] == [0, 4, 8, 12, 16, 24]


def test_type_codes_match_the_header():
    text = open(os.path.join(ROOT, "include", "iv.h")).read()
    codes = dict(re.findall(r"(IV_(?:F32|F16|BF16)) = (\d)", text))
    assert {"IV_F32": "0", "IV_F16": "1", "IV_BF16": "2"} == codes
    assert binding.DTYPES == {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}


def test_every_call_refuses_a_missing_context():
    lib = binding.load_library()
    none = None
    assert lib.iv_embedding(none, 16, 0, 1, 1, 1, 16, 8, 1, 1.0, 16, 0, 1, none) == binding.IV_ERR_INVALID_ARG
    assert lib.iv_embedding_grad(none, 16, 0, 1, 1, 16, 8, 1, 1, -1, 1.0, 0, 16, 0, 1, none) == binding.IV_ERR_INVALID_ARG
    assert lib.iv_embedding_grad_rows(none, 16, 0, 1, 1, 16, 8, 1, 1, -1, 1.0, 16, 16, 0, 1, 1, 16,
                                      none) == binding.IV_ERR_INVALID_ARG
    assert lib.iv_grad_norm(none, 16, 16, 16, none, 0, 1, none, 16, none) == binding.IV_ERR_INVALID_ARG
    assert lib.iv_grad_clip(none, 16, 16, 16, none, 0, 1, 1.0, none, none, -1, none, 16, none) == binding.IV_ERR_INVALID_ARG
    assert lib.iv_grad_scale(none, 16, 16, 16, none, 0, 1, 16, none, none, -1, none) == binding.IV_ERR_INVALID_ARG
