"""zero_log_probs's lists where their bound comes from few bins: logits that lie closer or farther apart than the histogram
of distances tells, long lists of short rows, rows with less to list than is asked for."""
import math
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import operator_checks as C  # noqa: E402
from test_gpu_log_probs import check, logits, zo  # noqa: E402,F401

pytestmark = pytest.mark.gpu
F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32


@pytest.mark.parametrize("vocab", (2048, 9001, 70001))
@pytest.mark.parametrize("k", (1, 20, 300, 1024))
def test_close_and_far_apart(zo, vocab, k):  # noqa: F811
    z, tokens = logits(8, vocab, F32, 21)
    z[0] = z[0] * 1e-6 + 5.0          # distances below the first bin
    z[1] = z[1] * 1e-5
    z[2] = z[2] * 1e9                 # beyond the last
    z[3] = torch.where(torch.arange(vocab) % 7 == 0, -3e38, 3e38)   # a difference past fp32's range
    z[4, 11:] = -3e38
    z[4, 3] = 3e38
    z[5] = z[5].abs().sqrt().sqrt()   # many near the largest
    z[6, :15] = torch.arange(15.0) * 1e-3 + 20
    check(zo, z, tokens, k)


@pytest.mark.parametrize("dtype", C.TYPES)
@pytest.mark.parametrize("vocab", (600, 5003, 66000))
def test_less_than_is_asked_for(zo, vocab, dtype):  # noqa: F811
    z, tokens = logits(6, vocab, dtype, 23)
    tokens[:] = 0
    z[0, 5:] = -math.inf
    z[1, 40:] = -math.inf
    z[1, 60] = math.nan
    z[2, 1:] = math.nan
    z[3, 2::3] = -math.inf
    z[4, ::2] = math.inf              # more of the largest than are listed
    z[5, 9] = math.inf
    for k in (1, 33, 128, 600):
        check(zo, z, tokens, k)
