"""zero_log_probs on rows so long that a thread adds up very many terms: the sums' error does not grow with the row."""
import math
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import operator_checks as C  # noqa: E402
from test_gpu_log_probs import check, logits  # noqa: E402
from test_gpu_operators import zo  # noqa: E402,F401

pytestmark = pytest.mark.gpu
F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32


@pytest.mark.parametrize("k", (0, 2))
@pytest.mark.parametrize("dtype,bits", ((BF16, 20), (BF16, 26), (BF16, 28), (F16, 26), (F32, 25)))
def test_sums_of_long_rows(zo, dtype, bits, k):  # noqa: F811
    """Logits 0 and -1 in turn, so that in one chain of fp32 every other rounding goes the same way.  The
    statistics from their closed form.  A thread's terms are rounded 512 times in turn, 30 steps follow; a term's
    exponent is held to 2 U and 2^x is off by 4 U."""
    vocab = (1 << bits) + 6
    z = torch.zeros(1, vocab, dtype=dtype, device="cuda")
    z[0, 1::2] = -1
    z[0, 3] = 2
    tokens = torch.tensor([7], dtype=torch.int32, device="cuda")
    lp, h, st = torch.empty(1, device="cuda"), torch.empty(1, device="cuda"), torch.empty(1, 3, device="cuda")
    kw = dict(top_index=torch.empty(1, k, dtype=torch.int32, device="cuda"), top_logp=torch.empty(1, k, device="cuda")) if k else {}
    zo.zero_log_probs(z, tokens, lp, entropy=h, stats=st, **kw)
    zeros, ones = vocab // 2, vocab // 2 - 1   # 2 below the largest, 3 below
    total = 1 + zeros * math.exp(-2) + ones * math.exp(-3)
    below = zeros * math.exp(-2) * 2 + ones * math.exp(-3) * 3
    entropy = math.log(total) + below / total
    adds = 512 + 30
    of_sum = (adds + 8 + 2 * 3 + 8 * math.log(total)) * C.U
    assert abs(st[0, 1].item() / total - 1) <= of_sum
    assert abs(lp.item() - (-3 - math.log(total))) <= of_sum + 4 * C.U * 3 + C.U * 30
    first = below / total
    assert abs(h.item() - entropy) <= of_sum + ((adds + 12) * first + 2 * 9) * C.U + first * of_sum + C.U * 30
    if k:
        assert kw["top_index"][0].tolist() == [3, 0]
        assert abs(kw["top_logp"][0, 0].item() + math.log(total)) <= of_sum + C.U * 30


@pytest.mark.parametrize("k", (0, 3))
def test_a_maximum_that_keeps_rising(zo, k):  # noqa: F811
    """Every sum is taken against a new maximum again and again, in 64 bits too."""
    vocab = 1 << 22
    z = (torch.arange(vocab, device="cuda", dtype=torch.float64) / vocab * 12).float()[None]
    lp, h, st = torch.empty(1, device="cuda"), torch.empty(1, device="cuda"), torch.empty(1, 3, device="cuda")
    kw = dict(top_index=torch.empty(1, k, dtype=torch.int32, device="cuda"), top_logp=torch.empty(1, k, device="cuda")) if k else {}
    zo.zero_log_probs(z, torch.tensor([5], dtype=torch.int32, device="cuda"), lp, entropy=h, stats=st, **kw)
    x = z[0].double().cpu() - z[0, -1].item()
    e = x.exp()
    total = e.sum().item()
    first = -(e * x).sum().item() / total
    # a move against another maximum costs 8 U; of a thread's 128 groups of vectors each may move the sums once
    of_sum = (512 + 30 + 8 + 8 * 128 + 2 * 12 + 8 * math.log(total)) * C.U
    assert abs(st[0, 1].item() / total - 1) <= of_sum
    assert abs(lp.item() - (x[5].item() - math.log(total))) <= of_sum + 4 * C.U * 12 + C.U * 30
    assert abs(h.item() - (math.log(total) + first)) <= 3 * of_sum + C.U * 30
    if k:
        assert kw["top_index"][0].tolist() == [vocab - 1, vocab - 2, vocab - 3]


@pytest.mark.parametrize("dtype", C.TYPES)
@pytest.mark.parametrize("rows,vocab", ((3, 60000), (64, 131072), (65, 131072), (3, 100000), (3, 28800), (65, 65536)))
def test_long_rows_without_a_list(zo, rows, vocab, dtype):  # noqa: F811
    """About the rows and lengths at which the kernel changes, for 8 and for 4 logits a vector."""
    check(zo, *logits(rows, vocab, dtype, 51), 0)
