"""The experts' products and their weights' gradient on each way of their operands to LDS, chosen by size and
alignment: through registers, and as aligned chunks; against the plain 64-bit implementations of expert_checks.py."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import expert_checks as E  # noqa: E402,F401
from test_gpu_experts import run_product, zo  # noqa: E402,F401

pytestmark = pytest.mark.gpu
F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32


# Through registers the copies are a step further ahead of the products than they are straight to LDS: with tiles
# of one step (64 columns of 16 bits) the third tile's rows are looked up before the first has ended.
@pytest.mark.parametrize("dtype", (F16, BF16))
@pytest.mark.parametrize("x_slots,y_slots", ((1, 0), (1, 1), (2, 0), (2, 1)))
@pytest.mark.parametrize("slots,experts,cin,cout,lead", (
    (1700, 12, 50, 17001, 1), (2600, 3, 64, 17000, 1), (2600, 3, 1, 17000, 0), (6000, 100, 63, 3700, 1)))
def test_product_tiles_of_one_step_through_registers(zo, slots, experts, cin, cout, lead, x_slots, y_slots, dtype):  # noqa: F811
    for transposed in (False, True):
        run_product(zo, slots // 2, 2, experts, cin, cout, dtype, x_slots, y_slots, transposed, 0, lead, 0.02)
