"""The example when a step has gone wrong: tokens whose router logits are NaN get no expert, the gradient is NaN, and the
shard step skips."""
import math
import os
import sys

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, os.path.join(ROOT, "examples"))

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("what", ("router", "token"))
def test_a_step_without_experts_is_skipped(what):
    import distill_experts as D
    student, teacher = D.Student("cuda"), D.Teacher("cuda")
    batch = teacher.batch()
    if what == "router":
        student.p["router"].fill_(math.nan)
        want = 0
    else:
        student.p["embed"][int(batch[0][3])] = math.nan
        want = D.CHOSEN * int((batch[0] != batch[0][3]).sum())
    before, scale = student.master.clone(), student.scaler.scale
    _, skipped = student.train_step(*batch)
    torch.cuda.synchronize()
    assert student.ends[D.EXPERTS] == want and len(student.slots) == want
    assert bool((student.slots >= 0).all())
    assert skipped == 1 and student.scaler.scale == scale / 2 and torch.equal(student.master, before)
    # the next step, from the parameters as they were, is an ordinary one
    student.p16.copy_(student.master)
    loss, _ = student.train_step(*teacher.batch())
    assert math.isfinite(loss) and student.ends[D.EXPERTS] == D.TOKENS * D.CHOSEN
