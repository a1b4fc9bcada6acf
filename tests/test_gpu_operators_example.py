"""The example that runs the operators together: a student with routed experts distilled through the shard step."""
import math
import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, os.path.join(ROOT, "examples"))

pytestmark = pytest.mark.gpu


def test_the_student_learns():
    import distill_experts as D
    losses, skips, e4m3, student = D.train(40)
    assert all(math.isfinite(x) for x in losses)
    assert skips <= 5, "a loss scale of 2^16 comes down in a few steps"
    # the teacher's table is learned: a third of the loss goes in 40 steps
    assert sum(losses[-5:]) < 0.67 * sum(losses[:5]), (losses[:5], losses[-5:])
    # rows in 8 bits carry 2^-4 of rounding each, of which a product over 128 columns leaves a few per cent
    assert abs(e4m3 / losses[-1] - 1) < 0.15, (e4m3, losses[-1])
    assert int(student.offsets[-1]) == D.TOKENS * D.CHOSEN


def test_the_gradient_is_the_losss():
    """The whole backward pass against automatic differentiation of the same student in float64, its choice of
    experts given.  On the way to a gradient lie at most eight roundings to fp16 (2^-11 of a value each): under 2 %
    in norm with room for sums that cancel; the router's is a difference of two such sums, of a tenth of
    their size where the chosen experts serve a token about alike."""
    import torch
    import distill_experts as D
    student, teacher = D.Student("cuda"), D.Teacher("cuda")
    tokens, index, logits, labels = teacher.batch()
    z = student.forward(tokens)
    D.zo.zero_distill_step(z, index, logits, student.loss, z, labels=labels, hard=D.HARD, temperature=D.TAU,
                           row_weight=student.row_weight, grad_scale=1024.0)
    student.backward(z, tokens)

    p = {k: t.double().cpu().requires_grad_(True) for k, t in student.p.items()}
    tokens, index, logits, labels, chosen = (t.cpu() for t in (tokens, index.long(), logits.double(), labels.long(),
                                                               student.index.long()))

    def norm(h, w):
        return h * (h.square().mean(1, keepdim=True) + D.EPS).rsqrt() * w

    x = p["embed"][tokens]
    y1 = norm(x, p["norm1"])
    w = torch.sigmoid((y1 @ p["router"]).gather(1, chosen))
    w = w / w.sum(1, keepdim=True)
    each = torch.stack([torch.relu(y1 @ p["up"][e]) @ p["down"][e] for e in range(D.EXPERTS)], 1)
    mixed = (each.gather(1, chosen[:, :, None].expand(-1, -1, D.HIDDEN)) * w[:, :, None]).sum(1)
    out = norm(x + mixed, p["norm2"]) @ p["head"].t()
    lp = torch.log_softmax(logits / D.TAU, 1)
    soft = D.TAU ** 2 * (lp.exp() * (lp - torch.log_softmax(out / D.TAU, 1).gather(1, index))).sum(1)
    hard = -torch.log_softmax(out, 1).gather(1, labels[:, None])[:, 0]
    loss = (soft + D.HARD * hard).mean()
    assert abs(float(student.loss.double().sum()) / float(loss.detach()) - 1) < 5e-3
    loss.backward()
    for name, t in p.items():
        got, want = student.g[name].double().cpu() / 1024.0, t.grad
        rel = float((got - want).norm() / want.norm())
        assert rel < (0.2 if name == "router" else 0.02), (name, rel)
