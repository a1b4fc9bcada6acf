"""A small student with routed experts, distilled from a teacher's top logits and trained with the shard step.

One transformer-like block without attention: embedding, norm, router, experts, residual, norm, head.  The
products are torch's; the norms, the routing, the loss and their gradients are the package's operators, and the
fp16 gradient, which carries the scaler's loss scale from the loss on, goes to zero_shard_step_scaled: an
overflow anywhere in the backward pass is found there, the step is skipped and the scale halved.  The teacher
is a table of next-token logits, of which the student sees the top few.

    python examples/distill_experts.py [--steps 60]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_1910_02054_amd import binding as zb  # noqa: E402
from paper_1910_02054_amd import operators as zo  # noqa: E402

VOCAB, HIDDEN, EXPERTS, CHOSEN, INNER, TOKENS, TOP = 2048, 128, 8, 2, 256, 1024, 16
EPS, TAU, HARD, BALANCE = 1e-6, 2.0, 0.1, 1e-3
SHAPES = {"embed": (VOCAB, HIDDEN), "norm1": (HIDDEN,), "router": (HIDDEN, EXPERTS), "up": (EXPERTS, HIDDEN, INNER),
          "down": (EXPERTS, INNER, HIDDEN), "norm2": (HIDDEN,), "head": (VOCAB, HIDDEN)}


class Student:
    """The parameters as one flat fp16 buffer (what the all-gather publishes), the gradient as another, the
    fp32 state of the only rank's shard, and the buffers that a step writes."""

    def __init__(self, device, seed=0):
        gen = torch.Generator(device=device).manual_seed(seed)
        self.n = sum(torch.Size(s).numel() for s in SHAPES.values())
        self.master = torch.empty(self.n, device=device).normal_(0.0, 0.05, generator=gen)
        self.m, self.v = torch.zeros_like(self.master), torch.zeros_like(self.master)
        self.p16 = torch.empty(self.n, dtype=torch.float16, device=device)
        self.g16 = torch.zeros_like(self.p16)
        self.p, self.g = self.views(self.p16), self.views(self.g16)
        for name, t in self.views(self.master).items():
            if name.startswith("norm"):
                t.fill_(1.0)
        self.p16.copy_(self.master)
        self.scaler = zb.Scaler(2.0 ** 16, window=200)
        self.step = zb.ShardStepCall([self.g16], self.master, self.m, self.v, self.p16, 2e-3, 0.9, 0.99, 1e-8, 0.0,
                                     clip=1.0)
        self.bias = torch.zeros(EXPERTS, device=device)

        def f16(*shape):
            return torch.empty(*shape, dtype=torch.float16, device=device)

        def f32(*shape):
            return torch.empty(*shape, device=device)

        def i32(*shape):
            return torch.empty(*shape, dtype=torch.int32, device=device)

        self.y1, self.rstd1 = f16(TOKENS, HIDDEN), f32(TOKENS)
        self.h2, self.y2, self.rstd2 = f16(TOKENS, HIDDEN), f16(TOKENS, HIDDEN), f32(TOKENS)
        self.q8 = torch.empty(TOKENS, HIDDEN, dtype=torch.float8_e4m3fn, device=device)
        self.q8_scale = f32(TOKENS, 1)
        self.index, self.weight = i32(TOKENS, CHOSEN), f32(TOKENS, CHOSEN)
        self.offsets, self.order = i32(EXPERTS + 1), i32(TOKENS * CHOSEN)
        self.loss = f32(TOKENS)
        self.dh2, self.dx, self.drouted = f16(TOKENS, HIDDEN), f16(TOKENS, HIDDEN), f16(TOKENS, EXPERTS)
        self.norm_room = f32(zo.zero_rms_norm_workspace(TOKENS, HIDDEN))
        self.order_room = i32(zo.zero_route_workspace(TOKENS * CHOSEN, EXPERTS))
        self.row_weight = torch.full((TOKENS,), 1.0 / TOKENS, device=device)

    @staticmethod
    def views(flat):
        out, at = {}, 0
        for name, shape in SHAPES.items():
            n = torch.Size(shape).numel()
            out[name] = flat[at:at + n].view(shape)
            at += n
        return out

    def forward(self, tokens):
        """The logits; leaves what the backward needs in `self`."""
        p = self.p
        self.x = p["embed"][tokens]
        zo.zero_rms_norm(self.x, p["norm1"], EPS, y=self.y1, rstd=self.rstd1)
        self.routed = self.y1 @ p["router"]
        zo.zero_route(self.routed, self.index, self.weight, score="sigmoid", bias=self.bias)
        zo.zero_route_order(self.index, EXPERTS, self.offsets, self.order, self.order_room)
        self.ends = self.offsets.tolist()
        # past the last expert's run are the slots that got no expert (a token whose logits are all NaN has none)
        self.slots = self.order[:self.ends[EXPERTS]].long()
        self.token = self.slots // CHOSEN
        self.ordered = self.y1[self.token]
        self.inner, self.out = [], []
        for e in range(EXPERTS):
            rows = slice(self.ends[e], self.ends[e + 1])
            self.inner.append(torch.relu(self.ordered[rows] @ p["up"][e]))
            self.out.append(self.inner[-1] @ p["down"][e])
        self.out = torch.cat(self.out)
        mixed = torch.zeros(TOKENS, HIDDEN, device=tokens.device)
        mixed.index_add_(0, self.token, self.out.float() * self.weight.view(-1)[self.slots, None])
        zo.zero_rms_norm(mixed.half(), p["norm2"], EPS, residual=self.x, h=self.h2, y=self.y2, q8=self.q8,
                         scale=self.q8_scale, rstd=self.rstd2)
        return self.y2 @ p["head"].t()

    def backward(self, dlogits, tokens):
        p, g = self.p, self.g
        g["head"].copy_(dlogits.t() @ self.y2)
        dy2 = dlogits @ p["head"]
        zo.zero_rms_norm_backward(dy2, self.h2, p["norm2"], self.rstd2, self.dh2, g["norm2"], self.norm_room)
        # the experts: the sum's gradient is the residual's and the mixture's alike
        arrived = self.dh2[self.token]
        w = self.weight.view(-1)[self.slots, None]
        dweight = torch.zeros_like(self.weight)
        dweight.view(-1)[self.slots] = (arrived.float() * self.out.float()).sum(1)
        dout = (arrived.float() * w).half()
        dordered = torch.empty_like(self.ordered)
        for e in range(EXPERTS):
            rows = slice(self.ends[e], self.ends[e + 1])
            g["down"][e].copy_(self.inner[e].t() @ dout[rows])
            dinner = (dout[rows] @ p["down"][e].t()) * (self.inner[e] > 0)
            g["up"][e].copy_(self.ordered[rows].t() @ dinner)
            dordered[rows] = dinner @ p["up"][e].t()
        zo.zero_route_backward(self.routed, self.index, dweight, self.drouted, score="sigmoid", bias=self.bias)
        g["router"].copy_(self.y1.t() @ self.drouted)
        dy1 = (self.drouted @ p["router"].t()).float().index_add_(0, self.token, dordered.float()).half()
        zo.zero_rms_norm_backward(dy1, self.x, p["norm1"], self.rstd1, self.dx, g["norm1"], self.norm_room,
                                  dh=self.dh2)
        dembed = torch.zeros(VOCAB, HIDDEN, device=tokens.device)
        g["embed"].copy_(dembed.index_add_(0, tokens, self.dx.float()))

    def train_step(self, tokens, teacher_index, teacher_logits, labels):
        """(loss, 1 if the step was skipped)."""
        logits = self.forward(tokens)
        # the gradient takes the logits' place
        zo.zero_distill_step(logits, teacher_index, teacher_logits, self.loss, logits, labels=labels, hard=HARD,
                             temperature=TAU, row_weight=self.row_weight, grad_scale=self.scaler.scale)
        loss = self.loss.sum()
        self.backward(logits, tokens)
        skipped = self.step.scaled(self.scaler)
        # experts with less than their share are preferred a little more
        load = self.offsets.diff().float()
        self.bias += BALANCE * torch.sign(load.mean() - load)
        return float(loss), skipped

    def loss_from_e4m3(self, tokens, teacher_index, teacher_logits, labels):
        """The loss with the head fed from the 8-bit rows, as a server would run it."""
        self.forward(tokens)
        rows = (self.q8.float() * self.q8_scale).half()
        zo.zero_distill_loss(rows @ self.p["head"].t(), teacher_index, teacher_logits, self.loss, labels=labels,
                             hard=HARD, temperature=TAU, row_weight=self.row_weight)
        return float(self.loss.sum())


class Teacher:
    """Next-token logits for each token: the top entries of a fixed table."""

    def __init__(self, device, seed=1):
        gen = torch.Generator(device=device).manual_seed(seed)
        u, v = (torch.randn(VOCAB, 16, generator=gen, device=device) for _ in range(2))
        top = torch.topk(u @ v.t(), TOP, dim=1)
        self.logits, self.index = top.values.half(), top.indices.int()
        self.gen = gen

    def batch(self):
        tokens = torch.randint(0, VOCAB, (TOKENS,), generator=self.gen, device=self.logits.device)
        return tokens, self.index[tokens], self.logits[tokens], self.index[tokens, 0].contiguous()


def train(steps, device="cuda", tell=None):
    """The losses of `steps` steps, the number of skipped ones, and the last batch's loss from 8-bit rows."""
    student, teacher = Student(device), Teacher(device)
    losses, skips = [], 0
    for k in range(steps):
        batch = teacher.batch()
        loss, skipped = student.train_step(*batch)
        losses.append(loss)
        skips += skipped
        if tell and (k % 10 == 0 or k == steps - 1):
            tell("step %3d loss %.4f%s" % (k, loss, " (skipped)" if skipped else ""))
    return losses, skips, student.loss_from_e4m3(*batch), student


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    ap.add_argument("--steps", type=int, default=60)
    losses, skips, e4m3, student = train(ap.parse_args().steps, tell=lambda s: print(s, flush=True))
    load = student.offsets.diff().tolist()
    print("skipped %d, loss scale %g, loss from e4m3 rows %.4f, slots of each expert %s"
          % (skips, student.scaler.scale, e4m3, load))
