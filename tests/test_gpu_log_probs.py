"""zero_log_probs and its gradient on the GPU against plain 64-bit implementations (log_prob_checks.py): sizes, types,
lists of every length, ties, masks, strides, graphs, and the teacher's list that the distillation takes."""
import math
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import log_prob_checks as L  # noqa: E402
import operator_checks as C  # noqa: E402
from test_gpu_operators import Out, put  # noqa: E402

pytestmark = pytest.mark.gpu
F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def zo():
    from paper_1910_02054_amd import operators
    assert torch.cuda.is_available()
    return operators


def logits(rows, vocab, dtype, seed, std=2.0):
    g = C.rng(seed, rows, vocab)
    z = C.normal(g, rows, vocab, std=std).to(dtype)
    tokens = torch.randint(0, vocab, (rows,), generator=g).int()
    if rows > 2:
        tokens[1], tokens[2] = -1, vocab
    return z, tokens


def check(zo, z, tokens, k, tau=1.0, pad=0, lead=0):
    rows, vocab = z.shape
    want = L.log_probs(z, tokens, k, tau)
    o = {n: Out(rows, 1, F32) for n in ("logp", "entropy")}
    o["stats"] = Out(rows, 3, F32)
    if k:
        o["top_index"], o["top_logp"] = Out(rows, k, torch.int32), Out(rows, k, F32)
    zo.zero_log_probs(put(z, pad, lead), tokens.cuda(), o["logp"].view, temperature=tau,
                      **{n: t.view for n, t in o.items() if n != "logp"})
    torch.cuda.synchronize()
    assert all(t.guards_intact() for t in o.values())
    for n in ("logp", "entropy"):
        C.within(o[n].view[:, 0], want[n][0], C.rounded(want[n][1], want[n][0].nan_to_num(nan=0.0, neginf=0.0), F32), n)
    C.within(o["stats"].view, want["stats"][0], C.rounded(want["stats"][1], want["stats"][0].nan_to_num(
        nan=0.0, posinf=0.0, neginf=0.0), F32), "stats")
    if k:
        assert torch.equal(o["top_index"].view.cpu().long(), want["top_index"])
        v, b = want["top_logp"]
        C.within(o["top_logp"].view, v, C.rounded(b, v.nan_to_num(nan=0.0, neginf=0.0), F32), "top_logp")
    return o


@pytest.mark.parametrize("dtype", C.TYPES)
@pytest.mark.parametrize("rows,vocab", ((1, 1), (3, 2), (4, 17), (5, 128), (3, 1000), (4, 1031), (3, 2048), (2, 5000), (3, 8193),
                                        (2, 20000), (3, 50257), (2, 65540), (2, 131072), (1, 150001)))
def test_sizes(zo, rows, vocab, dtype):
    z, tokens = logits(rows, vocab, dtype, 3)
    for k, tau, pad, lead in ((0, 1.0, 0, 0), (1, 0.7, 3, 1), (20, 2.0, 0, 0), (128, 1.0, 8, 0)):
        check(zo, z, tokens, k, tau, pad, lead)


@pytest.mark.parametrize("dtype", C.TYPES)
@pytest.mark.parametrize("k", (2, 63, 64, 65, 300, 511, 512, 513, 1000, 1024))
def test_lists(zo, k, dtype):
    for rows, vocab in ((2, 900), (3, 4000), (2, 30000)):
        z, tokens = logits(rows, vocab, dtype, 5)
        check(zo, z, tokens, k)


@pytest.mark.parametrize("dtype", C.TYPES)
def test_ties_and_sorted_rows(zo, dtype):
    """Equal logits by the lowest token, where more of them than the room for candidates stand at the list's end,
    too; rows in rising and falling order, whose largest logits lie side by side."""
    vocab = 9000
    z, tokens = logits(8, vocab, dtype, 7)
    z[0] = 1.0
    z[1] = (z[1].float() * 2).round().to(dtype) / 2
    z[2] = torch.where(torch.arange(vocab) % 3 == 0, 3.0, -1.0)
    z[3], z[4] = z[3].sort().values, z[4].sort(descending=True).values
    z[5] = 0.0
    z[5, 1::2] = -0.0
    z[6] = torch.where(torch.arange(vocab) < 4000, 2.0, z[6].float().clamp(max=2.0)).to(dtype)
    for k in (1, 20, 128, 700):
        check(zo, z, tokens, k)


@pytest.mark.parametrize("dtype", C.TYPES)
@pytest.mark.parametrize("vocab", (300, 6000, 140000))
def test_masks(zo, vocab, dtype):
    inf, low = math.inf, torch.finfo(dtype).min
    z, _ = logits(12, vocab, dtype, 9)
    z[0] = -inf                      # nothing is left
    z[1, 5:] = -inf                  # five are
    z[2] = low
    z[3, ::2] = low
    z[4, vocab // 2] = math.nan
    z[5, 7] = inf
    z[6, 1:] = -inf                  # one is: probability 1, entropy 0
    z[7] = math.nan
    z[8] = -inf
    z[8, 250] = low
    z[9] = torch.finfo(dtype).max
    z[10, 3] = torch.finfo(dtype).max
    tokens = torch.tensor([4, 4, 9, 0, 1, 7, 0, 0, 250, 17, 3, -5], dtype=torch.int32)
    for tau in (1.0, 0.01, 1e3):
        o = check(zo, z, tokens, 10, tau)
        assert o["logp"].view[0].item() == -inf and o["entropy"].view[0].item() == 0
        assert o["logp"].view[6].item() == 0 and o["entropy"].view[6].item() == 0
        assert (o["top_index"].view[0] == -1).all() and (o["top_index"].view[7] == -1).all()
    masked = tokens.clone()
    masked[1], masked[6] = 200, 12  # tokens that the mask has taken
    check(zo, z, masked, 0)


@pytest.mark.parametrize("tau", (1e-30, 1e-6, 1e6, 1e30))
def test_temperatures(zo, tau):
    for dtype in C.TYPES:
        z, tokens = logits(4, 3000, dtype, 11)
        z[0] = 0.0
        want = L.log_probs(z, tokens, 5, tau)
        out = {n: torch.empty(4, device="cuda") for n in ("logp", "entropy")}
        top = torch.empty(4, 5, dtype=torch.int32, device="cuda"), torch.empty(4, 5, device="cuda")
        zo.zero_log_probs(z.cuda(), tokens.cuda(), out["logp"], entropy=out["entropy"], top_index=top[0], top_logp=top[1],
                          temperature=tau)
        assert torch.equal(top[0].cpu().long(), want["top_index"])
        for n in out:
            C.within(out[n], want[n][0], want[n][1] + 8 * C.U * want[n][0].abs(), n)


@pytest.mark.parametrize("dtype", C.TYPES)
@pytest.mark.parametrize("rows,vocab", ((1, 1), (3, 5), (5, 128), (4, 1031), (2, 8193), (3, 50257), (1, 150001)))
def test_backward(zo, rows, vocab, dtype):
    z, tokens = logits(rows, vocab, dtype, 13)
    g = C.rng(17, rows)
    dlogp, dent = C.normal(g, rows).float(), C.normal(g, rows).float()
    for tau, scale, which, pad, lead in ((1.0, 1.0, "both", 0, 0), (0.7, 64.0, "logp", 3, 1), (2.0, 8.0, "entropy", 8, 0)):
        stats = L.log_probs(z, tokens, 0, tau)["stats"][0].float()
        a, b = dlogp if which != "entropy" else None, dent if which != "logp" else None
        want, bound = L.backward(z, tokens, a, b, tau, scale)
        out = Out(rows, vocab, dtype, pad, lead)
        dz = put(z, pad, lead)
        kw = dict(dlogp=None if a is None else a.cuda(), dentropy=None if b is None else b.cuda(), temperature=tau,
                  grad_scale=scale)
        zo.zero_log_probs_backward(dz, tokens.cuda(), stats.cuda(), out.view, **kw)
        torch.cuda.synchronize()
        assert out.guards_intact()
        C.within(out.view, want, C.rounded(bound, want, dtype), "dlogits")
        zo.zero_log_probs_backward(dz, tokens.cuda(), stats.cuda(), dz, **kw)  # in place
        assert torch.equal(dz, out.view)


@pytest.mark.parametrize("dtype", C.TYPES)
def test_backward_of_masked_rows(zo, dtype):
    inf, low = math.inf, torch.finfo(dtype).min
    z, _ = logits(6, 700, dtype, 19)
    z[0] = -inf
    z[1, 3:] = -inf
    z[2, ::2] = low
    z[3] = low
    z[4, 9] = math.nan
    tokens = torch.tensor([4, 1, 2, 5, 3, 700], dtype=torch.int32)
    stats = torch.empty(6, 3, device="cuda")
    zo.zero_log_probs(z.cuda(), None, None, stats=stats)
    d = torch.ones(6)
    want, bound = L.backward(z, tokens, d, d, 1.0, 1.0)
    out = torch.empty(6, 700, dtype=dtype, device="cuda")
    zo.zero_log_probs_backward(z.cuda(), tokens.cuda(), stats, out, dlogp=d.cuda(), dentropy=d.cuda())
    # the statistics are the kernel's own here: their error is that of the sums
    x, p, log_sum, _ = L.parts(z, 1.0)
    extra = torch.where(p > 0, 100 * C.U * p * (torch.where(p > 0, x.abs(), 0.0) + log_sum.abs() + 2), 0.0)
    extra = extra.nan_to_num(nan=0.0)
    C.within(out, want, C.rounded(bound + extra, want.nan_to_num(nan=0.0), dtype), "dlogits")
    assert (out[0] == 0).all() and torch.isnan(out[4]).all()


def test_gradient_against_differences(zo):
    """d (sum a logp + b entropy) / dz by central differences of the fp32 forward: step 2^-6, whose curvature term and
    rounding (2^-24 * 40 / 2^-6) stay under 2e-3."""
    z, tokens = logits(3, 60, F32, 23, std=1.0)
    tokens = torch.tensor([3, 59, 20], dtype=torch.int32)
    a, b = torch.tensor([1.0, -0.5, 0.7]), torch.tensor([0.3, 1.0, -2.0])
    lp, h, stats = torch.empty(3, device="cuda"), torch.empty(3, device="cuda"), torch.empty(3, 3, device="cuda")

    def value(z):
        zo.zero_log_probs(z.cuda(), tokens.cuda(), lp, entropy=h, temperature=0.8, stats=stats)
        return float((lp.cpu().double() * a + h.cpu().double() * b).sum())

    value(z)
    dz = torch.empty(3, 60, device="cuda")
    zo.zero_log_probs_backward(z.cuda(), tokens.cuda(), stats, dz, dlogp=a.cuda(), dentropy=b.cuda(), temperature=0.8)
    step = 2.0 ** -6
    for at in ((0, 3), (1, 0), (2, 20), (0, 59)):
        d = torch.zeros_like(z)
        d[at] = step
        assert abs((value(z + d) - value(z - d)) / (2 * step) - dz[at].item()) < 2e-3


def test_partial_outputs_and_no_rows(zo):
    # of the same array: where a row lies decides the order of its sums
    z, tokens = (t.cuda() for t in logits(4, 500, F16, 29))
    new = lambda *s, t=F32: torch.empty(*s, dtype=t, device="cuda")  # noqa: E731
    full = new(4), new(4), new(4, 7, t=torch.int32), new(4, 7)
    zo.zero_log_probs(z, tokens, full[0], entropy=full[1], top_index=full[2], top_logp=full[3])
    one, ti, tl = new(4), new(4, 7, t=torch.int32), new(4, 7)
    zo.zero_log_probs(z, None, None, entropy=one)
    assert torch.equal(one, full[1])
    zo.zero_log_probs(z, tokens, one)
    assert torch.equal(one, full[0])
    zo.zero_log_probs(z.view(2, 2, 500), None, None, top_index=ti, top_logp=tl)
    assert torch.equal(ti, full[2]) and torch.equal(tl, full[3])
    none = torch.empty(0, 500, dtype=F16, device="cuda")
    nothing = torch.empty(0, dtype=torch.int32, device="cuda")
    zo.zero_log_probs(none, nothing, torch.empty(0, device="cuda"))
    zo.zero_log_probs_backward(none, nothing, torch.empty(0, 3, device="cuda"), none.clone(),
                               dlogp=torch.empty(0, device="cuda"))


def test_lists_for_the_distillation(zo):
    """A teacher's list goes into zero_distill_step as it is: with the whole vocabulary listed the loss against the
    student's own logits is that of its log probabilities, 0, and its gradient too; padded entries are absent."""
    z, _ = logits(5, 40, F32, 31)
    z[3, 10:] = -math.inf
    index, lp = torch.empty(5, 40, dtype=torch.int32, device="cuda"), torch.empty(5, 40, device="cuda")
    zd = z.cuda()
    zo.zero_log_probs(zd, None, None, top_index=index, top_logp=lp)
    loss, dz = torch.empty(5, device="cuda"), torch.empty(5, 40, device="cuda")
    zo.zero_distill_step(zd, index, lp, loss, dz)
    assert (index[3, 10:] == -1).all()
    assert loss.abs().max() < 1e-5 and dz.abs().max() < 1e-5  # 40 terms of 2^-24, and logarithms of up to 8


@pytest.mark.parametrize("dtype", (F16, F32))
def test_graph_and_stream(zo, dtype):
    z, tokens = logits(6, 20000, dtype, 37)
    z, tokens = z.cuda(), tokens.cuda()
    new = lambda *s, t=F32: torch.zeros(*s, dtype=t, device="cuda")  # noqa: E731
    lp, h, ti, tl, st, dz = new(6), new(6), new(6, 30, t=torch.int32), new(6, 30), new(6, 3), torch.zeros_like(z)

    def go():
        zo.zero_log_probs(z, tokens, lp, entropy=h, top_index=ti, top_logp=tl, stats=st, temperature=0.9)
        zo.zero_log_probs_backward(z, tokens, st, dz, dlogp=lp, dentropy=h, temperature=0.9, grad_scale=4.0)

    outs = (lp, h, ti, tl, st, dz)
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        go()
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            go()
        for turn in range(4):
            z.mul_(0.8)
            go()
            want = [o.clone() for o in outs]
            for o in outs:
                o.zero_()
            graph.replay()
            stream.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(want, outs)), turn


def test_rows_past_one_launch_and_offsets_past_32_bits(zo):
    n = (1 << 20) + 3
    z = torch.randn(n, 8, device="cuda", dtype=F16)
    tokens = torch.randint(0, 8, (n,), device="cuda", dtype=torch.int32)
    lp, ti, tl = torch.empty(n, device="cuda"), torch.empty(n, 1, dtype=torch.int32, device="cuda"), torch.empty(n, 1, device="cuda")
    st, dz = torch.empty(n, 3, device="cuda"), torch.empty_like(z)
    zo.zero_log_probs(z, tokens, lp, top_index=ti, top_logp=tl, stats=st)
    want = torch.log_softmax(z.float(), 1)
    assert (lp - want.gather(1, tokens.long()[:, None])[:, 0]).abs().max() < 1e-5
    assert torch.equal(z.gather(1, ti.long()), z.amax(1, keepdim=True))
    zo.zero_log_probs_backward(z, tokens, st, dz, dlogp=torch.ones(n, device="cuda"))
    g = -want.exp()
    g.scatter_add_(1, tokens.long()[:, None], torch.ones(n, 1, device="cuda"))
    assert (dz.float() - g).abs().max() < 1e-3
    ld, rows = (1 << 31) + 64, 3
    buf = torch.zeros((rows - 1) * ld + 2048, dtype=F16, device="cuda")
    x, y = torch.as_strided(buf, (rows, 1000), (ld, 1)), torch.as_strided(buf, (rows, 1000), (ld, 1), 1024)
    x.copy_(torch.randn(rows, 1000, device="cuda"))
    t3, st3 = torch.tensor([1, 999, 5], dtype=torch.int32, device="cuda"), torch.empty(3, 3, device="cuda")
    zo.zero_log_probs(x, t3, lp[:3], stats=st3)
    want = torch.log_softmax(x.float(), 1)
    assert (lp[:3] - want.gather(1, t3.long()[:, None])[:, 0]).abs().max() < 1e-5
    zo.zero_log_probs_backward(x, t3, st3, y, dlogp=torch.ones(3, device="cuda"))
    g = -want.exp()
    g.scatter_add_(1, t3.long()[:, None], torch.ones(3, 1, device="cuda"))
    assert (y.float() - g).abs().max() < 1e-3
