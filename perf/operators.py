"""The training operators whose speed this framework answers for, each in its plain form and
through the package's public entry points.

Every case is one call, or the calls that belong together, as a training or serving loop
makes them:

  norm         root-mean-square norm with the residual's addition; the sum, the normalised rows
               and, where `group` says so, e4m3 rows with their scales
  norm_back    its gradients
  route        the choice of k experts a token, their weights, and the slots ordered by expert
  route_back   the gradient of the router's logits
  distill      `form` "step": loss and gradient of the logits in one call; "loss": the loss alone, as
               an evaluation takes it; "split": the loss, then the gradient from its statistics

`ld` is the row stride in elements (0: rows lie close together), `lead` the offset of the first
element from an aligned address.
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f16": 2, "bf16": 2}
E4M3_MAX = 448.0
TINY = 2.0 ** -100      # the least magnitude that a scale stands for
EPS = 1e-6
SCALE = 2.0 ** 16       # the loss scale that the gradient carries


def _norm(rows, cols, dtype, residual=True, y=True, group=-1, lead=0, ld=0, **kw):
    """group -1: no 8-bit rows; 0: one scale a row; else one scale for that many columns."""
    return dict(kw, op="norm", rows=rows, cols=cols, dtype=dtype, residual=residual, y=y, group=group, lead=lead,
                ld=ld)


def _norm_back(rows, cols, dtype, stream_grad=True, lead=0, ld=0, **kw):
    return dict(kw, op="norm_back", rows=rows, cols=cols, dtype=dtype, stream_grad=stream_grad, lead=lead, ld=ld)


def _route(op, rows, experts, k, dtype, score, bias=False, groups=1, top_groups=1, renorm=True, scale=1.0, **kw):
    return dict(kw, op=op, rows=rows, experts=experts, k=k, dtype=dtype, score=score, bias=bias, groups=groups,
                top_groups=top_groups, renorm=renorm, scale=scale)


def _distill(form, rows, vocab, k, dtype, tau, hard, lead=0, ld=0, **kw):
    return dict(kw, op="distill", form=form, rows=rows, vocab=vocab, k=k, dtype=dtype, tau=tau, hard=hard, lead=lead,
                ld=ld)


def listed():
    return [
        # one token of a served model of hidden size 8192, rows for 8-bit products: all latency
        _norm(1, 8192, "f16", y=False, group=0, name="norm_token"),
        # a micro-batch of 4 sequences of 1024 through a block of the 1.5B shape (hidden 1600)
        _norm(4096, 1600, "f16", name="norm_4k_1600"),
        # a long prompt batch at hidden 8192, with 8-bit rows in groups of 128 beside the 16-bit ones
        _norm(16384, 8192, "bf16", group=128, name="norm_16k_8192_e4m3"),
        # the gradient of a block of the 13B shape (hidden 4096), residual stream's gradient joined
        _norm_back(8192, 4096, "f16", name="norm_back_8k_4096"),
        # an odd hidden size in 32 bits, no residual stream
        _norm_back(1021, 1603, "f32", stream_grad=False, lead=1, name="norm_back_ragged"),
        # eight tokens being decoded over 64 experts
        _route("route", 8, 64, 6, "bf16", "softmax", renorm=False, name="route_decode"),
        # a training batch over 256 experts in 8 groups, balanced by a bias
        _route("route", 16384, 256, 8, "f32", "sigmoid", bias=True, groups=8, top_groups=4, scale=2.5,
               name="route_16k_256"),
        # its gradient
        _route("route_back", 16384, 256, 8, "f32", "sigmoid", bias=True, groups=8, top_groups=4, scale=2.5,
               name="route_back_16k_256"),
        # a small vocabulary, 37 rows of 32-bit logits: latency
        _distill("step", 37, 2048, 16, "f32", 1.0, 0.0, name="distill_small"),
        # a micro-batch of 4 sequences of 1024 at the vocabulary of 50257, soft and hard terms
        _distill("step", 4096, 50257, 64, "f16", 2.0, 0.5, name="distill_4k_50k"),
        # a large vocabulary, long teacher lists, soft term alone
        _distill("step", 1024, 131072, 128, "bf16", 1.0, 0.0, name="distill_1k_131k"),
        # loss and gradient as two calls, rows padded to whole lines
        _distill("split", 1024, 50257, 32, "bf16", 1.5, 0.0, ld=50304, name="distill_split_1k"),
    ]


def _log(rng, lo, hi):
    return int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))


def draw(rng):
    op = rng.choice(("norm", "norm", "norm_back", "route", "route_back", "distill", "distill"))
    dtype = rng.choice(("f16", "bf16", "f32"))
    if op in ("norm", "norm_back"):
        cols = rng.choice((rng.choice((128, 1600, 4096, 8192, 25600)), _log(rng, 64, 16384)))
        rows = min(_log(rng, 1, 16384), max(1, 134_000_000 // cols // (SIZE[dtype] // 2)))
        lead = rng.choice((0, 0, 0, 1, 3))
        ld = rng.choice((0, 0, cols + rng.choice((1, 8, 64))))
        if op == "norm":
            group = rng.choice((-1, -1, 0, 32, 128))
            return _norm(rows, cols, dtype, rng.random() < 0.7, group < 0 or rng.random() < 0.5, group, lead, ld)
        return _norm_back(rows, cols, dtype, rng.random() < 0.7, lead, ld)
    if op in ("route", "route_back"):
        groups = rng.choice((1, 1, 4, 8))
        experts = groups * max(2, _log(rng, 4, 384) // groups)
        k = rng.randint(1, min(10, experts))
        top = groups if groups == 1 else rng.randint(groups // 2, groups)
        return _route(op, _log(rng, 1, 32768), experts, k, dtype, rng.choice(("softmax", "sigmoid")),
                      rng.random() < 0.5, groups, top, rng.random() < 0.6, rng.choice((1.0, 2.5)))
    vocab = rng.choice((2048, 50257, _log(rng, 1000, 131072)))
    rows = _log(rng, 1, max(2, 100_000_000 // vocab // (SIZE[dtype] // 2)))
    return _distill(rng.choice(("step", "step", "loss", "split")), min(rows, 8192), vocab, rng.randint(1, 128), dtype,
                    rng.choice((1.0, 1.0, 2.0, 1.5)), rng.choice((0.0, 0.5)), rng.choice((0, 0, 1)),
                    rng.choice((0, 0, vocab + 47)))


def _rows(case, dtype, rows, cols, strided=True):
    """An uninitialised [rows, cols] array at the case's lead and stride."""
    lead, ld = (case.get("lead", 0), case.get("ld", 0) or cols) if strided else (0, cols)
    return torch.empty(lead + rows * ld, dtype=dtype, device="cuda")[lead:].view(rows, ld)[:, :cols]


def _normal(case, gen, rows, cols, std, mean=0.0, strided=True, boost=None):
    """Normal numbers in the case's type, drawn in 32 bits a slice of rows at a time."""
    out = _rows(case, TYPES[case["dtype"]], rows, cols, strided)
    step = max(1, (1 << 26) // cols)
    for a in range(0, rows, step):
        t = torch.empty(min(step, rows - a), cols, device="cuda").normal_(mean, std, generator=gen)
        out[a:a + step] = t if boost is None else t.mul_(boost)
    return out


def _norm_inputs(case, gen):
    rows, cols = case["rows"], case["cols"]
    # activations with some channels much larger than the rest, as trained models have them
    boost = torch.where(torch.rand(cols, device="cuda", generator=gen) < 0.01, 20.0, 1.0)
    s = {"w": (1.0 + 0.1 * torch.randn(cols, device="cuda", generator=gen)).to(TYPES[case["dtype"]])}
    if case["op"] == "norm":
        s["x"] = _normal(case, gen, rows, cols, 0.5)
        s["r"] = _normal(case, gen, rows, cols, 1.0, boost=boost) if case["residual"] else None
    else:
        s["h"] = _normal(case, gen, rows, cols, 1.0, boost=boost)
        s["dy"] = _normal(case, gen, rows, cols, 1.0)
        s["dh"] = _normal(case, gen, rows, cols, 1.0) if case["stream_grad"] else None
        hf = s["h"].float()
        s["rstd"] = 1.0 / torch.sqrt((hf * hf).mean(1) + EPS)
    return s


def _route_inputs(case, gen):
    rows, experts, k = case["rows"], case["experts"], case["k"]
    s = {"logits": _normal(case, gen, rows, experts, 1.5), "bias": None}
    if case["bias"]:  # whole steps of the balancing rate
        s["bias"] = torch.randint(-50, 51, (experts,), device="cuda", generator=gen).float() * 1e-3
    if case["op"] == "route_back":
        s["index"], s["weight"] = _route_plain(case, s["logits"], s["bias"])
        s["dweight"] = torch.randn(rows, k, device="cuda", generator=gen)
    return s


def _distill_inputs(case, gen):
    rows, vocab, k = case["rows"], case["vocab"], min(case["k"], case["vocab"])
    dt = TYPES[case["dtype"]]
    z = _normal(case, gen, rows, vocab, 2.0)
    u = torch.rand(rows, k, device="cuda", generator=gen)
    span = vocab // k  # one entry in each, so that a row's entries are distinct
    at = torch.arange(k, device="cuda") * span + (u * span).long().clamp_(max=span - 1)
    # the student agrees with the teacher in the main
    lift = torch.randn(rows, k, device="cuda", generator=gen) * 1.5 + 6.0
    z.scatter_(1, at, (z.gather(1, at).float() + lift).to(dt))
    mix = torch.argsort(torch.rand(rows, k, device="cuda", generator=gen), dim=1)
    tz = torch.sort(torch.randn(rows, k, device="cuda", generator=gen) * 2.0 + 10.0, dim=1, descending=True).values
    idx = at.gather(1, mix).int()
    # some lists are shorter than k
    kept = torch.randint(max(1, k // 2), k + 1, (rows, 1), device="cuda", generator=gen)
    idx[torch.arange(k, device="cuda") >= kept] = -1
    label = at.gather(1, mix)[:, 0].int()
    rare = torch.rand(rows, device="cuda", generator=gen)
    label = torch.where(rare < 0.3, torch.randint(0, vocab, (rows,), device="cuda", generator=gen).int(), label)
    label[rare > 0.95] = -1                      # no hard term there
    w = torch.full((rows,), 1.0 / rows, device="cuda")
    w[torch.rand(rows, device="cuda", generator=gen) < 0.06] = 0.0  # padding
    s = {"z": z, "idx": idx, "tz": tz.to(dt), "label": label if case["hard"] else None, "w": w}
    if case["form"] == "split":
        s["dloss"] = torch.rand(rows, device="cuda", generator=gen) + 0.5
    return s


def _inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    make = _norm_inputs if case["op"].startswith("norm") else _route_inputs if case["op"].startswith("route") else \
        _distill_inputs
    return make(case, gen)


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    op, dt = case["op"], TYPES[case["dtype"]]
    new = lambda shape, dtype: torch.empty(shape, dtype=dtype, device="cuda")  # noqa: E731
    # what a loop keeps from pass to pass: the buffers that its calls write
    if op == "norm":
        rows, cols, g = case["rows"], case["cols"], case["group"]
        s["out"] = {"rstd": new(rows, torch.float32)}
        if case["residual"]:
            s["out"]["h"] = _rows(case, dt, rows, cols)
        if case["y"]:
            s["out"]["y"] = _rows(case, dt, rows, cols, False)
        if g >= 0:
            s["out"]["q8"] = new((rows, cols), torch.float8_e4m3fn)
            s["out"]["scale"] = new((rows, -(-cols // g) if g else 1), torch.float32)
    elif op == "norm_back":
        s["out"] = {"dx": _rows(case, dt, case["rows"], case["cols"]), "dw": torch.empty_like(s["w"])}
        # partial sums of the weight's gradient, in 32 bits: room for the most that the call makes
        s["room"] = new(1024 * case["cols"], torch.float32)
    elif op == "route":
        rows, experts, k = case["rows"], case["experts"], case["k"]
        s["out"] = {"index": new((rows, k), torch.int32), "weight": new((rows, k), torch.float32),
                    "offsets": new(experts + 1, torch.int32), "order": new(rows * k, torch.int32)}
        s["room"] = new(1024 * (experts + 1), torch.int32)
    elif op == "route_back":
        s["out"] = {"dlogits": _rows(case, dt, case["rows"], case["experts"])}
    else:
        s["out"] = {"loss": new(case["rows"], torch.float32)}
        if case["form"] != "loss":
            s["out"]["dz"] = _rows(case, dt, case["rows"], case["vocab"])
        if case["form"] == "split":
            s["stats"] = new((case["rows"], 3), torch.float32)
    return s


# --- the plain forms ---------------------------------------------------------

def _norm_plain(s):
    c, dt = s["case"], TYPES[s["case"]["dtype"]]
    out = {}
    h = s["x"]
    if c["residual"]:
        h = out["h"] = (s["x"].float() + s["r"].float()).to(dt)
    hf = h.float()
    rstd = out["rstd"] = 1.0 / torch.sqrt((hf * hf).mean(1) + EPS)
    y = hf * rstd[:, None] * s["w"].float()
    if c["y"]:
        out["y"] = y.to(dt)
    if c["group"] >= 0:
        cols, g = c["cols"], c["group"] or c["cols"]
        n = -(-cols // g)
        padded = torch.zeros(c["rows"], n * g, device="cuda")
        padded[:, :cols] = y
        cut = padded.view(c["rows"], n, g)
        scale = out["scale"] = cut.abs().amax(2).clamp(min=TINY) / E4M3_MAX
        q = (cut / scale[:, :, None]).clamp(-E4M3_MAX, E4M3_MAX).view(c["rows"], n * g)
        out["q8"] = q[:, :cols].to(torch.float8_e4m3fn)
    return out


def _norm_back_plain(s):
    c, dt = s["case"], TYPES[s["case"]["dtype"]]
    dy, rstd = s["dy"].float(), s["rstd"][:, None]
    n = s["h"].float() * rstd
    g = dy * s["w"].float()
    dx = rstd * (g - n * (g * n).mean(1, keepdim=True))
    if c["stream_grad"]:
        dx = dx + s["dh"].float()
    return {"dx": dx.to(dt), "dw": (dy * n).sum(0).to(dt)}


def _chosen(case, key):
    """The k largest keys of each row, equal ones by the lowest expert; -1 where none is left."""
    groups, rows, experts = case["groups"], key.shape[0], case["experts"]
    if groups > 1:
        best = torch.sort(key.view(rows, groups, -1), dim=2, descending=True, stable=True).values
        score = best[:, :, 0] + best[:, :, 1] if case["score"] == "sigmoid" else best[:, :, 0]
        place = torch.argsort(torch.argsort(score, dim=1, descending=True, stable=True), dim=1)
        stays = (place < case["top_groups"]) & (score > -math.inf)
        key = torch.where(stays.repeat_interleave(experts // groups, 1), key, -math.inf)
    v, i = torch.sort(key, dim=1, descending=True, stable=True)
    v, i = v[:, :case["k"]], i[:, :case["k"]]
    return torch.where(v > -math.inf, i, -1)


def _route_plain(case, logits, bias):
    z = logits.float()
    b = bias if bias is not None else 0.0
    soft = case["score"] == "softmax"
    s = z if soft else 1.0 / (1.0 + torch.exp(-z))
    index = _chosen(case, s + b)
    there = index >= 0
    at = index.clamp(min=0)
    if soft:
        zs = torch.where(there, z.gather(1, at), -math.inf)
        over = zs if case["renorm"] else z
        m = over.amax(1, keepdim=True)
        w = torch.exp(zs - m) / torch.exp(over - m).sum(1, keepdim=True)
    else:
        w = torch.where(there, s.gather(1, at), 0.0)
        if case["renorm"]:
            w = w / w.sum(1, keepdim=True).clamp(min=2.0 ** -126)
    return index.int(), w * case["scale"]


def _route_whole_plain(s):
    c = s["case"]
    index, weight = _route_plain(c, s["logits"], s["bias"])
    flat = torch.where(index < 0, c["experts"], index).view(-1)
    ranked, order = torch.sort(flat, stable=True)
    offsets = torch.searchsorted(ranked, torch.arange(c["experts"] + 1, dtype=torch.int32, device="cuda"))
    order = torch.where(ranked < c["experts"], order, -1)
    return {"index": index, "weight": weight, "offsets": offsets.int(), "order": order.int()}


def _route_back_plain(s):
    c = s["case"]
    z, index, dw = s["logits"].float(), s["index"].long(), s["dweight"] * c["scale"]
    there = index >= 0
    at = index.clamp(min=0)
    dw = torch.where(there, dw, 0.0)
    zs = torch.where(there, z.gather(1, at), -math.inf)
    d = torch.zeros_like(z)
    if c["score"] == "softmax":
        over = zs if c["renorm"] else z
        m = over.amax(1, keepdim=True)
        total = torch.exp(over - m).sum(1, keepdim=True)
        p = torch.exp(zs - m) / total
        mean = (p * dw).sum(1, keepdim=True)
        if not c["renorm"]:
            d = -(torch.exp(z - m) / total) * mean
            return {"dlogits": d.scatter_add(1, at, p * dw).to(s["logits"].dtype)}
        dl = p * (dw - mean)
    else:
        p = torch.where(there, 1.0 / (1.0 + torch.exp(-zs)), 0.0)
        if c["renorm"]:
            total = p.sum(1, keepdim=True).clamp(min=2.0 ** -126)
            dw = (dw - (dw * p).sum(1, keepdim=True) / total) / total
        dl = dw * p * (1.0 - p)
    return {"dlogits": d.scatter_add(1, at, torch.where(there, dl, 0.0)).to(s["logits"].dtype)}


def _distill_plain(s):
    c, tau, hard = s["case"], s["case"]["tau"], s["case"]["hard"]
    z, idx, w = s["z"].float(), s["idx"].long(), s["w"]
    there = (idx >= 0) & (s["tz"] > -math.inf)
    at = idx.clamp(min=0)
    t = torch.where(there, s["tz"].float() / tau, -math.inf)
    any_there = there.any(1, keepdim=True)
    e = torch.where(there, torch.exp(t - torch.where(any_there, t.amax(1, keepdim=True), 0.0)), 0.0)
    p = e / e.sum(1, keepdim=True).clamp(min=2.0 ** -126)
    m = z.amax(1, keepdim=True)
    d = z - m
    x = d / tau
    q = torch.exp(x)
    total = q.sum(1, keepdim=True)
    logq = x.gather(1, at) - torch.log(total)
    term = torch.where(p > 0, p * (torch.log(torch.where(p > 0, p, 1.0)) - logq), 0.0)
    loss = tau * tau * term.sum(1)
    if hard:
        has = s["label"] >= 0
        label = s["label"].long().clamp(min=0)[:, None]
        q1 = torch.exp(d)
        total1 = q1.sum(1, keepdim=True)
        loss = loss + hard * torch.where(has, (torch.log(total1) - d.gather(1, label))[:, 0], 0.0)
    out = {"loss": torch.where(w != 0, w * loss, 0.0)}
    if c["form"] != "loss":
        up = w * SCALE if c["form"] == "step" else w * SCALE * s["dloss"]
        g = torch.where(any_there, q / total * tau, 0.0).scatter_add(1, at, -tau * p)
        if hard:
            g = g + torch.where(has[:, None], hard * (q1 / total1), 0.0)
            g.scatter_add_(1, label, torch.where(has, -hard, 0.0)[:, None])
        out["dz"] = torch.where(w[:, None] != 0, g * up[:, None], 0.0).to(s["z"].dtype)
    return out


PLAIN = {"norm": _norm_plain, "norm_back": _norm_back_plain, "route": _route_whole_plain,
         "route_back": _route_back_plain, "distill": _distill_plain}


# --- the framework's calls ---------------------------------------------------

def _own(s):
    from paper_1910_02054_amd import operators as zo
    c, out = s["case"], s["out"]
    op = c["op"]
    if op == "norm":
        zo.zero_rms_norm(s["x"], s["w"], EPS, residual=s["r"], h=out.get("h"), y=out.get("y"), q8=out.get("q8"),
                         scale=out.get("scale"), group=max(c["group"], 0), rstd=out["rstd"])
    elif op == "norm_back":
        zo.zero_rms_norm_backward(s["dy"], s["h"], s["w"], s["rstd"], out["dx"], out["dw"], s["room"], dh=s["dh"])
    elif op == "route":
        zo.zero_route(s["logits"], out["index"], out["weight"], score=c["score"], bias=s["bias"], groups=c["groups"],
                      top_groups=c["top_groups"], group_top=2 if c["score"] == "sigmoid" else 1,
                      renormalise=c["renorm"], scale=c["scale"])
        zo.zero_route_order(out["index"], c["experts"], out["offsets"], out["order"], s["room"])
    elif op == "route_back":
        zo.zero_route_backward(s["logits"], s["index"], s["dweight"], out["dlogits"], score=c["score"],
                               bias=s["bias"], renormalise=c["renorm"], scale=c["scale"])
    else:
        terms = dict(labels=s["label"], hard=c["hard"], temperature=c["tau"], row_weight=s["w"])
        if c["form"] == "step":
            zo.zero_distill_step(s["z"], s["idx"], s["tz"], out["loss"], out["dz"], grad_scale=SCALE, **terms)
        else:
            zo.zero_distill_loss(s["z"], s["idx"], s["tz"], out["loss"], stats=s.get("stats"), **terms)
        if c["form"] == "split":
            zo.zero_distill_backward(s["z"], s["idx"], s["tz"], s["stats"], out["dz"], dloss=s["dloss"],
                                     grad_scale=SCALE, **terms)
    return out


def run(state):
    return _own(state) if own else PLAIN[state["case"]["op"]](state)


def work(case):
    op, b = case["op"], SIZE[case["dtype"]]
    rows = case["rows"]
    if op == "norm":
        n, g = rows * case["cols"], case["group"]
        arrays = 1 + 2 * case["residual"] + case["y"]  # x, the residual and the sum, the output
        scales = rows * (-(-case["cols"] // g) if g else 1) * 4 if g >= 0 else 0
        return {"bytes": n * (arrays * b + (g >= 0)) + scales + 4 * rows + case["cols"] * b, "flops": 6.0 * n}
    if op == "norm_back":
        n = rows * case["cols"]
        return {"bytes": n * (3 + case["stream_grad"]) * b + 4 * rows + 2 * case["cols"] * b, "flops": 10.0 * n}
    if op == "route":
        slots = rows * case["k"]
        # logits; indices and weights written; the indices' order written
        return {"bytes": rows * case["experts"] * b + 12 * slots + 4 * (case["experts"] + 1),
                "flops": 8.0 * rows * case["experts"]}
    if op == "route_back":
        slots = rows * case["k"]
        read = rows * case["experts"] * b if case["score"] == "softmax" and not case["renorm"] else slots * b
        return {"bytes": rows * case["experts"] * b + read + 8 * slots, "flops": 2.0 * rows * case["experts"]}
    n, k = rows * case["vocab"], min(case["k"], case["vocab"])
    passes = {"step": 2, "loss": 1, "split": 3}[case["form"]]
    return {"bytes": n * passes * b + rows * k * (4 + b) + 12 * rows, "flops": (5.0 if passes == 1 else 10.0) * n}


# --- the definition in 64 bits -----------------------------------------------

def _exact_norm(case, s):
    dt = TYPES[case["dtype"]]
    x = s["x"].double()
    out = {}
    if case["residual"]:
        out["h"] = x + s["r"].double()
        x = out["h"].to(dt).double()
    out["rstd"] = (x.square().mean(dim=1) + EPS).rsqrt()
    y = torch.einsum("tc,t,c->tc", x, out["rstd"], s["w"].double())
    if case["y"]:
        out["y"] = y
    g = case["group"]
    if g >= 0:
        parts = y.split(g or case["cols"], dim=1)
        out["scale"] = torch.stack([p.abs().max(dim=1).values.clamp(min=TINY) / E4M3_MAX for p in parts], dim=1)
        out["q8"] = torch.cat([p / out["scale"][:, i:i + 1] for i, p in enumerate(parts)], dim=1)
    return out


def _exact_norm_back(case, s):
    h, dy, w = s["h"].double(), s["dy"].double(), s["w"].double()
    n = case["cols"]
    inv = s["rstd"].double()
    # d/dh of (h inv) w with inv = (mean h^2 + eps)^(-1/2): inv w dy - inv^3 h <w dy, h> / n
    along = (h * dy * w).sum(1) * inv.pow(3) / n
    dx = dy * w * inv[:, None] - h * along[:, None]
    if s["dh"] is not None:
        dx += s["dh"].double()
    return {"dx": dx, "dw": (dy * h * inv[:, None]).sum(0)}


def _exact_choice(case, key):
    rows, experts = key.shape
    if case["groups"] > 1:
        per = experts // case["groups"]
        two = key.view(rows, case["groups"], per).topk(2 if case["score"] == "sigmoid" else 1, dim=2).values.sum(2)
        keep = torch.zeros_like(two, dtype=torch.bool).scatter_(1, two.topk(case["top_groups"], dim=1).indices, True)
        key = key.masked_fill(~keep.repeat_interleave(per, 1), -math.inf)
    got = key.topk(case["k"], dim=1)
    return got.indices.masked_fill(got.values == -math.inf, -1)


def _exact_weights(case, z, index):
    none, at = index < 0, index.clamp(min=0)
    if case["score"] == "softmax":
        if case["renorm"]:
            return torch.softmax(z.gather(1, at).masked_fill(none, -math.inf), 1)
        return torch.softmax(z, 1).gather(1, at).masked_fill(none, 0.0)
    w = torch.sigmoid(z.gather(1, at)).masked_fill(none, 0.0)
    return w / w.sum(1, keepdim=True) if case["renorm"] else w


def _exact_route(case, s):
    z = s["logits"].double()
    score = torch.sigmoid(z) if case["score"] == "sigmoid" else z
    key = score + s["bias"].double() if s["bias"] is not None else score
    return {"index": None, "offsets": None, "order": None,
            "weight": case["scale"] * _exact_weights(case, z, _exact_choice(case, key))}


def _exact_route_back(case, s):
    with torch.enable_grad():
        z = s["logits"].double().requires_grad_(True)
        w = case["scale"] * _exact_weights(case, z, s["index"].long())
        return {"dlogits": torch.autograd.grad((w * s["dweight"].double()).sum(), z)[0]}


def _exact_distill(case, s):
    tau, hard, rows = case["tau"], case["hard"], case["rows"]
    loss = torch.zeros(rows, dtype=torch.float64, device="cuda")
    dz = torch.zeros(rows, case["vocab"], dtype=torch.float64, device="cuda") if case["form"] != "loss" else None
    step = max(1, (1 << 27) // case["vocab"])
    for a in range(0, rows, step):
        b = slice(a, min(rows, a + step))
        z = s["z"][b].double()
        absent = (s["idx"][b] < 0) | (s["tz"][b] == -math.inf)
        lp = torch.log_softmax((s["tz"][b].double() / tau).masked_fill(absent, -math.inf), 1)
        lp = lp.masked_fill(absent, -math.inf).nan_to_num(nan=-math.inf)
        p, at = lp.exp(), s["idx"][b].long().clamp(min=0)
        lq = torch.log_softmax(z / tau, 1)
        each = (p * (lp - lq.gather(1, at))).masked_fill(p == 0, 0.0)
        part = tau ** 2 * each.sum(1)
        g = lq.exp() * (tau * p.sum(1, keepdim=True))
        g.scatter_add_(1, at, -tau * p)
        if hard:
            l1 = torch.log_softmax(z, 1)
            has = (s["label"][b] >= 0).double()[:, None]
            label = s["label"][b].long().clamp(min=0)[:, None]
            part = part - hard * (l1.gather(1, label) * has)[:, 0]
            g += hard * has * l1.exp()
            g.scatter_add_(1, label, -hard * has)
        w = s["w"][b].double()
        loss[b] = part * w
        if dz is not None:
            up = w * SCALE * (s["dloss"][b].double() if "dloss" in s else 1.0)
            dz[b] = g * up[:, None]
    return {"loss": loss, "dz": dz}


EXACT = {"norm": _exact_norm, "norm_back": _exact_norm_back, "route": _exact_route, "route_back": _exact_route_back,
         "distill": _exact_distill}


def exact(case, seed):
    out = EXACT[case["op"]](case, _inputs(case, seed))
    return {k: v for k, v in out.items() if v is not None or k in ("index", "offsets", "order")}
