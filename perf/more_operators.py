"""Cases and plain forms of what stands around the products of an expert layer: the root-mean-square norm with the residual's
addition (rows in 16 or 32 bits, or in 8 bits with scales), the routing of tokens to experts (ids, weights and the rows'
places sorted by expert), and the rows' way to the experts and back, each with its gradients.

A case is a dict of plain values; `op` is "norm", "route" or "rows", `direction` says which call of it.  `run` computes the
plain form in elementary torch operations, or, where `own` is true, calls the library."""
import math

import torch

own = False

EPS = 1e-6


# ------------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # answering 16 tokens in 8 bits: the residual stream moves on, the rows go to a product of 8-bit integers
        dict(name="norm_i8_16_tokens", op="norm", direction="fwd", rows=16, width=1024, x="bf16", residual="bf16", gain=True, out="i8"),
        # a training batch at the width of the classifier's hidden layers
        dict(name="norm_8192", op="norm", direction="fwd", rows=8192, width=4096, x="bf16", residual="bf16", gain=True, out="bf16"),
        # an odd batch at the width of the last layer (1000 classes), the residual stream in float
        dict(name="norm_odd_float", op="norm", direction="fwd", rows=5003, width=1000, x="bf16", residual="f32", gain=True, out="f32"),
        # the training batch's gradients, the residual stream's own gradient added
        dict(name="norm_bwd_8192", op="norm", direction="bwd", rows=8192, width=4096, x="bf16", residual="bf16", gain=True, out="bf16"),
        # gradients of an odd batch, all in float, no residual
        dict(name="norm_bwd_odd_float", op="norm", direction="bwd", rows=4099, width=1001, x="f32", residual="none", gain=True, out="f32"),
        # answering 16 tokens: two of 64 experts each
        dict(name="route_16_tokens", op="route", direction="fwd", tokens=16, behind=0, experts=64, k=2, score="softmax", renormalise=True,
             bias=False, groups=1, top_groups=1, group_best=1, logits="f32"),
        # a padded training batch over many experts: sigmoid scores, a bias for balance, four of eight groups by their two best
        dict(name="route_groups_8192", op="route", direction="fwd", tokens=8150, behind=42, experts=256, k=8, score="sigmoid", renormalise=True,
             bias=True, groups=8, top_groups=4, group_best=2, logits="f32"),
        # its gradients where the weights are plain softmax scores: every logit gets one
        dict(name="route_bwd_8192", op="route", direction="bwd", tokens=8192, behind=0, experts=64, k=2, score="softmax", renormalise=False,
             bias=False, groups=1, top_groups=1, group_best=1, logits="bf16"),
        # a training batch's rows to two of eight experts each
        dict(name="dispatch_8192", op="rows", direction="dispatch", tokens=8192, behind=0, experts=8, k=2, width=4096, x="bf16"),
        # answering 16 tokens: the experts' results and the residual
        dict(name="combine_16_tokens", op="rows", direction="combine", tokens=16, behind=0, experts=64, k=2, width=4096, x="bf16", out="bf16",
             weights=True, residual=True),
        # the training batch's results
        dict(name="combine_8192", op="rows", direction="combine", tokens=8192, behind=0, experts=8, k=2, width=4096, x="bf16", out="bf16",
             weights=True, residual=True),
        # gradients of an odd, padded batch: four of 16 experts each
        dict(name="combine_bwd_odd", op="rows", direction="combine_bwd", tokens=5003, behind=37, experts=16, k=4, width=1000, x="bf16", out="bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    most = max(work(c)["bytes"] for c in listed())
    while True:
        c = _draw(rng)
        if work(c)["bytes"] <= most:
            return c


def _draw(rng):
    op = rng.choice(("norm", "route", "rows"))
    width = _log(rng, 8, 16384)
    if rng.random() < 0.7:
        width = (width + 7) // 8 * 8
    if op == "norm":
        c = dict(op=op, direction=rng.choice(("fwd", "fwd", "bwd")), rows=_log(rng, 1, 32768), width=width, x=rng.choice(("bf16", "f32")),
                 residual=rng.choice(("none", "bf16", "f32")), gain=rng.random() < 0.8)
        return dict(c, out=rng.choice(("bf16", "f32", "i8") if c["direction"] == "fwd" else ("bf16", "f32")))
    c = dict(op=op, tokens=_log(rng, 1, 16384), behind=rng.choice((0, 0, 3, 200)))
    if op == "rows":
        experts = _log(rng, 2, 256)
        c.update(direction=rng.choice(("dispatch", "combine", "combine_bwd")), experts=experts, k=rng.randint(1, min(8, experts)), width=width,
                 x=rng.choice(("bf16", "f32")))
        if c["direction"] == "dispatch":
            return dict(c, x=rng.choice(("bf16", "f32", "i8")))
        c.update(out=rng.choice(("bf16", "f32")))
        return dict(c, weights=rng.random() < 0.7, residual=rng.random() < 0.5) if c["direction"] == "combine" else c
    groups = rng.choice((1, 1, 2, 4, 8))
    experts = groups * _log(rng, 2, 512 // groups)
    top_groups = rng.randint(1, groups)
    return dict(c, direction=rng.choice(("fwd", "fwd", "bwd")), experts=experts, k=rng.randint(1, min(12, top_groups * experts // groups)),
                score=rng.choice(("softmax", "sigmoid")), renormalise=rng.random() < 0.6, bias=rng.random() < 0.5, groups=groups,
                top_groups=top_groups, group_best=rng.choice((1, 2)), logits=rng.choice(("bf16", "f32")))


_SIZE = {"i8": 1.0, "bf16": 2.0, "f32": 4.0, "none": 0.0}


def work(case):
    if case["op"] == "norm":
        n, res = case["rows"] * case["width"], _SIZE[case["residual"]]
        gain = 4.0 * case["width"] if case["gain"] else 0.0
        if case["direction"] == "fwd":
            scales = 4.0 * case["rows"] if case["out"] == "i8" else 0.0
            return {"bytes": n * (_SIZE[case["x"]] + 2.0 * res + _SIZE[case["out"]]) + gain + scales, "flops": 5.0 * n}
        held = res or _SIZE[case["x"]]
        return {"bytes": n * (_SIZE[case["out"]] + held + res + held) + 2.0 * gain, "flops": 10.0 * n}
    T, k = case["tokens"], case["k"]
    if case["op"] == "route":
        n, size = T * case["experts"], _SIZE[case["logits"]]
        if case["direction"] == "fwd":
            return {"bytes": n * size + 12.0 * T * k + 4.0 * case["experts"] * (2 if case["bias"] else 1), "flops": 10.0 * n}
        return {"bytes": n * size * 2.0 + 8.0 * T * k, "flops": 5.0 * n}
    n, size = T * case["width"], _SIZE[case["x"]]
    if case["direction"] == "dispatch":
        scales = 4.0 * T * (1 + k) if case["x"] == "i8" else 0.0
        return {"bytes": n * size * (1 + k) + 4.0 * T * k + scales, "flops": 1.0 * n}
    out = _SIZE[case["out"]]
    if case["direction"] == "combine":
        return {"bytes": n * (size * k + out * (2 if case["residual"] else 1)) + (8.0 if case["weights"] else 4.0) * T * k, "flops": 2.0 * n * k}
    return {"bytes": n * (out + 2.0 * size * k) + 12.0 * T * k, "flops": 3.0 * n * k}


# ------------------------------------------------------------------------------------------------------ inputs
_TYPE = {"i8": torch.int8, "bf16": torch.bfloat16, "f32": torch.float32}


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    s = {"case": case}
    if own:
        from paper_1712_04432_b200 import mbd
        s["mbd"] = mbd
        if case["op"] == "route":
            s["router"] = mbd.Router(case["experts"], case["k"], score=mbd.ROUTE_SOFTMAX if case["score"] == "softmax" else mbd.ROUTE_SIGMOID,
                                     renormalise=case["renormalise"], groups=case["groups"], top_groups=case["top_groups"],
                                     group_best=case["group_best"])

    def normal(*shape, scale=1.0, dtype=torch.float32):
        return (torch.randn(*shape, device="cuda", generator=gen) * scale).to(dtype)

    def empty(*shape, dtype=torch.float32):
        return torch.empty(*shape, dtype=dtype, device="cuda")

    if case["op"] == "norm":
        R, K = case["rows"], case["width"]
        held = _TYPE[case["x"] if case["residual"] == "none" else case["residual"]]
        s["gain"] = 1.0 + normal(K, scale=0.2) if case["gain"] else None
        if case["direction"] == "fwd":
            s["x"] = normal(R, K, scale=0.5, dtype=_TYPE[case["x"]])
            s["residual"] = normal(R, K, scale=2.0, dtype=held) if case["residual"] != "none" else None
            s["h"] = empty(R, K, dtype=held) if case["residual"] != "none" else None
            s["y"] = empty(R, K, dtype=_TYPE[case["out"]])
            s["scale"] = empty(R) if case["out"] == "i8" else None
            return s
        s["h"] = normal(R, K, scale=2.0, dtype=held)
        s["dy"] = normal(R, K, scale=0.01, dtype=_TYPE[case["out"]])
        s["d_residual"] = normal(R, K, scale=0.01, dtype=held) if case["residual"] != "none" else None
        s["dx"], s["d_gain"] = empty(R, K, dtype=held), empty(K) if case["gain"] else None
        return s

    T, k, E = case["tokens"] + case["behind"], case["k"], case["experts"]
    # logits as a router leaves them: some experts liked by all tokens
    logits = normal(T, E, scale=1.5) + normal(E)
    s["count"] = torch.full((1,), case["tokens"], dtype=torch.int32, device="cuda") if case["behind"] else None
    if case["op"] == "route":
        s["logits"] = logits.to(_TYPE[case["logits"]])
        s["bias"] = normal(E, scale=0.05) if case["bias"] else None
        if case["direction"] == "bwd":
            s["ids"] = _choose(case, s["logits"], s["bias"])[0]
            s["ids"][case["tokens"]:] = -1
            s["d_weights"] = normal(T, k, scale=0.1)
            s["d_logits"] = torch.empty_like(s["logits"])
            return s
        s["ids"], s["places"] = empty(T, k, dtype=torch.int32), empty(T, k, dtype=torch.int32)
        s["weights"], s["offsets"] = empty(T, k), empty(E + 1, dtype=torch.int32)
        return s

    K, d = case["width"], case["direction"]
    top, ids = torch.topk(logits, k, dim=1)
    s["places"], _ = _sorted(ids, case["tokens"], E)
    if d == "dispatch":
        s["x"] = torch.randint(-127, 128, (T, K), device="cuda", generator=gen).to(torch.int8) if case["x"] == "i8" else normal(T, K, dtype=_TYPE[case["x"]])
        s["scale"] = normal(T, scale=0.01).abs() if case["x"] == "i8" else None
        s["out_scale"] = normal(T * k) if case["x"] == "i8" else None
        s["out"] = torch.zeros(T * k, K, dtype=_TYPE[case["x"]], device="cuda")
        return s
    s["y"] = normal(T * k, K, dtype=_TYPE[case["x"]])
    s["weights"] = torch.softmax(top, 1) if d == "combine_bwd" or case["weights"] else None
    if d == "combine":
        s["residual"] = normal(T, K, scale=2.0, dtype=_TYPE[case["out"]]) if case["residual"] else None
        s["out"] = empty(T, K, dtype=_TYPE[case["out"]])
        return s
    s["d_out"] = normal(T, K, scale=0.01, dtype=_TYPE[case["out"]])
    s["dy"], s["d_weights"] = torch.zeros_like(s["y"]), empty(T, k)
    return s


# ------------------------------------------------------------------------------------------------------ the operators
def run(s):
    return {"norm": _run_norm, "route": _run_route, "rows": _run_rows}[s["case"]["op"]](s)


def _run_norm(s):
    case = s["case"]
    if case["direction"] == "bwd":
        if own:
            s["mbd"].rms_norm_backward(s["dy"], s["h"], s["dx"], gain=s["gain"], d_residual=s["d_residual"], d_gain=s["d_gain"], eps=EPS)
            return s["dx"], s["d_gain"]
        h, dy = s["h"].float(), s["dy"].float()
        r = torch.rsqrt((h * h).mean(1, keepdim=True) + EPS)
        g = dy * s["gain"] if s["gain"] is not None else dy
        dx = r * g - h * (r * r * r * (g * h).mean(1, keepdim=True))
        if s["d_residual"] is not None:
            dx = dx + s["d_residual"].float()
        s["dx"].copy_(dx)
        if s["gain"] is not None:
            s["d_gain"].copy_((dy * (h * r)).sum(0))
        return s["dx"], s["d_gain"]
    eight = case["out"] == "i8"
    if own:
        to = dict(q=s["y"], scale=s["scale"]) if eight else dict(y=s["y"])
        s["mbd"].rms_norm(s["x"], gain=s["gain"], residual=s["residual"], h=s["h"], eps=EPS, **to)
        return s["h"], s["y"], s["scale"]
    h = s["x"].float()
    if s["residual"] is not None:
        s["h"].copy_(h + s["residual"].float())
        h = s["h"].float()                               # the norm is of the stream as it is stored
    r = torch.rsqrt((h * h).mean(1, keepdim=True) + EPS)
    u = h * s["gain"] if s["gain"] is not None else h
    if eight:
        # the largest value of a row becomes 127; r is the same for the whole row and goes into its scale.  The quotients in 64 bits:
        # many lie next to half a step
        top = u.abs().amax(1) / torch.full((), 127.0, device="cuda")
        q = torch.round(u.double() / top.double().unsqueeze(1))
        s["y"].copy_(torch.where(top.unsqueeze(1) > 0, q, 0.0).clamp(-127.0, 127.0))
        s["scale"].copy_(top * r.squeeze(1))
    else:
        s["y"].copy_(u * r)
    return s["h"], s["y"], s["scale"]


def _choose(case, logits, bias):
    """ids [T, k] and the scores of all experts, in 64 bits: the choice is between values that may lie next to each other."""
    z = logits.double()
    T, E = z.shape
    if case["score"] == "softmax":
        p = torch.exp(z - z.amax(1, keepdim=True))
        p = p / p.sum(1, keepdim=True)
    else:
        p = 1.0 / (1.0 + torch.exp(-z))
    key = z if bias is None else p + bias.double()
    G, best = case["groups"], case["group_best"]
    if G > 1:
        # a group counts by its best expert or the sum of its two best
        in_group = (key if best == 1 or bias is not None else p).view(T, G, E // G)
        of_group = in_group.sort(dim=2, descending=True).values[:, :, :best].sum(2)
        rank = of_group.sort(dim=1, descending=True, stable=True).indices.argsort(1)
        key = torch.where((rank < case["top_groups"]).repeat_interleave(E // G, 1), key, -math.inf)
    return key.sort(dim=1, descending=True, stable=True).indices[:, :case["k"]].to(torch.int32), p


def _sorted(ids, tokens, experts):
    """Places of the slots [T, k] among the rows sorted by expert, in the order of the tokens within one; -1 behind the last
    token.  The experts' first rows [experts + 1]."""
    flat = ids[:tokens].reshape(-1)
    places = torch.full(ids.shape, -1, dtype=torch.int32, device="cuda")
    order = flat.sort(stable=True).indices
    places.view(-1)[order] = torch.arange(flat.numel(), dtype=torch.int32, device="cuda")
    offsets = torch.zeros(experts + 1, dtype=torch.int32, device="cuda")
    offsets[1:] = torch.cumsum((ids[:tokens].reshape(-1, 1) == torch.arange(experts, device="cuda")).sum(0), 0)
    return places, offsets


def _run_route(s):
    case, T = s["case"], s["case"]["tokens"]
    if own:
        if case["direction"] == "bwd":
            s["mbd"].expert_route_backward(s["router"], s["logits"], s["ids"], s["d_weights"], s["d_logits"])
            return s["d_logits"]
        s["mbd"].expert_route(s["router"], s["logits"], s["ids"], s["weights"], s["places"], s["offsets"], bias=s["bias"], count=s["count"])
        return s["ids"], s["weights"], s["places"], s["offsets"]
    if case["direction"] == "fwd":
        ids, p = _choose(case, s["logits"], s["bias"])
        w = p.gather(1, ids.long())
        if case["renormalise"]:
            w = w / w.sum(1, keepdim=True)
        s["ids"].copy_(ids)
        s["weights"].copy_(w)
        s["ids"][T:] = -1
        s["weights"][T:] = 0.0
        places, offsets = _sorted(ids, T, case["experts"])
        s["places"].copy_(places)
        s["offsets"].copy_(offsets)
        return s["ids"], s["weights"], s["places"], s["offsets"]
    z, dw = s["logits"].float(), s["d_weights"]
    there = s["ids"] >= 0
    at = s["ids"].clamp_min(0).long()
    if case["score"] == "softmax":
        p = torch.exp(z - z.amax(1, keepdim=True))
        p = p / p.sum(1, keepdim=True)
    else:
        p = 1.0 / (1.0 + torch.exp(-z))
    chosen = p.gather(1, at)
    if case["renormalise"]:
        total = chosen.sum(1, keepdim=True)
        dw = (dw - (chosen * dw).sum(1, keepdim=True) / total) / total
    dp = torch.zeros_like(z).scatter(1, at, torch.where(there, dw, 0.0))
    dz = p * (dp - (p * dp).sum(1, keepdim=True)) if case["score"] == "softmax" else p * (1.0 - p) * dp
    s["d_logits"].copy_(dz)
    return s["d_logits"]


def _run_rows(s):
    case, T, k, d = s["case"], s["case"]["tokens"], s["case"]["k"], s["case"]["direction"]
    if own:
        if d == "dispatch":
            s["mbd"].expert_dispatch(s["x"], s["places"], s["out"], scale=s["scale"], out_scale=s["out_scale"])
            return s["out"], s["out_scale"]
        if d == "combine":
            return s["mbd"].expert_combine(s["y"], s["places"], s["out"], weights=s["weights"], residual=s["residual"])
        s["mbd"].expert_combine_backward(s["d_out"], s["y"], s["places"], s["weights"], s["dy"], s["d_weights"])
        return s["dy"], s["d_weights"]
    at = s["places"][:T].reshape(-1).long()              # behind the last token there is nothing to bring
    if d == "dispatch":
        s["out"][at] = s["x"][:T].repeat_interleave(k, 0)
        if s["scale"] is not None:
            s["out_scale"][at] = s["scale"][:T].repeat_interleave(k, 0)
        return s["out"], s["out_scale"]
    y = s["y"][at].float().view(T, k, -1)
    if d == "combine":
        if s["weights"] is not None:
            y = y * s["weights"][:T].unsqueeze(2)
        r = torch.zeros(s["out"].shape, device="cuda") if s["residual"] is None else s["residual"].to(torch.float32, copy=True)
        r[:T] += y.sum(1)
        s["out"].copy_(r)
        return s["out"]
    d_out = s["d_out"][:T].float().unsqueeze(1)
    s["dy"][at] = (d_out * s["weights"][:T].unsqueeze(2)).view(T * k, -1).to(s["dy"].dtype)
    s["d_weights"].zero_()
    s["d_weights"][:T] = (d_out * y).sum(2)
    return s["dy"], s["d_weights"]


# ------------------------------------------------------------------------------------------------------ in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    D = torch.float64
    wide = lambda x: None if x is None else x.to(D)  # noqa: E731
    if case["op"] == "norm":
        g = s["gain"].to(D) if s["gain"] is not None else torch.ones(case["width"], dtype=D, device="cuda")
        if case["direction"] == "fwd":
            h = s["x"].to(D)
            if s["residual"] is not None:
                h = (h + s["residual"].to(D))
                held = h.to(torch.float32).to(s["h"].dtype).to(D)        # the sum of two floats, rounded once to the stream's type
            else:
                held = h
            y = held / (held.square().sum(1, keepdim=True) / case["width"] + EPS).sqrt() * g
            scale = y.abs().max(1).values / 127 if case["out"] == "i8" else None
            return (None if s["residual"] is None else h), (None if case["out"] == "i8" else y), scale
        h = s["h"].to(D).requires_grad_()
        g = g.requires_grad_()
        y = h / (h.square().sum(1, keepdim=True) / case["width"] + EPS).sqrt() * g
        dh, dg = torch.autograd.grad(y, (h, g), s["dy"].to(D))
        return dh if s["d_residual"] is None else dh + s["d_residual"].to(D), None if s["gain"] is None else dg
    T, k = case["tokens"], case["k"]
    if case["op"] == "route":
        return _exact_route(case, s)
    places, K, d = s["places"].long(), case["width"], case["direction"]
    if d == "dispatch":
        out, out_scale = s["out"].to(D), wide(s["out_scale"])
        for j in range(k):
            out[places[:T, j]] = s["x"][:T].to(D)
            if out_scale is not None:
                out_scale[places[:T, j]] = s["scale"][:T].to(D)
        return (None if case["x"] == "i8" else out), out_scale
    w = torch.ones(T, k, dtype=D, device="cuda") if s["weights"] is None else s["weights"][:T].to(D)
    if d == "combine":
        out = torch.zeros(T + case["behind"], K, dtype=D, device="cuda") if s["residual"] is None else s["residual"].to(D)
        for j in range(k):
            out[:T] += w[:, j:j + 1] * s["y"][places[:T, j]].to(D)
        return out
    dy, dw = s["dy"].to(D), torch.zeros(T + case["behind"], k, dtype=D, device="cuda")
    for j in range(k):
        dy[places[:T, j]] = w[:, j:j + 1] * s["d_out"][:T].to(D)
        dw[:T, j] = torch.einsum("td,td->t", s["d_out"][:T].to(D), s["y"][places[:T, j]].to(D))
    return dy, dw


def _exact_route(case, s):
    D = torch.float64
    z = s["logits"].to(D)
    T, E, k = case["tokens"], case["experts"], case["k"]
    score = (lambda x: torch.log_softmax(x, 1).exp()) if case["score"] == "softmax" else torch.special.expit

    def weights(x, ids):
        w = score(x).gather(1, ids)
        return w / w.sum(1, keepdim=True) if case["renormalise"] else w

    if case["direction"] == "bwd":
        z.requires_grad_()
        ids = s["ids"].long()
        dw = torch.where(ids >= 0, s["d_weights"].to(D), 0.0)
        return torch.autograd.grad(weights(z, ids.clamp_min(0)), z, dw)[0]
    p = score(z)
    key = p.clone() if s["bias"] is None else p + s["bias"].to(D)
    if case["groups"] > 1:
        member = torch.arange(E, device="cuda") // (E // case["groups"])
        of = []
        for g in range(case["groups"]):
            rest, best = key[:, member == g].clone(), torch.zeros(len(key), dtype=D, device="cuda")
            for _ in range(min(case["group_best"], rest.shape[1])):
                v, i = rest.max(1)
                best += v
                rest.scatter_(1, i[:, None], -math.inf)
            of.append(best)
        of, closed = torch.stack(of, 1), torch.ones(len(key), case["groups"], dtype=torch.bool, device="cuda")
        for _ in range(case["top_groups"]):
            i = of.argmax(1, keepdim=True)
            closed.scatter_(1, i, False)
            of.scatter_(1, i, -math.inf)
        key = key.masked_fill(closed[:, member], -math.inf)
    ids = []
    for _ in range(k):
        ids.append(key.argmax(1, keepdim=True))
        key.scatter_(1, ids[-1], -math.inf)
    w = weights(z, torch.cat(ids, 1))
    w[T:] = 0
    return None, w, None, None
