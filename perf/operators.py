"""Cases and plain forms of the operators an expert layer needs beside the dense ones: its three products grouped by
expert (forward, backward-data, backward-weight on ragged groups of rows), the AdamW step over all of a network's
tensors with moments in 32 or 8 bits, and the products of 8-bit integers that answer with the trained weights.

A case is a dict of plain values; `op` is "expert" (direction 0 / 1 / 2), "adamw" or "i8".  `run` computes the plain
form in elementary torch operations, or, where `own` is true, calls the library."""
import math

import torch

own = False

BLOCK = 256          # moments in 8 bits share one scale per so many consecutive elements of a tensor
E4M3_MAX = 448.0
E4M3_MIN = 2.0 ** -9
LR, BETA1, BETA2, EPS, DECAY = 1e-3, 0.9, 0.999, 1e-8, 0.01
T0 = 100             # steps taken before the first one here


# ------------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # answering 16 tokens, each sent to two of 64 experts: the weights of the touched experts are all the traffic
        dict(name="expert_fwd_16_tokens", op="expert", direction=0, experts=64, rows=32, behind=0, d_in=1024, d_out=4096,
             skew=0.5, relu=True, bias=True, out="bf16"),
        # a training batch through the hidden layer of the classifier (4096 -> 4096), as 8 experts
        dict(name="expert_fwd_8192", op="expert", direction=0, experts=8, rows=8192, behind=0, d_in=4096, d_out=4096,
             skew=0.3, relu=True, bias=True, out="bf16"),
        # the gradient that leaves the last layer (1000 classes) downwards, through the stored ReLU, padded batch
        dict(name="expert_bwd_data_ragged", op="expert", direction=1, experts=16, rows=5003, behind=37, d_in=4096, d_out=1000,
             skew=0.8, mask=True, out="bf16"),
        # the hidden layer's weight gradients, float as every weight gradient of the library
        dict(name="expert_bwd_weight_8192", op="expert", direction=2, experts=8, rows=8192, behind=0, d_in=4096, d_out=4096,
             skew=0.3, out="f32"),
        # many small experts, some without a row, one with most of them
        dict(name="expert_bwd_weight_skewed", op="expert", direction=2, experts=64, rows=4099, behind=5, d_in=1000, d_out=1024,
             skew=2.0, out="f32"),
        # the smallest network (784-512-512-10, float): six tensors, latency
        dict(name="adamw_small_f32", op="adamw", net="784,512,512,10", copies=1, param="f32", grad="f32", bits=32),
        # the classifier stack (9216-4096-4096-1000), bf16 weights with float masters
        dict(name="adamw_master_32bit", op="adamw", net="9216,4096,4096,1000", copies=1, param="bf16+master", grad="f32", bits=32),
        # the same with moments in 8 bits
        dict(name="adamw_master_8bit", op="adamw", net="9216,4096,4096,1000", copies=1, param="bf16+master", grad="f32", bits=8),
        # many tensors of odd sizes, bf16 weights alone and gradients in bf16
        dict(name="adamw_odd_8bit", op="adamw", net="1160,521,393,1001", copies=40, param="bf16", grad="bf16", bits=8),
        # answering 16 tokens with the first layer of the classifier
        dict(name="i8_16_tokens", op="i8", experts=0, rows=16, behind=0, d_in=9216, d_out=4096, skew=0.0, relu=True, bias=True,
             x="bf16", out="bf16"),
        # a batch of 8192 through a square layer
        dict(name="i8_8192", op="i8", experts=0, rows=8192, behind=0, d_in=8192, d_out=8192, skew=0.0, relu=False, bias=False,
             x="bf16", out="bf16"),
        # 8-bit experts on a ragged, padded batch
        dict(name="i8_experts_ragged", op="i8", experts=16, rows=5003, behind=37, d_in=4096, d_out=1000, skew=0.8, relu=False,
             bias=True, x="bf16", out="f32"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("expert", "expert", "adamw", "i8"))
    if op == "adamw":
        weights = 2 ** 30
        while weights > 50_000_000:
            dims = [_log(rng, 10, 9216) for _ in range(rng.randint(2, 4))]
            weights = sum(a * b + b for a, b in zip(dims, dims[1:]))
        return dict(op=op, net=",".join(map(str, dims)), copies=_log(rng, 1, max(1, min(60, 50_000_000 // weights))),
                    param=rng.choice(("f32", "bf16", "bf16+master")), grad=rng.choice(("f32", "bf16")), bits=rng.choice((32, 8)))
    step = 8 if op == "expert" else 16
    while True:
        rows, experts = _log(rng, 1, 16384), _log(rng, 1, 128)
        d_in, d_out = step * _log(rng, 2, 9216 // step), 8 * _log(rng, 1, 9216 // 8)
        if op == "i8" and rng.random() < 0.5:
            experts = 0
        if max(1, experts) * d_in * d_out <= 2 ** 28 and rows * d_in * d_out <= 2 ** 37:
            break
    c = dict(op=op, experts=experts, rows=rows, behind=rng.choice((0, 3, 200)), d_in=d_in, d_out=d_out, skew=rng.choice((0.0, 0.5, 1.0, 2.0)))
    if op == "i8":
        if not experts:
            c["behind"] = 0
        return dict(c, relu=rng.random() < 0.5, bias=rng.random() < 0.5, x=rng.choice(("bf16", "f32")), out=rng.choice(("bf16", "f32")))
    c["direction"] = rng.randrange(3)
    if c["direction"] == 0:
        c.update(relu=rng.random() < 0.5, bias=rng.random() < 0.5)
    if c["direction"] == 1:
        c.update(mask=rng.random() < 0.5)
    return dict(c, out=rng.choice(("bf16", "f32")))


def _shapes(case):
    dims = [int(d) for d in case["net"].split(",")]
    one = [s for a, b in zip(dims, dims[1:]) for s in ((b, a), (b,))]
    return one * case["copies"]


def work(case):
    if case["op"] == "adamw":
        n = sum(math.prod(s) for s in _shapes(case))
        moments = 16.0 if case["bits"] == 32 else 4.0 + 16.0 / BLOCK
        weights = {"f32": 8.0, "bf16": 4.0, "bf16+master": 10.0}[case["param"]]
        return {"bytes": n * (moments + weights + (4.0 if case["grad"] == "f32" else 2.0)), "flops": 20.0 * n}
    E, T, a, b = max(1, case["experts"]), case["rows"], case["d_in"], case["d_out"]
    touched = E * (1.0 - (1.0 - 1.0 / E) ** T)          # experts that get a row, were they equally likely
    out = 2.0 if case["out"] == "bf16" else 4.0
    flops = 2.0 * T * a * b
    if case["op"] == "i8":
        x = 2.0 if case["x"] == "bf16" else 4.0
        return {"bytes": T * a * (x + 1.0) + 4.0 * T + touched * (b * a + 4.0 * b) + T * b * out, "flops": flops}
    if case["direction"] == 0:
        return {"bytes": 2.0 * T * a + 2.0 * touched * a * b + out * T * b, "flops": flops}
    if case["direction"] == 1:
        return {"bytes": 2.0 * T * b + 2.0 * touched * a * b + out * T * a * (2.0 if case["mask"] else 1.0), "flops": flops}
    return {"bytes": 2.0 * T * (a + b) + out * E * a * b, "flops": flops}


# ------------------------------------------------------------------------------------------------------ inputs
def _type(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _groups(gen, experts, rows, skew):
    """Rows per expert as a router leaves them: expert e gets a row with a probability ~ exp(skew * normal).  The offsets
    of the groups [experts + 1] on the GPU, and the longest group (the plain form pads to it)."""
    p = torch.exp(skew * torch.randn(experts, device="cuda", generator=gen))
    got = torch.bincount(torch.multinomial(p / p.sum(), rows, replacement=True, generator=gen), minlength=experts)
    offsets = torch.zeros(experts + 1, dtype=torch.int32, device="cuda")
    offsets[1:] = torch.cumsum(got, 0).to(torch.int32)
    return offsets, int(got.max())


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    s = {"case": case}

    def normal(*shape, scale=1.0, dtype=torch.bfloat16):
        return (torch.randn(*shape, device="cuda", generator=gen) * scale).to(dtype)

    if case["op"] == "adamw":
        return _prepare_adamw(case, s, normal)
    E, T, a, b = case["experts"], case["rows"] + case["behind"], case["d_in"], case["d_out"]
    s["status"] = torch.zeros(1, dtype=torch.int32, device="cuda")
    s["offsets"], s["longest"] = _groups(gen, E, case["rows"], case["skew"]) if E else (None, case["rows"])
    if case["op"] == "i8":
        # post-ReLU features, weights already in 8 bits with one scale per output channel, as an answering program keeps them
        s["x"] = normal(T, a, dtype=torch.float32).clamp_min(0.0).to(_type(case["x"]))
        w = normal(*((E, b, a) if E else (b, a)), scale=a ** -0.5, dtype=torch.float32)
        s["w_scale"] = w.abs().amax(-1) / 127.0
        s["w"] = torch.round(w / s["w_scale"].unsqueeze(-1)).to(torch.int8)
        s["bias"] = normal(*((E, b) if E else (b,)), scale=0.1, dtype=torch.float32) if case["bias"] else None
        s["q"] = torch.empty(T, a, dtype=torch.int8, device="cuda")
        s["x_scale"] = torch.empty(T, dtype=torch.float32, device="cuda")
        s["y"] = normal(T, b, dtype=_type(case["out"]))
        return s
    d = case["direction"]
    if d != 1:
        s["x"] = normal(T, a, dtype=torch.float32).clamp_min(0.0).to(torch.bfloat16)
    if d != 0:
        s["dy"] = normal(T, b, scale=0.01)
    if d != 2:
        s["w"] = normal(E, b, a, scale=a ** -0.5)
    s["bias"] = normal(E, b, scale=0.1, dtype=torch.float32) if d == 0 and case["bias"] else None
    s["mask"] = normal(T, a, dtype=torch.float32).clamp_min(0.0).to(_type(case["out"])) if d == 1 and case["mask"] else None
    s["out"] = normal(*((E, b, a) if d == 2 else (T, b) if d == 0 else (T, a)), dtype=_type(case["out"]))
    return s


def _prepare_adamw(case, s, normal):
    """All tensors of one kind lie in one buffer, each from a multiple of BLOCK elements on; what lies between is zero."""
    shapes = _shapes(case)
    sizes = [math.prod(x) for x in shapes]
    blocks = [-(-n // BLOCK) for n in sizes]
    total = sum(blocks) * BLOCK
    starts = [BLOCK * sum(blocks[:i]) for i in range(len(blocks))]
    per = torch.tensor(blocks, device="cuda")
    ends = torch.tensor([x + n for x, n in zip(starts, sizes)], device="cuda").repeat_interleave(per)
    inside = torch.arange(total, device="cuda").view(-1, BLOCK) < ends.unsqueeze(1)
    decay = [DECAY if len(x) > 1 else 0.0 for x in shapes]
    s["decay"] = torch.tensor(decay, dtype=torch.float32, device="cuda").repeat_interleave(per).unsqueeze(1)
    s["t"] = T0

    def flat(scale, dtype=torch.float32):
        return torch.where(inside, normal(total // BLOCK, BLOCK, scale=scale, dtype=torch.float32), 0.0).view(-1).to(dtype)

    # weights, the moments after some steps, and the gradient as it comes: the sum over a batch of 256
    master = flat(0.02)
    s["p"] = master if case["param"] == "f32" else master.to(torch.bfloat16)
    s["master"] = master if case["param"] == "bf16+master" else None
    s["g"] = flat(0.256, _type(case["grad"]))
    m, r = flat(3e-4), flat(1e-3).abs()
    if case["bits"] == 8:
        s["m"], s["m_scale"] = _to_e4m3(m.view(-1, BLOCK), False)
        s["v"], s["v_scale"] = _to_e4m3(r.view(-1, BLOCK), True)
    else:
        s["m"], s["v"] = m, r * r
    if own:
        from paper_1712_04432_b200 import mbd

        def views(x, shaped=True):
            return None if x is None else [x[o:o + n].view(h) if shaped else x[o:o + n] for o, n, h in zip(starts, sizes, shapes)]

        def scales(x):
            return [x[o // BLOCK:o // BLOCK + k] for o, k in zip(starts, blocks)]

        more = dict(m_scales=scales(s["m_scale"]), v_scales=scales(s["v_scale"])) if case["bits"] == 8 else {}
        s["optimizer"] = mbd.AdamW(views(s["p"]), views(s["g"]), masters=views(s["master"]), weight_decay=decay, betas=(BETA1, BETA2),
                                   eps=EPS, state_bits=case["bits"], steps_done=T0, m=views(s["m"]), v=views(s["v"]), **more)
    return s


# ------------------------------------------------------------------------------------------------------ the operators
def run(s):
    case = s["case"]
    if case["op"] == "adamw":
        return _run_adamw(s)
    if case["op"] == "i8":
        return _run_i8(s)
    d = case["direction"]
    if own:
        from paper_1712_04432_b200 import mbd
        if d == 0:
            return mbd.expert_gemm(0, s["x"], s["w"], s["offsets"], s["out"], relu=case["relu"], bias=s["bias"], status=s["status"])
        if d == 1:
            return mbd.expert_gemm(1, s["dy"], s["w"], s["offsets"], s["out"], op=mbd.TAIL_MASK, mask=s["mask"], status=s["status"])
        return mbd.expert_gemm(2, s["dy"], s["x"], s["offsets"], s["out"], status=s["status"])
    o, longest, out = s["offsets"], s["longest"], s["out"]
    if d == 2:
        r = torch.bmm(_padded(s["dy"], o, longest).transpose(1, 2), _padded(s["x"], o, longest))
        out.copy_(r)
        return out
    w = s["w"].float()
    r = torch.bmm(_padded(s["x"], o, longest), w.transpose(1, 2)) if d == 0 else torch.bmm(_padded(s["dy"], o, longest), w)
    if d == 0 and s["bias"] is not None:
        r = r + s["bias"].unsqueeze(1)
    if d == 0 and case["relu"]:
        r = r.clamp_min(0.0)
    r = _rows(r, o, out.shape[0])
    if s["mask"] is not None:
        r = torch.where(s["mask"].float() > 0, r, 0.0)
    _put(out, r, o)
    return out


def _padded(x, offsets, longest):
    """[E, longest, d] float: the rows of each group, zeros behind them."""
    at = offsets[:-1].unsqueeze(1) + torch.arange(longest, device="cuda")
    return torch.where((at < offsets[1:].unsqueeze(1)).unsqueeze(2), x[at.clamp_max(x.shape[0] - 1)].float(), 0.0)


def _rows(r, offsets, rows):
    """[rows, d] of the padded groups [E, longest, d]; what lies behind the last group is of no meaning."""
    at = torch.arange(rows, device="cuda")
    e = (torch.searchsorted(offsets, at, right=True) - 1).clamp(0, r.shape[0] - 1)
    return r[e, (at - offsets[e]).clamp_max(r.shape[1] - 1)]


def _put(out, r, offsets):
    """Rows of a group are written, the rows behind the last group stay as they are."""
    inside = (torch.arange(out.shape[0], device="cuda") < offsets[-1]).unsqueeze(1)
    out.copy_(torch.where(inside, r.to(out.dtype), out))


def _run_i8(s):
    case = s["case"]
    if own:
        from paper_1712_04432_b200 import mbd
        mbd.quantize_rows(s["x"], s["q"], s["x_scale"])
        if case["experts"]:
            mbd.expert_gemm_i8(s["q"], s["x_scale"], s["w"], s["w_scale"], s["offsets"], s["y"], relu=case["relu"], bias=s["bias"], status=s["status"])
        else:
            mbd.gemm_i8(s["q"], s["x_scale"], s["w"], s["w_scale"], s["y"], relu=case["relu"], bias=s["bias"], status=s["status"])
        return s["q"], s["x_scale"], s["y"]
    # a token's scale maps its largest value to 127; a row of zeros has scale 0 and stays zero.  The quotients in 64 bits:
    # many lie next to half a step (a value of half the largest is 63.5 steps)
    x = s["x"].float()
    scale = x.abs().amax(-1) / torch.full((), 127.0, device="cuda")          # (a tensor: torch divides by a number through its reciprocal)
    q = torch.round(x.double() / scale.double().unsqueeze(-1)).float()
    q = torch.where(scale.unsqueeze(-1) > 0, q, 0.0).clamp(-127.0, 127.0)
    s["q"].copy_(q)
    s["x_scale"].copy_(scale)
    w = s["w"].float()
    if not case["experts"]:
        r = (q @ w.t()) * scale.unsqueeze(1) * s["w_scale"]
    else:
        r = torch.bmm(_padded(q, s["offsets"], s["longest"]), w.transpose(1, 2)) * s["w_scale"].unsqueeze(1)
    if not case["experts"]:
        r = r + s["bias"] if s["bias"] is not None else r
        s["y"].copy_(r.clamp_min(0.0) if case["relu"] else r)
        return s["q"], s["x_scale"], s["y"]
    r = _rows(r, s["offsets"], s["y"].shape[0]) * scale.unsqueeze(1)
    if s["bias"] is not None:
        at = torch.arange(r.shape[0], device="cuda")
        r = r + s["bias"][(torch.searchsorted(s["offsets"], at, right=True) - 1).clamp(0, case["experts"] - 1)]
    _put(s["y"], r.clamp_min(0.0) if case["relu"] else r, s["offsets"])
    return s["q"], s["x_scale"], s["y"]


def _to_e4m3(x, positive):
    """Blocks [n, BLOCK] in 8 bits: the largest of a block becomes 448.  positive: what is not zero does not become zero
    (it is divided by later), but the smallest number of the type."""
    scale = x.abs().amax(1) / torch.full((), E4M3_MAX, device="cuda")
    q = torch.where(scale.unsqueeze(1) > 0, x / scale.unsqueeze(1), 0.0).clamp(-E4M3_MAX, E4M3_MAX)
    if positive:
        q = torch.where(x > 0, q.clamp_min(E4M3_MIN), 0.0)
    return q.to(torch.float8_e4m3fn).view(-1), scale


def _run_adamw(s):
    case = s["case"]
    if own:
        s["optimizer"].step(LR, grad_scale=1.0 / 256)
    else:
        s["t"] += 1
        eight = case["bits"] == 8
        g = s["g"].float().view(-1, BLOCK) * (1.0 / 256)
        m, v = s["m"].float().view(-1, BLOCK), s["v"].float().view(-1, BLOCK)
        if eight:
            m = m * s["m_scale"].unsqueeze(1)
            v = v * s["v_scale"].unsqueeze(1)
            v = v * v                                    # held as its root
        m = m * BETA1 + g * (1.0 - BETA1)
        v = v * BETA2 + (g * g) * (1.0 - BETA2)
        root = torch.sqrt(v)
        denominator = root * (1.0 / math.sqrt(1.0 - BETA2 ** s["t"])) + EPS
        p = (s["p"] if s["master"] is None else s["master"]).float().view(-1, BLOCK)
        p = p * (1.0 - LR * s["decay"]) - (m / denominator) * (LR / (1.0 - BETA1 ** s["t"]))
        if eight:
            s["m"], s["m_scale"] = _to_e4m3(m, False)
            s["v"], s["v_scale"] = _to_e4m3(root, True)
        else:
            s["m"], s["v"] = m.view(-1), v.view(-1)
        if s["master"] is not None:
            s["master"] = p.view(-1)
        s["p"] = p.view(-1).to(s["p"].dtype)
    r = {k: s[k] for k in ("p", "master", "m", "v")}
    if case["bits"] == 8:
        r.update(m_scale=s["m_scale"], v_scale=s["v_scale"])
    return r


# ------------------------------------------------------------------------------------------------------ in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "adamw":
        return _exact_adamw(case, s)
    D = torch.float64
    bounds = s["offsets"].tolist() if s["offsets"] is not None else [0, case["rows"]]
    if case["op"] == "i8":
        x = s["x"].to(D)
        scale = x.abs().max(1).values / 127
        held = scale.to(torch.float32).to(D)          # the scale is a float: that is what a step of q stands for
        q = torch.zeros_like(x)
        some = held > 0
        q[some] = torch.round(x[some] / held[some, None])
        y = s["y"].to(D).clone()
        for e in range(len(bounds) - 1):
            at = slice(bounds[e], bounds[e + 1])
            w, ws = (s["w"][e], s["w_scale"][e]) if case["experts"] else (s["w"], s["w_scale"])
            z = torch.einsum("rk,nk->rn", q[at], w.to(D)) * held[at, None] * ws.to(D)[None]
            if s["bias"] is not None:
                z += (s["bias"][e] if case["experts"] else s["bias"]).to(D)
            y[at] = z.relu() if case["relu"] else z
        return None, scale, y
    d = case["direction"]
    out = torch.zeros_like(s["out"], dtype=D) if d == 2 else s["out"].to(D)
    for e in range(case["experts"]):
        at = slice(bounds[e], bounds[e + 1])
        if d == 0:
            z = torch.einsum("rk,nk->rn", s["x"][at].to(D), s["w"][e].to(D))
            if s["bias"] is not None:
                z += s["bias"][e].to(D)
            out[at] = z.relu() if case["relu"] else z
        elif d == 1:
            z = torch.einsum("rn,nk->rk", s["dy"][at].to(D), s["w"][e].to(D))
            out[at] = z * (s["mask"][at] > 0) if s["mask"] is not None else z
        else:
            out[e] = torch.einsum("rn,rk->nk", s["dy"][at].to(D), s["x"][at].to(D))
    return out


def _e4m3_values():
    """The 127 numbers of the type that are not negative, in rising order (the place of a number is its bits)."""
    return torch.tensor([(k % 8) * 2.0 ** -9 if k < 8 else (8 + k % 8) * 2.0 ** (k // 8 - 10) for k in range(127)], dtype=torch.float64, device="cuda")


def _nearest_e4m3(x):
    table = _e4m3_values()
    hi = torch.searchsorted(table, x.abs().contiguous()).clamp(0, 126)
    lo = (hi - 1).clamp_min(0)
    up, down = table[hi] - x.abs(), x.abs() - table[lo]
    at = torch.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    return table[at] * torch.sign(x)


def _exact_adamw(case, s):
    D = torch.float64
    rows = lambda x: x.to(torch.float32).to(D).reshape(-1, BLOCK)  # noqa: E731
    g = rows(s["g"]) / 256
    m, v = rows(s["m"]), rows(s["v"])
    if case["bits"] == 8:
        m = m * s["m_scale"].to(D)[:, None]
        v = (v * s["v_scale"].to(D)[:, None]).square()
    t = T0 + 1
    m = BETA1 * m + (1 - BETA1) * g
    v = BETA2 * v + (1 - BETA2) * g.square()
    p = rows(s["p"] if s["master"] is None else s["master"])
    p = p - LR * s["decay"].to(D) * p - LR * (m / (1 - BETA1 ** t)) / ((v / (1 - BETA2 ** t)).sqrt() + EPS)
    r = {"p": p.reshape(-1), "master": None if s["master"] is None else p.reshape(-1)}
    if case["bits"] == 32:
        return dict(r, m=m.reshape(-1), v=v.reshape(-1))
    root = v.sqrt()
    ms, vs = m.abs().max(1).values / E4M3_MAX, root.max(1).values / E4M3_MAX
    one = torch.ones((), dtype=D, device="cuda")
    mq = _nearest_e4m3(m / torch.where(ms > 0, ms, one)[:, None])
    vq = _nearest_e4m3(root / torch.where(vs > 0, vs, one)[:, None])
    vq = torch.where((root > 0) & (vq == 0), torch.full_like(vq, E4M3_MIN), vq)
    return dict(r, m=mq.reshape(-1), v=vq.reshape(-1), m_scale=ms, v_scale=vs)
