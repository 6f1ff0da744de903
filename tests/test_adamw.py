"""AdamW over a list of tensors (mbd_adamw_*) against its formulas in 64 bits: float and 8-bit moments, every pairing of weight,
master and gradient types, odd sizes and alignments, values that are not finite, several steps, capture."""
import ctypes as C

import numpy as np
import pytest

from paper_1712_04432_b200 import mbd

BLOCK = 256


# ---------------------------------------------------------------------------------------------------- refusals (no GPU needed)
def _entry(base=1 << 24, n=1000, **kw):
    e = dict(param_dev=base, master_dev=None, grad_dev=base + (1 << 20), m_dev=base + (2 << 20), v_dev=base + (3 << 20),
             m_scale_dev=base + (4 << 20), v_scale_dev=base + (5 << 20), n=n, weight_decay=0.0, param_bf16=0, grad_bf16=0, reserved=0)
    e.update(kw)
    return mbd.AdamWTensor(**e)


def _create(entries, bits=32, b1=0.9, b2=0.999, eps=1e-8, steps=0):
    table = (mbd.AdamWTensor * max(1, len(entries)))(*entries)
    h = C.c_void_p()
    return mbd.lib().mbd_adamw_create(table, len(entries), bits, b1, b2, eps, steps, C.byref(h))


@pytest.mark.parametrize("entries,args,status", [
    ([], {}, mbd.E_INVALID), ([_entry(n=0)], {}, mbd.E_INVALID), ([_entry(param_dev=None)], {}, mbd.E_INVALID),
    ([_entry(grad_dev=None)], {}, mbd.E_INVALID), ([_entry(m_dev=None)], {}, mbd.E_INVALID), ([_entry(v_dev=None)], {}, mbd.E_INVALID),
    ([_entry(weight_decay=-0.1)], {}, mbd.E_INVALID), ([_entry(weight_decay=float("nan"))], {}, mbd.E_INVALID),
    ([_entry(m_scale_dev=None)], dict(bits=8), mbd.E_INVALID), ([_entry(master_dev=1 << 28)], {}, mbd.E_INVALID),
    ([_entry()], dict(bits=16), mbd.E_UNSUPPORTED), ([_entry()], dict(b1=1.0), mbd.E_INVALID), ([_entry()], dict(b2=-0.1), mbd.E_INVALID),
    ([_entry()], dict(b1=float("nan")), mbd.E_INVALID), ([_entry()], dict(eps=0.0), mbd.E_INVALID), ([_entry()], dict(steps=-1), mbd.E_INVALID),
    ([_entry(), _entry()], {}, mbd.E_INVALID),                                                   # the same tensor twice
    ([_entry(), _entry(base=1 << 26, param_dev=(1 << 24) + 3996)], {}, mbd.E_INVALID),           # overlaps by one element
    ([_entry(), _entry(base=1 << 26, m_dev=(1 << 24) + (1 << 20))], {}, mbd.E_INVALID),          # a moment on a gradient
    ([_entry(v_dev=(1 << 24) + (2 << 20))], {}, mbd.E_INVALID),                                  # m and v on one buffer
    ([_entry(param_dev=(1 << 24) + 2)], {}, mbd.E_UNSUPPORTED), ([_entry(grad_dev=(1 << 25) + 1, grad_bf16=1)], {}, mbd.E_UNSUPPORTED),
    ([_entry(n=1 << 47)], {}, mbd.E_UNSUPPORTED),
])
def test_refusals(entries, args, status):
    assert _create(entries, **args) == status


def test_calls_without_a_list():
    L, n = mbd.lib(), C.c_int64()
    assert L.mbd_adamw_step(None, 1e-3, 1.0, None) == mbd.E_INVALID and L.mbd_adamw_destroy(None) == mbd.E_INVALID
    assert L.mbd_adamw_set_steps(None, 0) == mbd.E_INVALID and L.mbd_adamw_get_steps(None, C.byref(n)) == mbd.E_INVALID


# ---------------------------------------------------------------------------------------------------- the formulas in 64 bits
E4M3 = np.array([(k % 8) * 2.0 ** -9 if k < 8 else (8 + k % 8) * 2.0 ** (k // 8 - 10) for k in range(127)])


def _codes(x):
    """Values of a float8_e4m3fn tensor in 64 bits."""
    import torch
    return x.to(torch.float32).double().cpu().numpy().ravel()


def _spread(scale, n):
    return np.repeat(scale.double().cpu().numpy(), BLOCK)[:n]


def _step(p, g, m, v, t, lr, wd, b1=0.9, b2=0.999, eps=1e-8):
    m = b1 * m + (1 - b1) * g
    v = b2 * v + (1 - b2) * g * g
    return p * (1 - lr * wd) - lr * (m / (1 - b1 ** t)) / (np.sqrt(v / (1 - b2 ** t)) + eps), m, v


def _near(got, want, rel, floor=0.0):
    off = np.abs(got - want)
    slack = rel * np.abs(want) + floor
    assert (off <= slack).all(), (float((off - slack).max()), int((off > slack).sum()), np.flatnonzero(off > slack)[:5].tolist())


U = 2.0 ** -24                      # half a step of a float, relative


def _check_moments(opt, i, bits, m, v, n, before_m, before_v, g):
    """m and v in 64 bits against what is held.  Float: each of m's three and v's four operations rounds once, and a sum of terms of
    either sign is measured against their magnitudes.  8 bits: half a step of e4m3 (2^-4 relative, 2^-10 of the scale below the
    smallest normal number, a whole smallest number where the root is lifted off zero), and the scale itself."""
    from numpy import abs as a
    big_m = 0.9 * a(before_m) + 0.1 * a(g)
    if bits == 32:
        _near(opt.m[i].double().cpu().numpy().ravel(), m, 0, 4 * U * big_m + 1e-44)
        _near(opt.v[i].double().cpu().numpy().ravel(), v, 5 * U, 1e-44)
        return
    for what, held, scales, big in ((m, opt.m[i], opt.m_scales[i], big_m), (np.sqrt(v), opt.v[i], opt.v_scales[i], np.sqrt(v))):
        blocks = -(-n // BLOCK)
        top = np.array([a(what[k * BLOCK:(k + 1) * BLOCK]).max() for k in range(blocks)])
        slack = np.array([big[k * BLOCK:(k + 1) * BLOCK].max() for k in range(blocks)])
        _near(scales.double().cpu().numpy(), top / 448, 2 * U, 6 * U * slack / 448 + 1e-44)
        s = _spread(scales, n)
        codes = _codes(held)
        rounding = np.maximum(2.0 ** -4 * a(what), 2.0 ** -10 * s)
        if held is opt.v[i]:
            rounding = np.where((what > 0) & (what < 2.0 ** -9 * s), 2.0 ** -9 * s, rounding)
            assert ((codes > 0) == (what > 0)).all()                   # never rounded to zero
        _near(codes * s, what, 0, rounding * (1 + 8 * U) + 8 * U * big + 1e-44)
        for k in range(blocks):                                        # the largest of a block is held at 448
            c = a(codes[k * BLOCK:(k + 1) * BLOCK])
            assert top[k] == 0 or c.max() == 448


SIZES = [1, 3, 255, 256, 257, 1000, 4096, 70001]


def _make(sizes, param, grad, bits, seed, odd=False, decay=0.01, **kw):
    """Tensors with a history.  odd: each starts one element into its buffer."""
    import torch
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)

    def one(n, scale, dtype, values=None):
        buf = torch.zeros(n + 8, dtype=torch.float32 if dtype is None else dtype, device="cuda")
        x = buf[1:1 + n] if odd else buf[:n]
        x.copy_((torch.randn(n, device="cuda", generator=gen) * scale) if values is None else values)
        return x
    pt = torch.float32 if param == "f32" else torch.bfloat16
    gt = torch.float32 if grad == "f32" else torch.bfloat16
    masters = [one(n, 0.05, torch.float32) for n in sizes] if param == "bf16+master" else None
    params = [one(n, 0.05, pt, None if masters is None else masters[i]) for i, n in enumerate(sizes)]
    grads = [one(n, 3.0, gt) for n in sizes]
    if bits == 32:
        m = [one(n, 1e-2, torch.float32) for n in sizes]
        v = [one(n, 1e-2, torch.float32) for n in sizes]
        for x in v:
            x.copy_(x * x)
        more = {}
    else:
        blocks = lambda n: -(-n // BLOCK)  # noqa: E731
        code = lambda n, f: one(n, 1.0, torch.float8_e4m3fn, f(torch.randn(n, device="cuda", generator=gen) * 100).clamp(-448, 448).to(torch.float8_e4m3fn))  # noqa: E731
        m, v = [code(n, lambda x: x) for n in sizes], [code(n, torch.abs) for n in sizes]
        scale = lambda: [torch.rand(blocks(n), device="cuda", generator=gen) * 1e-4 for n in sizes]  # noqa: E731
        more = dict(m_scales=scale(), v_scales=scale())
    return mbd.AdamW(params, grads, masters=masters, weight_decay=decay, state_bits=bits, m=m, v=v, **more, **kw)


def _read(opt, i, bits):
    d = lambda x: x.double().cpu().numpy().ravel()  # noqa: E731
    n = opt.params[i].numel()
    p = d(opt.params[i] if opt.masters[i] is None else opt.masters[i])
    if bits == 32:
        return p, d(opt.grads[i]), d(opt.m[i]), d(opt.v[i])
    return p, d(opt.grads[i]), _codes(opt.m[i]) * _spread(opt.m_scales[i], n), (_codes(opt.v[i]) * _spread(opt.v_scales[i], n)) ** 2


@pytest.mark.gpu
@pytest.mark.parametrize("odd", [False, True])
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("param,grad", [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16"), ("bf16+master", "f32"), ("bf16+master", "bf16"), ("f32", "bf16")])
def test_steps_against_the_formulas(param, grad, bits, odd):
    import torch
    decay = [0.0 if n < 300 else 0.02 for n in SIZES]
    opt = _make(SIZES, param, grad, bits, seed=1, odd=odd, decay=decay, steps_done=3)
    lr, scale = 0.02, 1.0 / 64
    for t in (4, 5, 6):
        before = [_read(opt, i, bits) for i in range(len(SIZES))]
        opt.step(lr, grad_scale=scale)
        for i, n in enumerate(SIZES):
            p, g, m, v = before[i]
            g = g * scale
            want, wm, wv = _step(p, g, m, v, t, lr, decay[i])
            _check_moments(opt, i, bits, wm, wv, n, m, v, g)
            got = (opt.params[i] if opt.masters[i] is None else opt.masters[i]).double().cpu().numpy().ravel()
            # the quotient: m's roundings against the magnitudes of its terms, a few more for the root, the sum with eps, the
            # quotient, the rates; then the decayed weight and the difference
            root = np.sqrt(wv / (1 - 0.999 ** t)) + 1e-8
            move = lr * ((0.9 * np.abs(m) + 0.1 * np.abs(g)) / (1 - 0.9 ** t)) / root
            slack = 16 * U * move + 6 * U * np.abs(p)
            if param == "bf16":
                slack = slack + 2.0 ** -8 * (np.abs(want) + slack)
            _near(got, want, 0, slack + 1e-44)
            if param == "bf16+master":
                assert torch.equal(opt.params[i], opt.masters[i].to(torch.bfloat16))
    assert opt.steps_done == 6
    opt.close()


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [32, 8])
def test_many_steps_from_nothing(bits):
    # from zeroed buffers, twenty steps: the first moves every weight by lr (m / sqrt(v) is the sign of g), and the counter is right
    import torch
    gen = torch.Generator(device="cuda")
    gen.manual_seed(2)
    p = torch.zeros(3000, device="cuda")
    g = torch.randn(3000, device="cuda", generator=gen)
    g[::10] = 0.0
    opt = mbd.AdamW([p], [g], state_bits=bits)
    opt.step(0.01)
    want = -0.01 * torch.sign(g)
    assert ((p - want).abs() <= 0.01 * 1e-6 + 0.01 * 1e-8 / g.abs().clamp_min(1e-30) * (g != 0)).all()
    assert (p[::10] == 0).all()
    for _ in range(19):
        opt.step(0.01)
    assert opt.steps_done == 20
    if bits == 32:
        # a constant gradient keeps moving by lr each step: m and v are their own averages.  20 steps of a few roundings each.
        assert ((p - 20 * want).abs() <= 0.2 * 64 * 2.0 ** -24 + 20 * 0.01 * 1e-8 / g.abs().clamp_min(1e-30) * (g != 0)).all()
    else:
        # the moments are rounded at every step, by 2^-4 relative at most each; m and the root cannot drift further than the sum
        # of what is forgotten: m by 2^-4 * 9, so the bound is loose -- the sign and the order of the step stay
        moved = (p / want)[g != 0]
        assert (moved > 20 * (1 - 0.6)).all() and (moved < 20 * (1 + 1.2)).all()
    opt.steps_done = 0
    assert opt.steps_done == 0
    opt.close()


@pytest.mark.gpu
def test_small_roots_survive_next_to_large_ones():
    # one gradient 1e5 times the others in its block: their roots fall under the smallest number of the type and are lifted to it,
    # so no weight is moved by m / eps
    import torch
    g = torch.full((256,), 1e-3, device="cuda")
    g[17] = 1e3
    p = torch.zeros(256, device="cuda")
    opt = mbd.AdamW([p], [g], state_bits=8)
    for _ in range(5):
        opt.step(0.1)
    assert (opt.v[0].float() > 0).all()
    # after the first step a weight moves by at most lr |m| / root with root lifted, never lowered
    assert (p.abs() <= 5 * 0.1 * 1.2).all() and (p[17].abs() > 0.3)
    opt.close()


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [32, 8])
def test_what_is_not_finite_stays_its_own(bits):
    import torch
    opt = _make([600], "f32", "f32", bits, seed=4)
    clean = _make([600], "f32", "f32", bits, seed=4)
    opt.grads[0][[5, 300]] = float("nan")
    opt.grads[0][7] = float("inf")
    for o in (opt, clean):
        o.step(0.01)
        o.step(0.01)
    bad = torch.zeros(600, dtype=torch.bool, device="cuda")
    bad[[5, 7, 300]] = True
    assert opt.params[0][bad].isnan().all() and opt.m[0].float()[bad].isnan().any()
    # the others: as if the three were not in their blocks
    assert torch.isfinite(opt.params[0][~bad]).all() and torch.isfinite(opt.m[0].float()[~bad]).all() and torch.isfinite(opt.v[0].float()[~bad]).all()
    if bits == 32:
        assert torch.equal(opt.params[0][~bad], clean.params[0][~bad])
    else:
        assert torch.isfinite(opt.m_scales[0]).all() and torch.isfinite(opt.v_scales[0]).all()
    for o in (opt, clean):
        o.close()


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [32, 8])
def test_a_captured_step_counts_on(bits):
    import torch
    a, b = _make([700, 5], "bf16+master", "f32", bits, seed=5), _make([700, 5], "bf16+master", "f32", bits, seed=5)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        a.step(0.01, grad_scale=0.5)
    for _ in range(7):
        graph.replay()
        b.step(0.01, grad_scale=0.5)
    assert a.steps_done == b.steps_done == 7
    for x, y in zip(a.params + a.masters + a.m + a.v, b.params + b.masters + b.m + b.v):
        assert torch.equal(x.float(), y.float())
    a.close(); b.close()


@pytest.mark.gpu
def test_many_tensors_and_bad_rates():
    import torch
    sizes = [1 + (37 * k) % 600 for k in range(1500)]
    opt = _make(sizes, "bf16", "bf16", 8, seed=6)
    before = [_read(opt, i, 8) for i in (0, 1, 777, 1499)]
    others = [x.clone() for x in opt.params]
    opt.step(0.5)
    for j, i in enumerate((0, 1, 777, 1499)):
        p, g, m, v = before[j]
        want, _, _ = _step(p, g, m, v, 1, 0.5, 0.01)
        _near(opt.params[i].double().cpu().numpy(), want, 2.0 ** -8, 32 * U * (np.abs(p) + np.abs(want - p) * 10))
    assert sum(not torch.equal(x, y) for x, y in zip(opt.params, others)) > 1400
    for lr, gs in ((-1.0, 1.0), (float("nan"), 1.0), (0.1, float("inf"))):
        with pytest.raises(mbd.MbdError) as e:
            opt.step(lr, gs)
        assert e.value.status == mbd.E_INVALID
    assert opt.steps_done == 1
    opt.close()


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [32, 8])
def test_a_very_small_eps_and_very_small_gradients(bits):
    # eps beside roots that are themselves tiny: v is a denormal number, its root an ordinary one.  Four roundings in v near 1e-40 (its step
    # there is 1.4e-45: 7e-6 relative at 1e-40), halved by the root
    import torch
    g = torch.tensor([1e-18, -3e-19, 2e-18, 5e-19] * 64, device="cuda")
    p = torch.zeros(256, device="cuda")
    opt = mbd.AdamW([p], [g], eps=1e-20, state_bits=bits)
    opt.step(0.01)
    want, _, _ = _step(np.zeros(256), g.double().cpu().numpy(), np.zeros(256), np.zeros(256), 1, 0.01, 0.0, eps=1e-20)
    _near(p.double().cpu().numpy(), want, 1e-4)
    opt.close()


@pytest.mark.gpu
@pytest.mark.parametrize("grad", ["f32", "bf16"])
def test_moments_are_the_plain_float_formulas_bit_for_bit(grad):
    # each product and sum in float on the host; the codes by the type's own rounding of the float quotient
    import torch
    f = np.float32
    b1, c1, b2, c2 = f(0.9), f(1.0 - 0.9), f(0.999), f(1.0 - 0.999)
    for bits in (32, 8):
        opt = _make([200_000], "bf16+master", grad, bits, seed=9)
        g = opt.grads[0].float().cpu().numpy() * f(1 / 64)
        m, v = opt.m[0].float().cpu().numpy(), opt.v[0].float().cpu().numpy()
        if bits == 8:
            spread = lambda x: np.repeat(x.cpu().numpy(), BLOCK)[:200_000]  # noqa: E731
            m, v = m * spread(opt.m_scales[0]), v * spread(opt.v_scales[0])
            v = v * v
        m, v = m * b1 + g * c1, v * b2 + (g * g) * c2
        opt.step(0.01, grad_scale=1 / 64)
        if bits == 32:
            assert np.array_equal(opt.m[0].cpu().numpy(), m) and np.array_equal(opt.v[0].cpu().numpy(), v)
            opt.close()
            continue
        for x, held, scales in ((m, opt.m[0], opt.m_scales[0]), (np.sqrt(v), opt.v[0], opt.v_scales[0])):
            pad = np.zeros(-(-x.size // BLOCK) * BLOCK, f)
            pad[:x.size] = x
            s = np.abs(pad.reshape(-1, BLOCK)).max(1) / f(448)
            assert np.array_equal(scales.cpu().numpy(), s)
            q = torch.from_numpy((pad.reshape(-1, BLOCK) / s[:, None]).ravel()[:x.size]).cuda()
            if held is opt.v[0]:
                q = torch.where(q > 0, q.clamp_min(2.0 ** -9), q)
            assert torch.equal(held.view(torch.uint8), q.to(torch.float8_e4m3fn).view(torch.uint8))
        opt.close()
