"""Root-mean-square norm (mbd_rms_norm) and its gradients (mbd_rms_norm_backward) against 64 bits.

Tolerances count roundings, U = 2^-24 relative each: a row's sum of squares takes n of them (the values of one thread, then 10 steps of joining), half of that
in the root, and a handful for the quotient, the root and the products; then half a step of the result's type."""
import numpy as np
import pytest

from paper_1712_04432_b200 import mbd
from tests.test_i8 import _want_rows

U = 2.0 ** -24
EPS = 1e-6


def _n(K):
    """Float sums a value goes through on its way into a row's sum."""
    return 8 * max(2, -(-K // 8192)) + 10


# ---------------------------------------------------------------------------------------------------- refusals (no GPU needed)
MB = 1 << 20
FWD = dict(R=4, K=8, X=1 * MB, x_bf16=1, ldx=8, res=2 * MB, r_bf16=1, ldr=8, gain=3 * MB, eps=1e-6, H=4 * MB, ldh=8, Y=5 * MB, y_bf16=1, ldy=8, Q=6 * MB, ldq=8,
           scale=7 * MB)


@pytest.mark.parametrize("args,status", [
    (dict(R=-1), mbd.E_INVALID), (dict(K=0), mbd.E_INVALID), (dict(X=None), mbd.E_INVALID), (dict(Y=None, Q=None), mbd.E_INVALID),
    (dict(res=None), mbd.E_INVALID), (dict(scale=None), mbd.E_INVALID), (dict(ldx=7), mbd.E_INVALID), (dict(ldr=7), mbd.E_INVALID),
    (dict(ldh=7), mbd.E_INVALID), (dict(ldy=7), mbd.E_INVALID), (dict(ldq=7), mbd.E_INVALID), (dict(eps=0.0), mbd.E_INVALID),
    (dict(eps=1.0), mbd.E_INVALID), (dict(eps=float("nan")), mbd.E_INVALID), (dict(eps=-1e-6), mbd.E_INVALID),
    (dict(X=1 * MB + 1), mbd.E_UNSUPPORTED), (dict(gain=3 * MB + 2), mbd.E_UNSUPPORTED), (dict(scale=7 * MB + 2), mbd.E_UNSUPPORTED),
    (dict(H=4 * MB + 1), mbd.E_UNSUPPORTED), (dict(K=2 ** 31 - 1, ldx=2 ** 31, ldr=2 ** 31, ldh=2 ** 31, ldy=2 ** 31, ldq=2 ** 31), mbd.E_UNSUPPORTED),
    # results on each other, on other rows of an input, on an input of another type or stride
    (dict(H=5 * MB), mbd.E_INVALID), (dict(Q=5 * MB), mbd.E_INVALID), (dict(Q=1 * MB), mbd.E_INVALID), (dict(scale=1 * MB), mbd.E_INVALID),
    (dict(H=2 * MB + 16), mbd.E_INVALID), (dict(Y=1 * MB + 2), mbd.E_INVALID), (dict(Y=1 * MB, y_bf16=0), mbd.E_INVALID),
    (dict(H=2 * MB, ldh=16), mbd.E_INVALID), (dict(Y=3 * MB), mbd.E_INVALID), (dict(H=1 * MB, x_bf16=0), mbd.E_INVALID),
    (dict(R=0, X=None), mbd.OK),
])
def test_forward_refusals(args, status):
    a = {**FWD, **args}
    assert mbd.lib().mbd_rms_norm(*a.values(), None) == status


BWD = dict(R=4, K=8, dY=1 * MB, dy_bf16=1, lddy=8, H=2 * MB, h_bf16=1, ldh=8, gain=3 * MB, eps=1e-6, dres=4 * MB, lddres=8, dX=5 * MB, lddx=8, dg=6 * MB, scratch=7 * MB)


@pytest.mark.parametrize("args,status", [
    (dict(R=-1), mbd.E_INVALID), (dict(K=0), mbd.E_INVALID), (dict(dY=None), mbd.E_INVALID), (dict(H=None), mbd.E_INVALID), (dict(dX=None), mbd.E_INVALID),
    (dict(scratch=None), mbd.E_INVALID), (dict(lddy=7), mbd.E_INVALID), (dict(ldh=7), mbd.E_INVALID), (dict(lddres=7), mbd.E_INVALID),
    (dict(lddx=7), mbd.E_INVALID), (dict(eps=0.0), mbd.E_INVALID), (dict(dY=1 * MB + 1), mbd.E_UNSUPPORTED), (dict(dg=6 * MB + 2), mbd.E_UNSUPPORTED),
    (dict(scratch=7 * MB + 2), mbd.E_UNSUPPORTED), (dict(dX=2 * MB + 16), mbd.E_INVALID), (dict(dX=1 * MB, dy_bf16=0), mbd.E_INVALID),
    (dict(dX=3 * MB), mbd.E_INVALID), (dict(dg=3 * MB), mbd.E_INVALID), (dict(dg=7 * MB), mbd.E_INVALID), (dict(dg=5 * MB + 32), mbd.E_INVALID),
    (dict(scratch=2 * MB), mbd.E_INVALID), (dict(R=0, dY=None, dg=None), mbd.OK),
])
def test_backward_refusals(args, status):
    a = {**BWD, **args}
    assert mbd.lib().mbd_rms_norm_backward(*a.values(), None) == status


# ---------------------------------------------------------------------------------------------------- forward
def _type(name):
    import torch
    return torch.bfloat16 if name == "bf16" else torch.float32


def _gen(seed):
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _check(got, want, mag, rel, dtype):
    """rel * mag of float roundings, half a step of the type, and of its smallest denormals."""
    import torch
    slack = rel * mag + torch.finfo(dtype).eps / 2 * (want.abs() + rel * mag) + (2.0 ** -133 if dtype == torch.bfloat16 else 2.0 ** -148)
    off = (got.double() - want).abs()
    assert not (off > slack).any(), (float((off / slack).max()), (off > slack).nonzero()[:4].tolist())


def _norm64(h, gain, eps=EPS):
    h = h.double()
    r = 1.0 / ((h * h).mean(1, keepdim=True) + eps).sqrt()
    return h * r * (gain.double() if gain is not None else 1.0), r


def _run(R, K, x="bf16", res="none", out="bf16", eight=False, gain=True, seed=0, spread=True):
    import torch
    gen = _gen(seed + 31 * R + K)
    randn = lambda *s: torch.randn(*s, device="cuda", generator=gen)  # noqa: E731
    X = randn(R, K) * (torch.exp(3 * randn(R, 1)) if spread else 1.0)
    X = X.to(_type(x))
    residual = (randn(R, K) * 2).to(_type(res)) if res != "none" else None
    g = (1 + 0.3 * randn(K)) if gain else None
    h = torch.full((R, K), 5.0, dtype=residual.dtype, device="cuda") if residual is not None else None
    y = torch.full((R, K), 5.0, dtype=_type(out), device="cuda") if out != "none" else None
    q, s = (torch.full((R, K), 99, dtype=torch.int8, device="cuda"), torch.full((R,), -1.0, device="cuda")) if eight else (None, None)
    mbd.rms_norm(X, gain=g, residual=residual, h=h, y=y, q=q, scale=s, eps=EPS)
    held = X if residual is None else (X.float() + residual.float()).to(residual.dtype)
    if h is not None:
        assert torch.equal(h, held)
    want, r = _norm64(held, g)
    rel = (_n(K) / 2 + 8) * U
    if y is not None:
        _check(y, want, want.abs(), rel, y.dtype)
    if eight:
        u = held.float() * g if gain else held.float()
        ws, wq = _want_rows(u.cpu().numpy())
        assert np.array_equal(q.cpu().numpy(), wq)
        _check(s, torch.from_numpy(ws).cuda().double() * r[:, 0], torch.from_numpy(ws).cuda().double() * r[:, 0], rel, torch.float32)


SHAPES = [(1, 1), (1, 7), (3, 8), (5, 33), (2, 1001), (700, 64), (301, 1032), (4, 9216), (2, 32768), (1, 40008), (2, 32771), (600, 8192), (333, 24), (601, 1003),
          (1300, 513), (310, 8200), (300, 16384), (297, 512), (2000, 8), (299, 12001), (320, 4104), (400, 2047)]


@pytest.mark.gpu
@pytest.mark.parametrize("R,K", SHAPES)
@pytest.mark.parametrize("x,res", [("bf16", "none"), ("f32", "none"), ("bf16", "bf16"), ("f32", "f32"), ("bf16", "f32"), ("f32", "bf16")])
def test_forward(R, K, x, res):
    _run(R, K, x, res, out="bf16" if K % 3 else "f32", gain=K != 24)


@pytest.mark.gpu
@pytest.mark.parametrize("R,K", SHAPES)
@pytest.mark.parametrize("x,res,out", [("bf16", "none", "none"), ("f32", "bf16", "bf16"), ("bf16", "f32", "none"), ("f32", "none", "f32")])
def test_forward_in_8_bits(R, K, x, res, out):
    _run(R, K, x, res, out=out, eight=True, gain=K != 33)


@pytest.mark.gpu
def test_rows_at_the_ends_of_the_type():
    """Squares beyond and below float's range, zeros, infinities and NaN, the gain among them."""
    import torch
    for K in (40, 2056, 9000, 40000):
        rows = torch.ones(12, K, device="cuda") * (1 + torch.arange(K, device="cuda") % 7)
        rows[0] *= 1e19; rows[1] *= 4e37; rows[2] *= 1e-22; rows[3] *= 1e-40; rows[4] = 0.0
        rows[5, K // 2] = np.inf; rows[6, K - 1] = np.nan; rows[7, 0] = -np.inf
        rows[8, ::2] = 0.0
        rows[9] *= -3e18
        rows[10, 1:] *= 1e-10; rows[10, 0] = 3e38
        gain = torch.ones(K, device="cuda")
        gain[3], gain[5] = 0.0, -2.0
        y = torch.empty_like(rows)
        q, s = torch.empty(12, K, dtype=torch.int8, device="cuda"), torch.empty(12, device="cuda")
        mbd.rms_norm(rows, gain=gain, y=y, q=q, scale=s, eps=EPS)
        h = rows.double()
        r = 1.0 / ((h * h).mean(1, keepdim=True) + EPS).sqrt()
        want = h * r * gain.double()
        bad = [5, 6, 7]
        fine = [i for i in range(12) if i not in bad]
        assert torch.equal(torch.isnan(y[bad]), torch.isnan(want[bad])) and not torch.nan_to_num(y[bad]).any()      # an infinity: mean infinite, the others 0, itself NaN
        # a root below the smallest normal number (h of 1e38) has 2^-149 of steps: relative 2^-22 of about 3e-39
        _check(y[fine], want[fine], want[fine].abs(), (_n(K) / 2 + 8) * U + 2.0 ** -21, torch.float32)
        assert torch.isnan(s[bad]).all() and not q[bad].any()
        ws, wq = _want_rows((rows * gain).cpu().numpy())
        assert np.array_equal(q.cpu().numpy(), wq)
        ref = torch.from_numpy(ws).cuda().double() * r[:, 0]
        _check(s[fine], ref[fine], ref[fine].abs(), (_n(K) / 2 + 8) * U + 2.0 ** -21, torch.float32)


@pytest.mark.gpu
@pytest.mark.parametrize("K", [96, 101, 1024, 8200])
def test_views_places_of_inputs_and_streams(K):
    """Columns of wider buffers, h on the residual, y on x; on a stream of the caller's; nothing beside the columns is touched."""
    import torch
    gen = _gen(K)
    for R in (3, 700):
        wide = torch.randn(R, 3 * K + 5, device="cuda", generator=gen).to(torch.bfloat16)
        before = wide.clone()
        x, res, y = wide[:, 1:K + 1], wide[:, K + 2:2 * K + 2], wide[:, 2 * K + 3:3 * K + 3]
        gain = torch.randn(K, device="cuda", generator=gen)
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            mbd.rms_norm(x, gain=gain, residual=res, h=res, y=y, eps=EPS)
        s.synchronize()
        held = (before[:, 1:K + 1].float() + before[:, K + 2:2 * K + 2].float()).to(torch.bfloat16)
        assert torch.equal(res, held) and torch.equal(x, before[:, 1:K + 1])
        want, _ = _norm64(held, gain)
        _check(y, want, want.abs(), (_n(K) / 2 + 8) * U, torch.bfloat16)
        for c in (0, K + 1, 2 * K + 2, 3 * K + 3, 3 * K + 4):
            assert torch.equal(wide[:, c], before[:, c])
        a, b = torch.randn(R, K, device="cuda", generator=gen), torch.randn(R, K, device="cuda", generator=gen)
        held = a + b
        z = torch.empty_like(b)
        mbd.rms_norm(a, gain=gain, residual=b, h=a, y=b, eps=EPS)   # h on x, y on the residual
        want, _ = _norm64(held, gain)
        assert torch.equal(a, held)
        _check(b, want, want.abs(), (_n(K) / 2 + 8) * U, torch.float32)
        mbd.rms_norm(a, residual=a, h=z, eps=EPS, y=a)               # the same tensor twice
        assert torch.equal(z, held + held)
        dense = x.contiguous()
        want, _ = _norm64(dense, None)
        mbd.rms_norm(dense, y=dense, eps=EPS)                      # y on x
        _check(dense, want, want.abs(), (_n(K) / 2 + 8) * U, torch.bfloat16)


# ---------------------------------------------------------------------------------------------------- backward
def _backward64(dy, h, gain, dres, eps=EPS):
    dy, h = dy.double(), h.double()
    g = dy * gain.double() if gain is not None else dy
    r = 1.0 / ((h * h).mean(1, keepdim=True) + eps).sqrt()
    unit = h * r
    dx = r * (g - unit * (g * unit).mean(1, keepdim=True))
    mag = r * (g.abs() + unit.abs() * (g * unit).abs().mean(1, keepdim=True))
    if dres is not None:
        dx, mag = dx + dres.double(), mag + dres.double().abs()
    return dx, mag, (dy * unit).sum(0), (dy * unit).abs().sum(0)


def _run_backward(R, K, dy="bf16", h="bf16", dres=True, gain=True, want_gain=True):
    import torch
    gen = _gen(7 * R + K)
    randn = lambda *s: torch.randn(*s, device="cuda", generator=gen)  # noqa: E731
    H = (randn(R, K) * torch.exp(randn(R, 1))).to(_type(h))
    D = (randn(R, K) * 0.1).to(_type(dy))
    g = (1 + 0.3 * randn(K)) if gain else None
    res = (randn(R, K) * 0.1).to(H.dtype) if dres else None
    dx, dg = torch.full_like(H, 5.0), torch.full((K,), 5.0, device="cuda") if want_gain else None
    mbd.rms_norm_backward(D, H, dx, gain=g, d_residual=res, d_gain=dg, eps=EPS)
    want, mag, wg, magg = _backward64(D, H, g, res)
    _check(dx, want, mag, (_n(K) + 12) * U, dx.dtype)
    if want_gain:          # rows of a block one after the other, then the blocks' sums in eight strands
        _check(dg, wg, magg, (-(-R // 148) + 74 + 16 + _n(K) / 2 + 8) * U, torch.float32)


@pytest.mark.gpu
@pytest.mark.parametrize("R,K", SHAPES)
@pytest.mark.parametrize("dy,h,dres", [("bf16", "bf16", True), ("f32", "f32", False), ("bf16", "f32", True), ("f32", "bf16", False)])
def test_backward(R, K, dy, h, dres):
    _run_backward(R, K, dy, h, dres, gain=K != 24, want_gain=K != 64)


@pytest.mark.gpu
def test_backward_longer_than_shared_memory():
    _run_backward(3, 60008, "bf16", "f32")
    _run_backward(2, 70001, "f32", "bf16")


@pytest.mark.gpu
def test_backward_at_the_ends_of_the_type():
    import torch
    for K in (40, 2056, 9000):
        gen = _gen(K)
        H = torch.randn(6, K, device="cuda", generator=gen)
        H[0] *= 1e19; H[1] *= 4e37; H[2] *= 1e-22; H[3] = 0.0
        D = torch.randn(6, K, device="cuda", generator=gen)
        dx, dg = torch.empty_like(H), torch.empty(K, device="cuda")
        mbd.rms_norm_backward(D, H, dx, d_gain=dg, eps=EPS)
        want, mag, wg, magg = _backward64(D, H, None, None)
        _check(dx, want, mag, (_n(K) + 12) * U + 2.0 ** -21, torch.float32)
        _check(dg, wg, magg, (100 + _n(K)) * U + 2.0 ** -21, torch.float32)
        H[4, 1] = np.nan                                            # stays in its row, and in its columns' sums
        mbd.rms_norm_backward(D, H, dx, d_gain=dg, eps=EPS)
        assert torch.isnan(dx[4]).all() and not torch.isnan(dx[[0, 1, 2, 3, 5]]).any() and torch.isnan(dg).all()


@pytest.mark.gpu
def test_backward_in_place_and_no_rows():
    import torch
    gen = _gen(9)
    for K in (104, 1001, 8208):
        H, D, res = (torch.randn(500, K, device="cuda", generator=gen) for _ in range(3))
        gain, dg, dg2, dx = torch.randn(K, device="cuda", generator=gen), torch.empty(K, device="cuda"), torch.empty(K, device="cuda"), torch.empty_like(H)
        mbd.rms_norm_backward(D, H, dx, gain=gain, d_residual=res, d_gain=dg)
        for name in ("res", "D", "H"):
            t = dict(res=res.clone(), D=D.clone(), H=H.clone())
            mbd.rms_norm_backward(t["D"], t["H"], t[name], gain=gain, d_residual=t["res"], d_gain=dg2)
            assert torch.equal(t[name], dx) and torch.equal(dg, dg2)          # the same bits, in the same order
        none = torch.empty(0, K, device="cuda")
        mbd.rms_norm_backward(none, none, none, d_gain=dg)
        assert not dg.any()
        mbd.rms_norm(none, y=none)


@pytest.mark.gpu
def test_gradient_against_differences():
    """Along a direction v: (L(h + d v) - L(h - d v)) / 2d with L = <c, y>, y from the forward kernel in float.  y's roundings: 40 U of sum |c y| / d;
    the next term of the expansion: d^2 |v|^2 / |h|^2 of the slope's bound, with a factor below 4."""
    import torch
    for K in (64, 1001):
        gen = _gen(K)
        h, v, c = (torch.randn(5, K, device="cuda", generator=gen) for _ in range(3))
        gain = 1 + 0.2 * torch.randn(K, device="cuda", generator=gen)
        d = 2.0 ** -7
        y = [torch.empty_like(h) for _ in range(2)]
        sides = [h + d * v, h - d * v]
        for s, o in zip(sides, y):
            mbd.rms_norm(s, gain=gain, y=o, eps=EPS)
        slope = (c.double() * (y[0].double() - y[1].double())).sum(1) / (2 * d)
        dx = torch.empty_like(h)
        mbd.rms_norm_backward(c, h, dx, gain=gain, eps=EPS)
        got = (dx.double() * v.double()).sum(1)
        size = c.double().norm(dim=1) * v.double().norm(dim=1) * gain.abs().max() / h.double().square().mean(1).sqrt()
        slack = 40 * U * (c * y[0]).abs().double().sum(1) / d + (4 * d * d * 2 + 1e-5) * size
        assert ((slope - got).abs() <= slack).all()
        # the gain's: y is linear in it, so a step of one is exact but for roundings
        e = torch.randn(K, device="cuda", generator=gen)
        for sign, o in ((1, y[0]), (-1, y[1])):
            mbd.rms_norm(h, gain=gain + sign * e, y=o, eps=EPS)
        dg = torch.empty(K, device="cuda")
        mbd.rms_norm_backward(c, h, dx, gain=gain, d_gain=dg, eps=EPS)
        slope = float((c.double() * (y[0].double() - y[1].double())).sum() / 2)
        assert abs(slope - float((dg.double() * e.double()).sum())) <= 100 * U * float((c.double().abs() * (y[0].abs() + y[1].abs()).double()).sum())


@pytest.mark.gpu
def test_captured_and_replayed():
    import torch
    gen = _gen(11)
    R, K = 900, 1024
    x, res = torch.randn(R, K, device="cuda", generator=gen).to(torch.bfloat16), torch.randn(R, K, device="cuda", generator=gen).to(torch.bfloat16)
    gain, dy = torch.randn(K, device="cuda", generator=gen), torch.randn(R, K, device="cuda", generator=gen).to(torch.bfloat16)
    h, y, dx, dg = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x), torch.empty(K, device="cuda")

    def step():
        mbd.rms_norm(x, gain=gain, residual=res, h=h, y=y)
        mbd.rms_norm_backward(dy, h, dx, gain=gain, d_residual=y, d_gain=dg)

    step()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    x.mul_(2.0)
    step()
    want = [t.clone() for t in (h, y, dx, dg)]
    for t in (h, y, dx, dg):
        t.zero_()
    g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, (h, y, dx, dg)))


# ---------------------------------------------------------------------------------------------------- the forms of large batches
# More than 10 million values, or 2 rows for each of 148 SMs: rows in whole vectors through shared memory, several a block, each many times
# around its stages; the row of each width's end and one a vector shorter.
RING = [(24000, 512), (24000, 504), (24000, 1024), (24000, 1016), (12000, 2048), (12000, 2040), (6000, 4096), (6000, 4088), (3000, 8192), (3000, 8184),
        (1500, 16384), (1500, 16376)]


def _quotients(u):
    """scale and q of float rows, from the definition: a quotient in 64 bits is that of two floats on the right side of every half step."""
    import torch
    s = (u.abs().amax(1).double() / 127).float()                     # (24 bits by 7: 2^-32 from a half step at least)
    return s, torch.round(u.double() / s.double()[:, None]).clamp(-127, 127).to(torch.int8)


def _run_large(R, K, x, res, out, eight, in_place=False):
    import torch
    gen = _gen(R + K)
    randn = lambda *s: torch.randn(*s, device="cuda", generator=gen)  # noqa: E731
    X = (randn(R, K) * torch.exp(randn(R, 1))).to(_type(x))
    residual = (randn(R, K) * 2).to(_type(res)) if res != "none" else None
    g = 1 + 0.3 * randn(K)
    held = X.clone() if residual is None else (X.float() + residual.float()).to(residual.dtype)
    h = (residual if in_place else torch.full_like(residual, 5.0)) if residual is not None else None
    y = (X if in_place else torch.full((R, K), 5.0, dtype=_type(out), device="cuda")) if out != "none" else None
    q, s = (torch.full((R, K), 99, dtype=torch.int8, device="cuda"), torch.full((R,), -1.0, device="cuda")) if eight else (None, None)
    mbd.rms_norm(X, gain=g, residual=residual, h=h, y=y, q=q, scale=s, eps=EPS)
    if h is not None:
        assert torch.equal(h, held)
    want, r = _norm64(held, g)
    rel = (_n(K) / 2 + 8) * U
    if y is not None:
        _check(y, want, want.abs(), rel, y.dtype)
    if eight:
        ws, wq = _quotients(held.float() * g)
        assert torch.equal(q, wq)
        ws = ws.double() * r[:, 0]
        _check(s, ws, ws, rel, torch.float32)


@pytest.mark.gpu
@pytest.mark.parametrize("R,K", RING)
@pytest.mark.parametrize("x,res,out,eight", [("bf16", "none", "bf16", False), ("f32", "none", "bf16", False), ("bf16", "none", "none", True), ("f32", "none", "f32", True),
                                             ("bf16", "bf16", "bf16", True)])
def test_forward_of_large_batches_through_shared_memory(R, K, x, res, out, eight):
    _run_large(R, K, x, res, out, eight)


@pytest.mark.gpu
@pytest.mark.parametrize("R,K", RING[::2])
def test_forward_of_large_batches_in_place(R, K):
    _run_large(R, K, "bf16", "none", "bf16", False, in_place=True)
    _run_large(R, K, "bf16", "bf16", "bf16", True, in_place=True)


@pytest.mark.gpu
@pytest.mark.parametrize("R,K", [(2500, 4096), (700, 4088), (600, 2056), (501, 3001), (2500, 8192), (900, 8184), (300, 4097), (9001, 1024), (20000, 504), (2000, 4000), (401, 511), (401, 1021)])
@pytest.mark.parametrize("x,res,out", [("bf16", "bf16", "bf16"), ("f32", "f32", "f32"), ("bf16", "f32", "bf16"), ("f32", "bf16", "f32"), ("bf16", "none", "bf16"),
                                       ("f32", "none", "f32")])
def test_forward_of_large_batches_row_by_row(R, K, x, res, out):
    _run_large(R, K, x, res, out, False)
    if x == "bf16":
        _run_large(R, K, x, res, out, False, in_place=x == out)


@pytest.mark.gpu
@pytest.mark.parametrize("R,K", [(24000, 512), (24000, 504), (12000, 1024), (12000, 1016), (6000, 2048), (6000, 2040), (3000, 4096), (3000, 4088), (1500, 8192),
                                 (1500, 8184), (700, 16384), (700, 16376), (6000, 511), (5003, 1001), (3001, 2047), (1501, 4001), (1001, 8191), (450, 16383)])
@pytest.mark.parametrize("dy,h,dres", [("bf16", "bf16", True), ("bf16", "bf16", False), ("f32", "f32", False), ("f32", "f32", True), ("bf16", "f32", True), ("f32", "bf16", False)])
def test_backward_of_large_batches(R, K, dy, h, dres):
    """A block's row groups take many rows each.  dx: n / 2 + 2 roundings of r in three places, n of the dot product, eight of the products, sums and 1 / K.  d_gain: at most R / 148 rows one after the other in a group or, where a block has several groups, fewer
    and one step for each of at most 16 groups, then five blocks one after the other in each of 32 strands and five steps between those."""
    import torch
    gen = _gen(3 * R + K)
    randn = lambda *s: torch.randn(*s, device="cuda", generator=gen)  # noqa: E731
    H, D, g = (randn(R, K) * torch.exp(randn(R, 1))).to(_type(h)), (randn(R, K) * 0.1).to(_type(dy)), 1 + 0.3 * randn(K)
    res = (randn(R, K) * 0.1).to(H.dtype) if dres else None
    dx, dg = torch.full_like(H, 5.0), torch.full((K,), 5.0, device="cuda")
    mbd.rms_norm_backward(D, H, dx, gain=g, d_residual=res, d_gain=dg, eps=EPS)
    want, mag, wg, magg = _backward64(D, H, g, res)
    _check(dx, want, mag, (2.5 * _n(K) + 14) * U, dx.dtype)
    _check(dg, wg, magg, (-(-R // 148) + 16 + 10 + _n(K) / 2 + 8) * U, torch.float32)
    again = torch.empty_like(dg)
    mbd.rms_norm_backward(D, H, H if res is None else res, gain=g, d_residual=res, d_gain=again, eps=EPS)      # in place: the same bits
    assert torch.equal(H if res is None else res, dx) and torch.equal(again, dg)
