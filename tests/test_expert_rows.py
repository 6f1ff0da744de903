"""Rows to the experts and back (mbd_expert_dispatch, mbd_expert_combine, mbd_expert_combine_backward) against 64 bits: copies exactly, sums to
float roundings (U = 2^-24 each) and half a step of the result's type."""
import numpy as np
import pytest

from paper_1712_04432_b200 import mbd

U = 2.0 ** -24
MB = 1 << 20


# ---------------------------------------------------------------------------------------------------- refusals (no GPU needed)
DISPATCH = dict(T=10, k=2, K=8, size=2, X=1 * MB, ldx=8, scale=None, places=3 * MB, rows=20, out=4 * MB, ldo=8, out_scale=None)
COMBINE = dict(T=10, k=2, K=8, Y=1 * MB, y_bf16=1, ldy=8, rows=20, places=2 * MB, weights=3 * MB, res=4 * MB, ldres=8, out=5 * MB, out_bf16=1, ldo=8)
BACKWARD = dict(T=10, k=2, K=8, d_out=1 * MB, d_bf16=1, ldd=8, Y=2 * MB, y_bf16=1, ldy=8, rows=20, places=3 * MB, weights=4 * MB, dY=5 * MB, lddy=8, dw=6 * MB)

SIZES = [(dict(T=-1), mbd.E_INVALID), (dict(K=0), mbd.E_INVALID), (dict(k=0), mbd.E_INVALID), (dict(rows=-1), mbd.E_INVALID),
         (dict(places=None), mbd.E_INVALID), (dict(k=33), mbd.E_UNSUPPORTED), (dict(places=3 * MB + 2), mbd.E_UNSUPPORTED), (dict(T=0, places=None), mbd.OK),
         (dict(rows=2 ** 31), mbd.E_UNSUPPORTED), (dict(T=2 ** 31), mbd.E_UNSUPPORTED)]


@pytest.mark.parametrize("args,status", SIZES + [
    (dict(size=3), mbd.E_INVALID), (dict(size=8), mbd.E_INVALID), (dict(X=None), mbd.E_INVALID), (dict(out=None), mbd.E_INVALID), (dict(scale=7 * MB), mbd.E_INVALID),
    (dict(out_scale=7 * MB), mbd.E_INVALID), (dict(ldx=7), mbd.E_INVALID), (dict(ldo=7), mbd.E_INVALID), (dict(X=1 * MB + 1), mbd.E_UNSUPPORTED),
    (dict(out=1 * MB + 16), mbd.E_INVALID), (dict(out=3 * MB), mbd.E_INVALID), (dict(scale=7 * MB, out_scale=7 * MB + 8), mbd.E_INVALID),
    (dict(scale=7 * MB, out_scale=4 * MB), mbd.E_INVALID), (dict(scale=7 * MB, out_scale=8 * MB + 2), mbd.E_UNSUPPORTED)])
def test_dispatch_refusals(args, status):
    assert mbd.lib().mbd_expert_dispatch(*{**DISPATCH, **args}.values(), None) == status


@pytest.mark.parametrize("args,status", SIZES + [
    (dict(Y=None), mbd.E_INVALID), (dict(out=None), mbd.E_INVALID), (dict(ldy=7), mbd.E_INVALID), (dict(ldres=7), mbd.E_INVALID), (dict(ldo=7), mbd.E_INVALID),
    (dict(Y=1 * MB + 1), mbd.E_UNSUPPORTED), (dict(weights=3 * MB + 2), mbd.E_UNSUPPORTED), (dict(out=1 * MB), mbd.E_INVALID), (dict(out=4 * MB + 16), mbd.E_INVALID),
    (dict(out=3 * MB + 16), mbd.E_INVALID), (dict(out=4 * MB, ldo=16), mbd.E_INVALID)])
def test_combine_refusals(args, status):
    assert mbd.lib().mbd_expert_combine(*{**COMBINE, **args}.values(), None) == status


@pytest.mark.parametrize("args,status", SIZES + [
    (dict(d_out=None), mbd.E_INVALID), (dict(Y=None), mbd.E_INVALID), (dict(weights=None), mbd.E_INVALID), (dict(dY=None), mbd.E_INVALID), (dict(ldd=7), mbd.E_INVALID),
    (dict(ldy=7), mbd.E_INVALID), (dict(lddy=7), mbd.E_INVALID), (dict(dY=2 * MB + 16), mbd.E_INVALID), (dict(dY=1 * MB), mbd.E_INVALID), (dict(dw=4 * MB), mbd.E_INVALID),
    (dict(dw=5 * MB), mbd.E_INVALID), (dict(dw=6 * MB + 2), mbd.E_UNSUPPORTED), (dict(dY=5 * MB + 1), mbd.E_UNSUPPORTED)])
def test_combine_backward_refusals(args, status):
    assert mbd.lib().mbd_expert_combine_backward(*{**BACKWARD, **args}.values(), None) == status


# ---------------------------------------------------------------------------------------------------- inputs
def _type(name):
    import torch
    return dict(bf16=torch.bfloat16, f32=torch.float32, i8=torch.int8)[name]


def _places(T, k, rows, seed, empty=0.15):
    """Distinct places in [0, rows) in any order, some slots empty: -1, and numbers that are no rows."""
    import torch
    rng = np.random.default_rng(seed)
    p = rng.permutation(max(rows, T * k))[:T * k]
    p[p >= rows] = -1
    gone = rng.random(T * k) < empty
    p[gone] = rng.choice([-1, rows, rows + 7, -2 ** 31, 2 ** 31 - 1], gone.sum())
    return torch.from_numpy(p.astype(np.int32).reshape(T, k)).cuda()


def _normal(gen, *shape, dtype="f32"):
    import torch
    return torch.randn(*shape, device="cuda", generator=gen).to(_type(dtype))


def _gen(seed):
    import torch
    return torch.Generator(device="cuda").manual_seed(seed)


def _check(got, want, mag, rel):
    import torch
    slack = rel * mag + torch.finfo(got.dtype).eps / 2 * (want.abs() + rel * mag) + 2.0 ** -133
    off = (got.double() - want).abs()
    assert not (off > slack).any(), (float((off / slack).max()), (off > slack).nonzero()[:4].tolist())


SHAPES = [(1, 1, 1), (1, 2, 4096), (3, 4, 7), (16, 2, 1024), (17, 8, 129), (300, 1, 1000), (33, 32, 65), (5, 3, 9000), (700, 5, 264), (2, 2, 40007), (400, 2, 513)]


# ---------------------------------------------------------------------------------------------------- dispatch
@pytest.mark.gpu
@pytest.mark.parametrize("T,k,K", SHAPES)
@pytest.mark.parametrize("dtype", ["bf16", "f32", "i8"])
def test_dispatch(T, k, K, dtype):
    import torch
    gen = _gen(T + K)
    x = torch.randint(-127, 128, (T, K), device="cuda", generator=gen).to(torch.int8) if dtype == "i8" else _normal(gen, T, K, dtype=dtype)
    rows = T * k + 3
    places = _places(T, k, rows, K)
    scale = _normal(gen, T) if dtype == "i8" else None
    for pad in (0, 1, 8):                                            # row strides: whole vectors, single elements
        out = torch.full((rows, K + pad), 7, dtype=x.dtype, device="cuda")
        out_scale = torch.full((rows,), 7.0, device="cuda") if dtype == "i8" else None
        mbd.expert_dispatch(x, places, out[:, :K], scale=scale, out_scale=out_scale)
        want, want_scale = torch.full_like(out, 7), torch.full((rows,), 7.0, device="cuda")
        t, j = torch.nonzero((places >= 0) & (places < rows), as_tuple=True)
        want[places[t, j].long(), :K] = x[t]
        assert torch.equal(out, want)
        if scale is not None:
            want_scale[places[t, j].long()] = scale[t]
            assert torch.equal(out_scale, want_scale)


@pytest.mark.gpu
def test_dispatch_of_views_at_any_offset():
    import torch
    for dtype in ("i8", "bf16", "f32"):
        base = torch.arange(40 * 77, device="cuda").view(40, 77).to(torch.float32).remainder(100).to(_type(dtype))
        for first in (0, 1, 2, 3, 4, 8):
            for width in (1, 5, 16, 33, 64):
                x = base[:, first:first + width]
                places = _places(40, 2, 80, first * 100 + width, 0.0)
                buf = torch.full((80, 90), 55, dtype=x.dtype, device="cuda")
                mbd.expert_dispatch(x, places, buf[:, first + 3:first + 3 + width])
                want = torch.full_like(buf, 55)
                want[places.long().view(-1), first + 3:first + 3 + width] = x.repeat_interleave(2, 0)
                assert torch.equal(buf, want)


# ---------------------------------------------------------------------------------------------------- combine
def _combine64(y, places, weights, residual, T, K):
    import torch
    rows = y.shape[0]
    there = (places >= 0) & (places < rows)
    w = torch.where(there, weights.double() if weights is not None else 1.0, 0.0)
    picked = torch.where(there.unsqueeze(2), y.double()[places.long().clamp(0, max(rows - 1, 0))], 0.0) * w.unsqueeze(2)
    r = residual.double() if residual is not None else torch.zeros(T, K, dtype=torch.float64, device="cuda")
    return r + picked.sum(1), r.abs() + picked.abs().sum(1)


@pytest.mark.gpu
@pytest.mark.parametrize("T,k,K", SHAPES)
@pytest.mark.parametrize("y,out", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "bf16"), ("f32", "f32")])
def test_combine(T, k, K, y, out):
    import torch
    gen = _gen(T * 3 + K)
    rows = T * k + 2
    Y, places, w = _normal(gen, rows, K, dtype=y), _places(T, k, rows, K + 1), _normal(gen, T, k)
    unused = torch.ones(rows, dtype=torch.bool, device="cuda")
    unused[places[(places >= 0) & (places < rows)].long()] = False
    Y[unused] = float("nan")                                         # rows of nobody stay out
    w = torch.where((places >= 0) & (places < rows), w, float("nan"))  # so do weights of empty slots
    for weights in (w, None):
        for residual in (_normal(gen, T, K, dtype=out), None):
            O = torch.full((T, K), 5.0, dtype=_type(out), device="cuda")
            mbd.expert_combine(Y, places, O, weights=weights, residual=residual)
            Z = torch.nan_to_num(Y, nan=0.0)
            want, mag = _combine64(Z, places, weights, residual, T, K)
            _check(O, want, mag, (k + 1) * U)
            if residual is not None:
                mbd.expert_combine(Y, places, residual, weights=weights, residual=residual)      # in the residual's place
                assert torch.equal(residual, O)


@pytest.mark.gpu
def test_combine_of_views_and_of_no_rows():
    import torch
    gen = _gen(1)
    for K in (96, 101):
        big = _normal(gen, 64, 3 * K + 9, dtype="bf16")
        before = big.clone()
        Y, places = _normal(gen, 128, K + 8, dtype="bf16")[:, 3:K + 3], _places(64, 2, 128, K)
        res, out = big[:, 1:K + 1], big[:, 2 * K + 2:3 * K + 2]
        w = _normal(gen, 64, 2)
        mbd.expert_combine(Y, places, out, weights=w, residual=res)
        want, mag = _combine64(Y, places, w, before[:, 1:K + 1], 64, K)
        _check(out, want, mag, 3 * U)
        assert torch.equal(big[:, :2 * K + 2], before[:, :2 * K + 2]) and torch.equal(big[:, 3 * K + 2:], before[:, 3 * K + 2:])
        none = torch.empty(0, K, dtype=torch.bfloat16, device="cuda")
        o = torch.full((64, K), 3.0, dtype=torch.bfloat16, device="cuda")
        mbd.expert_combine(none, places, o, residual=res.contiguous())
        assert torch.equal(o, before[:, 1:K + 1])
        mbd.expert_combine(none, places, o)
        assert not o.any()


# ---------------------------------------------------------------------------------------------------- backward
@pytest.mark.gpu
@pytest.mark.parametrize("T,k,K", SHAPES)
@pytest.mark.parametrize("d,y", [("bf16", "bf16"), ("f32", "f32"), ("bf16", "f32"), ("f32", "bf16")])
def test_combine_backward(T, k, K, d, y):
    import torch
    gen = _gen(T * 5 + K)
    rows = T * k + 2
    D, Y, places, w = _normal(gen, T, K, dtype=d), _normal(gen, rows, K, dtype=y), _places(T, k, rows, K + 2), _normal(gen, T, k)
    dY, dw = torch.full_like(Y, 5.0), torch.full((T, k), 5.0, device="cuda")
    mbd.expert_combine_backward(D, Y, places, w, dY, dw)
    there = (places >= 0) & (places < rows)
    t, j = torch.nonzero(there, as_tuple=True)
    at = places[t, j].long()
    want = torch.full(Y.shape, 5.0, dtype=torch.float64, device="cuda")
    want[at] = D.double()[t] * w.double()[t, j][:, None]
    _check(dY, want, want.abs(), U)
    prod = torch.zeros(T, k, K, dtype=torch.float64, device="cuda")
    prod[t, j] = D.double()[t] * Y.double()[at]
    # eight products a thread, five steps within a warp, one more per piece of the row, the warps
    _check(dw, prod.sum(2), prod.abs().sum(2), (24 + K / 256) * U)
    assert not dw[~there].any()
    dY2 = torch.full_like(Y, 5.0)
    mbd.expert_combine_backward(D, None, places, w, dY2)
    assert torch.equal(dY2, dY)
    Z, dw2 = Y.clone(), torch.empty_like(dw)
    mbd.expert_combine_backward(D, Z, places, w, Z, dw2)             # in Y's place
    keep = torch.ones(rows, dtype=torch.bool, device="cuda")
    keep[at] = False
    assert torch.equal(Z[at], dY[at]) and torch.equal(Z[keep], Y[keep]) and torch.equal(dw2, dw)


@pytest.mark.gpu
def test_gradients_against_differences():
    """combine is linear in the rows and in the weights: differences of any size are its gradients but for roundings."""
    import torch
    gen = _gen(4)
    T, k, K = 9, 3, 200
    Y, places, w, c = _normal(gen, 27, K), _places(T, k, 27, 1), _normal(gen, T, k), _normal(gen, T, K)
    dY, dw = torch.zeros_like(Y), torch.empty_like(w)
    mbd.expert_combine_backward(c, Y, places, w, dY, dw)
    e, f = _normal(gen, 27, K), _normal(gen, T, k)

    def loss(Y, w):
        o = mbd.expert_combine(Y, places, torch.empty(T, K, device="cuda"), weights=w)
        return float((c.double() * o.double()).sum()), float((c.double() * o.double()).abs().sum())

    for (a, ma), (b, mb), got in ((loss(Y + e, w), loss(Y - e, w), float((dY.double() * e.double()).sum())), (loss(Y, w + f), loss(Y, w - f), float((dw.double() * f.double()).sum()))):
        assert abs((a - b) / 2 - got) <= 100 * U * (ma + mb)
    # dispatch: its gradient is combine without weights
    x, g = _normal(gen, T, K), _normal(gen, 27, K)
    out = mbd.expert_dispatch(x, places, torch.zeros(27, K, device="cuda"))
    dx = mbd.expert_combine(g, places, torch.empty(T, K, device="cuda"))
    a, b = (out.double() * g.double()), (x.double() * dx.double())
    assert abs(float(a.sum() - b.sum())) <= 10 * U * float(a.abs().sum())


@pytest.mark.gpu
def test_rows_behind_2_to_the_31_elements():
    import torch
    rows, K = 530000, 4104                                           # 2.17e9 bf16 elements
    Y = torch.empty(rows, K, dtype=torch.bfloat16, device="cuda")
    gen = _gen(2)
    x = _normal(gen, 3, K, dtype="bf16")
    places = torch.tensor([[rows - 1, 0], [rows - 2, 5], [rows - 9, -1]], dtype=torch.int32, device="cuda")
    mbd.expert_dispatch(x, places, Y)
    for t in range(3):
        assert torch.equal(Y[int(places[t, 0])], x[t])
    w = _normal(gen, 3, 2)
    out = mbd.expert_combine(Y, places, torch.empty(3, K, device="cuda"), weights=w)
    want = x.double() * torch.where(places >= 0, w.double(), 0.0).sum(1, keepdim=True)
    assert ((out.double() - want).abs() <= 4 * U * x.double().abs() * w.double().abs().sum(1, keepdim=True)).all()
    dw = torch.empty(3, 2, device="cuda")
    mbd.expert_combine_backward(x, Y, places, w, Y, dw)
    assert torch.equal(Y[rows - 1], (x[0].float() * w[0, 0]).to(torch.bfloat16))


# ---------------------------------------------------------------------------------------------------- the forms of large batches
# From 512 tokens and 512 columns on a thread has two or four vectors; the last one ragged, more columns than a block's threads have at once, and
# rows that move element by element.
LARGE = [(513, 1, 512), (513, 2, 4096), (600, 1, 1032), (520, 2, 520), (520, 3, 520), (515, 4, 1000), (513, 3, 4104), (514, 5, 1024), (515, 8, 1024), (513, 7, 4104),
         (512, 2, 16392), (512, 4, 9000), (512, 6, 9000), (513, 32, 520), (530, 2, 1001), (512, 5, 2049)]


@pytest.mark.gpu
@pytest.mark.parametrize("T,k,K", LARGE)
@pytest.mark.parametrize("y,out", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "bf16"), ("f32", "f32")])
def test_combine_of_large_batches(T, k, K, y, out):
    test_combine(T, k, K, y, out)


@pytest.mark.gpu
@pytest.mark.parametrize("T,k,K", LARGE)
@pytest.mark.parametrize("d,y", [("bf16", "bf16"), ("f32", "f32"), ("bf16", "f32"), ("f32", "bf16")])
def test_combine_backward_of_large_batches(T, k, K, d, y):
    test_combine_backward(T, k, K, d, y)


@pytest.mark.gpu
@pytest.mark.parametrize("T,k,K", LARGE)
@pytest.mark.parametrize("dtype", ["bf16", "f32", "i8"])
def test_dispatch_of_large_batches(T, k, K, dtype):
    test_dispatch(T, k, K, dtype)


@pytest.mark.gpu
def test_products_with_rows_behind_2_to_the_31_elements():
    """d_weights of rows at both ends of a tensor of 2.17e9 elements: eight products a thread, the steps within a warp and between the warps."""
    import torch
    rows, K = 530000, 4104
    Y = torch.empty(rows, K, dtype=torch.bfloat16, device="cuda")
    gen = _gen(6)
    places = torch.tensor([[rows - 1, 0], [rows - 2, 5], [rows - 9, -1]], dtype=torch.int32, device="cuda")
    for at in places.flatten().tolist():
        if at >= 0:
            Y[at] = _normal(gen, K, dtype="bf16")
    x, w, dw = _normal(gen, 3, K, dtype="bf16"), _normal(gen, 3, 2), torch.full((3, 2), 5.0, device="cuda")
    picked = torch.stack([torch.stack([Y[max(at, 0)] for at in row]) for row in places.tolist()]).double()
    mbd.expert_combine_backward(x, Y, places, w, Y, dw)
    prod = x.double()[:, None] * picked * (places >= 0).unsqueeze(2)
    _check(dw, prod.sum(2), prod.abs().sum(2), (24 + K / 256) * U)
    for t in range(3):
        for j in range(2):
            if int(places[t, j]) >= 0:
                assert torch.equal(Y[int(places[t, j])], (x[t].float() * w[t, j]).bfloat16())
