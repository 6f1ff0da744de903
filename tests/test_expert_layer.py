"""An expert layer as it is used: norm, routing, the rows to the experts, two products grouped by expert, the rows back onto the residual
stream; its gradients in the opposite order; the same layer answering in 8 bits.  Each step is compared with its formula in 64 bits on what the steps
before it left, so that every tolerance is that of one step: float roundings (U = 2^-24 each) and half a step of the result's type."""
import pytest

from paper_1712_04432_b200 import mbd

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
T, D, H, E, K_TOP = 200, 136, 72, 6, 2
LIVE = 187


def _close(got, want, mag, rel):
    import torch
    slack = rel * mag + torch.finfo(got.dtype).eps / 2 * (want.abs() + rel * mag) + 2.0 ** -133
    off = (got.double() - want).abs()
    assert not (off > slack).any(), float((off / slack).max())


class Layer:
    """Weights in bf16; all buffers made once, so that a step can be captured."""

    def __init__(self):
        import torch
        gen = torch.Generator(device="cuda").manual_seed(5)
        bf = dict(dtype=torch.bfloat16, device="cuda")
        f = dict(device="cuda")
        n = lambda *s: torch.randn(*s, device="cuda", generator=gen)  # noqa: E731
        self.gain, self.gate = 1 + 0.2 * n(D), (n(8, D) * D ** -0.5).bfloat16()      # the router's product wants multiples of 8: two experts of no one
        self.up, self.down = (n(E, H, D) * D ** -0.5).bfloat16(), (n(E, D, H) * H ** -0.5).bfloat16()
        self.router = mbd.Router(E, K_TOP, mbd.ROUTE_SOFTMAX, True)
        self.count = torch.tensor([LIVE], dtype=torch.int32, device="cuda")
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.x, self.stream = n(T, D).bfloat16(), (2 * n(T, D)).bfloat16()
        self.h, self.y = torch.empty(T, D, **bf), torch.empty(T, D, **bf)
        self.logits, self.bias = torch.empty(T, 8, **f), torch.zeros(E, **f)
        self.ids, self.places = torch.empty(T, K_TOP, dtype=torch.int32, **f), torch.empty(T, K_TOP, dtype=torch.int32, **f)
        self.w, self.offsets = torch.empty(T, K_TOP, **f), torch.empty(E + 1, dtype=torch.int32, **f)
        self.xs, self.a, self.ys = torch.zeros(T * K_TOP, D, **bf), torch.zeros(T * K_TOP, H, **bf), torch.zeros(T * K_TOP, D, **bf)
        self.out = torch.empty(T, D, **bf)
        self.d_out = (0.1 * n(T, D)).bfloat16()
        self.dys, self.da, self.dxs, self.dw = torch.zeros_like(self.ys), torch.zeros_like(self.a), torch.zeros_like(self.xs), torch.empty(T, K_TOP, **f)
        self.d_up, self.d_down = torch.empty(E, H, D, **f), torch.empty(E, D, H, **f)
        self.d_logits = torch.zeros(T, 8, **bf)
        self.dy_rows, self.dy, self.d_gate = torch.empty(T, D, **f), torch.empty(T, D, **f), torch.empty(8, D, **f)
        self.dx, self.d_gain, self.scratch = torch.empty(T, D, **bf), torch.empty(D, **f), torch.empty(T * D, **f)
        self.route_scratch = torch.empty(mbd.expert_route_scratch(T, E), dtype=torch.int32, **f)

    def forward(self):
        mbd.rms_norm(self.x, gain=self.gain, residual=self.stream, h=self.h, y=self.y)
        mbd.block_gemm(0, self.y, self.gate, self.logits, status=self.status)
        mbd.expert_route(self.router, self.logits[:, :E], self.ids, self.w, self.places, self.offsets, count=self.count, scratch=self.route_scratch)
        mbd.expert_dispatch(self.y, self.places, self.xs)
        mbd.expert_gemm(0, self.xs, self.up, self.offsets, self.a, relu=True, status=self.status)
        mbd.expert_gemm(0, self.a, self.down, self.offsets, self.ys, status=self.status)
        mbd.expert_combine(self.ys, self.places, self.out, weights=self.w, residual=self.h)

    def backward(self):
        mbd.expert_combine_backward(self.d_out, self.ys, self.places, self.w, self.dys, self.dw)
        mbd.expert_gemm(2, self.dys, self.a, self.offsets, self.d_down, status=self.status)
        mbd.expert_gemm(1, self.dys, self.down, self.offsets, self.da, op=mbd.TAIL_MASK, mask=self.a, status=self.status)
        mbd.expert_gemm(2, self.da, self.xs, self.offsets, self.d_up, status=self.status)
        mbd.expert_gemm(1, self.da, self.up, self.offsets, self.dxs, op=mbd.TAIL_MASK, status=self.status)
        mbd.expert_route_backward(self.router, self.logits[:, :E], self.ids, self.dw, self.d_logits[:, :E])
        mbd.block_gemm(2, self.d_logits, self.y, self.d_gate, status=self.status)
        mbd.block_gemm(1, self.d_logits, self.gate, self.dy_rows, status=self.status)
        mbd.expert_combine(self.dxs, self.places, self.dy, residual=self.dy_rows)        # both ways into y
        mbd.rms_norm_backward(self.dy, self.h, self.dx, gain=self.gain, d_residual=self.d_out, d_gain=self.d_gain, scratch=self.scratch)

    def results(self):
        return [self.out, self.h, self.offsets, self.places, self.d_up, self.d_down, self.d_gate, self.dx, self.d_gain]


def _groups(offsets):
    o = offsets.tolist()
    return [slice(o[e], o[e + 1]) for e in range(E)]


def test_layer_forward_and_gradients():
    import torch
    L = Layer()
    L.forward()
    L.backward()
    torch.cuda.synchronize()
    assert int(L.status) == 0
    d = lambda t: t.double()  # noqa: E731
    # forward
    assert torch.equal(L.h, (L.x.float() + L.stream.float()).bfloat16())
    r = 1 / (d(L.h).square().mean(1, keepdim=True) + 1e-6).sqrt()
    _close(L.y, d(L.h) * r * d(L.gain), (d(L.h) * r * d(L.gain)).abs(), 30 * U)
    _close(L.logits, d(L.y) @ d(L.gate).T, d(L.y).abs() @ d(L.gate).abs().T, 2 * D * U)
    top = torch.topk(L.logits[:LIVE, :E], K_TOP, dim=1)
    assert torch.equal(L.ids[:LIVE], top.indices.int()) and (L.ids[LIVE:] == -1).all()
    w = torch.softmax(d(top.values), 1)
    _close(L.w[:LIVE], w, w, 100 * U)
    assert L.offsets[-1] == LIVE * K_TOP and torch.equal(L.xs[L.places[:LIVE].long()], L.y[:LIVE, None].expand(-1, K_TOP, -1)) and not L.xs[LIVE * K_TOP:].any()
    for e, at in enumerate(_groups(L.offsets)):
        _close(L.a[at], (d(L.xs[at]) @ d(L.up[e]).T).relu(), d(L.xs[at]).abs() @ d(L.up[e]).abs().T, 2 * D * U)
        _close(L.ys[at], d(L.a[at]) @ d(L.down[e]).T, d(L.a[at]).abs() @ d(L.down[e]).abs().T, 2 * H * U)
    y = d(L.ys)[L.places[:LIVE].long()]
    want, mag = d(L.h).clone(), d(L.h).abs()
    want[:LIVE] += (y * d(L.w)[:LIVE, :, None]).sum(1)
    mag[:LIVE] += (y * d(L.w)[:LIVE, :, None]).abs().sum(1)
    _close(L.out, want, mag, 3 * U)
    # gradients
    _close(L.dw[:LIVE], (d(L.d_out)[:LIVE, None] * y).sum(2), (d(L.d_out)[:LIVE, None] * y).abs().sum(2), 40 * U)
    assert not L.dw[LIVE:].any() and not L.dys[LIVE * K_TOP:].any()
    g = d(L.d_out)[:LIVE, None] * d(L.w)[:LIVE, :, None]
    _close(L.dys[L.places[:LIVE].long()], g, g.abs(), U)
    for e, at in enumerate(_groups(L.offsets)):
        n = max(1, at.stop - at.start)
        _close(L.d_down[e], d(L.dys[at]).T @ d(L.a[at]), d(L.dys[at]).abs().T @ d(L.a[at]).abs(), 2 * n * U)
        _close(L.da[at], (d(L.dys[at]) @ d(L.down[e])) * (L.a[at] > 0), d(L.dys[at]).abs() @ d(L.down[e]).abs(), 2 * D * U)
        _close(L.d_up[e], d(L.da[at]).T @ d(L.xs[at]), d(L.da[at]).abs().T @ d(L.xs[at]).abs(), 2 * n * U)
        _close(L.dxs[at], d(L.da[at]) @ d(L.up[e]), d(L.da[at]).abs() @ d(L.up[e]).abs(), 2 * H * U)
    l = d(L.logits)[:LIVE, :E].clone().requires_grad_()
    s = torch.softmax(l.gather(1, top.indices), 1)
    (gl,) = torch.autograd.grad(s, l, d(L.dw)[:LIVE])
    ml = torch.zeros_like(gl).scatter_(1, top.indices, w * (d(L.dw)[:LIVE].abs() + (w * d(L.dw)[:LIVE].abs()).sum(1, keepdim=True)))
    _close(L.d_logits[:LIVE, :E], gl, ml, 100 * U)
    assert not L.d_logits[LIVE:].any() and not L.d_logits[:, E:].any()
    _close(L.d_gate, d(L.d_logits).T @ d(L.y), d(L.d_logits).abs().T @ d(L.y).abs(), 2 * T * U)
    rows, mag = d(L.dy_rows).clone(), d(L.dy_rows).abs()
    rows[:LIVE] += d(L.dxs)[L.places[:LIVE].long()].sum(1)
    mag[:LIVE] += d(L.dxs)[L.places[:LIVE].long()].abs().sum(1)
    _close(L.dy, rows, mag, 3 * U)
    unit, g = d(L.h) * r, d(L.dy) * d(L.gain)
    _close(L.dx, r * (g - unit * (g * unit).mean(1, keepdim=True)) + d(L.d_out), r * (g.abs() + unit.abs() * (g * unit).abs().mean(1, keepdim=True)) + d(L.d_out).abs(), 40 * U)
    _close(L.d_gain, (d(L.dy) * unit).sum(0), (d(L.dy) * unit).abs().sum(0), 150 * U)


def test_layer_captured_and_replayed_with_another_batch():
    import torch
    L = Layer()
    L.forward()                                                        # the first call on a device sets kernels up
    L.backward()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        L.forward()
        L.backward()
    for live in (LIVE, 3, 0, T):
        L.count.fill_(live)
        L.x.copy_(torch.randn(T, D, device="cuda"))
        for t in (L.xs, L.a, L.ys, L.dys, L.da, L.dxs):
            t.zero_()
        L.forward()
        L.backward()
        want = [t.clone() for t in L.results()]
        for t in L.results() + [L.xs, L.a, L.ys, L.dys, L.da, L.dxs]:
            t.zero_()
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(want, L.results()))
    assert int(L.status) == 0


@pytest.mark.parametrize("tokens", [1, 16, T])
def test_layer_answering_in_8_bits(tokens):
    """The norm leaves rows in 8 bits with scales, dispatch takes both along, the experts' products read them."""
    import torch
    L = Layer()
    L.forward()
    width = 144                                                        # int8 rows: strides of 16 bytes
    up_q, up_s = torch.zeros(E, H, width, dtype=torch.int8, device="cuda"), torch.empty(E, H, device="cuda")
    dense = torch.empty(E, H, D, dtype=torch.int8, device="cuda")
    mbd.quantize_rows(L.up, dense, up_s)
    up_q[..., :D] = dense
    x, res = L.x[:tokens], L.stream[:tokens]
    h, q, s = torch.empty_like(x), torch.zeros(tokens, width, dtype=torch.int8, device="cuda"), torch.empty(tokens, device="cuda")
    mbd.rms_norm(x, gain=L.gain, residual=res, h=h, q=q[:, :D], scale=s)
    ids, w, places, offsets = L.ids[:tokens].clone(), L.w[:tokens].clone(), L.places[:tokens].clone(), torch.empty(E + 1, dtype=torch.int32, device="cuda")
    mbd.expert_route(L.router, L.logits[:tokens, :E], ids, w, places, offsets, scratch=L.route_scratch)
    rows = tokens * K_TOP
    qs, ss, a = torch.zeros(rows, width, dtype=torch.int8, device="cuda"), torch.empty(rows, device="cuda"), torch.empty(rows, H, dtype=torch.float32, device="cuda")
    mbd.expert_dispatch(q, places, qs, scale=s, out_scale=ss)
    mbd.expert_gemm_i8(qs, ss, up_q, up_s, offsets, a)
    back = mbd.expert_combine(a, places, torch.empty(tokens, H, device="cuda"), weights=w)
    d = lambda t: t.double()  # noqa: E731
    assert int(offsets[-1]) == rows
    want = torch.zeros(tokens, H, dtype=torch.float64, device="cuda")
    mag = torch.zeros_like(want)
    for t in range(tokens):
        for j in range(K_TOP):
            e = int(ids[t, j])
            v = (d(q[t]) @ d(up_q[e]).T) * d(s[t]) * d(up_s[e]) * d(w[t, j])
            want[t] += v
            mag[t] += v.abs()
    _close(back, want, mag, 8 * U)
    # and the rows in 8 bits are the norm's, to half a step of each row's scale
    r = 1 / (d(h).square().mean(1, keepdim=True) + 1e-6).sqrt()
    assert ((d(q[:, :D]) * d(s)[:, None] - d(h) * r * d(L.gain)).abs() <= d(s)[:, None] * (0.5 + 130 * 40 * U)).all()
