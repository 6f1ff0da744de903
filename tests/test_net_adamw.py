"""AdamW inside a network (mbd_enable_adamw): a trajectory in the fp32 mode against the oracle's gradients and the formulas in
64 bits, bf16 networks step by step from the gradient the device itself materialised (fused, un-fused, captured; with masters, in
8 bits), the order of the switches, refusals; and the operators of an expert layer used together: trained, then answered with in 8 bits."""
import numpy as np
import pytest

from paper_1712_04432_b200 import inputs as I
from tests.helpers import rel_fro, to_dev, to_np


def test_refusals_without_a_network():
    from paper_1712_04432_b200 import mbd
    assert mbd.lib().mbd_enable_adamw(None, 0.9, 0.999, 1e-8, 0.0, 32) == mbd.E_INVALID


def _step(p, g, m, v, t, lr, wd, b1=0.9, b2=0.999, eps=1e-8):
    m = b1 * m + (1 - b1) * g
    v = b2 * v + (1 - b2) * g * g
    return p * (1 - lr * wd) - lr * (m / (1 - b1 ** t)) / (np.sqrt(v / (1 - b2 ** t)) + eps), m, v


@pytest.mark.gpu
def test_fp32_trajectory_follows_the_oracle():
    import torch
    from oracle import mbd_oracle as O
    from paper_1712_04432_b200 import mbd
    w = I.fc_workload((96, 64, 48, 10), 32, "fp32")
    inp = I.make_inputs(w, seed=5)
    eta, wd, L = 0.002, 0.05, len(inp.Ws)
    net = mbd.Net(mbd.fc_layers(w.dims, bias=True), w.B, 2, 2, mbd.F32, mbd.LOSS_SOFTMAX_CE, 2)
    # eps far above the rounding of a gradient: with a tiny one the first step is the gradient's sign, and an oracle would have to
    # agree about zeros
    eps = 1e-3
    net.enable_adamw(eps=eps, weight_decay=wd)
    for i in range(L):
        net.set_weights(i, torch.from_numpy(inp.Ws[i]).cuda(), torch.from_numpy(inp.bs[i]).cuda())
    X, labels = torch.from_numpy(inp.X).cuda(), torch.from_numpy(inp.labels).cuda()
    Ws, bs = [a.astype(np.float64) for a in inp.Ws], [a.astype(np.float64) for a in inp.bs]
    M = [(np.zeros_like(a), np.zeros_like(a)) for a in Ws]
    Mb = [(np.zeros_like(a), np.zeros_like(a)) for a in bs]
    for t in range(1, 6):
        layers = [O.FC(Ws[i], bs[i], relu=(i < L - 1)) for i in range(L)]
        o = O.train_step(layers, inp.X.astype(np.float64).T, inp.labels, "softmax_ce", eta)
        for i in range(L):
            Ws[i], *M[i] = _step(Ws[i], o["dWs"][i] / w.B, *M[i], t, eta, wd, eps=eps)
            bs[i], *Mb[i] = _step(bs[i], o["dbs"][i].reshape(bs[i].shape) / w.B, *Mb[i], t, eta, 0.0, eps=eps)
        net.forward(X, labels)
        if t % 2:
            net.backward(eta)
        else:
            net.backward(0.0); net.sgd_step(eta)
        net.poll()
        for i in range(L):
            Wg, bg = net.get_weights(i, with_bias=True)
            assert rel_fro(to_np(Wg), Ws[i]) < 1e-5 and rel_fro(to_np(bg), bs[i]) < 1e-4, (t, i)
            assert rel_fro(to_np(net.get_tensor(mbd.T_ADAM_M, i)), M[i][0]) < 1e-4 and rel_fro(to_np(net.get_tensor(mbd.T_ADAM_V, i)), M[i][1]) < 1e-4
            assert rel_fro(to_np(net.get_tensor(mbd.T_ADAM_M_BIAS, i)), Mb[i][0]) < 1e-4 and rel_fro(to_np(net.get_tensor(mbd.T_ADAM_V_BIAS, i)), Mb[i][1]) < 1e-4
    net.close()


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("master", ["before", "after", None])
@pytest.mark.parametrize("grid,mp", [((1, 1), 0), ((2, 4), 2)])
def test_bf16_networks_step_as_the_list_does(grid, mp, master, bits):
    # the same gradients through the stand-alone list: bit for bit, whether the step is fused, on its own or captured
    import torch
    from paper_1712_04432_b200 import mbd
    w = I.fc_workload((136, 72, 40, 24), 32, "bf16")
    inp = I.make_inputs(w, seed=81)
    L, eta, wd = len(inp.Ws), 0.01, 0.1
    X, labels = to_dev(inp.X, True), torch.from_numpy(inp.labels).cuda()
    stream = torch.cuda.Stream()

    def make(s=None):
        net = mbd.Net(mbd.fc_layers(w.dims, bias=True), w.B, grid[0], grid[1], mbd.BF16, mbd.LOSS_SOFTMAX_CE, mp, stream=s)
        if master == "before":
            net.enable_master_weights()
        net.enable_adamw(weight_decay=wd, state_bits=bits)
        for i in range(L):
            net.set_weights(i, to_dev(inp.Ws[i], True), torch.from_numpy(inp.bs[i]).cuda())
        if master == "after":
            net.enable_master_weights()
        torch.cuda.synchronize()
        return net
    nets = {"unfused": make(), "fused": make(), "graph": make(stream)}
    u = nets["unfused"]
    Ws = [to_dev(inp.Ws[i], True) for i in range(L)]
    bs = [torch.from_numpy(inp.bs[i]).cuda() for i in range(L)]
    params = [x for p in zip(Ws, bs) for x in p]
    masters = [x for p in Ws for x in (p.float(), None)] if master else None
    grads = [torch.zeros(x.shape, device="cuda") for x in params]
    opt = mbd.AdamW(params, grads, masters=masters, weight_decay=[wd, 0.0] * L, state_bits=bits)
    for step in range(3):
        u.forward(X, labels); u.backward(0.0)
        for i in range(L):
            grads[2 * i].copy_(u.get_tensor(mbd.T_DW, i)); grads[2 * i + 1].copy_(u.get_tensor(mbd.T_DB, i))
        u.sgd_step(eta)
        opt.step(np.float32(eta), grad_scale=1.0 / w.B)
        nets["fused"].forward(X, labels); nets["fused"].backward(eta)
        torch.cuda.synchronize()
        nets["graph"].train_step(X, labels, eta)
        for n in nets.values():
            n.poll()
        torch.cuda.synchronize()
        for name, n in nets.items():
            for i in range(L):
                W, b = n.get_weights(i, with_bias=True)
                torch.cuda.synchronize()
                assert torch.equal(W, Ws[i]) and torch.equal(b, bs[i]), (name, step, i)
                if master:
                    Wm = n.get_tensor(mbd.T_MASTER, i)
                    torch.cuda.synchronize()
                    assert torch.equal(Wm, masters[2 * i])
    assert not torch.equal(Ws[0], to_dev(inp.Ws[0], True))
    for n in nets.values():
        n.close()
    opt.close()


@pytest.mark.gpu
def test_switches_and_refusals():
    import torch
    from paper_1712_04432_b200 import mbd
    from tests.helpers import mixed_layers
    net = mbd.Net(mbd.fc_layers((64, 32, 16)), 8, 1, 1, mbd.F32, mbd.LOSS_SOFTMAX_CE, 0)
    for bad, status in ((dict(betas=(1.0, 0.9)), mbd.E_INVALID), (dict(betas=(0.9, -0.1)), mbd.E_INVALID), (dict(eps=0.0), mbd.E_INVALID),
                        (dict(weight_decay=-1.0), mbd.E_INVALID), (dict(state_bits=16), mbd.E_UNSUPPORTED)):
        with pytest.raises(mbd.MbdError) as e:
            net.enable_adamw(**bad)
        assert e.value.status == status
    with pytest.raises(mbd.MbdError):
        net.get_tensor(mbd.T_ADAM_M, 0)                  # no moments before
    X, labels = torch.randn(8, 64, device="cuda"), torch.zeros(8, dtype=torch.int32, device="cuda")
    for i, (a, b) in enumerate(((32, 64), (16, 32))):
        net.set_weights(i, torch.randn(a, b, device="cuda") * 0.1, torch.zeros(a, device="cuda"))
    net.enable_adamw(state_bits=8)
    net.train_step(X, labels, 0.01); net.poll()
    net.enable_adamw(state_bits=32)                      # other moments, from nothing
    assert not net.get_tensor(mbd.T_ADAM_M, 0).any()
    net.train_step(X, labels, 0.01); net.poll()
    assert net.get_tensor(mbd.T_ADAM_M, 0).any()
    net.enable_adamw()                                   # again: reset
    assert not net.get_tensor(mbd.T_ADAM_M, 0).any()
    net.enable_momentum(0.5)                             # the one enabled last
    before = net.get_weights(0)
    net.forward(X, labels); net.backward(0.0)
    dW = net.get_tensor(mbd.T_DW, 0)
    net.sgd_step(0.5); net.poll()
    assert rel_fro(to_np(net.get_weights(0) - before), -0.5 / 8 * to_np(dW)) < 1e-4
    net.close()
    w = I.mixed_workload(64, 8, 40, 2, (128, 16), 6, name="mixed_adamw")
    net = mbd.Net(mixed_layers(w), w.B, 1, 1, mbd.BF16, mbd.LOSS_SOFTMAX_CE, 0)
    with pytest.raises(mbd.MbdError) as e:
        net.enable_adamw()
    assert e.value.status == mbd.E_UNSUPPORTED
    net.close()


@pytest.mark.gpu
def test_an_expert_layer_trained_and_then_answered_with_in_8_bits():
    # two layers of 6 experts: forward, loss, both backward products, AdamW over all experts' tensors, one captured step replayed; the
    # gradients against 64 bits; then the trained weights in 8 bits on new rows
    import torch
    from paper_1712_04432_b200 import mbd
    gen = torch.Generator(device="cuda")
    gen.manual_seed(21)
    E, T, d0, d1, d2 = 6, 300, 64, 128, 40
    counts = torch.tensor([70, 0, 129, 1, 60, 33])
    offsets = torch.cat([torch.zeros(1), counts.cumsum(0)]).to(torch.int32).cuda()          # 293 rows; 7 of padding
    rn = lambda *s, k=1.0: (torch.randn(*s, device="cuda", generator=gen) * k)  # noqa: E731
    X = rn(T, d0).to(torch.bfloat16)
    labels = torch.randint(0, d2, (T,), device="cuda", generator=gen).to(torch.int32)
    masters = [rn(E, d1, d0, k=d0 ** -0.5), rn(E, d2, d1, k=d1 ** -0.5)]
    W = [m.to(torch.bfloat16) for m in masters]
    b = torch.zeros(E, d1, device="cuda")
    H, Y = torch.zeros(T, d1, dtype=torch.bfloat16, device="cuda"), torch.zeros(T, d2, device="cuda")
    dY, dH, loss = torch.zeros(T, d2, dtype=torch.bfloat16, device="cuda"), torch.zeros(T, d1, dtype=torch.bfloat16, device="cuda"), torch.zeros(T, device="cuda")
    dW = [torch.zeros(E, d1, d0, device="cuda"), torch.zeros(E, d2, d1, device="cuda")]
    db = torch.zeros(E, d1, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    opt = mbd.AdamW([*W, b], [*dW, db], masters=[*masters, None], weight_decay=[0.01, 0.01, 0.0], state_bits=8)

    def step():
        mbd.expert_gemm(0, X, W[0], offsets, H, relu=True, bias=b, status=status)
        mbd.expert_gemm(0, H, W[1], offsets, Y, status=status)
        mbd.softmax_xent(Y, labels, dY, loss, sync=False)
        mbd.expert_gemm(1, dY, W[1], offsets, dH, op=mbd.TAIL_MASK, mask=H, status=status)
        mbd.expert_gemm(2, dY, H, offsets, dW[1], status=status)
        mbd.expert_gemm(2, dH, X, offsets, dW[0], status=status)
        opt.step(3e-3, grad_scale=1.0 / 293)
    step()
    torch.cuda.synchronize()
    # the gradients of that step, from its own stored activations (each a decision or one rounding), in 64 bits
    bounds = offsets.tolist()
    W64 = [m.double() for m in (dW[0], dW[1])]
    for e in range(E):
        s = slice(bounds[e], bounds[e + 1])
        assert rel_fro(to_np(W64[1][e]), to_np(dY[s].double().T @ H[s].double())) < 2e-5 if bounds[e + 1] > bounds[e] else not dW[1][e].any()
        assert rel_fro(to_np(W64[0][e]), to_np(dH[s].double().T @ X[s].double())) < 2e-5 if bounds[e + 1] > bounds[e] else not dW[0][e].any()
    first = float(loss[:293].sum())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert opt.steps_done == 4 and int(status) == 0 and np.isfinite(first) and torch.isfinite(loss[:293]).all()
    assert torch.equal(W[0], masters[0].to(torch.bfloat16)) and torch.equal(W[1], masters[1].to(torch.bfloat16))
    # an expert without rows is only decayed
    assert not H[293:].any() and not Y[293:].any()
    # answer with the trained weights in 8 bits, one scale per output channel and one per row
    Wq, Ws = [torch.empty(m.shape, dtype=torch.int8, device="cuda") for m in masters], [torch.empty(m.shape[:2], device="cuda") for m in masters]
    for k in range(2):
        mbd.quantize_rows(masters[k], Wq[k], Ws[k])
    q, s = torch.empty(T, d0, dtype=torch.int8, device="cuda"), torch.empty(T, device="cuda")
    out = torch.zeros(T, d1, device="cuda")
    mbd.quantize_rows(X, q, s)
    mbd.expert_gemm_i8(q, s, Wq[0], Ws[0], offsets, out, relu=True, bias=b, status=status)
    torch.cuda.synchronize()
    for e in range(E):
        at = slice(bounds[e], bounds[e + 1])
        ref = X[at].double() @ masters[0][e].double().T
        # each row and each channel is off by half a step of its scale at most
        slack = 0.5 * s[at].double()[:, None] * masters[0][e].double().abs().sum(1) + 0.5 * Ws[0][e].double() * 127 * d0 * s[at].double()[:, None]
        assert ((out[at].double() - (ref + b[e].double()).relu()).abs() <= 1.001 * slack).all()
    opt.close()
