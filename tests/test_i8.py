"""Rows in 8 bits (mbd_quantize_rows) and the products of 8-bit integers (mbd_gemm_i8, mbd_expert_gemm_i8) against 64 bits:
the integers and their sums exactly, the scaled results to the roundings of the last few operations."""
import numpy as np
import pytest

from paper_1712_04432_b200 import mbd


# ---------------------------------------------------------------------------------------------------- refusals (no GPU needed)
def _gemm(M=16, N=32, K=64, A=1 << 20, lda=64, sa=2 << 20, B=3 << 20, ldb=64, sb=4 << 20, out=5 << 20, ldo=32, op=mbd.TAIL_STORE, bias=None,
          experts=0, stride=64 * 32, offsets=7 << 20):
    import ctypes as C
    t = mbd.Tail(op, 1, 0, 0, out, ldo, bias, None, 0, 0.0)
    if experts:
        return mbd.lib().mbd_expert_gemm_i8(experts, offsets, M, N, K, A, lda, sa, B, ldb, stride, sb, C.byref(t), 6 << 20, None)
    return mbd.lib().mbd_gemm_i8(M, N, K, A, lda, sa, B, ldb, sb, C.byref(t), 6 << 20, None)


@pytest.mark.parametrize("args,status", [
    (dict(M=0), mbd.E_INVALID), (dict(N=0), mbd.E_INVALID), (dict(K=0), mbd.E_INVALID), (dict(A=None), mbd.E_INVALID),
    (dict(B=None), mbd.E_INVALID), (dict(sa=None), mbd.E_INVALID), (dict(sb=None), mbd.E_INVALID), (dict(out=None), mbd.E_INVALID),
    (dict(lda=48), mbd.E_INVALID), (dict(ldb=48), mbd.E_INVALID), (dict(ldo=24), mbd.E_INVALID),
    (dict(lda=72), mbd.E_UNSUPPORTED), (dict(ldb=72), mbd.E_UNSUPPORTED), (dict(ldo=36), mbd.E_UNSUPPORTED),
    (dict(A=(1 << 20) + 8), mbd.E_UNSUPPORTED), (dict(B=(3 << 20) + 8), mbd.E_UNSUPPORTED), (dict(sa=(2 << 20) + 2), mbd.E_UNSUPPORTED),
    (dict(K=131072, lda=131072, ldb=131072), mbd.E_UNSUPPORTED), (dict(op=mbd.TAIL_MASK), mbd.E_UNSUPPORTED),
    (dict(op=mbd.TAIL_SGD), mbd.E_UNSUPPORTED), (dict(experts=2, stride=64 * 31), mbd.E_INVALID),
    (dict(experts=2, stride=64 * 32 + 8), mbd.E_UNSUPPORTED), (dict(experts=513), mbd.E_UNSUPPORTED),
    (dict(experts=2, offsets=None), mbd.E_INVALID), (dict(experts=2, M=-1), mbd.E_INVALID),
])
def test_product_refusals(args, status):
    assert _gemm(**args) == status


@pytest.mark.parametrize("args,status", [
    (dict(R=-1), mbd.E_INVALID), (dict(K=0), mbd.E_INVALID), (dict(ldx=7), mbd.E_INVALID), (dict(ldq=7), mbd.E_INVALID),
    (dict(X=None), mbd.E_INVALID), (dict(Q=None), mbd.E_INVALID), (dict(S=None), mbd.E_INVALID),
    (dict(X=(1 << 20) + 1), mbd.E_UNSUPPORTED), (dict(S=(3 << 20) + 2), mbd.E_UNSUPPORTED), (dict(R=0, X=None), mbd.OK),
])
def test_quantize_refusals(args, status):
    a = dict(X=1 << 20, R=4, K=8, ldx=8, Q=2 << 20, ldq=8, S=3 << 20)
    a.update(args)
    assert mbd.lib().mbd_quantize_rows(a["X"], 1, a["R"], a["K"], a["ldx"], a["Q"], a["ldq"], a["S"], 0, None) == status


# ---------------------------------------------------------------------------------------------------- rows in 8 bits
def _want_rows(X):
    """scale and q of float32 rows on the host, from the definition in 64 bits (the scale is then a float)."""
    X = X.astype(np.float64)
    top = np.abs(X).max(1)
    with np.errstate(invalid="ignore", over="ignore"):
        s = (top.astype(np.float32) / np.float32(127)).astype(np.float32)
    s[~np.isfinite(top)] = np.nan
    q = np.zeros(X.shape, np.int8)
    some = s > 0
    q[some] = np.clip(np.rint(X[some] / s[some, None].astype(np.float64)), -127, 127)
    return s, q


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("R,K", [(1, 1), (1, 7), (3, 8), (5, 33), (2, 1001), (700, 64), (300, 1032), (4, 9216), (2, 32768), (1, 40007), (400, 8200),
                                 (700, 8192), (3000, 24), (601, 1003), (1300, 2056), (650, 16384), (2000, 8)])
def test_rows(R, K, dtype):
    import torch
    gen = torch.Generator(device="cuda")
    gen.manual_seed(R * 7 + K)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    X = (torch.randn(R, K, device="cuda", generator=gen) * torch.exp(3 * torch.randn(R, 1, device="cuda", generator=gen))).to(dt)
    X[:, ::5] = X[:, ::5].clamp_min(0.0)
    X[R // 2, : K // 2] = X[R // 2].abs().max() / 2              # half the largest: 63.5 steps, next to half a step
    q = torch.full((R, K), 99, dtype=torch.int8, device="cuda")
    s = torch.full((R,), -1.0, device="cuda")
    mbd.quantize_rows(X, q, s, sync=True)
    ws, wq = _want_rows(X.float().cpu().numpy())
    assert np.array_equal(s.cpu().numpy(), ws) and np.array_equal(q.cpu().numpy(), wq)


@pytest.mark.gpu
def test_rows_at_half_steps_and_at_the_ends_of_the_type():
    import torch
    steps = np.arange(-254, 255, dtype=np.float32) / 2             # every half step of a row whose scale is 1, 3, 1/3, a third's float
    rows = [np.concatenate([steps * np.float32(f), [127 * np.float32(f)]]) for f in (1.0, 3.0, 1 / 3, 0.1, 7e-31, 1e-38, 1.2e-36, 2.0 ** 120)]
    rows.append(np.zeros(510, np.float32))
    rows.append(np.full(510, 1e-45, np.float32))                   # the scale underflows
    rows.append(np.full(510, 2e-43, np.float32))
    bad = np.ones((3, 510), np.float32)
    bad[0, 3], bad[1, 5], bad[2, 0] = np.inf, np.nan, -np.inf
    X = np.concatenate([np.stack(rows).astype(np.float32), bad])
    # neighbours of the half steps, one unit away on each side
    X = np.concatenate([X, np.nextafter(X[:4], np.float32(np.inf)), np.nextafter(X[:4], np.float32(-np.inf))])
    q = torch.empty(X.shape, dtype=torch.int8, device="cuda")
    s = torch.empty(len(X), device="cuda")
    mbd.quantize_rows(torch.from_numpy(X).cuda(), q, s, sync=True)
    ws, wq = _want_rows(X)
    assert np.array_equal(s.cpu().numpy(), ws, equal_nan=True) and np.array_equal(q.cpu().numpy(), wq)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_of_views_at_any_offset(dtype):
    import torch
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    gen = torch.Generator(device="cuda")
    gen.manual_seed(3)
    base = torch.randn(9, 117, device="cuda", generator=gen).to(dt)
    X = base[:, 3:104]
    qbase = torch.full((9, 131), 77, dtype=torch.int8, device="cuda")
    q = qbase[:, 5:106]
    s = torch.empty(9, device="cuda")
    mbd.quantize_rows(X, q, s, sync=True)
    ws, wq = _want_rows(X.float().cpu().numpy())
    assert np.array_equal(s.cpu().numpy(), ws) and np.array_equal(q.cpu().numpy(), wq)
    assert (qbase[:, :5] == 77).all() and (qbase[:, 106:] == 77).all()
    W = torch.randn(3, 16, 40, device="cuda", generator=gen).to(dt)     # channels of a stack of matrices
    q, s = torch.empty(3, 16, 40, dtype=torch.int8, device="cuda"), torch.empty(3, 16, device="cuda")
    mbd.quantize_rows(W, q, s, sync=True)
    ws, wq = _want_rows(W.float().cpu().numpy().reshape(48, 40))
    assert np.array_equal(s.cpu().numpy().ravel(), ws) and np.array_equal(q.cpu().numpy().reshape(48, 40), wq)


# ---------------------------------------------------------------------------------------------------- products
def _ints(shape, gen, ld=None):
    import torch
    x = torch.randint(-127, 128, shape, device="cuda", generator=gen).to(torch.int8)
    if ld is None or ld == shape[-1]:
        return x
    wide = torch.full((*shape[:-1], ld), 101, dtype=torch.int8, device="cuda")
    wide[..., :shape[-1]] = x
    return wide[..., :shape[-1]]


def _close(got, ref, dtype, mag):
    """float(sum), times a scale, times a scale, plus a bias: four float roundings, then half a step of the result's type."""
    import torch
    slack = 4 * 2.0 ** -24 * mag + torch.finfo(dtype).eps / 2 * (ref.abs() + 4 * 2.0 ** -24 * mag) + 1e-30
    off = (got.double() - ref).abs()
    assert not (off > slack).any(), (float((off / slack).max()), (off > slack).nonzero()[:4].tolist())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M,N,K", [(1, 1, 1), (1, 8, 16), (16, 128, 4096), (3, 1000, 200), (64, 72, 1040), (65, 264, 128), (300, 520, 272),
                                   (513, 131, 1001), (2, 4096, 9216), (1000, 24, 48), (128, 520, 9216), (250, 264, 4112), (700, 136, 8208)])
def test_dense(M, N, K, dtype):
    import torch
    gen = torch.Generator(device="cuda")
    gen.manual_seed(M + N + K)
    up = lambda d, m: -(-d // m) * m  # noqa: E731
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    A, B = _ints((M, K), gen, up(K, 16)), _ints((N, K), gen, up(K, 16))
    sa, sb = torch.rand(M, device="cuda", generator=gen) + 0.01, torch.rand(N, device="cuda", generator=gen) + 0.01
    bias = torch.randn(N, device="cuda", generator=gen) * 1000
    whole = torch.full((M, up(N, 8)), float("nan"), dtype=dt, device="cuda")
    ref = (A.double() @ B.double().T) * sa.double()[:, None] * sb.double()
    mbd.gemm_i8(A, sa, B, sb, whole[:, :N])
    _close(whole[:, :N], ref, dt, ref.abs())
    assert whole[:, N:].isnan().all()
    mbd.gemm_i8(A, sa, B, sb, whole[:, :N], relu=True, bias=bias)
    _close(whole[:, :N], (ref + bias.double()).relu(), dt, ref.abs() + bias.abs().double())


@pytest.mark.gpu
def test_the_longest_sum_does_not_overflow():
    # every product at its largest, 128 * 128, over the longest row: the sum is just below 2^31 and exact
    import torch
    K = 131071
    A = torch.full((2, 131072), -128, dtype=torch.int8, device="cuda")[:, :K]
    B = torch.full((9, 131072), -128, dtype=torch.int8, device="cuda")[:, :K]
    B[1] = 127
    one = lambda n: torch.ones(n, device="cuda")  # noqa: E731
    out = torch.empty((2, 16), dtype=torch.float32, device="cuda")[:, :9]
    mbd.gemm_i8(A, one(2), B, one(9), out)
    want = np.full(9, float(np.float32(128 * 128 * K)), np.float32)
    want[1] = np.float32(-128 * 127 * K)
    assert np.array_equal(out.cpu().numpy(), np.stack([want, want]))


@pytest.mark.gpu
@pytest.mark.parametrize("counts,before,behind,d_in,d_out", [([1, 0, 2], 0, 0, 2048, 136), ([5, 300, 257], 3, 9, 144, 264), ([0, 0], 0, 4, 32, 8),
                                                            ([64, 65, 1, 0, 33], 1, 0, 1001, 520), ([900, 31, 260], 0, 0, 512, 1000)])
def test_grouped_by_expert(counts, before, behind, d_in, d_out):
    import torch
    gen = torch.Generator(device="cuda")
    gen.manual_seed(sum(counts))
    E, T = len(counts), before + sum(counts) + behind
    A, B = _ints((T, d_in), gen, -(-d_in // 16) * 16), _ints((E, d_out, d_in), gen, -(-d_in // 16) * 16)
    sa, sb = torch.rand(T, device="cuda", generator=gen), torch.rand(E, d_out, device="cuda", generator=gen)
    sa[:before] = float("nan")
    sa[T - behind:] = float("inf")
    bias = torch.randn(E, d_out, device="cuda", generator=gen)
    bounds = before + np.concatenate([[0], np.cumsum(counts)])
    offsets = torch.from_numpy(bounds.astype(np.int32)).cuda()
    for dt in (torch.bfloat16, torch.float32):
        out = torch.randn(T, d_out, device="cuda", generator=gen).to(dt)
        old = out.clone()
        mbd.expert_gemm_i8(A, sa, B, sb, offsets, out, bias=bias)
        for e in range(E):
            s = slice(int(bounds[e]), int(bounds[e + 1]))
            ref = (A[s].double() @ B[e].double().T) * sa[s].double()[:, None] * sb[e].double()
            _close(out[s], ref + bias[e].double(), dt, ref.abs() + bias[e].abs().double())
        assert torch.equal(out[:before], old[:before]) and torch.equal(out[before + sum(counts):], old[before + sum(counts):])


@pytest.mark.gpu
def test_a_row_that_is_not_finite_is_nan_alone():
    import torch
    gen = torch.Generator(device="cuda")
    gen.manual_seed(4)
    X = torch.randn(40, 256, device="cuda", generator=gen).to(torch.bfloat16)
    X[7, 3], X[9, 200] = float("inf"), float("nan")
    X[11] = 0
    W = torch.randn(24, 256, device="cuda", generator=gen).to(torch.bfloat16)
    q, s, wq, ws = torch.empty(40, 256, dtype=torch.int8, device="cuda"), torch.empty(40, device="cuda"), torch.empty(24, 256, dtype=torch.int8, device="cuda"), torch.empty(24, device="cuda")
    mbd.quantize_rows(X, q, s)
    mbd.quantize_rows(W, wq, ws)
    out = mbd.gemm_i8(q, s, wq, ws, torch.empty(40, 24, device="cuda"))
    bad = torch.zeros(40, dtype=torch.bool, device="cuda")
    bad[[7, 9]] = True
    assert out[bad].isnan().all() and torch.isfinite(out[~bad]).all() and not out[11].any()
    # 8 bits against the product itself: each value is off by half a step of its row's scale at most
    ref = X[~bad].double() @ W.double().T
    slack = 0.5 * s[~bad].double()[:, None] * W.double().abs().sum(1) + 0.5 * ws.double() * (127 * 256) * s[~bad].double()[:, None]
    assert ((out[~bad].double() - ref).abs() <= slack * 1.001).all()


@pytest.mark.gpu
def test_captured_and_replayed():
    import torch
    gen = torch.Generator(device="cuda")
    gen.manual_seed(6)
    X = torch.randn(16, 4096, device="cuda", generator=gen).to(torch.bfloat16)
    B, sb = _ints((256, 4096), gen), torch.rand(256, device="cuda", generator=gen)
    q, s = torch.empty(16, 4096, dtype=torch.int8, device="cuda"), torch.empty(16, device="cuda")
    out, status = torch.empty(16, 256, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")

    def go():
        mbd.quantize_rows(X, q, s)
        return mbd.gemm_i8(q, s, B, sb, out, status=status)
    go()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        go()
    for k in range(3):
        X.copy_(torch.randn(16, 4096, device="cuda", generator=gen) * (k + 1))
        graph.replay()
        got = out.clone()
        go()
        assert torch.equal(got, out)
        ref = (q.double() @ B.double().T) * s.double()[:, None] * sb.double()
        _close(out, ref, torch.float32, ref.abs())
    assert int(status) == 0


@pytest.mark.gpu
def test_the_binding_refuses_what_it_would_misread():
    import torch
    X, q, s = torch.randn(4, 32, device="cuda"), torch.empty(4, 32, dtype=torch.int8, device="cuda"), torch.empty(4, device="cuda")
    mbd.quantize_rows(X, q, s)
    for bad in ((X.t(), q.t(), torch.empty(32, device="cuda")), (X.half(), q, s), (X, q, s[:2]), (X, q.short(), s), (X.cpu(), q, s), (X[:2], q, s), (X, q, s.double())):
        with pytest.raises(AssertionError):
            mbd.quantize_rows(*bad)
    with pytest.raises(mbd.MbdError) as e:
        mbd.quantize_rows(X[:1].expand(4, 32), q, s)                # rows on top of each other
    assert e.value.status == mbd.E_INVALID
    B, sb, out = torch.zeros(8, 32, dtype=torch.int8, device="cuda"), torch.ones(8, device="cuda"), torch.empty(4, 8, device="cuda")
    mbd.gemm_i8(q, s, B, sb, out)
    for bad in (dict(A=X), dict(B=B[None]), dict(B=B[:, :16]), dict(a_scale=s[:3]), dict(b_scale=sb[:4]), dict(out=out.t()), dict(out=out.half()), dict(bias=sb[:4]),
                dict(status=s)):
        with pytest.raises(AssertionError):
            mbd.gemm_i8(**{**dict(A=q, a_scale=s, B=B, b_scale=sb, out=out), **bad})


def test_no_rows_is_no_work_without_a_device():
    # row tensors of no rows may be null, their scales too; the weights' scales are there all the same
    assert _gemm(experts=2, M=0) == mbd.OK and _gemm(experts=2, M=0, A=None, sa=None, out=None) == mbd.OK
    assert _gemm(experts=2, M=0, sb=None) == mbd.E_INVALID and _gemm(experts=2, M=1, sa=None) == mbd.E_INVALID


@pytest.mark.gpu
@pytest.mark.parametrize("K", [764, 33000])
def test_half_steps_of_very_small_scales(K):
    # scales with few bits (denormal numbers) and around the border of the special path: every half step and the floats next to it on both
    # sides.  The quotient in 64 bits tells them apart: x / s is a half step or 2^-25 of it away at least
    import torch
    rng = np.random.default_rng(K)
    tops = np.concatenate([rng.integers(1, 2 ** 23, 60) * 2.0 ** -149 * 127, rng.integers(1, 4000, 20) * 2.0 ** -149, [4.605892889927633e-39 * 127],
                           127e-30 * rng.uniform(0.5, 2.0, 40), 127 * 2.0 ** -126 * rng.uniform(0.5, 2.0, 20)]).astype(np.float32)
    X = np.zeros((len(tops), K), np.float32)
    for row, top in zip(X, tops):
        s = np.float64(np.float32(top) / np.float32(127))
        half = (np.arange(-127, 127, dtype=np.float64) + 0.5) * s
        x = half.astype(np.float32)
        x = np.concatenate([x, np.nextafter(x, np.float32(np.inf)), np.nextafter(x, np.float32(-np.inf))])
        row[1:len(x) + 1] = np.clip(x, -top, top)
        row[0] = top
    q, s = torch.empty(X.shape, dtype=torch.int8, device="cuda"), torch.empty(len(X), device="cuda")
    mbd.quantize_rows(torch.from_numpy(X).cuda(), q, s, sync=True)
    ws, wq = _want_rows(X)
    assert np.array_equal(s.cpu().numpy(), ws) and np.array_equal(q.cpu().numpy(), wq)


@pytest.mark.gpu
def test_an_empty_batch_through_the_binding():
    import torch
    X, W = torch.randn(5, 64, device="cuda"), torch.randn(3, 24, 64, device="cuda")
    wq, ws = torch.empty(3, 24, 64, dtype=torch.int8, device="cuda"), torch.empty(3, 24, device="cuda")
    mbd.quantize_rows(W, wq, ws)
    q, s = torch.empty(0, 64, dtype=torch.int8, device="cuda"), torch.empty(0, device="cuda")
    mbd.quantize_rows(X[:0], q, s)
    for dt in (torch.bfloat16, torch.float32):
        out = mbd.expert_gemm_i8(q, s, wq, ws, torch.zeros(4, dtype=torch.int32, device="cuda"), torch.empty(0, 24, dtype=dt, device="cuda"))
        assert out.shape == (0, 24)
