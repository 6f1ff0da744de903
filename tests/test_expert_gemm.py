"""The products grouped by expert (mbd_expert_gemm_bf16) against the same products in 64 bits, element by element: ragged and
empty groups, single rows, odd sizes, strides, every tail operation, rows outside the groups, infinities and NaN next to a
group, offsets that make no sense, captured and concurrent calls."""
import numpy as np
import pytest

from paper_1712_04432_b200 import mbd


# ---------------------------------------------------------------------------------------------------- refusals (no GPU needed)
def _call(variant=0, E=2, T=64, d_out=32, d_in=48, lda=None, ldb=None, stride=None, A=1 << 20, B=2 << 20, offsets=3 << 20, out=4 << 20,
          op=mbd.TAIL_STORE, out_bf16=1, relu=0, ldo=None, bias=None, mask=None, ldmask=0):
    """The status of a call on addresses that are never used: every refusal comes before the device is touched."""
    import ctypes as C
    lda = lda if lda is not None else (d_in if variant == 0 else d_out)
    ldb = ldb if ldb is not None else d_in
    ldo = ldo if ldo is not None else (d_out if variant == 0 else d_in)
    stride = stride if stride is not None else d_out * d_in
    t = mbd.Tail(op, out_bf16, relu, 0, out, ldo, bias, mask, ldmask, 0.5)
    return mbd.lib().mbd_expert_gemm_bf16(variant, E, offsets, T, d_out, d_in, A, lda, B, ldb, stride, C.byref(t), 5 << 20, None)


@pytest.mark.parametrize("args,status", [
    (dict(variant=3), mbd.E_INVALID), (dict(variant=-1), mbd.E_INVALID), (dict(E=0), mbd.E_INVALID), (dict(T=-1), mbd.E_INVALID),
    (dict(d_out=0), mbd.E_INVALID), (dict(d_in=0), mbd.E_INVALID), (dict(A=None), mbd.E_INVALID), (dict(B=None), mbd.E_INVALID),
    (dict(offsets=None), mbd.E_INVALID), (dict(out=None), mbd.E_INVALID), (dict(op=7), mbd.E_INVALID),
    (dict(lda=40), mbd.E_INVALID), (dict(ldb=40), mbd.E_INVALID), (dict(ldo=24), mbd.E_INVALID),        # rows would overlap
    (dict(stride=48 * 31), mbd.E_INVALID), (dict(stride=0), mbd.E_INVALID),                             # experts would overlap
    (dict(variant=2, ldo=56), mbd.E_INVALID),
    (dict(lda=52), mbd.E_UNSUPPORTED), (dict(ldb=52, stride=52 * 32), mbd.E_UNSUPPORTED), (dict(ldo=36), mbd.E_UNSUPPORTED),
    (dict(stride=48 * 32 + 4), mbd.E_UNSUPPORTED), (dict(E=513), mbd.E_UNSUPPORTED),
    (dict(A=(1 << 20) + 8), mbd.E_UNSUPPORTED), (dict(B=(2 << 20) + 8), mbd.E_UNSUPPORTED), (dict(out=(4 << 20) + 8), mbd.E_UNSUPPORTED),
    (dict(offsets=(3 << 20) + 2), mbd.E_UNSUPPORTED), (dict(bias=(6 << 20) + 2), mbd.E_UNSUPPORTED),
    (dict(variant=1, bias=6 << 20), mbd.E_UNSUPPORTED), (dict(variant=2, relu=1), mbd.E_UNSUPPORTED),
    (dict(op=mbd.TAIL_MASK, mask=6 << 20, ldmask=32), mbd.E_UNSUPPORTED), (dict(variant=1, op=mbd.TAIL_SGD), mbd.E_UNSUPPORTED),
    (dict(variant=1, op=mbd.TAIL_MASK, mask=6 << 20, ldmask=40), mbd.E_INVALID),
    (dict(variant=1, op=mbd.TAIL_MASK, mask=(6 << 20) + 8, ldmask=48), mbd.E_UNSUPPORTED),
    (dict(T=2 ** 31), mbd.E_UNSUPPORTED), (dict(d_in=2 ** 31, stride=2 ** 37), mbd.E_UNSUPPORTED),
])
def test_refusals(args, status):
    assert _call(**args) == status


def test_no_rows_is_no_work_without_a_device():
    assert _call(T=0) == mbd.OK and _call(variant=1, T=0, A=None) == mbd.OK


# ---------------------------------------------------------------------------------------------------- against 64 bits
def _bf(shape, gen, scale=1.0, ld=None):
    """bf16 tensor on the GPU with rows `ld` apart; what lies between the rows is NaN."""
    import torch
    x = torch.randn(*shape, device="cuda", generator=gen) * scale
    return _spread(x.to(torch.bfloat16), ld)


def _spread(x, ld):
    import torch
    if ld is None:
        return x
    wide = torch.full((*x.shape[:-1], ld), float("nan"), dtype=x.dtype, device="cuda")
    wide[..., :x.shape[-1]] = x
    return wide[..., :x.shape[-1]]


def _bounds(counts, before=0):
    return np.concatenate([[before], before + np.cumsum(counts)]).astype(np.int64)


def _reference(variant, A, B, bounds, E):
    """The product and the sum of its terms' magnitudes, in 64 bits; rows in no group stay NaN."""
    import torch
    A, B = A.double(), B.double()
    if variant == 2:
        pairs = [(A[bounds[e]:bounds[e + 1]].T, B[bounds[e]:bounds[e + 1]]) for e in range(E)]
        return torch.stack([a @ b for a, b in pairs]), torch.stack([a.abs() @ b.abs() for a, b in pairs])
    out = torch.full((A.shape[0], B.shape[1] if variant == 0 else B.shape[2]), float("nan"), dtype=torch.float64, device="cuda")
    mag = out.clone()
    for e in range(E):
        s = slice(int(bounds[e]), int(bounds[e + 1]))
        w = B[e].T if variant == 0 else B[e]
        out[s] = A[s] @ w
        mag[s] = A[s].abs() @ w.abs()
    return out, mag


def _slack(K, mag, ref, dtype):
    """An accumulation step of the tensor core takes 16 products and cuts what lies below 2^-23 of the largest addend: at most
    2^-23 of the sum of magnitudes for the products and as much for the addition, K / 16 times; the result is then rounded once to
    `dtype` (half a step), plus one float rounding per segment of 4096 (K / 4096 + 1)."""
    import torch
    acc = (2.0 * (K / 16 + 1) + K / 4096 + 1) * 2.0 ** -23 * mag
    return acc + torch.finfo(dtype).eps / 2 * (ref.abs() + acc) + 1e-30


def _check(got, ref, slack):
    off = (got.double() - ref).abs()
    bad = off > slack
    assert not bad.any(), (int(bad.sum()), float((off / slack)[bad].max()), bad.nonzero()[:4].tolist())
    import torch
    assert torch.isfinite(got.double()).all()


CASES = [
    # counts, rows before the first group, rows behind the last, d_in, d_out, extra row stride
    ([1], 0, 0, 8, 8, 0),
    ([3], 0, 2, 64, 1000, 0),                               # one group, many channels, K cut over a cluster or not
    ([16], 0, 0, 2048, 128, 0),                             # one tile of channels, long K: the split form
    ([0, 1, 33, 0], 0, 0, 72, 40, 0),
    ([0, 0, 0], 0, 5, 16, 24, 0),                           # nobody gets a row
    ([5, 300, 257], 3, 9, 136, 264, 0),
    ([513, 0, 96, 1, 700], 0, 37, 200, 328, 8),
    ([2, 1, 0, 7, 1, 64, 65, 31, 32, 33], 1, 1, 1024, 520, 16),
    ([17, 129], 0, 0, 37, 41, None),                        # odd sizes in padded rows
    ([1, 255, 256, 257, 1], 2, 2, 1001, 131, None),
    ([1000], 0, 24, 16, 8, 0),
    ([120, 70], 0, 3, 4096, 256, 0),                        # long K and few tiles of 65 - 256 rows: the other split forms
    ([200], 5, 0, 256, 4104, 0),
    ([2000, 1100], 0, 0, 136, 72, 0),                       # variant 2: long groups, few tiles
]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("variant", [0, 1, 2])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_ragged_groups(variant, dtype, case):
    import torch
    counts, before, behind, d_in, d_out, extra = CASES[case]
    gen = torch.Generator(device="cuda")
    gen.manual_seed(100 * case + variant)
    up = lambda d: -(-d // 8) * 8  # noqa: E731
    ld = (lambda d: up(d)) if extra is None else (lambda d: d + extra)
    E, T = len(counts), before + sum(counts) + behind
    bounds = _bounds(counts, before)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    offsets = torch.from_numpy(bounds.astype(np.int32)).cuda()
    X, dY, W = _bf((T, d_in), gen, ld=ld(d_in)), _bf((T, d_out), gen, ld=ld(d_out)), _bf((E, d_out, d_in), gen, ld=ld(d_in))
    A, B = ((X, W), (dY, W), (dY, X))[variant]
    shape = ((T, d_out), (T, d_in), (E, d_out, d_in))[variant]
    # rows of no group hold infinities and NaN: they must reach nothing
    inside = torch.zeros(T, dtype=torch.bool, device="cuda")
    inside[before:before + sum(counts)] = True
    for t in (X, dY):
        t[~inside] = float("nan")
        t[~inside, ::2] = float("inf")
    out = _spread(torch.randn(*shape, device="cuda", generator=gen).to(dt), ld(shape[-1]))
    old = out.clone()
    mbd.expert_gemm(variant, A, B, offsets, out)
    ref, mag = _reference(variant, A, B, bounds, E)
    K = {0: d_in, 1: d_out, 2: max(counts)}[variant]
    if variant == 2:
        _check(out, ref, _slack(K, mag, ref, dt))
    else:
        assert torch.equal(out[~inside], old[~inside])       # rows of no group stay
        if inside.any():
            _check(out[inside], ref[inside], _slack(K, mag[inside], ref[inside], dt))
    if out.stride(-2) > out.shape[-1] and out.dim() == 2 and T > 1:
        whole = torch.as_strided(out, (T - 1, out.stride(0)), (out.stride(0), 1))
        assert whole[:, out.shape[1]:].isnan().all()         # what lies between the rows is not written


@pytest.mark.gpu
@pytest.mark.parametrize("variant", [0, 1, 2])
def test_long_sums_in_float(variant):
    # K beyond a segment of 4096: a float result keeps the accuracy of segments summed in float, whatever K is
    import torch
    gen = torch.Generator(device="cuda")
    gen.manual_seed(5)
    K = 20488
    counts = [K, 4097] if variant == 2 else [70, 3]
    d_in, d_out = (72, 136) if variant == 2 else ((K, 72) if variant == 0 else (72, K))
    T, bounds = sum(counts), _bounds(counts)
    X, dY, W = _bf((T, d_in), gen), _bf((T, d_out), gen), _bf((2, d_out, d_in), gen)
    A, B = ((X, W), (dY, W), (dY, X))[variant]
    out = torch.empty(((T, d_out), (T, d_in), (2, d_out, d_in))[variant], dtype=torch.float32, device="cuda")
    mbd.expert_gemm(variant, A, B, torch.from_numpy(bounds.astype(np.int32)).cuda(), out)
    ref, mag = _reference(variant, A, B, bounds, 2)
    _check(out, ref, _slack(4096, mag, ref, torch.float32) + (K / 4096 + 1) * 2.0 ** -23 * mag)
    # random terms: a truncating sum over all of K would be off by 1.1e-9 K = 2.2e-5, one over a segment by 4.5e-6
    assert float((out.double() - ref).norm() / ref.norm()) < 1e-5


@pytest.mark.gpu
@pytest.mark.parametrize("counts", [[3, 0, 20], [130, 0, 200, 7]])
def test_tails(counts):
    import torch
    gen = torch.Generator(device="cuda")
    gen.manual_seed(9)
    E, T, d_in, d_out = len(counts), sum(counts), 264, 136
    bounds = _bounds(counts)
    offsets = torch.from_numpy(bounds.astype(np.int32)).cuda()
    owner = torch.from_numpy(np.repeat(np.arange(E), counts)).cuda()
    X, dY, W = _bf((T, d_in), gen), _bf((T, d_out), gen), _bf((E, d_out, d_in), gen)
    for dt in (torch.bfloat16, torch.float32):
        eps = torch.finfo(dt).eps
        # bias + ReLU of the forward product
        bias = torch.randn(E, d_out, device="cuda", generator=gen) * 10
        out = torch.empty((T, d_out), dtype=dt, device="cuda")
        mbd.expert_gemm(0, X, W, offsets, out, relu=True, bias=bias)
        ref, mag = _reference(0, X, W, bounds, E)
        want = ref + bias[owner].double()
        _check(out, want.relu(), _slack(d_in, mag + bias[owner].abs().double(), want, dt))
        # the ReLU mask of backward-data: NaN, zeros, minus zero and the type's lowest value let nothing through
        mask = torch.randn(T, d_in, device="cuda", generator=gen).to(dt)
        mask[:, 0::7], mask[:, 1::7], mask[:, 2::7], mask[:, 3::7] = 0.0, -0.0, float("nan"), torch.finfo(dt).min
        mask[:, 4::7] = float("inf")
        mask[1] = -1.0                                       # a row that the mask leaves empty
        out = torch.empty((T, d_in), dtype=dt, device="cuda")
        mbd.expert_gemm(1, dY, W, offsets, out, op=mbd.TAIL_MASK, mask=mask)
        ref, mag = _reference(1, dY, W, bounds, E)
        keep = mask > 0
        assert (out[~keep] == 0).all() and keep.any() and (~keep).any()
        _check(out, ref * keep, _slack(d_out, mag, ref, dt))
        # Eq. 1 in the backward-weight product
        w = torch.randn(E, d_out, d_in, device="cuda", generator=gen).to(dt)
        w0 = w.clone()
        mbd.expert_gemm(2, dY, X, offsets, w, op=mbd.TAIL_SGD, scale=-0.25)
        ref, mag = _reference(2, dY, X, bounds, E)
        want = w0.double() - 0.25 * ref
        _check(w, want, _slack(max(counts), 0.25 * mag, want, dt) + eps / 2 * want.abs())
        empty = [e for e in range(E) if counts[e] == 0]
        assert empty and all(torch.equal(w[e], w0[e]) for e in empty)


@pytest.mark.gpu
def test_sgd_tail_over_several_segments():
    import torch
    gen = torch.Generator(device="cuda")
    gen.manual_seed(10)
    counts = [9001]
    X, dY = _bf((9001, 72), gen), _bf((9001, 200), gen)
    w = torch.randn(1, 200, 72, device="cuda", generator=gen)
    w0 = w.double()
    mbd.expert_gemm(2, dY, X, torch.tensor([0, 9001], dtype=torch.int32, device="cuda"), w, op=mbd.TAIL_SGD, scale=0.5)
    ref, mag = _reference(2, dY, X, _bounds(counts), 1)
    want = w0 + 0.5 * ref
    _check(w, want, _slack(4096, 0.5 * mag, want, torch.float32) + 4 * 2.0 ** -24 * (want.abs() + 0.5 * mag))


@pytest.mark.gpu
@pytest.mark.parametrize("counts", [[40, 50, 60], [300, 77, 500]])
@pytest.mark.parametrize("variant", [0, 1, 2])
def test_what_is_not_finite_stays_in_its_group(variant, counts):
    import torch
    gen = torch.Generator(device="cuda")
    gen.manual_seed(11)
    E, T, d_in, d_out = 3, sum(counts), 72, 136
    bounds = _bounds(counts)
    X, dY, W = _bf((T, d_in), gen), _bf((T, d_out), gen), _bf((E, d_out, d_in), gen)
    s = slice(int(bounds[1]), int(bounds[2]))
    X[s], dY[s] = float("inf"), float("nan")
    A, B = ((X, W), (dY, W), (dY, X))[variant]
    out = torch.zeros(((T, d_out), (T, d_in), (E, d_out, d_in))[variant], dtype=torch.float32, device="cuda")
    mbd.expert_gemm(variant, A, B, torch.from_numpy(bounds.astype(np.int32)).cuda(), out)
    ref, mag = _reference(variant, A, B, bounds, E)
    others = [0, 2] if variant == 2 else [r for r in range(T) if not s.start <= r < s.stop]
    _check(out[others], ref[others], _slack(max(max(counts), 136), mag[others], ref[others], torch.float32))
    assert not torch.isfinite(out[1] if variant == 2 else out[s]).any()


@pytest.mark.gpu
@pytest.mark.parametrize("variant", [0, 1, 2])
@pytest.mark.parametrize("offsets", [[-5, 10, 20], [0, 50, 10, 60], [0, 1000000, 5], [30, 20, 10], [2147483647, -2147483648, 7], [0, 40, 40, 70]])
def test_offsets_that_make_no_sense(variant, offsets):
    # clamped to the rows there are, a falling one counts as the largest before it: no row belongs to two groups
    import torch
    gen = torch.Generator(device="cuda")
    gen.manual_seed(12)
    E, T, d_in, d_out = len(offsets) - 1, 64, 40, 72
    bounds = np.maximum.accumulate(np.clip(np.array(offsets, np.int64), 0, T))
    X, dY, W = _bf((T, d_in), gen), _bf((T, d_out), gen), _bf((E, d_out, d_in), gen)
    A, B = ((X, W), (dY, W), (dY, X))[variant]
    out = torch.randn(((T, d_out), (T, d_in), (E, d_out, d_in))[variant], device="cuda", generator=gen)
    old = out.clone()
    mbd.expert_gemm(variant, A, B, torch.tensor(offsets, dtype=torch.int32, device="cuda"), out)
    ref, mag = _reference(variant, A, B, bounds, E)
    if variant != 2:
        free = ref.isnan().all(1)
        assert torch.equal(out[free], old[free])
        out, ref, mag = out[~free], ref[~free], mag[~free]
    if out.numel():
        _check(out, ref, _slack(72, mag, ref, torch.float32))


@pytest.mark.gpu
def test_views_of_larger_buffers():
    # experts with a stride of their own, results in a slice of columns, no rows at all
    import torch
    gen = torch.Generator(device="cuda")
    gen.manual_seed(13)
    counts = [90, 20]
    bounds = _bounds(counts)
    offsets = torch.from_numpy(bounds.astype(np.int32)).cuda()
    bank = _bf((4, 80, 192), gen)
    W = bank[::2, 8:72, 64:128]                              # [2, 64, 64]
    X = _bf((110, 64), gen)
    wide = torch.zeros((110, 128), dtype=torch.bfloat16, device="cuda")
    mbd.expert_gemm(0, X, W, offsets, wide[:, 64:])
    ref, mag = _reference(0, X, W, bounds, 2)
    _check(wide[:, 64:], ref, _slack(64, mag, ref, torch.bfloat16))
    assert not wide[:, :64].any()
    dW = torch.ones((3, 64, 64), dtype=torch.float32, device="cuda")
    mbd.expert_gemm(2, X[:0], X[:0], torch.zeros(4, dtype=torch.int32, device="cuda"), dW)
    assert not dW.any()
    mbd.expert_gemm(0, X[:0], W, torch.zeros(3, dtype=torch.int32, device="cuda"), torch.empty((0, 64), dtype=torch.float32, device="cuda"))


@pytest.mark.gpu
def test_the_same_bits_every_time_and_from_a_graph():
    # eager on two streams at once, and captured and replayed on changed inputs and offsets
    import torch
    gen = torch.Generator(device="cuda")
    gen.manual_seed(14)
    T, d_in, d_out = 700, 264, 520
    X, dY, W = _bf((T, d_in), gen), _bf((T, d_out), gen), _bf((4, d_out, d_in), gen)
    few = _bf((9, 2048), gen)
    Wf = _bf((4, 256, 2048), gen)

    def run(offsets, small, status):
        outs = [torch.zeros((T, d_out), dtype=torch.bfloat16, device="cuda"), torch.zeros((T, d_in), dtype=torch.float32, device="cuda"),
                torch.zeros((4, d_out, d_in), dtype=torch.float32, device="cuda"), torch.zeros((9, 256), dtype=torch.float32, device="cuda")]
        return outs, lambda: (mbd.expert_gemm(0, X, W, offsets, outs[0], status=status), mbd.expert_gemm(1, dY, W, offsets, outs[1], status=status),
                              mbd.expert_gemm(2, dY, X, offsets, outs[2], status=status), mbd.expert_gemm(0, few, Wf, small, outs[3], status=status))
    offsets = torch.tensor([0, 100, 100, 431, 690], dtype=torch.int32, device="cuda")
    small = torch.tensor([0, 2, 3, 9, 9], dtype=torch.int32, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    first, go = run(offsets, small, status)
    go()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    pairs = []
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            outs, go = run(offsets, small, status)
            for _ in range(3):
                go()
            pairs.append(outs)
    torch.cuda.synchronize()
    for outs in pairs:
        assert all(torch.equal(a, b) for a, b in zip(outs, first))
    captured, go = run(offsets, small, status)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        go()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(captured, first))
    offsets.copy_(torch.tensor([0, 300, 301, 600, 700], dtype=torch.int32))
    X.copy_(X.flip(0))
    for o in captured:
        o.zero_()
    graph.replay()
    again, go = run(offsets, small, status)
    go()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(captured, again)) and not torch.equal(captured[0], first[0])
    assert int(status) == 0


@pytest.mark.gpu
def test_gradients_against_differences():
    # J = sum(C * Y): dX and dW from the products, against central differences of the forward product on power-of-two steps
    import torch
    gen = torch.Generator(device="cuda")
    gen.manual_seed(15)
    counts = [5, 0, 20]
    bounds = _bounds(counts)
    offsets = torch.from_numpy(bounds.astype(np.int32)).cuda()
    ints = lambda *s: torch.randint(-4, 5, s, device="cuda", generator=gen).to(torch.bfloat16)  # noqa: E731
    X, C, W = ints(25, 16), ints(25, 24), ints(3, 24, 16)     # small integers: every product and sum is exact
    forward = lambda x, w: mbd.expert_gemm(0, x, w, offsets, torch.zeros((25, 24), dtype=torch.float32, device="cuda"))  # noqa: E731
    dX = mbd.expert_gemm(1, C, W, offsets, torch.zeros((25, 16), dtype=torch.float32, device="cuda"))
    dW = mbd.expert_gemm(2, C, X, offsets, torch.zeros((3, 24, 16), dtype=torch.float32, device="cuda"))
    J = lambda x, w: float((forward(x, w).double() * C.double()).sum())  # noqa: E731
    for r, k in [(0, 0), (4, 15), (5, 3), (24, 7)]:
        up, down = X.clone(), X.clone()
        up[r, k] += 1
        down[r, k] -= 1
        assert (J(up, W) - J(down, W)) / 2 == float(dX[r, k])
    for e, n, k in [(0, 0, 0), (1, 3, 3), (2, 23, 15)]:
        up, down = W.clone(), W.clone()
        up[e, n, k] += 1
        down[e, n, k] -= 1
        assert (J(X, up) - J(X, down)) / 2 == float(dW[e, n, k])


@pytest.mark.gpu
def test_the_binding_refuses_what_it_would_misread():
    import torch
    X, W, out = torch.zeros(8, 16, dtype=torch.bfloat16, device="cuda"), torch.zeros(2, 24, 16, dtype=torch.bfloat16, device="cuda"), torch.zeros(8, 24, device="cuda")
    ok = torch.tensor([0, 3, 8], dtype=torch.int32, device="cuda")
    call = lambda **k: mbd.expert_gemm(**{**dict(variant=0, A=X, B=W, offsets=ok, out=out), **k})  # noqa: E731
    call()
    for bad in (dict(offsets=ok.long()), dict(offsets=ok.repeat_interleave(2)[::2]), dict(offsets=ok[:2]), dict(offsets=ok.cpu()), dict(variant=3),
                dict(A=X.float()), dict(A=X[:, :8]), dict(A=X.t()), dict(B=W.transpose(1, 2)), dict(B=W[0]), dict(out=out[:4]), dict(out=out.half()),
                dict(out=torch.zeros(24, 8, device="cuda").t()), dict(bias=torch.zeros(24, device="cuda")), dict(bias=torch.zeros(2, 24, device="cuda").half()),
                dict(status=torch.zeros(1, device="cuda")), dict(op=mbd.TAIL_MASK, mask=torch.zeros(8, 24, dtype=torch.bfloat16, device="cuda"))):
        with pytest.raises(AssertionError):
            call(**bad)
    with pytest.raises(mbd.MbdError) as e:
        call(A=torch.zeros(8, 20, dtype=torch.bfloat16, device="cuda")[:, :16])          # rows 40 bytes apart
    assert e.value.status == mbd.E_UNSUPPORTED


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["bfloat16", "float32"])
@pytest.mark.parametrize("d_in", [2056, 100, 4096])
@pytest.mark.parametrize("d_out", [64, 1000])
def test_masks_over_many_boxes_are_the_product_where_positive(kind, d_in, d_out):
    """Tiles of up to eight boxes, many tiles per SM, groups that end inside a box, empty groups; the mask in rows of its own stride, and in
    the result's own memory.  The sums do not depend on the mask: every element is the unmasked one or zero, bit for bit."""
    import torch
    dt = getattr(torch, kind)
    gen = torch.Generator(device="cuda").manual_seed(d_in + d_out)
    counts = [0, 1, 255, 256, 257, 0, 700, 33, 1031, 31, 513, 2, 0]
    T, E = sum(counts), len(counts)
    offsets = torch.tensor([0] + counts).cumsum(0).int().cuda()
    ld = (d_in + 7) // 8 * 8
    dY = torch.randn(T, d_out, device="cuda", generator=gen).bfloat16()
    W = torch.randn(E, d_out, ld, device="cuda", generator=gen).bfloat16()[:, :, :d_in]
    mask = torch.randn(T, ld + 16, device="cuda", generator=gen).to(dt)[:, :d_in]
    plain = torch.full((T, ld), 7.0, device="cuda", dtype=dt)
    mbd.expert_gemm(1, dY, W, offsets, plain[:, :d_in])
    want = torch.where(mask > 0, plain[:, :d_in], torch.zeros((), device="cuda", dtype=dt))
    out = torch.full((T + 3, ld), 7.0, device="cuda", dtype=dt)
    for _ in range(3):
        out[:, :] = 7.0
        mbd.expert_gemm(1, dY, W, offsets, out[:T, :d_in], op=mbd.TAIL_MASK, mask=mask)
        assert torch.equal(out[:T, :d_in], want)
        assert (out[T:] == 7.0).all() and (out[:, d_in:] == 7.0).all()
    out[:T, :d_in] = mask
    mbd.expert_gemm(1, dY, W, offsets, out[:T, :d_in], op=mbd.TAIL_MASK, mask=out[:T, :d_in])
    assert torch.equal(out[:T, :d_in], want)


@pytest.mark.parametrize("args,status", [
    (dict(mask=(4 << 20) + 16), mbd.E_INVALID),                          # eight columns on
    (dict(mask=(4 << 20) + 96), mbd.E_INVALID), (dict(mask=(4 << 20) - 96), mbd.E_INVALID),      # a row on, a row back
    (dict(mask=4 << 20, ldmask=64), mbd.E_INVALID),                      # the same address, other rows
    (dict(mask=(4 << 20) + 64 * 96 - 16), mbd.E_INVALID),                # the last eight elements
    (dict(mask=(4 << 20) + 2 * 40, ldmask=96, ldo=96), mbd.E_INVALID),   # columns 40 .. 87 beside columns 0 .. 47
    (dict(mask=(4 << 20) + 2 * 56, ldmask=96, ldo=96), mbd.E_INVALID),   # columns 56 .. 103: into the next row
    (dict(T=1, mask=(4 << 20) + 16, ldmask=96), mbd.E_INVALID),
    (dict(T=0, mask=(4 << 20) + 16), mbd.OK),
])
def test_a_mask_laid_over_the_result_in_another_way(args, status):
    a = dict(variant=1, op=mbd.TAIL_MASK, ldmask=48)
    a.update(args)
    assert _call(**a) == status


def test_a_mask_beside_the_result_passes_the_check():
    # accepted calls end in the search for a device, or in a product on memory that is not there: the check alone, by what it lets through
    # to the refusal behind it (a bias belongs to the forward product)
    for args in (dict(mask=4 << 20), dict(mask=(4 << 20) + 64 * 96), dict(mask=(4 << 20) - 64 * 96), dict(mask=(4 << 20) + 96, ldmask=96, ldo=96),
                 dict(mask=4 << 20, ldmask=96, ldo=96), dict(T=1, mask=(4 << 20) + 96, ldmask=480), dict(T=1, mask=4 << 20, ldmask=480)):
        assert _call(**{**dict(variant=1, op=mbd.TAIL_MASK, ldmask=48, bias=6 << 20), **args}) == mbd.E_UNSUPPORTED


# few tiles and many (the form of 64 rows a tile, and the pairs of CTAs), sizes of whole 16 bytes and odd ones
SEVERAL_SEGMENTS = [([0, 3, 70, 0, 33], 264), ([0, 3, 70, 0, 33], 131), ([300, 257, 1, 0, 513], 264), ([300, 257, 1, 0, 513], 131),
                    ([700, 1, 0, 900, 390], 2056), ([700, 1, 0, 900, 390], 2055)]


@pytest.mark.gpu
@pytest.mark.parametrize("counts,d_in", SEVERAL_SEGMENTS)
def test_masks_over_several_segments(counts, d_in):
    """A float result whose K is more than eight pieces of 4096, so that no form keeps it in one accumulation: the mask in memory of its
    own and in the result's.  Every element is the unmasked one or zero, bit for bit."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(d_in + sum(counts))
    d_out, E, T, ld = 33000, len(counts), sum(counts) + 7, -(-d_in // 8) * 8
    bounds = _bounds(counts, 2)
    offsets = torch.from_numpy(bounds.astype(np.int32)).cuda()
    inside = slice(2, 2 + sum(counts))
    dY, W = _bf((T, d_out), gen), _bf((E, d_out, d_in), gen, ld=ld)
    plain = torch.full((T, ld), 7.0, device="cuda")
    mbd.expert_gemm(1, dY, W, offsets, plain[:, :d_in])
    ref, mag = _reference(1, dY, W, bounds, E)
    _check(plain[inside, :d_in], ref[inside], _slack(4096, mag[inside], ref[inside], torch.float32) + (d_out / 4096 + 1) * 2.0 ** -23 * mag[inside])
    mask = torch.randn(T, ld, device="cuda", generator=gen)[:, :d_in]
    mask[:, 0::7], mask[:, 1::7], mask[:, 2::7], mask[:, 3::7] = 0.0, -0.0, float("nan"), torch.finfo(torch.float32).min
    mask[:, 4::7] = float("inf")
    mask[4] = -1.0                                           # a row that the mask leaves empty
    want = torch.where(mask > 0, plain[:, :d_in], torch.zeros((), device="cuda"))
    out = torch.full((T, ld), 7.0, device="cuda")
    mbd.expert_gemm(1, dY, W, offsets, out[:, :d_in], op=mbd.TAIL_MASK, mask=mask)
    assert torch.equal(out[inside, :d_in], want[inside])
    out[:, :d_in] = mask
    mbd.expert_gemm(1, dY, W, offsets, out[:, :d_in], op=mbd.TAIL_MASK, mask=out[:, :d_in])
    assert torch.equal(out[inside, :d_in], want[inside])
    outside = [0, 1, *range(T - 5, T)]
    assert torch.equal(out[outside, :d_in].nan_to_num(nan=5.0), mask[outside].nan_to_num(nan=5.0)) and (out[:, d_in:] == 7.0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("counts,d_out", SEVERAL_SEGMENTS)
def test_bias_and_relu_over_several_segments(counts, d_out):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(d_out + sum(counts))
    d_in, E, T = 33000, len(counts), sum(counts)
    bounds = _bounds(counts)
    X, W = _bf((T, d_in), gen), _bf((E, d_out, d_in), gen)
    bias = torch.randn(E, d_out, device="cuda", generator=gen) * 100
    out = _spread(torch.empty(T, d_out, device="cuda"), -(-d_out // 8) * 8)
    mbd.expert_gemm(0, X, W, torch.from_numpy(bounds.astype(np.int32)).cuda(), out, relu=True, bias=bias)
    ref, mag = _reference(0, X, W, bounds, E)
    b = bias[torch.from_numpy(np.repeat(np.arange(E), counts)).cuda()].double()
    want = ref + b
    _check(out, want.relu(), _slack(4096, mag, want, torch.float32) + (d_in / 4096 + 2) * 2.0 ** -23 * (mag + b.abs()))


@pytest.mark.gpu
@pytest.mark.parametrize("variant", [0, 1, 2])
def test_the_most_experts_there_may_be(variant):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(variant)
    E, d_in, d_out = 512, 72, 40
    counts = torch.randint(0, 4, (E,), device="cuda", generator=gen).tolist()
    counts[17], counts[511] = 300, 70
    bounds, T = _bounds(counts, 1), sum(counts) + 3
    X, dY, W = _bf((T, d_in), gen), _bf((T, d_out), gen), _bf((E, d_out, d_in), gen)
    A, B = ((X, W), (dY, W), (dY, X))[variant]
    out = torch.zeros(((T, d_out), (T, d_in), (E, d_out, d_in))[variant], device="cuda")
    mbd.expert_gemm(variant, A, B, torch.from_numpy(bounds.astype(np.int32)).cuda(), out)
    ref, mag = _reference(variant, A, B, bounds, E)
    rows = slice(None) if variant == 2 else slice(1, 1 + sum(counts))
    _check(out[rows], ref[rows], _slack(300, mag[rows], ref[rows], torch.float32))
    assert variant == 2 or not (out[0].any() or out[-2:].any())
