"""Routing to experts (mbd_expert_route) and its gradient against the definition in 64 bits: the experts, places and offsets exactly, the
weights and gradients to float roundings (U = 2^-24 each)."""
import ctypes as C
import math

import numpy as np
import pytest

from paper_1712_04432_b200 import mbd

U = 2.0 ** -24
MB = 1 << 20


# ---------------------------------------------------------------------------------------------------- refusals (no GPU needed)
ROUTER = dict(experts=16, top_k=2, score=0, renormalise=1, groups=4, top_groups=2, group_best=2, scale=1.0)
FWD = dict(T=100, logits=1 * MB, bf16=0, ld=16, bias=2 * MB, count=3 * MB, ids=4 * MB, weights=5 * MB, places=6 * MB, offsets=7 * MB, scratch=8 * MB)
BWD = dict(T=100, logits=1 * MB, bf16=0, ld=16, ids=2 * MB, dw=3 * MB, out=4 * MB, out_bf16=1, ldd=16)


@pytest.mark.parametrize("router,args,status", [
    (dict(experts=0), {}, mbd.E_INVALID), (dict(top_k=0), {}, mbd.E_INVALID), (dict(score=2), {}, mbd.E_INVALID), (dict(groups=0), {}, mbd.E_INVALID),
    (dict(groups=3), {}, mbd.E_INVALID), (dict(top_groups=0), {}, mbd.E_INVALID), (dict(top_groups=5), {}, mbd.E_INVALID),
    (dict(group_best=0), {}, mbd.E_INVALID), (dict(group_best=3), {}, mbd.E_INVALID), (dict(top_k=9), {}, mbd.E_INVALID),
    (dict(scale=math.nan), {}, mbd.E_INVALID), (dict(scale=math.inf), {}, mbd.E_INVALID),
    (dict(experts=516), dict(ld=516), mbd.E_UNSUPPORTED), (dict(experts=256, top_k=33), dict(ld=256), mbd.E_UNSUPPORTED),
    (dict(experts=128, groups=64), dict(ld=128), mbd.E_UNSUPPORTED),
    ({}, dict(T=-1), mbd.E_INVALID), ({}, dict(logits=None), mbd.E_INVALID), ({}, dict(ids=None), mbd.E_INVALID), ({}, dict(weights=None), mbd.E_INVALID),
    ({}, dict(places=None), mbd.E_INVALID), ({}, dict(offsets=None), mbd.E_INVALID), ({}, dict(scratch=None), mbd.E_INVALID), ({}, dict(ld=15), mbd.E_INVALID),
    ({}, dict(logits=1 * MB + 2), mbd.E_UNSUPPORTED), ({}, dict(logits=1 * MB + 1, bf16=1), mbd.E_UNSUPPORTED), ({}, dict(ids=4 * MB + 2), mbd.E_UNSUPPORTED),
    ({}, dict(count=3 * MB + 2), mbd.E_UNSUPPORTED), ({}, dict(scratch=8 * MB + 8), mbd.E_UNSUPPORTED), ({}, dict(T=2 ** 27), mbd.E_UNSUPPORTED),
    ({}, dict(places=4 * MB), mbd.E_INVALID), ({}, dict(weights=1 * MB + 64), mbd.E_INVALID), ({}, dict(offsets=6 * MB), mbd.E_INVALID),
    ({}, dict(ids=2 * MB), mbd.E_INVALID), ({}, dict(scratch=5 * MB + 16), mbd.E_INVALID), ({}, dict(offsets=3 * MB - 8), mbd.E_INVALID),
])
def test_forward_refusals(router, args, status):
    r = mbd.Router(**{**ROUTER, **router})
    assert mbd.lib().mbd_expert_route(C.byref(r), *{**FWD, **args}.values(), None) == status


def test_no_router_is_refused():
    assert mbd.lib().mbd_expert_route(None, *FWD.values(), None) == mbd.E_INVALID
    assert mbd.lib().mbd_expert_route_backward(None, *BWD.values(), None) == mbd.E_INVALID


@pytest.mark.parametrize("router,args,status", [
    (dict(experts=0), {}, mbd.E_INVALID), (dict(top_k=33, experts=512), dict(ld=512, ldd=512), mbd.E_INVALID), ({}, dict(T=-1), mbd.E_INVALID), ({}, dict(logits=None), mbd.E_INVALID), ({}, dict(ids=None), mbd.E_INVALID),
    ({}, dict(dw=None), mbd.E_INVALID), ({}, dict(out=None), mbd.E_INVALID), ({}, dict(ld=15), mbd.E_INVALID), ({}, dict(ldd=15), mbd.E_INVALID),
    ({}, dict(out=4 * MB + 1), mbd.E_UNSUPPORTED), ({}, dict(logits=1 * MB + 2), mbd.E_UNSUPPORTED), ({}, dict(out=1 * MB), mbd.E_INVALID),
    ({}, dict(out=2 * MB), mbd.E_INVALID), ({}, dict(T=0, logits=None), mbd.OK),
])
def test_backward_refusals(router, args, status):
    r = mbd.Router(**{**ROUTER, "groups": 1, "top_groups": 1, **router})
    if router.get("top_k") == 33:
        status = mbd.E_UNSUPPORTED
    assert mbd.lib().mbd_expert_route_backward(C.byref(r), *{**BWD, **args}.values(), None) == status


def test_scratch_grows_slowly():
    assert mbd.expert_route_scratch(0, 8) == 0 and mbd.expert_route_scratch(mbd.ROUTE_ONE_BLOCK, 512) == 0 and mbd.expert_route_scratch(100, 0) == 0
    assert mbd.expert_route_scratch(mbd.ROUTE_ONE_BLOCK + 1, 7) > 0
    for T in (100, 5000, 16384, 10 ** 6, 2 ** 26 - 1):
        assert 0 < mbd.expert_route_scratch(T, 512) <= 256 * max(4, -(-T // (256 * 65472)) * 4) * 256


# ---------------------------------------------------------------------------------------------------- the definition
def _scores(l, sigmoid):
    l = l.astype(np.float64)
    with np.errstate(invalid="ignore", over="ignore"):
        if sigmoid:
            return 1 / (1 + np.exp(-l))
        top = np.max(np.where(np.isnan(l), -np.inf, l), 1, keepdims=True)
        p = np.where(l == -np.inf, 0.0, np.exp(l - top))
        return p / p.sum(1, keepdims=True)


def _choice(l, bias, r):
    """ids [T, k] (-1: empty) from float64 logits, by sorting."""
    p = _scores(l, r.score)
    key = l.astype(np.float64) if bias is None else p + bias.astype(np.float64)
    there = (l != -np.inf) & (key != -np.inf)
    T, E = l.shape
    rank = lambda v: -np.inf if math.isnan(v) else v  # noqa: E731

    def best(values, n):            # indices of the n best, numbers before NaN, equal ones by rising index
        return sorted(values, key=lambda iv: (math.isnan(iv[1]), -rank(iv[1]) if not math.isnan(iv[1]) else 0.0, iv[0]))[:n]

    ids = np.full((T, r.top_k), -1, np.int32)
    S = E // r.groups
    for t in range(T):
        of = p[t] if bias is None and r.group_best == 2 else key[t]
        allowed = range(r.groups)
        if r.groups > 1:
            scores = []
            for g in range(r.groups):
                two = best([(e, float(of[e])) for e in range(g * S, g * S + S) if there[t, e]], r.group_best)
                if two:
                    scores.append((g, two[0][1] + (two[1][1] if len(two) > 1 else 0.0)))
            allowed = [g for g, _ in best(scores, r.top_groups)]
        chosen = best([(e, float(key[t, e])) for g in allowed for e in range(g * S, g * S + S) if there[t, e]], r.top_k)
        ids[t, :len(chosen)] = [e for e, _ in chosen]
    return ids


def _weights(l, ids, r):
    p = _scores(l, r.score)
    there = ids >= 0
    at = np.maximum(ids, 0)
    z = np.where(there, np.take_along_axis(l.astype(np.float64), at, 1), -np.inf)
    w = np.where(there, np.take_along_axis(p, at, 1), 0.0)
    if r.renormalise:
        with np.errstate(invalid="ignore", over="ignore", divide="ignore"):
            top = z.max(1, keepdims=True)
            if r.score:             # relative to the largest, in logarithms
                s = -np.logaddexp(0, -z)
                w = np.where(there, np.exp(s - s.max(1, keepdims=True)), 0.0)
            else:
                w = np.where(there, np.exp(z - top), 0.0)
            w = np.where(there, w / w.sum(1, keepdims=True), 0.0)
    return w * r.scale


def _order(ids, E):
    """places and offsets by a stable sort."""
    flat = ids.ravel()
    slots = np.flatnonzero(flat >= 0)
    order = slots[np.argsort(flat[slots], kind="stable")]
    places = np.full(flat.size, -1, np.int32)
    places[order] = np.arange(order.size, dtype=np.int32)
    offsets = np.concatenate([[0], np.cumsum(np.bincount(flat[slots], minlength=E))]).astype(np.int32)
    return places.reshape(ids.shape), offsets


def _route(r, logits, bias=None, count=None, ld=None, scratch=None):
    import torch
    T, E = logits.shape
    k = r.top_k
    dev = dict(device="cuda")
    ids, places = torch.full((T, k), 77, dtype=torch.int32, **dev), torch.full((T, k), 77, dtype=torch.int32, **dev)
    weights, offsets = torch.full((T, k), 7.0, **dev), torch.full((E + 1,), 77, dtype=torch.int32, **dev)
    mbd.expert_route(r, logits, ids, weights, places, offsets, bias=bias, count=count, scratch=scratch)
    return ids, weights, places, offsets


def _compare(r, logits, bias=None, live=None, count=None):
    """One call against the definition."""
    import torch
    got = [x.cpu().numpy() for x in _route(r, logits, bias, count)]
    l = logits.float().cpu().numpy()
    want = _choice(l, None if bias is None else bias.cpu().numpy(), r)
    w = _weights(l, want, r)
    if live is not None:
        want[live:], w[live:] = -1, 0.0
    assert np.array_equal(got[0], want), np.argwhere(got[0] != want)[:5]
    places, offsets = _order(want, r.experts)
    assert np.array_equal(got[2], places) and np.array_equal(got[3], offsets)
    # the exponent's rounding (|z - top| U) twice, exponentials (2 U each), sums over 512 numbers in a warp, quotients, the scale; below the
    # smallest normal number the steps are 2^-149
    spread = np.minimum(np.float64(300), np.ptp(np.where(np.isfinite(l), l, 0.0).astype(np.float64), 1))[:, None]   # (beyond 300 there is nothing left)
    slack = (2 * spread + 60) * U * np.abs(w) + 2.0 ** -145
    with np.errstate(invalid="ignore"):
        off = np.abs(got[1] - w)
    assert np.array_equal(np.isnan(got[1]), np.isnan(w)) and not (off > slack).any(), float(np.nanmax(off / slack))
    return got


def _logits(T, E, dtype, seed, scale=1.5):
    import torch
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    x = torch.randn(T, E, device="cuda", generator=gen) * scale + torch.randn(E, device="cuda", generator=gen)
    return x.to(torch.bfloat16 if dtype == "bf16" else torch.float32), torch.randn(E, device="cuda", generator=gen) * 0.05


# ---------------------------------------------------------------------------------------------------- forward
@pytest.mark.gpu
@pytest.mark.parametrize("T,E,k", [(1, 1, 1), (1, 64, 2), (2, 3, 3), (16, 64, 2), (33, 33, 5), (63, 160, 8), (64, 512, 32), (65, 32, 4), (128, 257, 7), (129, 31, 1),
                                   (700, 256, 8), (1000, 100, 12), (3001, 8, 2), (5, 512, 1), (300, 511, 17)])
@pytest.mark.parametrize("dtype,score,renormalise,with_bias", [("f32", 0, True, False), ("bf16", 0, False, True), ("bf16", 1, True, True), ("f32", 1, False, False),
                                                               ("f32", 1, True, True), ("bf16", 0, True, False), ("f32", 0, False, True)])
def test_choice(T, E, k, dtype, score, renormalise, with_bias):
    logits, bias = _logits(T, E, dtype, 7 * T + E)
    _compare(mbd.Router(E, k, score, renormalise, scale=2.5), logits, bias if with_bias else None)


@pytest.mark.gpu
@pytest.mark.parametrize("T,E,k,G,top,best", [(16, 64, 2, 8, 2, 1), (70, 256, 8, 8, 4, 2), (300, 256, 8, 8, 4, 2), (100, 160, 6, 8, 3, 1), (40, 512, 8, 32, 7, 2), (65, 96, 3, 3, 1, 2),
                                              (20, 32, 8, 32, 8, 2), (33, 60, 20, 5, 5, 2), (200, 510, 9, 17, 6, 2), (50, 12, 1, 2, 1, 1)])
@pytest.mark.parametrize("dtype,score,with_bias", [("f32", 1, True), ("bf16", 0, False), ("bf16", 1, True), ("f32", 0, True), ("f32", 1, False)])
def test_groups(T, E, k, G, top, best, dtype, score, with_bias):
    logits, bias = _logits(T, E, dtype, T + E + G)
    _compare(mbd.Router(E, k, score, True, G, top, best), logits, bias if with_bias else None)


@pytest.mark.gpu
def test_many_tokens():
    """Several hundred blocks, blocks of several hundred tokens; the choice checked by its keys, the order exactly."""
    import torch
    for T, E, k in ((20011, 37, 3), (70000, 128, 2)):
        logits, _ = _logits(T, E, "f32", E)
        ids, w, places, offsets = (x.cpu().numpy() for x in _route(mbd.Router(E, k), logits))
        top = torch.topk(logits, k, dim=1)
        assert np.array_equal(ids, top.indices.cpu().numpy())       # (no two of them equal, by far)
        want = _order(ids, E)
        assert np.array_equal(places, want[0]) and np.array_equal(offsets, want[1])


@pytest.mark.gpu
@pytest.mark.parametrize("score", [0, 1])
def test_keys_that_floats_cannot_tell_apart(score):
    """Biases that bring all keys of a token's experts to within a few 2^-26 of each other: the order is that of the exact values."""
    import torch
    rng = np.random.default_rng(5 + score)
    for E, k, G, top, best in ((64, 4, 1, 1, 1), (256, 8, 8, 3, 2), (37, 2, 1, 1, 1), (512, 6, 16, 2, 1)):
        l = rng.normal(size=E).astype(np.float32)
        p = _scores(l[None], score)[0]
        bias = (0.7 - p).astype(np.float32)                          # rounded: keys spread over some 2^-25
        rows = np.repeat(l[None], 40, 0)
        assert len(np.unique((p.astype(np.float32) + bias).astype(np.float32))) < E / 2
        _compare(mbd.Router(E, k, score, True, G, top, best), torch.from_numpy(rows).cuda(), torch.from_numpy(bias).cuda())


@pytest.mark.gpu
@pytest.mark.parametrize("score", [0, 1])
@pytest.mark.parametrize("level", [0.0, 0.6, 6.0])
def test_pairs_of_keys_that_floats_cannot_tell_apart(score, level):
    """Experts in pairs whose keys are a few 2^-26 apart, the pairs far from each other: at small biases, and at ones beyond one."""
    import torch
    rng = np.random.default_rng(int(level * 10) + score)
    for E, k, G, top, best in ((64, 5, 1, 1, 1), (256, 8, 8, 4, 2), (100, 12, 4, 2, 1), (512, 32, 1, 1, 1)):
        l = rng.normal(size=E).astype(np.float32)
        p = _scores(l[None], score)[0]
        bias = (level + 0.3 * rng.random(E)).astype(np.float32)
        other = rng.permutation(E)
        for a, b in zip(other[::2], other[1::2]):                    # b's key becomes a's, as near as a float bias goes
            bias[b] = np.float32(p[a] + np.float64(bias[a]) - p[b])
        rows = np.repeat(l[None], 30, 0)
        _compare(mbd.Router(E, k, score, True, G, top, best), torch.from_numpy(rows).cuda(), torch.from_numpy(bias).cuda())


@pytest.mark.gpu
@pytest.mark.parametrize("G,top,best", [(1, 1, 1), (8, 3, 1), (8, 3, 2), (5, 2, 1)])
def test_logits_a_bit_apart(G, top, best):
    """Neighbouring floats, some of them equal, in many clusters: the order is that of the floats, to the last bit."""
    import torch
    rng = np.random.default_rng(G + best)
    E = 160
    centre = rng.normal(size=(200, 12)).astype(np.float32) * 3
    l = np.take_along_axis(centre, rng.integers(0, 12, (200, E)), 1)
    l = (l.view(np.int32) + rng.integers(-3, 4, l.shape)).astype(np.int32).view(np.float32)
    _compare(mbd.Router(E, 8, 0, True, G, top, best), torch.from_numpy(l).cuda())


@pytest.mark.gpu
def test_two_best_of_groups_that_floats_cannot_tell_apart():
    """Without a bias: sums of two scores that differ by about 1e-9, with the larger expert in the group of the smaller sum."""
    import torch
    E, G = 32, 4
    l = np.full((50, E), -3.0, np.float32)
    rng = np.random.default_rng(3)
    for t in range(50):
        base = rng.uniform(0.2, 0.4)
        for g in range(G):
            a = base + rng.uniform(-0.1, 0.1)
            b = 2 * base - a
            l[t, g * 8 + rng.integers(0, 4)] = math.log(a / (1 - a))
            l[t, g * 8 + 4 + rng.integers(0, 4)] = math.log(b / (1 - b))
    _compare(mbd.Router(E, 3, 1, True, G, 2, 2), torch.from_numpy(l).cuda())


@pytest.mark.gpu
@pytest.mark.parametrize("score", [0, 1])
@pytest.mark.parametrize("level", [4.0, 16.0, 100.0, 1000.0])
def test_two_best_of_groups_whose_keys_cancel(score, level):
    """Biases of both signs, one expert of a group near `level` and the others near -level: sums of two keys next to zero that differ by less than
    a float has at `level`."""
    import torch
    rng = np.random.default_rng(int(level) + score)
    for E, k, G, top in ((256, 8, 8, 4), (64, 3, 4, 2), (96, 2, 3, 1), (512, 8, 16, 5), (510, 6, 17, 6)):
        S, part = E // G, 1.0 if score else 1.0 / G
        first = np.arange(G) * S + rng.integers(0, S // 2, G)
        second = np.arange(G) * S + rng.integers(S // 2, S, G)
        bias = (-level - 2 - rng.random(E)).astype(np.float32)
        bias[first] = level + 0.1 * part * rng.random(G)
        bias[second] = -level - 0.1 * part * rng.random(G)
        both = bias[first].astype(np.float64) + bias[second]
        rows = []
        for _ in range(40):
            pa = part * rng.uniform(0.3, 0.4, G)
            pb = 0.8 * part - both - pa + 3e-8 * level * rng.normal(size=G)
            if score:
                l = rng.normal(size=E)
                l[first], l[second] = np.log(pa / (1 - pa)), np.log(pb / (1 - pb))
            else:
                l = np.full(E, np.log((1 - pa.sum() - pb.sum()) / (E - 2 * G)))
                l[first], l[second] = np.log(pa), np.log(pb)
            rows.append(l)
        _compare(mbd.Router(E, k, score, True, G, top, 2), torch.from_numpy(np.array(rows, np.float32)).cuda(), torch.from_numpy(bias).cuda())


@pytest.mark.gpu
@pytest.mark.parametrize("score", [0, 1])
@pytest.mark.parametrize("level", [0.5, 10.0, 100.0, -100.0, 1000.0])
def test_two_best_of_groups_among_logits_a_few_bits_apart(score, level):
    """Without a bias: the best experts of each group up to 15 units of a float apart, next to each other and far from each other in the group; the
    differences reach the scores where the logits have a common offset."""
    import torch
    rng = np.random.default_rng(int(abs(level)) + score)
    unit = np.spacing(np.float32(level) * np.float32(0.99))
    for E, k, G, top in ((256, 8, 8, 4), (512, 8, 8, 1), (512, 6, 16, 3), (128, 4, 8, 2), (64, 4, 4, 2), (160, 5, 5, 2), (510, 6, 3, 1)):
        S = E // G
        l = np.full((40, E), level - 20.0, np.float64)
        for t in range(40):
            for g in range(G):
                near = g * S + rng.integers(0, S - 4) + np.arange(4)            # neighbours
                far = g * S + rng.choice(S, 2, replace=False)
                for e in (*near, *far):
                    l[t, e] = level + unit * rng.integers(-15, 1)
        l = l.astype(np.float32)
        # Groups whose sums doubles do not tell apart are nobody's to order: a + b units over two experts give the same sum but for s'' u^2 (a^2 - b^2) / 2,
        # at 0.5 (u = 2^-25, s'' = 0.058, a^2 - b^2 <= 225) 6e-15 and mostly below 1e-16, where a double of two sums with three roundings
        # of 2^-53 each has 7e-16 < 2^-50 of itself.  Such tokens are left out, but not those whose scores are one in doubles, too: equal keys.
        sums = np.sort(np.sort(_scores(l, score).reshape(40, G, S), 2)[:, :, -2:].sum(2), 1)
        l = l[(sums[:, -top] - sums[:, -top - 1] >= 2.0 ** -50 * sums[:, -top]) | (sums[:, -top - 1] == 2.0)]
        assert len(l) > 10
        _compare(mbd.Router(E, k, score, True, G, top, 2), torch.from_numpy(l).cuda())


@pytest.mark.gpu
@pytest.mark.parametrize("top", [-1e-3, -1.0, -30.0, -59.0, -61.0, -85.0, 0.0, 5.0])
def test_renormalised_sigmoids_on_both_sides_of_the_smallest_float(top):
    """Chosen scores that are numbers of full precision beside scores that are not (below e^-87): their quotients are, and so are the gradients."""
    import torch
    E, k, T = 32, 6, 30
    rng = np.random.default_rng(int(abs(top)))
    l = np.full((T, E), -400.0, np.float32)
    for t in range(T):
        at = rng.permutation(E)[:k]
        l[t, at] = np.concatenate([[top], rng.uniform(-104.0, min(top, -70.0), k - 1)])
    r = mbd.Router(E, k, 1, True)
    logits = torch.from_numpy(l).cuda()
    got = _compare(r, logits)
    dw = torch.randn(T, k, device="cuda", generator=torch.Generator(device="cuda").manual_seed(3))
    ids = torch.from_numpy(got[0]).cuda()
    _close(_backward(r, logits, ids, dw), l, got[0], dw.cpu().numpy(), r)


@pytest.mark.gpu
@pytest.mark.parametrize("score,renormalise,G", [(0, True, 1), (0, False, 1), (1, True, 1), (1, False, 4), (0, True, 4)])
def test_equal_keys_masks_and_numbers_that_are_none(score, renormalise, G):
    import torch
    E, k = 64, 6
    rng = np.random.default_rng(1)
    l = np.round(rng.normal(size=(120, E)) * 2).astype(np.float32) / 2       # many equal logits
    l[0] = 0.0
    l[1] = -0.0
    l[1, ::3] = 0.0
    l[2] = -np.inf                                                  # nobody
    l[3] = -np.inf; l[3, 40] = 1.0                                  # one
    l[4] = -np.inf; l[4, [3, 17, 18]] = [2.0, 2.0, 5.0]             # fewer than k
    l[5] = -1e30                                                    # all equally hopeless
    l[6] = np.finfo(np.float32).min
    l[7] = np.finfo(np.float32).min; l[7, 9] = -100.0
    l[8] = -200.0 - np.arange(E)                                    # below float's exponentials
    l[9] = 200.0 + np.arange(E)
    l[10, 5] = np.nan
    l[11] = np.nan
    l[12] = np.nan; l[12, :4] = -np.inf
    l[13] = -np.inf; l[13, [8, 50]] = [np.nan, 1.0]
    bias = np.zeros(E, np.float32)
    for b in (None, bias):
        for best in (1, 2):
            if G == 1 and best == 2:
                continue
            r = mbd.Router(E, k, score, renormalise, G, max(1, G // 2), best)
            rows = l
            if score == 0 and not (renormalise and b is None and best == 1):
                rows = l.copy(); rows[[5, 6]] = 0.25                # (as logits of equal experts: their softmax is the same)
            if score == 0 and renormalise:                          # a softmax over the chosen logits alone: a NaN elsewhere does not reach it
                rows = rows.copy(); rows[10, 5] = 0.0
            if score == 1 and b is not None:
                rows = rows.copy(); rows[9] = 3.0                   # (sigmoids that are one even in 64 bits are equal keys; a test of its own)
            _compare(r, torch.from_numpy(rows).cuda(), None if b is None else torch.from_numpy(b).cuda())


@pytest.mark.gpu
def test_saturated_sigmoids_with_a_bias_are_equal_keys():
    import torch
    l = torch.full((3, 40), 60.0, device="cuda")
    l[1] += torch.arange(40, device="cuda")
    l[2, :20] = 10.0
    ids, w, places, offsets = _route(mbd.Router(40, 4, 1), l, torch.zeros(40, device="cuda"))
    assert ids.tolist() == [[0, 1, 2, 3], [0, 1, 2, 3], [20, 21, 22, 23]] and torch.equal(w, torch.full((3, 4), 0.25, device="cuda"))


@pytest.mark.gpu
def test_biases_that_are_infinite():
    import torch
    logits, bias = _logits(90, 24, "f32", 4)
    bias[[3, 20]] = -np.inf
    bias[7] = np.inf
    for score in (0, 1):
        got = _compare(mbd.Router(24, 5, score), logits, bias)
        assert not np.isin(got[0], [3, 20]).any() and (got[0][:, 0] == 7).all()
    got = _compare(mbd.Router(24, 24, 1), logits, bias)             # two can never be chosen
    assert (got[0][:, 22:] == -1).all() and (got[2][:, 22:] == -1).all() and got[3][-1] == 90 * 22


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 50, 64, 65, 200, 1500])
def test_padded_batches_and_views(T):
    import torch
    base, bias = _logits(T, 100, "bf16", T)
    logits = base[:, 3:83]                                          # 80 experts of a wider product
    r = mbd.Router(80, 4, 1, groups=4, top_groups=2, group_best=2)
    for count, live in ((0, 0), (-5, 0), (1, 1), (T // 2, T // 2), (T, T), (T + 9, T)):
        _compare(r, logits, bias[:80].contiguous(), live, torch.tensor([count], dtype=torch.int32, device="cuda"))


@pytest.mark.gpu
def test_no_tokens_leave_zero_offsets():
    import torch
    got = _route(mbd.Router(9, 2), torch.empty(0, 9, device="cuda"))
    assert not got[3].any()


@pytest.mark.gpu
def test_two_streams_and_a_captured_call_that_counts_on():
    import torch
    T, E = 900, 64
    r = mbd.Router(E, 4, 1)
    (a, bias), (b, _) = _logits(T, E, "f32", 1), _logits(T, E, "f32", 2)
    want = [_route(r, x, bias) for x in (a, b)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(5):
        got = []
        for s, x in zip(streams, (a, b)):
            with torch.cuda.stream(s):
                got.append(_route(r, x, bias))
        torch.cuda.synchronize()
        assert all(torch.equal(g, w) for gs, ws in zip(got, want) for g, w in zip(gs, ws))
    count, x = torch.tensor([T], dtype=torch.int32, device="cuda"), a.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = _route(r, x, bias, count)
    for n, src in ((T, a), (333, b), (0, a), (T, b)):
        count.fill_(n)
        x.copy_(src)
        graph.replay()
        ids = (want[0] if src is a else want[1])[0].cpu().numpy().copy()
        ids[n:] = -1
        places, offsets = _order(ids, E)
        assert np.array_equal(got[0].cpu().numpy(), ids) and np.array_equal(got[2].cpu().numpy(), places) and np.array_equal(got[3].cpu().numpy(), offsets)


# ---------------------------------------------------------------------------------------------------- backward
def _grad64(l, ids, dw, r):
    """By the formulas, one slot after the other; and the sum of the magnitudes that meet in each element."""
    T, E = l.shape
    p = _scores(l, r.score)
    g, mag = np.zeros((T, E)), np.zeros((T, E))
    for t in range(T):
        slots = [j for j in range(ids.shape[1]) if 0 <= ids[t, j] < E]
        if not slots:
            continue
        at = ids[t, slots]
        d = dw[t, slots].astype(np.float64) * r.scale
        pj = p[t, at]
        if r.renormalise:
            one = np.repeat(at[None], 1, 0)
            s = _weights(l[t:t + 1], one, mbd.Router(E, len(slots), r.score, True))[0]
            slope = 1 / (1 + np.exp(l[t, at].astype(np.float64))) if r.score else 1.0
            mean = (s * d).sum()
            np.add.at(g[t], at, s * slope * (d - mean))
            np.add.at(mag[t], at, s * slope * (np.abs(d) + (s * np.abs(d)).sum()))
        elif r.score:
            slope = 1 / (1 + np.exp(l[t, at].astype(np.float64)))          # 1 - p, which cancels next to one
            np.add.at(g[t], at, pj * slope * d)
            np.add.at(mag[t], at, pj * slope * np.abs(d))
        else:
            dp = np.zeros(E); np.add.at(dp, at, d)
            da = np.zeros(E); np.add.at(da, at, np.abs(d))
            g[t] = p[t] * (dp - (pj * d).sum())
            mag[t] = p[t] * (da + (pj * np.abs(d)).sum())
    return g, mag


def _backward(r, logits, ids, dw, out_dtype=None):
    import torch
    out = torch.full(logits.shape, 9.0, dtype=out_dtype or logits.dtype, device="cuda")
    return mbd.expert_route_backward(r, logits, ids, dw, out)


def _close(got, l, ids, dw, r):
    import torch
    g, mag = _grad64(l, ids, dw, r)
    spread = (np.where(np.isfinite(l), l, 0).max(1) - np.where(np.isfinite(l), l, 0).min(1))[:, None]
    rel = (3 * spread + 100) * U
    step = torch.finfo(got.dtype).eps / 2
    off = np.abs(got.double().cpu().numpy() - g)
    slack = rel * mag + step * (np.abs(g) + rel * mag) + 2.0 ** -133
    assert not (off > slack).any(), float((off / slack).max())


@pytest.mark.gpu
@pytest.mark.parametrize("T,E,k", [(1, 1, 1), (1, 64, 2), (16, 64, 2), (33, 33, 5), (100, 160, 8), (65, 512, 32), (300, 257, 7), (7, 31, 3), (3000, 64, 2)])
@pytest.mark.parametrize("score", [0, 1])
@pytest.mark.parametrize("renormalise", [True, False])
def test_gradient(T, E, k, score, renormalise):
    import torch
    for dtype, out in (("f32", torch.float32), ("bf16", torch.bfloat16), ("bf16", torch.float32)):
        r = mbd.Router(E, k, score, renormalise, scale=1.7)
        logits, _ = _logits(T, E, dtype, T + E)
        gen = torch.Generator(device="cuda")
        gen.manual_seed(T)
        dw = torch.randn(T, k, device="cuda", generator=gen)
        ids = _route(r, logits)[0]
        ids[T // 2:T // 2 + 3, k // 2:] = -1                           # empty slots
        _close(_backward(r, logits, ids, dw, out), logits.float().cpu().numpy(), ids.cpu().numpy(), dw.cpu().numpy(), r)


@pytest.mark.gpu
@pytest.mark.parametrize("score", [0, 1])
def test_one_expert_renormalised_has_weight_one_and_no_gradient(score):
    """Exactly: the weight does not depend on the logits."""
    import torch
    for dtype in ("f32", "bf16"):
        r = mbd.Router(70, 1, score, True, scale=2.5)
        logits, _ = _logits(500, 70, dtype, 3, scale=20.0)
        ids, w, _, _ = _route(r, logits)
        assert (w == 2.5).all()
        dw = torch.randn(500, 1, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
        assert not _backward(r, logits, ids, dw).any()


@pytest.mark.gpu
@pytest.mark.parametrize("score,renormalise", [(0, True), (0, False), (1, True), (1, False)])
def test_gradient_of_given_ids(score, renormalise):
    """Ids out of range, an expert named twice, masked experts, a row of nothing, far logits."""
    import torch
    E, k = 40, 4
    logits, _ = _logits(8, E, "f32", 2)
    ids = torch.tensor([[3, 3, 5, 9], [-1, 40, 1000, 2], [-1, -1, -1, -1], [0, 39, 7, 8], [1, 2, 3, 4], [1, 2, 3, 4], [5, 6, 7, 8], [1, 1, 1, 1]], dtype=torch.int32, device="cuda")
    logits[3, 7] = -np.inf
    logits[4] = -300.0 - torch.arange(E, device="cuda")
    logits[5] = 60.0 - torch.arange(E, device="cuda")
    logits[6] = -np.inf
    dw = torch.randn(8, k, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    r = mbd.Router(E, k, score, renormalise)
    got = _backward(r, logits, ids, dw)
    assert not got[6].any() and not got[2].any() and torch.isfinite(got).all()
    keep = [0, 1, 2, 3, 4, 5, 7]
    _close(got[keep], logits.cpu().numpy()[keep], ids.cpu().numpy()[keep], dw.cpu().numpy()[keep], r)


@pytest.mark.gpu
@pytest.mark.parametrize("score,renormalise", [(0, True), (0, False), (1, True), (1, False)])
def test_gradient_against_differences(score, renormalise):
    """Along a direction v with the choice held: (w(l + d v) - w(l - d v)) / 2d; weights are off by 60 U, the expansion's next term is below d^2 |v|_max^2
    (third derivatives of these scores are below 6)."""
    import torch
    E, k, T = 12, 3, 6
    gen = torch.Generator(device="cuda").manual_seed(8)
    l = torch.randn(T, E, device="cuda", generator=gen)
    top = torch.topk(l, k, dim=1).indices
    l.scatter_add_(1, top, torch.ones(T, k, device="cuda") * torch.tensor([6.0, 4.0, 2.0], device="cuda"))   # the choice stays
    v, dw = torch.randn(T, E, device="cuda", generator=gen).clamp(-2, 2), torch.randn(T, k, device="cuda", generator=gen)
    r = mbd.Router(E, k, score, renormalise)
    d = 2.0 ** -7
    a, b = _route(r, l + d * v), _route(r, l - d * v)
    ids = _route(r, l)[0]
    assert torch.equal(a[0], ids) and torch.equal(b[0], ids)
    slope = (dw.double() * (a[1].double() - b[1].double())).sum(1) / (2 * d)
    got = (_backward(r, l, ids, dw).double() * v.double()).sum(1)
    slack = dw.double().abs().sum(1) * (60 * U / d + 8 * 6 * d * d)
    assert ((slope - got).abs() <= slack).all()
