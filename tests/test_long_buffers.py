"""Buffers of more than 2^31 elements: the places behind that border are computed, and computed right."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


def test_products_and_rows_behind_2_to_the_31():
    import torch
    from paper_1712_04432_b200 import mbd
    T, wide, narrow = 66000, 32776, 24                          # 2.16e9 elements
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    big = torch.empty((T, wide), dtype=torch.bfloat16, device="cuda")
    X, W = torch.randn(T, narrow, device="cuda", generator=gen).to(torch.bfloat16), torch.randn(2, wide, narrow, device="cuda", generator=gen).to(torch.bfloat16)
    offsets = torch.tensor([0, T - 40, T - 3], dtype=torch.int32, device="cuda")
    big[-3:] = 7.0
    mbd.expert_gemm(0, X, W, offsets, big)
    tail = big[-40:].double()
    ref = torch.cat([X[-40:-3].double() @ W[1].double().T, torch.full((3, wide), 7.0, dtype=torch.float64, device="cuda")])
    assert ((tail - ref).abs() <= 2.0 ** -8 * ref.abs() + 1e-3).all()          # 24 products of up to ~20, one rounding to bf16
    # backward-data and backward-weight read the same long rows
    dX = mbd.expert_gemm(1, big, W, offsets, torch.zeros(T, narrow, dtype=torch.float32, device="cuda"))
    want = big[-40:-3].double() @ W[1].double()
    assert ((dX[-40:-3].double() - want).abs() <= 1e-4 * (big[-40:-3].double().abs() @ W[1].double().abs())).all() and not dX[-3:].any()
    dW = mbd.expert_gemm(2, big, X, offsets, torch.zeros(2, wide, narrow, dtype=torch.float32, device="cuda"))
    want = big[-40:-3].double().T @ X[-40:-3].double()
    assert ((dW[1].double() - want).abs() <= 1e-5 * (big[-40:-3].double().abs().T @ X[-40:-3].double().abs())).all()
    q, s = torch.empty((T, wide), dtype=torch.int8, device="cuda"), torch.empty(T, device="cuda")
    mbd.quantize_rows(big, q, s)
    x = big[-5:].double()
    top = (x.abs().amax(1).float() / torch.full((), 127.0, device="cuda"))
    assert torch.equal(s[-5:], top) and torch.equal(q[-5:], torch.round(x / top.double()[:, None]).to(torch.int8))


def test_a_tensor_of_more_than_2_to_the_31_elements():
    import torch
    from paper_1712_04432_b200 import mbd
    n = 2 ** 31 + 700
    p, g = torch.zeros(n, dtype=torch.bfloat16, device="cuda"), torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    g[-900:] = 2.0
    g[:300] = -1.0
    opt = mbd.AdamW([p], [g], state_bits=8)
    opt.step(0.5)
    torch.cuda.synchronize()
    assert torch.equal(p[-900:].float(), torch.full((900,), -0.5, device="cuda")) and torch.equal(p[:300].float(), torch.full((300,), 0.5, device="cuda"))
    assert not p[300:-900].any() and (opt.m[0][-900:].float() == 448).all() and not opt.m[0][300:-900].view(torch.uint8).any()
    assert torch.equal(opt.m_scales[0][-3:], torch.full((3,), float(np.float32(np.float32(2.0) * np.float32(1 - 0.9)) / np.float32(448)), device="cuda"))
    opt.close()
