"""How many bits the adapters' products of the 4-bit layer carry.

Parts: T (f32 results) and G (dA) enter their products in three bf16 parts, 24 bits, so whole numbers below 2^24 pass through exactly; two
parts hold 17.

Chains: an accumulator of the tensor core adds up at most 32 MMAs of sixteen products.  With operands of one sign each step loses less than 2^-23 of the
running sum, and as much again inside the sixteen; the running sums of a chain average half of its result, so 33 2^-23 of it.  Sets of accumulators, slices and
parts are then added up in fp32, one rounding each: one per 512 products of the contraction and at most 24 more."""
import numpy as np
import pytest

import torch

pytestmark = pytest.mark.gpu


def digits(t):
    """Whole numbers below 2^24 as three digits of base 256."""
    return torch.stack([t % 256, t // 256 % 256, t // 65536], -1).float()


def two_parts(t):
    hi = t.float().to(torch.bfloat16).float()
    return hi.double() + (t.float() - hi).to(torch.bfloat16).double()


def numbers(M, r, seed):
    g = torch.Generator().manual_seed(seed)
    t = torch.randint(1 << 23, 1 << 24, (M, r), generator=g)
    assert (two_parts(t) != t).double().mean() > 0.9
    return t


@pytest.mark.parametrize("M", [4, 20, 60, 200, 700])
@pytest.mark.parametrize("r", [8, 64])
def test_an_f32_result_holds_all_bits_of_t(M, r):
    from paper_2505_14742_b200.layer import Mx4Linear
    K, N = 256, 128
    t = numbers(M, r, M)
    X, A, B = torch.zeros((M, K)), torch.zeros((K, r)), torch.zeros((r, N))
    X[:, : 3 * r] = digits(t).reshape(M, -1)
    for j in range(r):
        A[3 * j: 3 * j + 3, j] = torch.tensor([1.0, 256.0, 65536.0])
        B[j, 2 * j] = 1.0
    X, A, B = (a.to(torch.bfloat16).cuda() for a in (X, A, B))
    layer = Mx4Linear(torch.zeros((N, K), dtype=torch.bfloat16, device="cuda"), A, B, 1.0, M, y_dtype=torch.float32, train=False)
    Y = layer.forward(X)
    assert torch.equal(Y[:, 0: 2 * r: 2].double().cpu(), t.double()) and not Y[:, 1::2].any()


@pytest.mark.parametrize("M", [64, 1000, 4096])
@pytest.mark.parametrize("r", [8, 16, 40, 64])
def test_da_holds_all_bits_of_g(M, r):
    from paper_2505_14742_b200.layer import Mx4Linear
    K, N = (M + 7) // 8 * 8, 256
    t = numbers(M, r, M + r)
    dY, A, B = torch.zeros((M, N)), torch.zeros((K, r)), torch.zeros((r, N))
    dY[:, : 3 * r] = digits(t).reshape(M, -1)
    for j in range(r):
        B[j, 3 * j: 3 * j + 3] = torch.tensor([1.0, 256.0, 65536.0])
    X = torch.eye(M, K)
    X, A, B, dY = (a.to(torch.bfloat16).cuda() for a in (X, A, B, dY))
    layer = Mx4Linear(torch.zeros((N, K), dtype=torch.bfloat16, device="cuda"), A, B, 1.0, M)
    layer.forward(X)
    _, dA, _ = layer.backward(dY)
    assert torch.equal(dA[:M].double().cpu(), t.double()) and not dA[M:].any()


def eps(products):
    return 33 * 2.0 ** -23 + (products / 512 + 24) * 2.0 ** -24


def positive(g, *shape):
    return (0.25 + torch.rand(shape, generator=g, device="cuda")).to(torch.bfloat16)


@pytest.mark.parametrize("M,K,N,r", [(16384, 11008, 256, 64), (16384, 11008, 256, 24), (16384, 11000, 264, 8), (40000, 1024, 256, 40), (16384, 1024, 11008, 64),
                                     (40000, 256, 520, 64), (2000, 2048, 2048, 64), (515, 1000, 1544, 8)])
def test_long_sums_keep_their_bits(M, K, N, r):
    """Contractions over many tokens: the error stays that of one short chain, and the sums repeat bit for bit."""
    from paper_2505_14742_b200.layer import Mx4Linear
    g = torch.Generator(device="cuda").manual_seed(M + N + r)
    X, W, A, B, dY = positive(g, M, K), positive(g, N, K), positive(g, K, r), positive(g, r, N), positive(g, M, N)
    layer = Mx4Linear(W, A, B, 1.0, M)
    layer.forward(X)
    _, dA, dB = layer.backward(dY, need_dX=False)
    G = dY.double() @ B.double().t()
    want = X.double().t() @ G
    assert ((dA.double() - want).abs() <= (eps(M) + eps(N) + 2.0 ** -24) * want).all(), ((dA.double() - want).abs() / want).max()
    want = layer.T.double().t() @ dY.double()
    assert ((dB.double() - want).abs() <= eps(M) * want).all(), ((dB.double() - want).abs() / want).max()
    a, b = dA.clone(), dB.clone()
    for _ in range(3):
        layer.ws.fill_(0xEE)
        layer.backward(dY, need_dX=False)
        assert torch.equal(layer.dA, a) and torch.equal(layer.dB, b)


@pytest.mark.parametrize("M,K,r", [(16384, 16384, 64), (4096, 20000, 64), (300, 16384, 40), (12800, 20000, 8)])
def test_long_rows_keep_the_bits_of_t(M, K, r):
    """T over long rows, seen through an f32 result; the codes of X ride along and are those of quaff_mx4_quantize."""
    from paper_2505_14742_b200 import binding as Q
    from paper_2505_14742_b200.layer import Mx4Linear
    g = torch.Generator(device="cuda").manual_seed(M + K + r)
    N = 64
    X, A = positive(g, M, K), positive(g, K, r)
    B = torch.eye(r, N, device="cuda").to(torch.bfloat16)
    layer = Mx4Linear(torch.zeros((N, K), dtype=torch.bfloat16, device="cuda"), A, B, 1.0, M, y_dtype=torch.float32, train=False)
    first = layer.forward(X).clone()
    want = X.double() @ A.double()
    assert ((first[:, :r].double() - want).abs() <= (eps(K) + 2.0 ** -22) * want).all(), ((first[:, :r].double() - want).abs() / want).max()
    W = positive(g, N, K)
    Q.quaff_mx4_quantize(W, layer.Wc, layer.Ws)
    layer.B.zero_()
    codes, scales = Q.mx4_empty(M, K)
    Q.quaff_mx4_quantize(X, codes, scales)
    Y = torch.empty((M, N), device="cuda")
    Q.quaff_mx4_matmul(codes, scales, layer.Wc, layer.Ws, K, Y)
    for _ in range(3):
        layer.ws.fill_(0xEE)
        assert torch.equal(layer.forward(X), Y)
