"""The 4-bit layer where the adapters' inner results T and G leave the range of bf16: infinities come out as the formula has them."""
import numpy as np
import pytest

import torch

pytestmark = pytest.mark.gpu

INF = float("inf")


def positive_layer(M, K, N, r, **kw):
    """Every operand positive and none of W's elements rounded to zero, so an infinity is never multiplied by zero or cancelled."""
    from paper_2505_14742_b200.layer import Mx4Linear
    g = torch.Generator().manual_seed(M + K)
    some = lambda *s: (0.5 + 0.5 * torch.rand(s, generator=g)).to(torch.bfloat16).cuda()
    layer = Mx4Linear(some(N, K), some(K, r), some(r, N), 1.0, M, **kw)
    return layer, some(M, K), some(M, N)


@pytest.mark.parametrize("M,r", [(4, 16), (20, 8), (200, 16), (700, 40)])
@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32])
def test_an_infinite_t_makes_its_row_infinite(M, r, out):
    layer, X, _ = positive_layer(M, 256, 320, r, y_dtype=out, train=False)
    plain = layer.forward(X).clone()
    X[1, 3:10] = 3e38                                          # T overflows; the product of the quantized operands need not
    Y = layer.forward(X)
    rest = [m for m in range(M) if m != 1]
    assert (layer.T[1] == INF).all() and (Y[1] == INF).all()
    assert torch.equal(Y[rest], plain[rest])


@pytest.mark.parametrize("M,r", [(4, 16), (200, 16), (300, 40)])
def test_an_infinite_gradient_stays_infinite(M, r):
    layer, X, dY = positive_layer(M, 256, 320, r, keep_G=True)
    layer.forward(X)
    plain = layer.backward(dY)[0].clone()
    dY[1, 3] = INF
    dX, dA, dB = layer.backward(dY)
    rest = [m for m in range(M) if m != 1]
    assert (layer.G[1] == INF).all() and (dX[1] == INF).all() and (dA == INF).all()
    assert torch.equal(dX[rest], plain[rest])
    assert (dB[:, 3] == INF).all() and torch.isfinite(dB[:, :3]).all() and torch.isfinite(dB[:, 4:]).all()


@pytest.mark.parametrize("M", [3, 200])
def test_a_g_between_the_largest_bf16_and_the_largest_f32_is_a_number(M):
    """G = (2 - 2^-7) 2^127 + 3/4 2^120 has no finite bf16 next to it, but its products with A have: as the sum of its parts, each of 8 bits."""
    from paper_2505_14742_b200.layer import Mx4Linear
    K, N, r = 64, 64, 8
    W = torch.zeros((N, K), dtype=torch.bfloat16, device="cuda")
    A = torch.full((K, r), 2.0 ** -30, dtype=torch.bfloat16, device="cuda")
    B = torch.zeros((r, N), dtype=torch.bfloat16, device="cuda")
    B[:, 0], B[:, 1] = 2.0 - 2.0 ** -7, 0.75 * 2.0 ** -7
    dY = torch.zeros((M, N), dtype=torch.bfloat16, device="cuda")
    dY[1, :2] = 2.0 ** 127
    X = torch.full((M, K), 2.0 ** -30, dtype=torch.bfloat16, device="cuda")
    layer = Mx4Linear(W, A, B, 1.0, M, keep_G=True)
    layer.forward(X)
    dX, dA, _ = layer.backward(dY)
    G = (2.0 - 2.0 ** -7) * 2.0 ** 127 + 0.75 * 2.0 ** 120
    # one rounding of dX to bf16 (2^-8); dA is f32: parts of 8 bits each and eight truncated sums
    assert (np.abs(dX[1].double().cpu().numpy() - r * G * 2.0 ** -30) <= 2.0 ** -8 * r * G * 2.0 ** -30).all()
    assert (np.abs(dA.double().cpu().numpy() - G * 2.0 ** -30) <= 2.0 ** -20 * G * 2.0 ** -30).all()
