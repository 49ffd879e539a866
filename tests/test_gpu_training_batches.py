"""The persistent kernels at the sizes they are persistent for: products with several tiles per pair of CTAs, rows of logits with several per CTA,
against plain 64-bit forms.

Limits are those of test_gpu_mx4.py and test_gpu_logits.py: a product is off by (K / 64 + r / 8 + 4) 2^-22 of the sum of its terms' magnitudes, and one
rounding of the result; T by (K / 16 + 200) 2^-22 of its own; the parts of s T carry 2^-16.  Loss and gradient of a row: 1e-5 of the terms they are sums of,
2e-5 w tau at listed tokens."""
import pytest

import torch

from paper_2505_14742_b200 import binding as Q

pytestmark = pytest.mark.gpu

BF, F = torch.bfloat16, torch.float32
INF = float("inf")


def rows_of(t, pad):
    w = 16 // t.element_size()
    buf = torch.full((t.shape[0], (t.shape[1] + pad + w - 1) // w * w), float("nan"), dtype=t.dtype, device="cuda")
    buf[:, : t.shape[1]] = t
    return buf[:, : t.shape[1]]


def quantize(X):
    c, s = Q.mx4_empty(*X.shape)
    Q.quaff_mx4_quantize(X, c, s)
    v = torch.empty((X.shape[0], (X.shape[1] + 7) // 8 * 8), dtype=BF, device="cuda")[:, : X.shape[1]]
    Q.quaff_mx4_dequantize(c, s, v)                            # (bit for bit right: test_gpu_mx4.py)
    return (c, s), v.double()


# Tiles of 256 x 256 for at most 74 pairs: 132 to 520 of them; stages per tile from 1 to 9, so that the ring of six stages, the four slots of
# block scales and the two accumulators stand everywhere relative to one another from tile to tile
@pytest.mark.parametrize("M,K,N", [(3000, 200, 2600), (3001, 512, 2603), (2560, 700, 5000), (8192, 1000, 4096), (5000, 1400, 6600), (2600, 2300, 4095)])
@pytest.mark.parametrize("out", [BF, F])
def test_product_over_many_tiles(M, K, N, out):
    g = torch.Generator(device="cuda").manual_seed(M + K + N)
    X, W = rows_of(torch.randn((M, K), generator=g, device="cuda").to(BF), 0), rows_of((torch.randn((N, K), generator=g, device="cuda") * 0.05).to(BF), 8)
    (xq, Xv), (wq, Wv) = quantize(X), quantize(W)
    want = Xv @ Wv.t()
    lim = (K / 64 + 4) * 2.0 ** -22 * (Xv.abs() @ Wv.abs().t()) + (2.0 ** -8 * want.abs() if out == BF else 0.0)
    status = torch.zeros(4, dtype=torch.int32, device="cuda")
    first = None
    for pad in (0, 3, 0, 8):                                  # whole-line stores where the pitch allows them, else row by row
        ld = (N + 7) // 8 * 8 + pad
        Y = torch.full((M + 1, ld), 5.0, dtype=out, device="cuda")
        Q.quaff_mx4_matmul(*xq, *wq, K, Y[:M, :N], None, status)
        assert int(status[0]) == 0
        assert (Y[M] == 5.0).all() and (Y[:, N:] == 5.0).all()
        Y = Y[:M, :N].contiguous()
        assert first is None or torch.equal(Y, first)
        if first is None:
            assert ((Y.double() - want).abs() <= lim).all()
        first = Y


@pytest.mark.parametrize("M,K,N,r", [(3000, 512, 2600, 16), (4096, 200, 2560, 64), (8192, 1000, 4096, 8), (2600, 1800, 5000, 40), (515, 96, 32000, 16)])
@pytest.mark.parametrize("out", [BF, F])
def test_layer_over_many_tiles(M, K, N, r, out):
    """With the stages of the adapters (two for bf16, three for f32) between those of the tiles; the last is an output head."""
    from paper_2505_14742_b200.layer import Mx4Linear
    g = torch.Generator(device="cuda").manual_seed(M + r)
    rn = lambda *s: torch.randn(s, generator=g, device="cuda")
    X, W, A, B = rn(M, K).to(BF), (rn(N, K) * 0.05).to(BF), (rn(K, r) * 0.1).to(BF), (rn(r, N) * 0.1).to(BF)
    layer = Mx4Linear(W, A, B, 0.5, M, y_dtype=out)
    Y = layer.forward(X)
    assert int(layer.status[0]) == 0
    (_, Xv), (_, Wv) = quantize(X), quantize(W)
    t, absB = X.double() @ A.double(), B.double().abs()
    dT = (K / 16 + 200) * 2.0 ** -22 * (X.double().abs() @ A.double().abs())
    want = Xv @ Wv.t() + 0.5 * t @ B.double()
    lim = (K / 64 + r / 8 + 4) * 2.0 ** -22 * (Xv.abs() @ Wv.abs().t()) + 0.5 * dT @ absB
    lim += (2.0 ** -16 + (K / 64 + r / 8 + 4) * 2.0 ** -22) * 0.5 * (t.abs() @ absB) + (2.0 ** -8 * want.abs() if out == BF else 0.0)
    assert ((Y.double() - want).abs() <= lim).all()
    assert ((layer.T.double() - t).abs() <= 2.0 ** -8 * t.abs() + dT).all()
    again = Y.clone()
    for _ in range(3):
        layer.ws.fill_(0xFF)
        assert torch.equal(layer.forward(X), again)
    # and the gradient through it
    dY = (rn(M, N) * 0.1).to(BF)
    dX, _, _ = layer.backward(dY)
    dy, G = dY.double(), 0.5 * dY.double() @ B.double().t()
    dG = (N / 16 + 200) * 2.0 ** -22 * 0.5 * (dy.abs() @ absB.t()) + 2.0 ** -16 * G.abs()
    want = dy @ Wv + G @ A.double().t()
    lim = (N / 16 + r / 16 + 4) * 2.0 ** -22 * (dy.abs() @ Wv.abs()) + ((N / 16 + r / 16 + 4) * 2.0 ** -22 * G.abs() + dG) @ A.double().abs().t()
    assert ((dX.double() - want).abs() <= lim + 2.0 ** -8 * want.abs()).all()


# Rows of one CTA each, up to three on an SM: the 445th is some CTA's second
def batch_of_logits(M, V, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    z = torch.randn((M, V), generator=g, device="cuda") * 3.0
    z.scatter_add_(1, torch.randint(0, V, (M, 12), generator=g, device="cuda"), torch.full((M, 12), 9.0, device="cuda"))
    z[5::97] = -INF
    z[6::97, ::3] = -INF
    z[7::97] = 0.25
    return rows_of(z.to(dtype), 8), g


@pytest.mark.parametrize("M,V,k", [(2000, 3001, 20), (1500, 9000, 100), (1400, 16000, 256), (5000, 500, 1)])
@pytest.mark.parametrize("dtype", [BF, F])
def test_top_logits_of_many_rows(M, V, k, dtype):
    Z, _ = batch_of_logits(M, V, dtype, V + k)
    tau = 1.5
    val, idx, lse = torch.empty((M, k), device="cuda"), torch.empty((M, k), dtype=torch.int32, device="cuda"), torch.empty(M, device="cuda")
    Q.quaff_topk_logits(Z, tau, val, idx, lse)
    z = Z.double()
    order = torch.argsort(-z, dim=1, stable=True)[:, :k]
    want = torch.gather(z, 1, order)
    assert torch.equal(val.double(), want)
    assert torch.equal(idx.long(), torch.where(want > -INF, order, torch.full_like(order, -1)))
    ref = torch.logsumexp(z / tau, 1)
    assert ((lse.double() - ref).abs() <= 1e-5 + 1e-6 * ref.abs())[ref > -INF].all() and (lse[ref == -INF] == -INF).all()


def distill_definition(Z, val, idx, lse, tau, w):
    """Loss, gradient, and the sums of their terms' magnitudes, for lists without holes."""
    z = Z.double() / tau
    live, at = idx >= 0, idx.long().clamp_min(0)
    logq = z - torch.logsumexp(z, 1, keepdim=True)
    t = torch.where(live, val.double() / tau, torch.full_like(val, -INF, dtype=torch.float64))
    logp = t - (torch.logsumexp(t, 1, keepdim=True) if lse is None else lse.double()[:, None])
    p = logp.exp()
    terms = torch.where(live & (p > 0), p * (logp - torch.gather(logq, 1, at)), torch.zeros_like(p))
    R = torch.zeros_like(w, dtype=torch.float64) if lse is None else (1.0 - p.sum(1)).clamp_min(0.0)
    listed = torch.zeros_like(z, dtype=torch.int32).scatter_add_(1, at, live.int()) > 0
    rest = torch.where(listed, torch.full_like(z, -INF), logq)
    logr = torch.logsumexp(rest, 1)
    more = torch.where(R > 0, R * (R.clamp_min(1e-300).log() - logr), torch.zeros_like(R))
    c = (p.sum(1) + R)[:, None]
    wt = (w.double() * tau)[:, None]
    a, b = wt * c * logq.exp(), wt * torch.where(R[:, None] > 0, R[:, None] * (rest - logr[:, None]).exp(), torch.zeros_like(rest))
    pv = torch.zeros_like(z).scatter_add_(1, at, torch.where(live, p, torch.zeros_like(p)))
    grad = torch.where(listed, a - wt * pv, a - b)
    lim = torch.where(listed, 2e-5 * wt.expand_as(z), 2e-5 * (a + b) + 1e-15 * wt)
    s = w.double() * tau * tau
    return s * (terms.sum(1) + more), s * (terms.abs().sum(1) + more.abs()), grad, lim


@pytest.mark.parametrize("M,V,k", [(2000, 3001, 20), (1500, 9000, 100), (1300, 16000, 256), (5000, 500, 4)])
@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("in_place", [False, True])
def test_distillation_of_many_rows(M, V, k, dtype, rest, in_place):
    tau = 2.0
    T, g = batch_of_logits(M, V, dtype, V)
    val, idx, lse = torch.empty((M, k), device="cuda"), torch.empty((M, k), dtype=torch.int32, device="cuda"), torch.empty(M, device="cuda")
    Q.quaff_topk_logits(T, tau, val, idx, lse)
    Z = rows_of((T.float() + torch.randn((M, V), generator=g, device="cuda")).to(dtype), 8)
    w = torch.rand(M, generator=g, device="cuda")
    w[torch.rand(M, generator=g, device="cuda") < 0.2] = 0.0
    w[700:760] = 0.0                                          # runs of rows without a loss, the last ones among them
    w[-40:] = 0.0
    alive = (T > -INF).any(1)
    loss, mag, grad, lim = distill_definition(Z, val, idx, lse if rest else None, tau, w)
    got, alone = torch.full((M,), 9.0, device="cuda"), torch.full((M,), 9.0, device="cuda")
    Q.quaff_distill_topk(Z, val, idx, lse if rest else None, tau, w, alone)
    dZ = Z if in_place else torch.empty_strided(Z.shape, Z.stride(), dtype=dtype, device="cuda").fill_(7.0)
    Q.quaff_distill_topk(Z, val, idx, lse if rest else None, tau, w, got, dZ)
    assert torch.equal(got, alone)
    dead = ~alive | (w == 0)
    assert not got[dead].any() and not dZ[dead].any()
    if dtype == BF:
        lim = lim + 2.0 ** -8 * grad.abs()
    assert ((got.double() - loss).abs() <= 1e-5 * mag + 5e-6 * w.double() * tau * tau)[~dead].all()
    assert ((dZ.double() - grad).abs() <= lim)[~dead].all()
