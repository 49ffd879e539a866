"""Mx4Linear as it is strung together with the loss: its results are what quaff_distill_topk and its own backward take, whatever the vocabulary."""
import numpy as np
import pytest

import torch

from paper_2505_14742_b200 import binding as Q

pytestmark = pytest.mark.gpu


def teacher_list(M, V, k, seed):
    g = torch.Generator().manual_seed(seed)
    t = torch.zeros((M, (V + 7) // 8 * 8), device="cuda")[:, :V]
    t.copy_((torch.randn((M, V), generator=g) * 3.0).cuda())
    val, idx, lse = torch.empty((M, k), device="cuda"), torch.empty((M, k), dtype=torch.int32, device="cuda"), torch.empty(M, device="cuda")
    Q.quaff_topk_logits(t, 1.0, val, idx, lse)
    return val, idx, lse


@pytest.mark.parametrize("N", [1, 7, 1000, 1003])
@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("M", [1, 5, 130])
def test_logits_of_any_vocabulary_go_into_the_loss(M, N, out):
    from paper_2505_14742_b200.layer import Mx4Linear
    g = torch.Generator().manual_seed(N + M)
    K = 96
    X, W = (torch.randn(s, generator=g).to(torch.bfloat16).cuda() for s in ((M, K), (N, K)))
    layer = Mx4Linear(W, None, None, 1.0, max(M, 4), y_dtype=out)
    Z = layer.forward(X)
    assert Z.shape == (M, N)
    val, idx, lse = teacher_list(M, N, min(N, 8), N)
    loss, dZ = torch.empty(M, device="cuda"), torch.empty_strided(Z.shape, Z.stride(), dtype=out, device="cuda")
    Q.quaff_distill_topk(Z, val, idx, lse, 1.0, None, loss, dZ)
    assert torch.isfinite(loss).all() and torch.isfinite(dZ).all()
    if out == torch.bfloat16:                                  # and the gradient, in place of the logits, into the backward
        Q.quaff_distill_topk(Z, val, idx, lse, 1.0, None, loss, Z)
        assert torch.equal(Z, dZ)
        dX, dA, dB = layer.backward(Z)
        Wd = torch.zeros((N, K), dtype=torch.bfloat16, device="cuda")
        Q.quaff_mx4_dequantize(layer.Wc, layer.Ws, Wd)
        want = dZ.double() @ Wd.double()
        lim = 2.0 ** -8 * want.abs() + (N / 16 + 4) * 2.0 ** -22 * (dZ.double().abs() @ Wd.double().abs())
        assert dA is None and dB is None and ((dX.double() - want).abs() <= lim).all()


def test_an_odd_vocabulary_is_trained_in_a_head_padded_to_eight():
    """What the class says for adapters and a vocabulary that is no multiple of 8: rows of zeros in W, the loss over the real columns, the
    padding's gradient cleared."""
    from paper_2505_14742_b200.layer import Mx4Linear
    g = torch.Generator().manual_seed(4)
    M, K, V, N, r = 70, 128, 1003, 1008, 8
    X = torch.randn((M, K), generator=g).to(torch.bfloat16).cuda()
    W = torch.zeros((N, K), dtype=torch.bfloat16, device="cuda")
    W[:V] = (torch.randn((V, K), generator=g) * 0.2).to(torch.bfloat16).cuda()
    A = (torch.randn((K, r), generator=g) * 0.1).to(torch.bfloat16).cuda()
    B = torch.zeros((r, N), dtype=torch.bfloat16, device="cuda")
    B[:, :V] = (torch.randn((r, V), generator=g) * 0.1).to(torch.bfloat16).cuda()
    val, idx, lse = teacher_list(M, V, 16, 5)
    layer = Mx4Linear(W, A, B, 1.0, M)
    loss = torch.empty(M, device="cuda")
    Z = layer.forward(X)
    Q.quaff_distill_topk(Z[:, :V], val, idx, lse, 1.0, None, loss, Z[:, :V])
    Z[:, V:].zero_()
    dX, dA, dB = layer.backward(Z)
    dz, T = Z[:, :V].double().cpu().numpy(), layer.T.double().cpu().numpy()
    want = T.T @ dz
    assert (np.abs(dB[:, :V].double().cpu().numpy() - want) <= (M / 16 + 200) * 2.0 ** -22 * (np.abs(T).T @ np.abs(dz))).all()
    assert not dB[:, V:].any() and torch.isfinite(loss).all() and torch.isfinite(dX).all() and torch.isfinite(dA).all()


def test_a_backward_that_cannot_be_says_so():
    from paper_2505_14742_b200.layer import Mx4Linear
    W = torch.ones((64, 64), dtype=torch.bfloat16, device="cuda")
    X = torch.ones((4, 64), dtype=torch.bfloat16, device="cuda")
    A, B = torch.ones((64, 8), dtype=torch.bfloat16, device="cuda"), torch.ones((8, 64), dtype=torch.bfloat16, device="cuda")
    serve = Mx4Linear(W, A, B, 1.0, 4, train=False)
    for M in (2, 4):                                           # fewer rows than the layer was made for, and as many
        dY = serve.forward(X[:M]).clone()
        with pytest.raises(RuntimeError, match="train"):
            serve.backward(dY)
    layer = Mx4Linear(W, A, B, 1.0, 4)
    with pytest.raises(RuntimeError, match="forward"):
        layer.backward(torch.ones((4, 64), dtype=torch.bfloat16, device="cuda"))
    layer.forward(X[:2])
    with pytest.raises(ValueError):                            # the batch of another forward
        layer.backward(torch.ones((4, 64), dtype=torch.bfloat16, device="cuda"))
    for bad in (torch.ones((5, 64), dtype=torch.bfloat16, device="cuda"), torch.ones((4, 32), dtype=torch.bfloat16, device="cuda")):
        with pytest.raises(ValueError):
            layer.forward(bad)
