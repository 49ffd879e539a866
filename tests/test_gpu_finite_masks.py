"""Rows of logits masked with finite values of any size (-1e4 to the type's lowest), through the top logits and the distillation, against 64-bit forms.

Within a row the masked tokens weigh nothing beside a visible one, so the limits are those of the visible tokens (test_gpu_logits.py, test_gpu_distill_extremes.py);
rows of nothing but masks are uniform over their largest value."""
import numpy as np
import pytest

import torch

from paper_2505_14742_b200 import binding as Q
from test_gpu_distill_extremes import check, device_rows, lse64

pytestmark = pytest.mark.gpu

MASKS = [-1e4, -1e6, -3e7, -1e9, -3e9, -1e10, -1e15, -1e20, -1e30, -1e37, -1e38, -3e38]


def masked(M, V, mask, tau, seed):
    """Logits whose masked tokens fill whole blocks of a thread's work, every other token, all but one, everything."""
    g = np.random.default_rng(seed)
    z = tau * g.standard_normal((M, V)) * 2.0
    z[0::6, V // 3:] = mask
    z[1::6, : V - 5] = mask
    z[2::6, ::2] = mask
    z[3::6] = mask
    z[3::6, V // 2] = 1.0
    z[4::6] = mask
    return z


@pytest.mark.parametrize("mask", MASKS)
@pytest.mark.parametrize("tau", [0.25, 1.0, 3.0, 10.0, 40.0])
@pytest.mark.parametrize("M,V", [(12, 3000), (600, 3000), (6, 40001)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_log_sum_exp_beside_finite_masks(mask, tau, M, V, dtype):
    Z = device_rows(masked(M, V, mask, tau, 5), dtype)
    k = 9
    val, idx, lse = torch.empty((M, k), device="cuda"), torch.empty((M, k), dtype=torch.int32, device="cuda"), torch.empty(M, device="cuda")
    Q.quaff_topk_logits(Z, tau, val, idx, lse)
    z = Z.double()
    order = torch.argsort(-z, dim=1, stable=True)[:, :k]
    assert torch.equal(idx.long(), order) and torch.equal(val.double(), torch.gather(z, 1, order))
    m = z.amax(1, keepdim=True)
    want = (torch.exp((z - m) / tau).sum(1).log() + m[:, 0] / tau).cpu().numpy()
    ok = np.abs(want) < 3.4e38                                 # (a row of masks over a small temperature leaves the floats)
    got = lse.double().cpu().numpy()
    assert (np.abs(got - want) <= 1e-5 + 1e-6 * np.abs(want))[ok].all(), (got[ok], want[ok])
    assert (got[~ok] == -np.inf).all()


@pytest.mark.parametrize("mask", MASKS)
@pytest.mark.parametrize("tau", [0.5, 1.0, 3.0, 10.0, 40.0])
@pytest.mark.parametrize("M,V", [(12, 3000), (600, 3000), (6, 40001)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rest", [False, True])
def test_distillation_beside_finite_masks(mask, tau, M, V, dtype, rest):
    g = np.random.default_rng(6)
    z = masked(M, V, mask, tau, 5)
    k = 7
    idx = np.argsort(g.random((M, V)), axis=1)[:, :k].astype(np.int32)
    np.put_along_axis(z, idx[:, : k - 1].astype(np.int64), tau * g.standard_normal((M, k - 1)), 1)       # the last of the list may be masked
    z[4::6] = mask                                             # (rows of nothing else, the list included)
    val = (tau * g.standard_normal((M, k))).astype(np.float32)
    lse = (lse64(val.astype(np.float64) / tau) - np.log(0.75)).astype(np.float32) if rest else None
    check(device_rows(z, dtype), val, idx, lse, tau, np.linspace(0.1, 0.3, M).astype(np.float32))


@pytest.mark.parametrize("top", [1e6, 1e9, 3e9, 1e15, 1e30])
@pytest.mark.parametrize("tau", [1.0, 7.0])
def test_one_logit_far_above_all(top, tau):
    M, V, k = 3, 5000, 4
    g = np.random.default_rng(2)
    z = g.standard_normal((M, V))
    z[:, 77] = top
    Z = device_rows(z, torch.float32)
    val, idx, lse = torch.empty((M, k), device="cuda"), torch.empty((M, k), dtype=torch.int32, device="cuda"), torch.empty(M, device="cuda")
    Q.quaff_topk_logits(Z, tau, val, idx, lse)
    want = float(np.float32(top)) / tau
    assert (idx[:, 0] == 77).all() and ((lse.double() - want).abs() <= 1e-6 * want).all()
