"""Distillation where the student's unlisted tokens carry next to nothing, and teacher rows at the edge of their definition,
against the definition in 64 bits and in logarithms.

Tolerances.  The gradient of an unlisted token is w tau (c q_v - R s_v), s_v its share of the unlisted mass: two exponentials whose arguments
(a nats below their maximum) carry about 2e-7 a, so each term is held to 2e-5 of itself down to a = 100, and to 1e-15 w tau below; a
listed one is the difference of two terms of at most w tau, 2e-5 of that.  The loss is a sum of p (log p - log q) and R (log R - log r), each
held to 1e-5 of its magnitude and 5e-6 w tau^2.  bf16 gradients: one rounding more, 2^-8."""
import numpy as np
import pytest

import torch

from paper_2505_14742_b200 import binding as Q

pytestmark = pytest.mark.gpu

INF = float("inf")


def lse64(x, axis=-1):
    m = x.max(axis, keepdims=True)
    m = np.where(np.isfinite(m), m, 0.0)
    with np.errstate(divide="ignore"):
        return np.log(np.exp(x - m).sum(axis)) + m.squeeze(axis)


def reference(Z, val, idx, lse, tau, w):
    """Loss, gradient and what bounds their errors; every row has a visible student logit."""
    z = Z.double().cpu().numpy() / tau
    M, V = z.shape
    loss, mag, grad, lim = np.zeros(M), np.zeros(M), np.zeros((M, V)), np.zeros((M, V))
    for m in range(M):
        z[m] -= z[m].max()                                    # (beside a mask of 1e15 a double holds no logarithm)
        ok = (idx[m] >= 0) & (idx[m] < V) & (val[m] > -np.inf)
        at, t = idx[m][ok], val[m][ok].astype(np.float64) / tau
        logp = t - (lse64(t) if lse is None else float(lse[m]))
        p = np.exp(logp)
        R = 0.0 if lse is None else max(0.0, 1.0 - p.sum())
        c = p.sum() + R
        unl = np.ones(V, bool)
        unl[at] = False
        total = lse64(z[m])
        lq = z[m] - total
        terms = p * (logp - lq[at])
        grad[m, unl] = w[m] * tau * c * np.exp(lq[unl])
        lim[m, unl] = np.abs(grad[m, unl])
        if R > 0:
            lu = lse64(z[m][unl])
            share = np.exp(z[m][unl] - z[m][unl].max())       # (lu itself holds no logarithm of their number beside a mask of 1e38)
            rest = w[m] * tau * R * share / share.sum()
            grad[m, unl] -= rest
            lim[m, unl] += rest
            terms = np.append(terms, R * (np.log(R) - (lu - total)))
        lim[m, unl] = 2e-5 * lim[m, unl] + 1e-15 * w[m] * tau
        grad[m, at] = w[m] * tau * (c * np.exp(lq[at]) - p)
        lim[m, at] = 2e-5 * w[m] * tau
        loss[m] = w[m] * tau * tau * terms.sum()
        mag[m] = w[m] * tau * tau * np.abs(terms).sum()
    return loss, mag, grad, lim


def run(Z, val, idx, lse, tau, w):
    dev = lambda a: None if a is None else torch.from_numpy(np.ascontiguousarray(a)).cuda()
    loss = torch.full((Z.shape[0],), 9.0, device="cuda")
    dZ = torch.empty_strided(Z.shape, Z.stride(), dtype=Z.dtype, device="cuda").fill_(5.0)
    Q.quaff_distill_topk(Z, dev(val), dev(idx), dev(lse), tau, dev(w), loss, dZ)
    alone = torch.empty_like(loss)
    Q.quaff_distill_topk(Z, dev(val), dev(idx), dev(lse), tau, dev(w), alone)
    assert torch.equal(loss.view(torch.int32), alone.view(torch.int32))
    return loss.double().cpu().numpy(), dZ.double().cpu().numpy()


def check(Z, val, idx, lse, tau, w):
    loss, dZ = run(Z, val, idx, lse, tau, w)
    want, mag, grad, lim = reference(Z, val, idx, lse, tau, w)
    if Z.dtype == torch.bfloat16:
        lim = lim + 2.0 ** -8 * np.abs(grad)
    assert np.isfinite(want).all() and np.isfinite(grad).all()
    over = mag > 3.4e38                                        # beyond the floats
    assert (loss[over] == INF).all()
    assert (np.abs(loss - want) <= 1e-5 * mag + 5e-6 * w * tau * tau)[~over].all(), (loss, want)
    bad = ~(np.abs(dZ - grad) <= lim)
    assert not bad.any(), (np.argwhere(bad)[:4], dZ[bad][:4], grad[bad][:4])


def device_rows(z, dtype):
    V = z.shape[1]
    buf = torch.zeros((z.shape[0], (V + 7) // 8 * 8), dtype=dtype, device="cuda")
    buf[:, :V] = torch.as_tensor(z, dtype=torch.float32).to(dtype).cuda()
    return buf[:, :V]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("M,V", [(6, 1001), (500, 1001), (3, 20000), (2, 70003)])
@pytest.mark.parametrize("low,tau", [(-9.0, 0.1), (-8.0, 0.1), (-30.0, 0.4), (-80.0, 1.0), (-95.0, 1.0), (-200.0, 1.0), (-1e4, 1.0), (-1e4, 3.0), ("lowest", 1.0),
                                     ("lowest", 0.5)])
@pytest.mark.parametrize("rest", [False, True])
def test_unlisted_tokens_far_below_the_list(dtype, M, V, low, tau, rest):
    """Their share of the student's mass may be far below the smallest float: its logarithm and their shares of it are not."""
    g = np.random.default_rng(V + M)
    k = 5
    if low == "lowest":
        z = np.full((M, V), torch.finfo(dtype).min)
    else:
        z = low + tau * g.standard_normal((M, V))
        if low < -1000.0:
            z[:, : V // 2] = low                              # (equal ones beside others a little apart)
    idx = np.argsort(g.random((M, V)), axis=1)[:, :k].astype(np.int32)
    np.put_along_axis(z, idx.astype(np.int64), tau * g.standard_normal((M, k)), 1)
    val = (tau * g.standard_normal((M, k))).astype(np.float32)
    # the teacher leaves 10 % unlisted
    lse = (lse64(val.astype(np.float64) / tau) - np.log(0.9)).astype(np.float32) if rest else None
    check(device_rows(z, dtype), val, idx, lse, tau, np.linspace(0.25, 1.0, M).astype(np.float32))


@pytest.mark.parametrize("gap", [0.0, 40.0, 85.0, 87.0, 88.0, 90.0, 103.0, 150.0])
def test_unlisted_mass_across_the_smallest_float(gap):
    M, V, k = 4, 3000, 8
    g = np.random.default_rng(7)
    z = g.standard_normal((M, V)) * 0.5
    z[:, :k] += gap
    val = g.standard_normal((M, k)).astype(np.float32)
    idx = np.tile(np.arange(k, dtype=np.int32), (M, 1))
    lse = (lse64(val.astype(np.float64)) - np.log([0.999999, 0.99, 0.5, 1e-3])).astype(np.float32)
    check(device_rows(z, torch.float32), val, idx, lse, 1.0, np.ones(M, np.float32))


def test_listed_tokens_at_the_lowest_value_of_the_type():
    """The student masks a listed token with a finite value: the loss is as large as that and finite."""
    M, V, k = 2, 900, 4
    g = np.random.default_rng(8)
    z = g.standard_normal((M, V))
    z[:, 2] = torch.finfo(torch.float32).min
    val = g.standard_normal((M, k)).astype(np.float32)
    idx = np.tile(np.arange(k, dtype=np.int32), (M, 1))
    for tau in (1.0, 0.5, 0.25):
        check(device_rows(z, torch.float32), val, idx, None, tau, np.full(M, 0.5, np.float32))


# ---------------------------------------------------------------- nothing visible is left unlisted
def restricted(M, V, n, seed, spread=3.0):
    """Rows with n visible tokens each."""
    g = np.random.default_rng(seed)
    z = np.full((M, V), -INF)
    at = np.argsort(g.random((M, V)), axis=1)[:, :n]
    np.put_along_axis(z, at, g.standard_normal((M, n)) * spread, 1)
    return z


@pytest.mark.parametrize("V,n,k", [(1, 1, 1), (5, 5, 5), (60, 60, 64), (200, 200, 256), (4000, 1, 1), (4000, 20, 20), (4000, 20, 64), (70000, 33, 64)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("tau", [0.3, 1.0, 2.0])
def test_a_list_of_all_visible_tokens_leaves_no_rest(V, n, k, dtype, tau):
    """Teacher and student see the same few tokens and all of them are listed: what 1 - sum p has left is the rounding of the
    teacher's log-sum-exp, which no logit of the student can carry.  Loss and gradient as from the renormalised list, which
    rounding changes by at most the 2^-16 + 2^-20 |lse| that the rule allows; lse is below 64 here."""
    M = 64
    t = device_rows(restricted(M, V, n, V + n, 4.0 * tau), dtype)
    g = np.random.default_rng(n)
    z = t.double().cpu().numpy()
    z = device_rows(np.where(np.isfinite(z), z + g.standard_normal(z.shape) * tau, z), dtype)
    val, idx, lse = torch.empty((M, k), device="cuda"), torch.empty((M, k), dtype=torch.int32, device="cuda"), torch.empty(M, device="cuda")
    Q.quaff_topk_logits(t, tau, val, idx, lse)
    w = np.ones(M, np.float32)
    loss, dZ = run(z, val.cpu().numpy(), idx.cpu().numpy(), lse.cpu().numpy(), tau, w)
    want, grad = run(z, val.cpu().numpy(), idx.cpu().numpy(), None, tau, w)
    assert np.isfinite(loss).all() and np.isfinite(dZ).all()
    step = 2.0 ** -16 + 2.0 ** -20 * 64
    # p changes by that share of itself, |log p - log q| <= 40
    assert (np.abs(loss - want) <= 40 * step * tau * tau).all(), (loss, want)
    assert (np.abs(dZ - grad) <= (step + (2.0 ** -7 if dtype == torch.bfloat16 else 0.0)) * tau).all()


def test_a_rest_that_the_student_cannot_carry_is_still_an_infinite_loss():
    """Beyond the resolution of the log-sum-exp the definition holds: the teacher gives mass to tokens that the student rules out."""
    M, V, k = 3, 4000, 8
    z = restricted(M, V, k, 3)
    idx = np.stack([np.flatnonzero(np.isfinite(r)) for r in z]).astype(np.int32)
    val = np.zeros((M, k), np.float32)
    lse = (np.log(k) - np.log([0.999, 0.9, 0.1])).astype(np.float32)
    loss, dZ = run(device_rows(z, torch.float32), val, idx, lse, 1.0, np.ones(M, np.float32))
    assert (loss == INF).all() and np.isfinite(dZ).all()


# ---------------------------------------------------------------- teacher rows that are not finite
@pytest.mark.parametrize("V", [900, 70003])
@pytest.mark.parametrize("bad", [float("nan"), INF])
def test_a_teacher_row_with_nan_or_inf_makes_the_loss_nan(V, bad):
    """Through the teacher's own list: quaff_topk_logits makes the row's log-sum-exp NaN or +inf."""
    M, k = 4, 12
    g = np.random.default_rng(V)
    t = device_rows(g.standard_normal((M, V)), torch.float32)
    z = device_rows(g.standard_normal((M, V)), torch.float32)
    t[1, 7] = bad
    t[3] = bad if np.isnan(bad) else t[3]                     # a row of nothing else: an empty list
    val, idx, lse = torch.empty((M, k), device="cuda"), torch.empty((M, k), dtype=torch.int32, device="cuda"), torch.empty(M, device="cuda")
    Q.quaff_topk_logits(t, 1.0, val, idx, lse)
    w = np.ones(M, np.float32)
    loss, dZ = run(z, val.cpu().numpy(), idx.cpu().numpy(), lse.cpu().numpy(), 1.0, w)
    rows = [1, 3] if np.isnan(bad) else [1]
    rest = [m for m in range(M) if m not in rows]
    assert np.isnan(loss[rows]).all() and np.isnan(dZ[rows]).all()
    assert np.isfinite(loss[rest]).all() and np.isfinite(dZ[rest]).all()
    if not np.isnan(bad):                                     # the list renormalised: +inf / +inf
        loss, dZ = run(z, val.cpu().numpy(), idx.cpu().numpy(), None, 1.0, w)
        assert np.isnan(loss[1]) and np.isnan(dZ[1]).all()
        assert np.isfinite(loss[rest]).all() and np.isfinite(dZ[rest]).all()


def test_a_nan_log_sum_exp_does_not_reach_rows_that_are_not_trained():
    M, V, k = 3, 500, 4
    g = np.random.default_rng(1)
    z = g.standard_normal((M, V))
    z[1] = -INF
    val, idx = g.standard_normal((M, k)).astype(np.float32), np.tile(np.arange(k, dtype=np.int32), (M, 1))
    lse = np.array([np.nan, np.nan, 3.0], np.float32)
    loss, dZ = run(device_rows(z, torch.float32), val, idx, lse, 1.0, np.array([0.0, 1.0, 1.0], np.float32))
    assert loss[0] == 0.0 and loss[1] == 0.0 and not dZ[:2].any() and np.isfinite(loss[2])
