"""Logits masked with a finite value (-1e9 and its like) or far from zero, where such a value is all
that is left outside the list: top logits and the distillation loss on the GPU against float64.

Bounds.  u = 2^-24, EPS and the logarithms' bounds are those of ``test_gpu_distill``.  Where the
arguments in use and their logarithms are at most 60 in size, 4 u (60 + 60) <= EPS and every logarithm is off
by d <= 2 EPS.  An unlisted class at the mask value has the share 1 / n of the rest exactly but for the sum and
its reciprocal (EPS), and log s = (mask - m) / T - ... is off by 4 u of itself and 2 EPS.  So
    J:     soft / T (q d + p d + (s + rho) / n (d + EPS)) 1.01 + hard (q d + 2 u)
    loss:  p (2 d + 1.01 d |log p - log q|) + rho (d + 4 u |log s| + 2 EPS + 1.01 d |log rho - log s|) + hard d
"""
import numpy as np
import pytest
import torch

from oracle import ops
from test_gpu_distill import DT, EPS, U, call, check_top, log_error, logits, matrix, put, top

pytestmark = pytest.mark.gpu

# (mask value, temperature): the usual constants, and what makes |mask| / T pass 2^30 with few or many bits to spare
MASKS = [(-1e9, 0.3), (-1e10, 1.0), (-1e10, 2.0), (-1e12, 1.0), (-1e9, 1.0), (-1e9, 2.5), (-1e15, 0.7), (-1e18, 1.0), (-1e30, 1.0), (-3e38, 2.0)]


def rounded(x, dtype):
    return float(torch.tensor(x, dtype=DT[dtype]).float())


def masked_rows(rng, rows, C, left, mask, dtype):
    """Rows with `left` classes unmasked, and those classes."""
    z = np.full((rows, C), rounded(mask, dtype))
    at = np.stack([rng.permutation(C)[:left] for _ in range(rows)])
    np.put_along_axis(z, at, logits(rng, rows, left, 1.2), 1)
    return z, at


# a wave, a workgroup and parts to a row
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("C,K", [(41, 8), (390, 71), (5000, 64), (9000, 200), (40000, 64), (131072, 50)])
@pytest.mark.parametrize("mask,T", MASKS)
def test_top_logits_beside_a_finite_mask(C, K, mask, T, dtype):
    rng = np.random.default_rng(C + K)
    for left in (K - 1, K, K + 1):
        z, _ = masked_rows(rng, 2, C, left, mask, dtype)
        check_top(matrix(z, dtype), C, K, T, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("mask,T", MASKS)
def test_top_logits_of_many_rows_beside_a_finite_mask(mask, T, dtype):
    """The same rows often enough for a thread each."""
    rng = np.random.default_rng(3)
    z = np.concatenate([masked_rows(rng, 2, 41, left, mask, dtype)[0] for left in (7, 8, 9)])
    Z = matrix(np.tile(z, (10000, 1)), dtype)
    v, i, t = (x.reshape(10000, 6, -1) for x in top(Z, 41, 8, T, dtype))
    assert (v == v[0]).all() and (i == i[0]).all() and (t == t[0]).all()
    rv, ri, rt = ops.top_logits(Z[:6, :41].float().cpu().numpy().astype(np.float64), 8, T)
    assert np.array_equal(v[0], rv) and np.array_equal(i[0], ri)
    assert (np.abs(t[0, :, 0] - rt) <= log_error(4 * abs(mask) / T, rt)).all()


@pytest.mark.parametrize("C,K", [(41, 8), (390, 71), (5000, 64), (40000, 64)])
@pytest.mark.parametrize("at,T", [(1e6, 1e-4), (5e5, 1e-4), (-3e7, 0.01), (2.0 ** 40, 1.0), (-(2.0 ** 31), 1.0)])
def test_top_logits_far_from_zero(C, K, at, T):
    """Whole rows whose neighbouring values are more than a temperature apart."""
    rng = np.random.default_rng(C)
    step = float(np.spacing(np.float32(abs(at)))) / 2            # of the binade below, too
    z = at - 2 * step * rng.integers(0, 4, (3, C))
    check_top(matrix(z, "f32"), C, K, T, "f32")


def rest_of(z, listed, T):
    """(log of the sum over the unlisted classes relative to their maximum, that maximum, their shares) of z / T."""
    r = z[~listed]
    e = np.exp((r - r.max()) / T)
    within = np.zeros(len(z))
    within[~listed] = e / e.sum()
    return np.log(e.sum()), r.max(), within


def reference(z, v, i, tail, y, T, soft, hard):
    """(loss, J, bound of the loss, bounds of J) of a row whose unlisted classes have a far lower maximum than the listed ones.
    Differences are formed before the division by T: float64 holds them exactly."""
    C, m = len(z), z.max()
    listed = np.zeros(C, bool)
    listed[i] = True
    t = (v - v.max()) / T
    total = np.logaddexp(np.log(np.exp(t).sum()), tail - v.max() / T)
    log_p, log_rho = t - total, tail - v.max() / T - total
    log_all = np.log(np.exp((z - m) / T).sum())
    log_q = (z - m) / T - log_all
    log_rest, top_rest, within = rest_of(z, listed, T)
    log_s = (top_rest - m) / T + log_rest - log_all
    q, p, rho, s = np.exp(log_q), np.zeros(C), np.exp(log_rho), np.exp(log_s)
    p[i] = np.exp(log_p)
    on = np.exp(log_p) > 0
    diff = (log_p - log_q[i])[on]
    d = 2 * EPS
    loss = (p[i][on] * diff).sum() + (rho * (log_rho - log_s) if rho > 0 else 0.0)
    bound = (p[i][on] * (2 * d + 1.01 * d * np.abs(diff))).sum()
    if rho > 0:
        bound += rho * (d + 4 * U * abs(log_s) + 2 * EPS + 1.01 * d * abs(log_rho - log_s))
    J = soft / T * np.where(listed, q - p, within * (s - rho))
    jb = 1.01 * soft / T * (q * d + p * d + within * (s + rho) * (d + EPS))
    loss, bound = soft * loss, soft * bound
    if y >= 0:
        h = np.exp(z - m - np.log(np.exp(z - m).sum()))
        loss += hard * (m - z[y] + np.log(np.exp(z - m).sum()))
        bound += hard * d
        J += hard * h
        J[y] -= hard
        jb += hard * (h * d + 2 * U)
    return loss, J, bound, jb


# a few lanes, a wave, a workgroup, parts to a row
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,C,K", [(40, 41, 8), (9, 1500, 30), (5, 2500, 64), (4, 30000, 200), (130, 30000, 64), (2, 70000, 40),
                                      (150, 70000, 8)])
@pytest.mark.parametrize("mask,T", MASKS)
def test_distill_beside_a_finite_mask(rows, C, K, mask, T, dtype):
    rng = np.random.default_rng(C + K)
    if rows > 100 and (mask, T) not in MASKS[:4]:
        rows = 3
    for left in (K - 1, K, K + 1):
        z, at = masked_rows(rng, rows, C, left, mask, dtype)
        Z = matrix(z, dtype)
        z = Z[:, :C].float().cpu().numpy().astype(np.float64)
        low = z.min()
        lists = np.sort(at, axis=1)[:, :K]                         # K - 1 left: a masked class takes the last slot
        if left < K:
            lists = np.concatenate([lists, [[next(c for c in range(C) if c not in set(r))] for r in lists]], 1)
        v = (np.take_along_axis(z, lists, 1) + 0.5 * rng.standard_normal(lists.shape)).astype(np.float32).astype(np.float64)
        v[np.take_along_axis(z, lists, 1) == low] = low
        tail = (v.max(1) / T - 1.0).astype(np.float32).astype(np.float64)
        if left == K:                                              # the teacher's own log-sum of its masked classes
            tail[::2] = np.float32(low / T)
        y = np.where(rng.random(rows) < 0.3, -1, at[:, 0])
        soft, hard = float(np.float32(0.9 / rows)), float(np.float32(0.4 / rows))
        T32 = float(np.float32(T))
        vt, it, tt = put(v, lists, tail)
        J, loss = call(Z, C, vt, it, tt, torch.from_numpy(y.astype(np.int32)).cuda(), T, soft, hard, dtype)
        torch.cuda.synchronize()
        j = J[:, :C].float().cpu().numpy().astype(np.float64)
        want, lb = 0.0, 0.0
        for r in range(rows):
            l, ref, b, jb = reference(z[r], v[r], lists[r], tail[r], int(y[r]), T32, soft, hard)
            jb = jb + 4 * U * np.abs(ref) + 2.0 ** -126
            if dtype == "bf16":
                jb = jb * (1 + 2.0 ** -8) + 2.0 ** -8 * np.abs(ref)
            assert (np.abs(j[r] - ref) <= jb).all(), (left, r, np.abs(j[r] - ref).max())
            want, lb = want + l, lb + b
        assert abs(float(loss[0]) - want) <= lb + 2 * U * abs(want), (left, float(loss[0]), want, lb)


def test_the_masks_agree_over_kernels():
    """A row has the same tail whichever kernel the number of rows selects."""
    rng = np.random.default_rng(0)
    for mask in (-1e9, -1e10, -1e12):
        z, _ = masked_rows(rng, 1, 41, 8, mask, "f32")
        one = top(matrix(z, "f32"), 41, 8, 0.3, "f32")
        many = top(matrix(np.tile(z, (60000, 1)), "f32"), 41, 8, 0.3, "f32")
        assert np.array_equal(one[1][0], many[1][0]) and abs(float(one[2][0]) - float(many[2][0])) <= 16 * U * abs(mask) / 0.3
