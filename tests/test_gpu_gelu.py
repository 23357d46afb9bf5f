"""GELU and its slope in the group norm's kernels, against 64 bits at the very u that the kernel forms: fp32
operations one after another on the mean and rstd that the call returns, which numpy's float32 gives bit by bit.

Bounds.  V = 2^-24, P = Phi(u), Q = Phi(-|u|).
Q, where it is formed as e^{-u^2/2} t poly(t), t = 1 / (1 + 0.3 |u|): the fit 2.5 V; t is off by 3 V (a reciprocal within
one unit, a rounding), and d log(t poly) / d log t <= 2.7 on [0, 14]: 8 V; the polynomial's seven steps, whose terms are
at most twice their sum: 4 V a step at the innermost, less each time t or the sum outweighs it, in all 4 V; the exponent -u^2/2
log2 e has two roundings of itself, u^2 V, and the exponential and two products 4 V.  So dQ <= (20 + u^2) V Q, and P's own rounding
(1 - Q) adds V / 2.  In fp32 P for |u| <= 1.25 is 1/2 + u S(u^2): off by 3 V of |u S| <= 0.4 and V P; the above covers it
there too (Q >= 0.1: 2 V), so one bound serves both.
    y = u P:        |u| dP + V |y| + 2^-126 |u| (a tail below the smallest normal may be flushed)
    P + u phi:      dP + (u^2 + 6) V |u| phi + 2 V (P + |u| phi);  times J in the sum for beta: V more.
A bf16 result is rounded once: 2^-8 of itself."""
import math

import numpy as np
import pytest
import torch

from test_gpu_group_norm import U as V, TINY, backward, forward, host, matrix, spread

pytestmark = pytest.mark.gpu

erfc = np.vectorize(math.erfc, otypes=[np.float64])


def u_of(X, f, G, samples, R, mean, rstd, ga, be):
    """The kernel's u."""
    S = lambda t: spread(host(t[:-1]).reshape(samples, G), samples, R, G, f).astype(np.float32)
    d = (X[:, :f].float().cpu().numpy() - S(mean)) * S(rstd)
    return (d * ga + be).astype(np.float64)


def inputs(samples, R, f, dtype, seed):
    rng = np.random.default_rng(seed)
    X = matrix(0.3 * rng.standard_normal((samples * R, f)), dtype)
    ga = np.full(f, 0.5, np.float32)
    be = rng.permutation(np.linspace(-14.0, 14.0, f)).astype(np.float32)      # u over the whole range
    return rng, X, ga, be, torch.from_numpy(ga).cuda(), torch.from_numpy(be).cuda()


def cdf(u):
    """(Phi, its bound, phi)."""
    q = 0.5 * erfc(np.abs(u) / math.sqrt(2.0))
    return 0.5 * erfc(-u / math.sqrt(2.0)), q * (20 + u * u) * V + np.where(u > 0, V / 2, 0.0), np.exp(-0.5 * u * u) / math.sqrt(2 * math.pi)


# rows in registers, through LDS, in chunks
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("samples,R,f,G", [(9, 1, 1024, 1), (7, 1, 1023, 3), (2, 3, 500, 5), (1, 3000, 64, 2), (5, 1, 8192, 8)])
def test_gelu(samples, R, f, G, dtype):
    rng, X, ga, be, gt, bt = inputs(samples, R, f, dtype, f)
    Y, mean, rstd = forward(X, f, G, samples, R, gt, bt, "gelu", dtype)
    torch.cuda.synchronize()
    u = u_of(X, f, G, samples, R, mean, rstd, ga, be)
    p, dp, _ = cdf(u)
    bound = np.abs(u) * dp + V * np.abs(u * p) + TINY * np.abs(u)
    if dtype == "bf16":
        bound = bound * (1 + 2.0 ** -8) + 2.0 ** -8 * np.abs(u * p) + TINY
    err = np.abs(host(Y[:samples * R, :f]) - u * p)
    assert (err <= bound).all(), (u[err > bound][:5], err[err > bound][:5], bound[err > bound][:5])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("f,G", [(1024, 1), (1023, 3), (300, 100), (8192, 8)])
def test_gelu_slope(f, G, dtype):
    """One row: beta's gradient is J times the slope."""
    rng, X, ga, be, gt, bt = inputs(1, 1, f, dtype, f)
    J = matrix(rng.standard_normal((1, f)), dtype)
    _, mean, rstd = forward(X, f, G, 1, 1, gt, bt, "gelu", dtype)
    db = backward(X, J, f, G, 1, 1, gt, bt, mean, rstd, "gelu", dtype)[2]
    torch.cuda.synchronize()
    u, j = u_of(X, f, G, 1, 1, mean, rstd, ga, be)[0], host(J[0, :f])
    p, dp, phi = cdf(u)
    a = np.abs(u) * phi
    bound = np.abs(j) * (dp + (u * u + 6) * V * a + 3 * V * (p + a) + TINY * (1 + np.abs(u)))
    err = np.abs(host(db[:f]) - j * (p + u * phi))
    assert (err <= bound).all(), (u[err > bound][:5], err[err > bound][:5], bound[err > bound][:5])
