"""Group normalisation with an activation on the GPU against ``oracle.ops`` (float64).

Bounds.  u = 2^-24; a value is read exactly.  A mean of n elements is a recurrence of at most
CHAIN = 64 steps per lane and 32 joins, each off by at most 4 u of the largest |x| (a difference,
a weight, a product, a sum): E_mu = 4 (CHAIN + 32) u max|x|.  M2 gains at most 8 roundings per step
relative to itself (its terms are squares), and what the mean's error adds: (E_mu / sigma)^2 in the
relative; the root and the quotient 4 u: E_r = r (4 (CHAIN + 32) u + (E_mu r)^2 + 4 u).
With d = x - mean:  |xhat error| <= r (E_mu + u |d|) + |d| E_r + u |xhat|,
u's: |gamma| that + u |gamma xhat| + u |u|.  An activation's slope is below 1.13 in size, its second
derivative below 1; its own evaluation costs 16 u (1 + |u|).  A bf16 result is rounded once: 2^-8 of itself.
The backward takes mean and rstd as given, so xhat is off by 3 u |xhat| only; sums over rows are chains
of CHAIN + 256 additions at most: (CHAIN + 256) u of the sum of the terms' sizes.
ReLU's slope is decided from u as the interface forms it: fp32 operations one after another, which
numpy's float32 gives bit by bit.
"""
import numpy as np
import pytest
import torch

from oracle import ops
from paper_2203_10428_amd import binding as B

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
CHAIN = 64
TINY = 2.0 ** -126
CODE = {"f32": B.PGCN_F32, "bf16": B.PGCN_BF16}
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
ACT = {"none": B.PGCN_ACT_NONE, "relu": B.PGCN_ACT_RELU, "silu": B.PGCN_ACT_SILU, "gelu": B.PGCN_ACT_GELU}


def matrix(x, dtype, pad=8):
    rows, cols = x.shape
    m = torch.full((rows, (cols + 7) // 8 * 8 + pad), float("nan"), dtype=DT[dtype], device="cuda")
    m[:, :cols] = torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).cuda().to(DT[dtype])
    return m


def host(t):
    return t.float().cpu().numpy().astype(np.float64)


def params(rng, f, affine=True):
    if not affine:
        return None, None, np.ones(f), np.zeros(f)
    g, b = (1 + 0.3 * rng.standard_normal(f)).astype(np.float32), (0.3 * rng.standard_normal(f)).astype(np.float32)
    return torch.from_numpy(g).cuda(), torch.from_numpy(b).cuda(), g.astype(np.float64), b.astype(np.float64)


def workspace(dtype, f, G, samples, rows):
    n = B.pgcn_group_norm_workspace_size(CODE[dtype], f, G, samples, rows)
    return torch.full((max(16, n),), 255, dtype=torch.uint8, device="cuda")


def forward(X, f, G, samples, R, ga, be, kind, dtype, eps=1e-5, stats=True, stream=None, Y=None, ws=None, out=None, pad=16):
    rows = samples * R
    if Y is None:
        Y = torch.full((rows + 1, (f + 7) // 8 * 8 + pad), 5.0, dtype=DT[dtype], device="cuda")
    mean, rstd = out or [torch.full((samples * G + 1,), 7.0, device="cuda") if stats else None for _ in range(2)]
    ws = workspace(dtype, f, G, samples, R) if ws is None else ws
    B.pgcn_group_norm_fwd(dtype=CODE[dtype], act=ACT[kind], channels=f, groups=G, samples=samples, sample_rows=R,
                          ld_x=X.stride(0), ld_y=Y.stride(0), eps=eps, X=X, gamma=ga, beta=be, Y=Y, mean=mean, rstd=rstd,
                          workspace=ws, workspace_bytes=ws.numel(), stream=stream)
    return Y, mean, rstd


def backward(X, J, f, G, samples, R, ga, be, mean, rstd, kind, dtype, stream=None, dX=None, out=None, ws=None, want=(1, 1, 1),
             pad=24):
    rows = samples * R
    if dX is None and want[0]:
        dX = torch.full((rows + 1, (f + 7) // 8 * 8 + pad), 5.0, dtype=DT[dtype], device="cuda")
    dg, db = out or [torch.full((f + 1,), 7.0, device="cuda") if w else None for w in want[1:]]
    ws = workspace(dtype, f, G, samples, R) if ws is None else ws
    B.pgcn_group_norm_bwd(dtype=CODE[dtype], act=ACT[kind], channels=f, groups=G, samples=samples, sample_rows=R,
                          ld_x=X.stride(0), ld_j_out=J.stride(0), ld_j_in=dX.stride(0) if dX is not None else 0, X=X, J_out=J,
                          gamma=ga, beta=be, mean=mean, rstd=rstd, J_in=dX, dgamma=dg, dbeta=db, workspace=ws,
                          workspace_bytes=ws.numel(), stream=stream)
    return dX, dg, db


def spread(v, samples, R, G, f):
    """[samples, G] values at every element of [rows, f]."""
    return np.repeat(np.repeat(v, R, axis=0), f // G, axis=1)


def check_forward(x, f, G, samples, R, kind, dtype, eps=1e-5, affine=True, seed=0):
    rng = np.random.default_rng(seed)
    X = matrix(x, dtype)
    x = host(X[:, :f])
    ga, be, g64, b64 = params(rng, f, affine)
    Y, mean, rstd = forward(X, f, G, samples, R, ga, be, kind, dtype, eps)
    torch.cuda.synchronize()
    rows = samples * R
    assert (Y[rows] == 5.0).all() and (Y[:, f:] == 5.0).all() and mean[-1] == 7.0 and rstd[-1] == 7.0
    ref, mu, rs = ops.group_norm_forward(x, g64, b64, samples, G, float(np.float32(eps)), kind)
    top = np.abs(x).reshape(samples, R, G, f // G).max(axis=(1, 3))
    e_mu = 4 * (CHAIN + 32) * U * top
    e_r = rs * (4 * (CHAIN + 32) * U + (e_mu * rs) ** 2 + 4 * U)
    assert (np.abs(host(mean[:-1]).reshape(mu.shape) - mu) <= e_mu).all()
    assert (np.abs(host(rstd[:-1]).reshape(mu.shape) - rs) <= e_r).all()
    S = lambda v: spread(v, samples, R, G, f)
    d = np.abs(x - S(mu))
    xhat = d * S(rs)
    e_x = S(rs) * (S(e_mu) + U * d) + (d + S(e_mu)) * S(e_r) + U * xhat
    u = (x - S(mu)) * S(rs) * g64 + b64
    e_u = np.abs(g64) * (e_x + U * xhat) + U * np.abs(u) + TINY
    bound = 1.13 * e_u + 16 * U * (1 + np.abs(u)) * (kind in ("silu", "gelu")) + U * np.abs(ref)
    if dtype == "bf16":
        bound = bound * (1 + 2.0 ** -8) + 2.0 ** -8 * np.abs(ref)
    err = np.abs(host(Y[:rows, :f]) - ref)
    assert (err <= bound).all(), (err - bound).max()
    return X, ga, be, mean, rstd, g64, b64


def check_backward(x, f, G, samples, R, kind, dtype, eps=1e-5, affine=True, seed=0):
    X, ga, be, mean, rstd, g64, b64 = check_forward(x, f, G, samples, R, kind, dtype, eps, affine, seed)
    rng = np.random.default_rng(seed + 1)
    rows = samples * R
    J = matrix(rng.standard_normal((rows, f)), dtype, pad=16)
    dX, dg, db = backward(X, J, f, G, samples, R, ga, be, mean, rstd, kind, dtype)
    torch.cuda.synchronize()
    assert (dX[rows] == 5.0).all() and (dX[:, f:] == 5.0).all() and dg[-1] == 7.0 and db[-1] == 7.0
    x, j = host(X[:, :f]), host(J[:, :f])
    mu, rs = host(mean[:-1]).reshape(samples, G), host(rstd[:-1]).reshape(samples, G)
    S = lambda v: spread(v, samples, R, G, f)
    u32 = ((x.astype(np.float32) - S(mu).astype(np.float32)) * S(rs).astype(np.float32)) * g64.astype(np.float32) + b64.astype(np.float32)
    slope = (u32 > 0).astype(np.float64) if kind == "relu" else None
    ref, rg, rb = ops.group_norm_backward(x, j, g64, b64, mu, rs, samples, G, kind, slope)
    xhat = (x - S(mu)) * S(rs)
    u = xhat * g64 + b64
    sl = ops.act_slope(u, kind) if slope is None else slope
    e_u = 4 * U * (np.abs(g64 * xhat) + np.abs(u)) + TINY
    e_s = (e_u + 16 * U * (1 + np.abs(u))) * (kind in ("silu", "gelu"))
    du = np.abs(j * sl)
    e_du = np.abs(j) * e_s + U * du
    chain = (CHAIN + 256) * U
    n = R * (f // G)
    grp = lambda v: v.reshape(samples, R, G, f // G).sum(axis=(1, 3))
    ax = np.abs(xhat)
    assert (np.abs(host(db[:-1]) - rb) <= (e_du + chain * du).sum(0) + TINY).all()
    assert (np.abs(host(dg[:-1]) - rg) <= (ax * (e_du + (chain + 4 * U) * du)).sum(0) + TINY).all()
    ag = np.abs(g64)
    e_c1 = grp(ag * (e_du + (chain + 4 * U) * du)) / n
    e_c2 = grp(ag * ax * (e_du + (chain + 8 * U) * du)) / n
    c1, c2 = grp(ag * du) / n, grp(ag * ax * du) / n
    bound = S(rs) * (ag * e_du + S(e_c1) + ax * S(e_c2) + 8 * U * (ag * du + S(c1) + ax * S(c2))) + TINY
    if dtype == "bf16":
        bound = bound * (1 + 2.0 ** -8) + 2.0 ** -8 * np.abs(ref)
    err = np.abs(host(dX[:rows, :f]) - ref)
    assert (err <= bound).all(), (err - bound).max()


# (samples, rows of a sample, channels, groups): every node by itself, whole samples, odd and ragged widths, groups that
# straddle vectors, one channel, widths past a workgroup's lanes
SHAPES = [(1, 1, 1, 1), (1, 1, 32, 4), (37, 1, 8, 2), (1000, 1, 256, 1), (513, 1, 256, 8), (70, 1, 602, 1), (33, 1, 602, 14), (65, 1, 41, 1),
          (50, 1, 300, 4), (9, 1, 300, 100), (21, 1, 512, 512), (5, 1, 2048, 1), (7, 1, 2052, 3), (3, 1, 8192, 32), (2, 1, 8191, 1),
          (2, 7, 16, 4), (3, 64, 320, 32), (5, 33, 60, 5), (1, 5000, 256, 8), (2, 1025, 7, 1), (40, 3, 130, 13), (1, 3001, 1, 1),
          (4, 256, 1000, 8), (600, 2, 24, 3), (2, 500, 2100, 7), (1, 40, 8192, 2), (17, 100, 4, 2), (2, 9, 8192, 8192),
          (1500, 5, 16, 2), (700, 2, 4, 4), (90, 3, 1, 1), (33, 128, 64, 4), (20, 32, 256, 1), (7, 30, 260, 4), (9, 8, 1000, 8),
          (3, 2, 4096, 64), (3, 8192, 1, 1), (2, 2049, 4, 2), (5, 129, 64, 4), (2500, 1, 16, 16), (1300, 1, 12, 3), (37, 1, 4100, 4), (1, 3000, 257, 257), (1, 2000, 24, 3),
          (3, 1, 8000, 5), (3, 1, 8192, 8192), (300, 1, 300, 4), (5, 1, 1200, 2), (5, 1, 2048, 4), (9, 1, 1024, 4), (3, 1, 6000, 1), (2, 1, 5000, 50),
          (70, 2, 100, 25), (3, 1, 4096, 4096), (3, 4, 2000, 8)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("i", range(len(SHAPES)), ids=[str(s) for s in SHAPES])
def test_group_norm(i, dtype):
    samples, R, f, G = SHAPES[i]
    rng = np.random.default_rng(i)
    x = 1.5 * rng.standard_normal((samples * R, f)) + 0.5
    for k in (i, i + 1) if samples * R * f < 200000 else (i,):
        check_backward(x, f, G, samples, R, ["none", "relu", "silu", "gelu"][k % 4], dtype, affine=(i + k) % 5 != 0, seed=i)


@pytest.mark.parametrize("samples,R,f,G", [(40, 1, 256, 8), (2, 300, 48, 4), (3, 20, 33, 3), (6, 1, 4096, 2)])
@pytest.mark.parametrize("kind", ["far_mean", "constant", "tiny", "one_large", "big"])
def test_group_norm_numerics(samples, R, f, G, kind):
    """A mean far from zero keeps the variance's digits; constants, tiny values; one value that outweighs all."""
    rng = np.random.default_rng(f)
    x = rng.standard_normal((samples * R, f))
    if kind == "far_mean":
        x = x + 4096.0
    elif kind == "constant":
        x[:] = 3.25
    elif kind == "tiny":
        x *= 2.0 ** -20
    elif kind == "one_large":
        x[0, :] = 1e4
        x[-1, 0] = -1e4
    else:
        x *= 2.0 ** 40
    check_backward(x, f, G, samples, R, "silu" if kind != "big" else "none", "f32", eps=1e-12 if kind == "tiny" else 1e-5, seed=3)


def test_nan_stays_in_its_group():
    rng = np.random.default_rng(2)
    for samples, R, f, G in ((30, 1, 256, 8), (3, 50, 64, 4), (2, 4, 90, 9)):
        x = rng.standard_normal((samples * R, f))
        x[0, 1] = np.nan
        for kind in ACT:
            X = matrix(x, "f32")
            Y = forward(X, f, G, samples, R, None, None, kind, "f32")[0]
            torch.cuda.synchronize()
            bad = torch.isnan(Y[:samples * R, :f]).cpu().numpy().reshape(samples, R, G, f // G)
            assert bad[0, :, 0].all() and bad.sum() == R * (f // G), kind


def test_optional_outputs_and_no_samples():
    rng = np.random.default_rng(1)
    samples, R, f, G = 3, 40, 64, 4
    X, J = matrix(rng.standard_normal((120, f)), "f32"), matrix(rng.standard_normal((120, f)), "f32")
    ga, be, _, _ = params(rng, f)
    Y, mean, rstd = forward(X, f, G, samples, R, ga, be, "silu", "f32")
    Y2, _, _ = forward(X, f, G, samples, R, ga, be, "silu", "f32", stats=False)
    dX, dg, db = backward(X, J, f, G, samples, R, ga, be, mean, rstd, "silu", "f32")
    torch.cuda.synchronize()
    assert torch.equal(Y, Y2)
    for want in ((1, 0, 0), (0, 1, 1), (0, 0, 1), (0, 1, 0), (1, 1, 0), (0, 0, 0)):
        a, b, c = backward(X, J, f, G, samples, R, ga, be, mean, rstd, "silu", "f32", want=want)
        torch.cuda.synchronize()
        assert (a is None or torch.equal(a, dX)) and (b is None or torch.equal(b, dg)) and (c is None or torch.equal(c, db))
    dg, db = torch.full((f,), 7.0, device="cuda"), torch.full((f,), 7.0, device="cuda")
    B.pgcn_group_norm_bwd(dtype=B.PGCN_F32, act=0, channels=f, groups=G, samples=0, sample_rows=R, ld_x=f, ld_j_out=f, ld_j_in=f,
                          X=None, J_out=None, gamma=None, beta=None, mean=None, rstd=None, J_in=None, dgamma=dg, dbeta=db)
    torch.cuda.synchronize()
    assert (dg == 0).all() and (db == 0).all()


@pytest.mark.parametrize("samples,R,f,G", [(3000, 1, 256, 8), (1, 4000, 256, 8), (20, 50, 60, 5)])
def test_reproducible_on_any_stream_and_in_a_graph(samples, R, f, G):
    rng = np.random.default_rng(9)
    rows = samples * R
    X, J = matrix(rng.standard_normal((rows, f)), "f32"), matrix(rng.standard_normal((rows, f)), "f32")
    ga, be, _, _ = params(rng, f)
    Y, mean, rstd = forward(X, f, G, samples, R, ga, be, "gelu", "f32")
    dX, dg, db = backward(X, J, f, G, samples, R, ga, be, mean, rstd, "gelu", "f32")
    torch.cuda.synchronize()
    outs = (Y, mean, rstd, dX, dg, db)
    want = [t.clone() for t in outs]
    ws = workspace("f32", f, G, samples, R)
    side = torch.cuda.Stream()

    def run(stream):
        forward(X, f, G, samples, R, ga, be, "gelu", "f32", stream=stream, Y=Y, ws=ws, out=(mean, rstd))
        backward(X, J, f, G, samples, R, ga, be, mean, rstd, "gelu", "f32", stream=stream, dX=dX, out=(dg, db), ws=ws)

    def same():
        torch.cuda.synchronize()
        for t, w, keep in zip(outs, want, (Y, mean, rstd, dX, dg, db)):
            assert torch.equal(t, w)
        Y[:rows, :f] = 1.0
        dX[:rows, :f] = 1.0
        for t in (mean, rstd, dg, db):
            t[:-1] = 1.0
        ws.fill_(255)
        torch.cuda.synchronize()

    run(side)
    same()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        run(torch.cuda.current_stream())
    for _ in range(3):
        g.replay()
        same()
        run(torch.cuda.current_stream())
        same()


def test_gradient_against_differences():
    """J_in, dgamma and dbeta against differences of sum(Y J), fp32, in steps far above the rounding."""
    rng = np.random.default_rng(12)
    samples, R, f, G = 1, 5, 12, 3
    x, j = rng.standard_normal((R, f)), rng.standard_normal((R, f))
    ga, be, g64, b64 = params(rng, f)
    X = matrix(x, "f32")
    Y, mean, rstd = forward(X, f, G, samples, R, ga, be, "silu", "f32")
    dX, dg, db = backward(X, matrix(j, "f32"), f, G, samples, R, ga, be, mean, rstd, "silu", "f32")

    def value(x_, g_, b_):
        y = forward(matrix(x_, "f32"), f, G, samples, R, torch.from_numpy(g_.astype(np.float32)).cuda(),
                    torch.from_numpy(b_.astype(np.float32)).cuda(), "silu", "f32")[0]
        torch.cuda.synchronize()
        return float((host(y[:R, :f]) * j).sum())

    h = 2.0 ** -6
    # 20 elements a group: chains of 5 steps and 8 joins, so the module notes' bound of Y is below 1e-5 here; the
    # difference divides two such errors by 2 h, and the third derivative (below 6 per unit of J) adds h^2
    tol = np.abs(j).sum() * (1e-5 / h + h * h)
    ref, rg, rb = ops.group_norm_backward(x.astype(np.float32).astype(np.float64), j, g64, b64, host(mean[:-1]).reshape(1, G),
                                          host(rstd[:-1]).reshape(1, G), 1, G, "silu")
    for a, b in ((0, 0), (2, 5), (4, 11)):
        e = np.zeros_like(x)
        e[a, b] = h
        d = (value(x + e, g64, b64) - value(x - e, g64, b64)) / (2 * h)
        assert abs(d - float(dX[a, b])) <= tol and abs(ref[a, b] - float(dX[a, b])) <= 1e-4
    for c in (0, 7):
        e = np.zeros(f)
        e[c] = h
        assert abs((value(x, g64 + e, b64) - value(x, g64 - e, b64)) / (2 * h) - float(dg[c])) <= tol
        assert abs((value(x, g64, b64 + e) - value(x, g64, b64 - e)) / (2 * h) - float(db[c])) <= tol
