"""Group norm of matrices whose element offsets pass 2^31, and two calls at once.

Bounds are those of ``test_gpu_group_norm`` with the chains of these sizes: a thread adds up STEPS values or joins STEPS batches
(rows / (workgroups x row slots), and four rows to a batch where a sample goes in chunks)."""
import numpy as np
import pytest
import torch

from test_gpu_group_norm import TINY, U, backward, forward, matrix, params, workspace

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("samples,R,G,steps", [(300_000_001, 1, 1, 300_000_001 // (1024 * 64) + 1),
                                               (1, 300_000_001, 2, 300_000_001 // (512 * 128) + 1)], ids=["rows", "one_sample"])
def test_offsets_past_32_bits(samples, R, G, steps):
    f, rows = 8, samples * R
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("needs 60 GiB of device memory")
    gen = torch.Generator(device="cuda").manual_seed(3)
    X = torch.randn(rows, f, generator=gen, device="cuda").mul_(1.5).add_(0.25)
    J = torch.randn(rows, f, generator=gen, device="cuda")
    rng = np.random.default_rng(3)
    ga, be, g64, b64 = params(rng, f)
    Y = torch.full((rows + 1, f), 5.0, device="cuda")
    Y, mean, rstd = forward(X, f, G, samples, R, ga, be, "silu", "f32", Y=Y)
    dX = torch.full((rows + 1, f), 5.0, device="cuda")
    dX, dg, db = backward(X, J, f, G, samples, R, ga, be, mean, rstd, "silu", "f32", dX=dX)
    torch.cuda.synchronize()
    assert (Y[rows] == 5.0).all() and (dX[rows] == 5.0).all()
    g, b = torch.from_numpy(g64).cuda(), torch.from_numpy(b64).cuda()
    per = f // G
    wide = lambda v: v.double().reshape(-1, G).repeat_interleave(per, 1)

    def sums(step=30_000_000):
        """Over all rows: of du, du xhat and their sizes, for every channel."""
        out = torch.zeros(4, f, dtype=torch.float64, device="cuda")
        for r0 in range(0, rows, step):
            s = slice(r0, min(rows, r0 + step))
            xh = (X[s].double() - (wide(mean[:-1][s]) if R == 1 else wide(mean[:G]))) * (wide(rstd[:-1][s]) if R == 1 else wide(rstd[:G]))
            sg = torch.sigmoid(xh * g + b)
            du = J[s] * sg * (1 + (xh * g + b) * (1 - sg))
            for k, v in enumerate((du, du * xh, du.abs(), (du * xh).abs())):
                out[k] += v.sum(0)
        return out

    total = sums()
    chain = (steps + 256 + 32) * U                        # and 16 u of each term's slope, a few of its factors
    assert ((db[:-1] - total[0]).abs() <= (chain + 64 * U) * total[2]).all()
    assert ((dg[:-1] - total[1]).abs() <= (chain + 64 * U) * total[3]).all()
    if R > 1:
        x64 = torch.zeros(f, dtype=torch.float64, device="cuda")
        for r0 in range(0, rows, 30_000_000):
            x64 += X[r0:r0 + 30_000_000].double().sum(0)
        mu = x64.reshape(G, per).sum(1) / (rows * per)
        m2 = torch.zeros(f, dtype=torch.float64, device="cuda")
        for r0 in range(0, rows, 30_000_000):
            m2 += (X[r0:r0 + 30_000_000].double() - mu.repeat_interleave(per)).square().sum(0)
        rs = ((m2.reshape(G, per).sum(1) / (rows * per)) + 1e-5).rsqrt()
        e_mu = 4 * (steps / 4 + 32) * U * 12.0            # |x| < 12
        assert ((mean[:G] - mu).abs() <= e_mu).all() and ((rstd[:G] - rs).abs() <= rs * (4 * (steps / 4 + 32) * U + (e_mu * rs) ** 2 + 4 * U)).all()
        c1, c2 = ((t * g).reshape(G, per).sum(1) / (rows * per) for t in (total[0], total[1]))
    border = 2 ** 31 // f
    for r0 in (0, border - 500, rows - 1000):
        s = slice(r0, r0 + 1000)
        x, j = X[s].double(), J[s].double()
        m, r = (wide(mean[:-1][s]), wide(rstd[:-1][s])) if R == 1 else (wide(mean[:G]), wide(rstd[:G]))
        if R == 1:
            mu = x.mean(1, keepdim=True)
            assert ((m[:, :1] - mu).abs() <= 64 * U * 12).all()
        xh = (x - m) * r
        u = xh * g + b
        sg = torch.sigmoid(u)
        bound = 1.13 * (8 * U * ((xh * g).abs() + u.abs())) + 16 * U * (1 + u.abs()) + TINY
        assert ((Y[s] - u * sg).abs() <= bound + U * (u * sg).abs()).all()
        du = j * sg * (1 + u * (1 - sg))
        dx = du * g
        if R == 1:
            p1, p2 = dx.mean(1, keepdim=True), (dx * xh).mean(1, keepdim=True)
        else:
            p1, p2 = c1.repeat_interleave(per), c2.repeat_interleave(per)
        ref = r * (dx - p1 - xh * p2)
        e = 64 * U * (1 + u.abs()) * j.abs() * g.abs()
        tol = r * (e + (e.mean(1, keepdim=True) + chain) * (1 + xh.abs()) * 2 + 16 * U * (dx.abs() + xh.abs()))
        assert ((dX[s] - ref).abs() <= tol + TINY).all()
    del X, Y, J, dX
    torch.cuda.empty_cache()


@pytest.mark.parametrize("samples,R,f,G", [(3000, 1, 256, 1), (3000, 1, 300, 4), (1, 4000, 256, 8)])
def test_two_calls_at_once(samples, R, f, G):
    """Two streams, a workspace each."""
    rng = np.random.default_rng(5)
    rows, sets = samples * R, []
    for _ in range(2):
        X, J = matrix(rng.standard_normal((rows, f)), "f32"), matrix(rng.standard_normal((rows, f)), "f32")
        ga, be, _, _ = params(rng, f)
        Y, mean, rstd = forward(X, f, G, samples, R, ga, be, "gelu", "f32")
        dX, dg, db = backward(X, J, f, G, samples, R, ga, be, mean, rstd, "gelu", "f32")
        torch.cuda.synchronize()
        outs = (Y, mean, rstd, dX, dg, db)
        sets.append((X, J, ga, be, outs, [t.clone() for t in outs], workspace("f32", f, G, samples, R), torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(4):
        for X, J, ga, be, (Y, mean, rstd, dX, dg, db), _, ws, st in sets:
            forward(X, f, G, samples, R, ga, be, "gelu", "f32", stream=st, Y=Y, ws=ws, out=(mean, rstd))
            backward(X, J, f, G, samples, R, ga, be, mean, rstd, "gelu", "f32", stream=st, dX=dX, out=(dg, db), ws=ws)
    torch.cuda.synchronize()
    for *_, outs, want, ws, st in sets:
        assert all(torch.equal(a, b) for a, b in zip(outs, want))
