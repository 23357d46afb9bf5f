"""The product of rows in 4 bits on the GPU, against ``oracle.mx`` (float64).

Bounds, u = 2^-24: a term a b is exact (4 bits times 4 bits times a power of two); a sum of k terms in fp32, in any
order, rounded or cut off at each of at most k + 64 steps, is off by at most 2 (k + 64) u sum |a b|.  A bf16 result is
rounded once more, by half a step: 2^-8 of itself."""
import numpy as np
import pytest
import torch

from mx_helpers import U, host, matmul, quantize, matrix, upload
from oracle import mx
from paper_2203_10428_amd import binding as B

pytestmark = pytest.mark.gpu


def rows_of(rng, rows, k, spread=1.0):
    return mx.quantize(rng.standard_normal((rows, k)) * np.exp(spread * rng.standard_normal((rows, 1))), "fp4")


def check(C, a, b, m, n, k, dtype, relu):
    torch.cuda.synchronize()
    va, vb = mx.values(*a, k, "fp4"), mx.values(*b, k, "fp4")
    want, size = mx.product(va, vb, relu), np.abs(va) @ np.abs(vb).T
    tol = 2 * (k + 64) * U * size + (2.0 ** -8 * np.abs(want) if dtype == "bf16" else 0) * (1 + 2.0 ** -7) + 2.0 ** -120
    assert (np.abs(host(C[:m], n) - want) <= tol).all()
    assert (C[:m, n:] == 77).all() and (C[m:] == 77).all()


SHAPES = [(1, 1, 1), (1, 8, 32), (1, 100, 4096), (1, 1000, 33), (2, 17, 64), (3, 513, 1000), (8, 64, 129), (15, 16, 17), (16, 16, 128),
          (17, 31, 127), (33, 1000, 160), (64, 64, 512), (65, 130, 515), (100, 41, 602), (129, 257, 96), (255, 256, 257), (256, 512, 1024),
          (300, 300, 300), (700, 47, 100), (257, 8, 2000), (2000, 1, 70), (5, 3000, 256), (513, 769, 1030)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m,n,k", SHAPES)
def test_product(m, n, k, dtype):
    rng = np.random.default_rng(m + n + k)
    a, b = rows_of(rng, m, k), rows_of(rng, n, k)
    A, SA = upload(*a, "fp4", (16, 4))
    Bq, SB = upload(*b, "fp4", (0, 0))
    relu = (m + n) % 2 == 0
    check(matmul(A, SA, Bq, SB, m, n, k, dtype, relu), a, b, m, n, k, dtype, relu)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m,n,k", [(2050, 2100, 290), (4100, 4000, 70), (4090, 4200, 300)])
def test_many_tiles(m, n, k, dtype):
    """Enough rows and columns for the larger tiles, with ragged edges; an even and an odd number of slabs, part of one."""
    test_product(m, n, k, dtype)


@pytest.mark.parametrize("k", [32, 256, 257, 500, 512, 600, 768, 1000, 1024, 1030, 1280, 1500, 1800, 2048, 2100, 2400])
@pytest.mark.parametrize("m,n", [(70, 3), (1, 90), (16, 16)])
def test_every_number_of_slabs(m, n, k):
    """One slab to more than all stages hold, with whole and part last ones; groups for one wave to more than all."""
    test_product(m, n, k, "f32")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m,n,k", [(1, 40, 20000), (1, 1, 70000), (9, 130, 9001), (16, 33, 16384), (100, 90, 9000), (17, 5, 40000), (129, 200, 4100),
                                   (64, 64, 2048)])
def test_long_rows_in_parts(m, n, k, dtype):
    """Blocks split among workgroups, the last part shorter; one part fewer than asked for."""
    assert B.pgcn_mx_matmul_workspace_size(B.PGCN_F32, m, n, k) >= 2 * 4 * m * n
    test_product(m, n, k, dtype)


@pytest.mark.parametrize("m,n,k", [(4100, 4000, 600), (4090, 4200, 1100), (2050, 2100, 600), (2049, 2176, 1200), (16400, 4100, 40)])
def test_many_tiles_of_more_slabs(m, n, k):
    test_product(m, n, k, "bf16")


@pytest.mark.parametrize("m", [1, 20, 300])
def test_scales_far_apart(m):
    rng = np.random.default_rng(m)
    e = rng.integers(-90, 90, (1, 10))
    both = [mx.quantize(np.ldexp(rng.standard_normal((r, 320)), np.repeat(sign * e, 32, axis=1)), "fp4") for r, sign in ((m, 1), (70, -1))]
    C = matmul(*upload(*both[0], "fp4"), *upload(*both[1], "fp4"), m, 70, 320, "f32")
    check(C, *both, m, 70, 320, "f32", False)


@pytest.mark.parametrize("m,n,k", [(1, 40, 300), (70, 300, 300), (300, 40, 70)])
def test_nan_blocks_show_in_their_rows_alone(m, n, k):
    rng = np.random.default_rng(2)
    a, b = rows_of(rng, m, k), rows_of(rng, n, k)
    a[1][m - 1, 1], b[1][n - 2, 0] = 255, 255
    for relu in (False, True):
        C = matmul(*upload(*a, "fp4"), *upload(*b, "fp4"), m, n, k, "f32", relu)
        torch.cuda.synchronize()
        bad = np.zeros((m, n), bool)
        bad[m - 1], bad[:, n - 2] = True, True
        got = host(C[:m], n)
        assert np.isnan(got[bad]).all() and np.isfinite(got[~bad]).all()


def test_zero_rows():
    a, b = mx.quantize(np.zeros((5, 100)), "fp4"), rows_of(np.random.default_rng(3), 6, 100)
    C = matmul(*upload(*a, "fp4"), *upload(*b, "fp4"), 5, 6, 100, "bf16")
    torch.cuda.synchronize()
    assert (C[:5, :6] == 0).all()


@pytest.mark.parametrize("m,n,k", [(1, 600, 2000), (40, 300, 515), (600, 520, 700), (2, 90, 20000), (100, 90, 9000), (2100, 2060, 1100)])
def test_the_same_bits_every_time_and_from_a_graph(m, n, k):
    """Quantised activations times held weights, on another stream, replayed with eager calls between."""
    rng = np.random.default_rng(4)
    X, side = matrix(rng.standard_normal((m, k))), torch.cuda.Stream()
    Bq, SB = upload(*rows_of(rng, n, k), "fp4")
    held = quantize(X, k, "fp4")
    want = matmul(*held, Bq, SB, m, n, k, "f32")
    torch.cuda.synchronize()
    out, ws = torch.full_like(want, 77.0), torch.full((1 << 24,), 255, dtype=torch.uint8, device="cuda")
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        quantize(X, k, "fp4", out=held, stream=torch.cuda.current_stream())
        matmul(*held, Bq, SB, m, n, k, "f32", out=out, ws=ws, stream=torch.cuda.current_stream())
    for _ in range(3):
        out.fill_(77.0)
        ws.fill_(255)
        held[0].fill_(255)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
        again = matmul(*held, Bq, SB, m, n, k, "f32", stream=side)
        torch.cuda.synchronize()
        assert torch.equal(again, want)
