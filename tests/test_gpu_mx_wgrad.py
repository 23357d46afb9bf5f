"""The weight gradient from rows in 8 bits on the GPU, against ``oracle.mx`` (float64).

Bounds, u = 2^-24: a product of the fp32 arithmetic is exact in its three parts but for what the split's last part
rounds away (below 2^-24 of J), and every addition of a chain of at most rows + 128 rounds once or is cut off (2 u of the
running sum, which the sum of absolute terms bounds).  So |error| <= (2 rows + 260) u sum |v J|.  bf16: J o mask is
first rounded to nearest (the oracle does so too), then the same."""
import numpy as np
import pytest
import torch

from mx_helpers import U, host, matrix, upload, wgrad
from oracle import mx

pytestmark = pytest.mark.gpu


def inputs(seed, rows, f_in, f_out, masked):
    rng = np.random.default_rng(seed)
    x = np.maximum(rng.standard_normal((rows, f_in)), 0) * np.exp(rng.standard_normal((rows, 1)))
    code, s = mx.quantize(x, "int8")
    J = (1e-3 * rng.standard_normal((rows, f_out))).astype(np.float32).astype(np.float64)
    H = np.maximum(rng.standard_normal((rows, f_out)), 0) if masked else None
    return code, s, J, H


def check(dW, code, s, J, H, f_in, f_out, dtype):
    torch.cuda.synchronize()
    v = mx.values(code, s, f_in, "int8")
    if H is not None:
        J = np.where(H > 0, J, 0.0)
    if dtype == "bf16":
        J = torch.from_numpy(J).float().to(torch.bfloat16).double().numpy()
    want, size = mx.wgrad(v, J), np.abs(v).T @ np.abs(J)
    got = dW[:f_in * f_out].view(f_in, f_out).cpu().numpy().astype(np.float64)
    assert (np.abs(got - want) <= (2 * len(J) + 260) * U * size + 2.0 ** -126).all()
    assert (dW[f_in * f_out:] == 77).all()


SHAPES = [(1, 1, 1), (1, 33, 7), (2, 64, 64), (15, 5, 100), (16, 32, 16), (17, 129, 65), (33, 96, 128), (100, 602, 41), (257, 256, 256),
          (1000, 32, 16), (1500, 100, 130), (4099, 300, 47), (3000, 513, 260), (700, 1025, 8), (64, 40, 1500), (20000, 128, 128),
          (2000, 300, 130), (999, 540, 200), (50, 384, 100), (35, 257, 65)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("masked", [True, False])
@pytest.mark.parametrize("rows,f_in,f_out", SHAPES)
def test_weight_gradient(rows, f_in, f_out, masked, dtype):
    code, s, J, H = inputs(rows + f_out, rows, f_in, f_out, masked)
    Q, S = upload(code, s, "int8")
    dW = wgrad(Q, S, matrix(J), None if H is None else matrix(H, pad=16), rows, f_in, f_out, dtype)
    check(dW, code, s, J, H, f_in, f_out, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_no_rows(dtype):
    Q, S = torch.zeros(1, 64, dtype=torch.uint8, device="cuda"), torch.zeros(1, 4, dtype=torch.uint8, device="cuda")
    dW = wgrad(Q, S, torch.zeros(1, 8, device="cuda"), None, 0, 40, 7, dtype)
    torch.cuda.synchronize()
    assert (dW[:280] == 0).all() and (dW[280:] == 77).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_masks_that_leave_nothing_and_what_they_hide(dtype):
    """Rows without any unmasked place; NaN and infinities in masked places; a mask of negative and zero values."""
    code, s, J, H = inputs(3, 300, 70, 40, True)
    H[10:200] = 0.0
    H[:, 3] = -1.0
    J[H <= 0] = np.resize([np.nan, np.inf, -np.inf], int((H <= 0).sum()))
    Q, S = upload(code, s, "int8")
    check(wgrad(Q, S, matrix(J), matrix(H), 300, 70, 40, dtype), code, s, np.where(H > 0, J, 0.0), None, 70, 40, dtype)
    dW = wgrad(Q, S, matrix(J), matrix(np.zeros_like(H)), 300, 70, 40, dtype)
    torch.cuda.synchronize()
    assert (dW[:2800] == 0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_nan_blocks_and_gradients_show_where_they_count(dtype):
    code, s, J, _ = inputs(4, 130, 70, 40, False)
    s[100, 1] = 255                                        # features 32 .. 63 of a row
    J[7, 5] = np.nan
    Q, S = upload(code, s, "int8")
    dW = wgrad(Q, S, matrix(J), None, 130, 70, 40, dtype)
    torch.cuda.synchronize()
    got = dW[:2800].view(70, 40).cpu().numpy()
    bad = np.zeros((70, 40), bool)
    bad[32:64], bad[:, 5] = True, True
    assert np.isnan(got[bad]).all() and np.isfinite(got[~bad]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_scales_far_apart(dtype):
    """Rows whose scales span the range of floats, paired with gradients that bring them back."""
    rng = np.random.default_rng(5)
    e = rng.integers(-100, 100, (64, 1))
    code, s = mx.quantize(np.ldexp(rng.standard_normal((64, 40)), e), "int8")
    J = np.ldexp(rng.standard_normal((64, 24)), -e).astype(np.float32).astype(np.float64)
    Q, S = upload(code, s, "int8")
    check(wgrad(Q, S, matrix(J), None, 64, 40, 24, dtype), code, s, J, None, 40, 24, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("scale", [0, 1, 6, 133, 253, 254])
def test_every_element_at_the_ends_of_the_scales(dtype, scale):
    """Elements -128 .. 127 with the smallest and largest scales; J brings the products to where floats are."""
    rows, f_in, f_out = 40, 256, 8
    code = np.tile(np.arange(-128, 128), (rows, 1))
    if scale == 254:
        code = np.maximum(code, -127)                      # -128 with the largest scale is no float
    s = np.full((rows, 8), scale)
    J = np.zeros((rows, f_out))
    J[np.arange(rows), np.arange(rows) % f_out] = np.ldexp(1.0 + np.arange(rows) / 64.0, -60 if scale > 133 else 60)
    Q, S = upload(code, s, "int8")
    dW = wgrad(Q, S, matrix(J), None, rows, f_in, f_out, dtype)
    if scale >= 6:                                         # below, values are less than 2^-126
        check(dW, code, s, J, None, f_in, f_out, dtype)
    torch.cuda.synchronize()
    assert torch.isfinite(dW).all()


def test_the_same_bits_every_time_and_from_a_graph():
    code, s, J, H = inputs(6, 5000, 100, 72, True)
    Q, S = upload(code, s, "int8")
    Jd, Hd, side = matrix(J), matrix(H), torch.cuda.Stream()
    for dtype in ("f32", "bf16"):
        want = wgrad(Q, S, Jd, Hd, 5000, 100, 72, dtype)
        torch.cuda.synchronize()
        out = torch.full_like(want, 77.0)
        ws = torch.full((1 << 24,), 255, dtype=torch.uint8, device="cuda")
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            wgrad(Q, S, Jd, Hd, 5000, 100, 72, dtype, out=out, ws=ws, stream=torch.cuda.current_stream())
        for k in range(3):
            out.fill_(77.0)
            ws.fill_(255)
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, want)
            again = wgrad(Q, S, Jd, Hd, 5000, 100, 72, dtype, stream=side)
            torch.cuda.synchronize()
            assert torch.equal(again, want)


def test_against_differences():
    """dW of a loss sum (v W) J that is linear in W: a difference over one weight is the sum that the gradient names."""
    code, s, J, _ = inputs(7, 50, 33, 9, False)
    Q, S = upload(code, s, "int8")
    dW = wgrad(Q, S, matrix(J), None, 50, 33, 9, "f32")
    v = mx.values(code, s, 33, "int8")
    torch.cuda.synchronize()
    W = np.random.default_rng(1).standard_normal((33, 9))
    for at in ((0, 0), (32, 8), (17, 4)):
        e = np.zeros_like(W)
        e[at] = 0.5
        d = ((v @ (W + e)) * J).sum() - ((v @ (W - e)) * J).sum()
        assert abs(d - float(dW[at[0] * 9 + at[1]])) <= 360 * U * np.abs(v[:, at[0]] * J[:, at[1]]).sum() + 1e-12
    assert host(matrix(J), 9).shape == J.shape
