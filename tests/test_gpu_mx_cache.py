"""Rows quantised as they are written and read back on the GPU, against ``oracle.mx``.

Scales and elements have to be those of the oracle, byte for byte, and so have the values read back in fp32; they
are exact in bf16 too.  The moving average g out + (1 - g) v is formed from fp32 g and 1 - g (rounded once), one
product and one product-sum: off by at most 2 u |(1 - g) v| + u |result|, u = 2^-24, and 2^-149 where it is subnormal."""
import numpy as np
import pytest
import torch

from mx_helpers import FMT, U, check_held, dequantize, held, host, matrix, quantize, upload
from oracle import mx
from paper_2203_10428_amd import binding as B

pytestmark = pytest.mark.gpu
FMTS = ["int8", "fp4"]


def rows_of(rng, rows, cols, dtype="f32"):
    """Rows of different sizes, half of the elements 0, one row of zeros; values that the type has."""
    x = np.maximum(rng.standard_normal((rows, cols)), 0) * np.exp(2 * rng.standard_normal((rows, 1)))
    x *= np.sign(rng.standard_normal((rows, cols)))
    if rows > 2:
        x[1] = 0.0
    return torch.from_numpy(x).to(torch.bfloat16 if dtype == "bf16" else torch.float32).double().numpy()


COLS = [1, 7, 8, 9, 31, 32, 33, 63, 64, 65, 100, 256, 602, 2049]


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("cols", COLS)
def test_write_and_read(fmt, dtype, cols):
    rng = np.random.default_rng(cols)
    for rows in (1, 3, 131):
        x = rows_of(rng, rows, cols, dtype)
        Q, S = quantize(matrix(x, dtype), cols, fmt, dtype)
        code, s = check_held(Q, S, x, fmt)
        for out in ("f32", "bf16"):
            y = dequantize(Q, S, rows, cols, fmt, out)
            torch.cuda.synchronize()
            assert np.array_equal(host(y[:rows], cols), mx.values(code, s, cols, fmt))
            assert (y[:rows, cols:] == 77).all() and (y[rows:] == 77).all()


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", [(1, 1), (31, 5), (32, 64), (33, 257), (100, 300), (1000, 17), (65, 1025), (255, 33), (257, 129),
                                       (600, 258)])
def test_write_transposed(fmt, dtype, rows, cols):
    x = rows_of(np.random.default_rng(rows), rows, cols, dtype)
    Q, S = quantize(matrix(x, dtype), cols, fmt, dtype, transpose=True)
    check_held(Q, S, np.ascontiguousarray(x.T), fmt)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("cols", [5, 64, 602])
def test_write_gathered(fmt, cols):
    """Repeated, missing (negative) and impossible rows; more rows than the source has, and none."""
    rng = np.random.default_rng(cols)
    x = rows_of(rng, 40, cols)
    index = np.concatenate((rng.integers(0, 40, 90), [-1, 39, 0, 0, 40, 2 ** 31 - 1, -2 ** 31, 39]))
    Q, S = quantize(matrix(x), cols, fmt, index=index)
    check_held(Q, S, mx.gather(x, index), fmt)
    Q, S = held(3, cols, fmt)
    B.pgcn_mx_quantize(format=FMT[fmt], dtype=B.PGCN_F32, rows=3, cols=cols, src_rows=0, ld_x=(cols + 3) // 4 * 4, ld_q=Q.stride(0),
                       ld_s=S.stride(0), X=None, index=torch.tensor([-1, 0, -5], dtype=torch.int32, device="cuda"), Q=Q, S=S)
    check_held(Q, S, np.stack([np.zeros(cols), np.full(cols, np.nan), np.zeros(cols)]), fmt)


def test_source_views():
    """A view into a wider matrix, whose last row ends with the columns; fewer rows than the source has."""
    rng = np.random.default_rng(4)
    x = rows_of(rng, 21, 36)
    flat = torch.zeros(21 * 64, device="cuda")
    wide = flat.as_strided((21, 36), (64, 1), 20)                      # ends 8 floats before its buffer does
    wide.copy_(torch.from_numpy(x.astype(np.float32)).cuda())
    for fmt in FMTS:
        Q, S = quantize(wide, 36, fmt, rows=13)
        check_held(Q, S, x[:13], fmt)
        Q, S = quantize(wide, 36, fmt, transpose=True)
        check_held(Q, S, np.ascontiguousarray(x.T), fmt)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("transpose", [False, True])
def test_scales_over_the_whole_range(fmt, transpose):
    """Largest magnitudes at every exponent and around every border of a scale, ties among the others."""
    rng = np.random.default_rng(5)
    tops = np.float32([1.0, 1.5, 1.75, 1.9921875, 127.5 / 64, 1.25]).view(np.uint32) & 0x7FFFFF
    near = (tops.astype(np.int64)[:, None] + [-1, 0, 1]) % (1 << 23)
    bits = ((np.arange(256)[:, None, None] << 23) + near[None]).astype(np.uint32)
    top = np.unique(np.concatenate((bits.reshape(-1), np.uint32([0, 1, 2, 0x7F7FFF, 0x7F8000, 0x7FFFFF, 0x7F7FFFFF, 0x7F800000]))))
    x = np.zeros((len(top), 32))
    with np.errstate(over="ignore", invalid="ignore"):
        t = top.view(np.float32).astype(np.float64)
        x[:, 0] = t * rng.choice([-1, 1], len(t))
        grid = np.where(rng.random((len(t), 31)) < 0.7, rng.integers(-256, 257, (len(t), 31)) / 256.0, rng.uniform(-1, 1, (len(t), 31)))
        x[:, 1:] = np.where(np.isfinite(t), 2.0 ** np.floor(np.log2(np.maximum(t, 2.0 ** -149))), 1.0)[:, None] * grid
        x = x.astype(np.float32).astype(np.float64)
    x[3::7, 5] = -0.0
    if transpose:
        Q, S = quantize(matrix(np.ascontiguousarray(x.T)), len(x), fmt, transpose=True)
    else:
        Q, S = quantize(matrix(x), 32, fmt)
    check_held(Q, S, x, fmt)


@pytest.mark.parametrize("fmt", FMTS)
def test_what_is_not_finite(fmt):
    x = rows_of(np.random.default_rng(6), 9, 100)
    x[0, 5], x[2, 99], x[3, 31], x[4, 32], x[5] = np.nan, np.inf, -np.inf, np.nan, np.inf
    for dtype in ("f32", "bf16"):
        v = torch.from_numpy(x).to(torch.bfloat16).double().numpy() if dtype == "bf16" else x.astype(np.float32).astype(np.float64)
        Q, S = quantize(matrix(v, dtype), 100, fmt, dtype)
        code, s = check_held(Q, S, v, fmt)
        y = dequantize(Q, S, 9, 100, fmt)
        torch.cuda.synchronize()
        assert np.array_equal(host(y[:9], 100), mx.values(code, s, 100, fmt), equal_nan=True)
        Q, S = quantize(matrix(np.ascontiguousarray(v.T), dtype), 9, fmt, dtype, transpose=True)
        check_held(Q, S, v, fmt)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("out", ["f32", "bf16"])
def test_read_every_byte_at_every_scale(fmt, out):
    """Also those that no block is written with: q = -128, scales past the largest."""
    per = 32 if fmt == "int8" else 16
    b = np.tile(np.arange(256, dtype=np.uint8), 256).reshape(-1, per)
    s = np.repeat(np.arange(256), 256 // per)
    code = mx.from_bytes(b, fmt)
    Q, S = upload(code, s[:, None], fmt)
    y = dequantize(Q, S, len(code), 32, fmt, out)
    torch.cuda.synchronize()
    with np.errstate(over="ignore"):
        want = mx.values(code, s[:, None], 32, fmt).astype(np.float32).astype(np.float64)
    assert np.array_equal(host(y[:-1], 32), want, equal_nan=True)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("rows,cols", [(1, 1), (5, 33), (300, 100), (64, 512)])
def test_moving_average(fmt, rows, cols):
    rng = np.random.default_rng(cols)
    x, state = rows_of(rng, rows, cols), rng.standard_normal((rows, cols))
    Q, S = quantize(matrix(x), cols, fmt)
    v = mx.values(*mx.quantize(x, fmt), cols, fmt)
    for gamma in (0.95, 0.3, 1.0, 1e-30):
        out = matrix(state, fill=77.0)
        before = host(out, cols)
        g = float(np.float32(gamma))
        dequantize(Q, S, rows, cols, fmt, gamma=gamma, out=out)
        torch.cuda.synchronize()
        want = mx.average(before, v, g)
        tol = 2 * U * np.abs((1 - g) * v) + U * np.abs(want) + 2.0 ** -149
        assert (np.abs(host(out, cols) - want) <= tol).all()
        assert (out[:, cols:] == 77).all()


def test_gamma_zero_does_not_read_what_was_there():
    x = rows_of(np.random.default_rng(8), 4, 40)
    Q, S = quantize(matrix(x), 40, "int8")
    out = torch.full((4, 40), float("nan"), device="cuda")
    dequantize(Q, S, 4, 40, "int8", out=out)
    torch.cuda.synchronize()
    assert torch.isfinite(out).all()


def test_streams_and_graphs():
    """On another stream than the current one, and replayed from a graph with eager calls between the replays."""
    rng = np.random.default_rng(9)
    x, index = rows_of(rng, 50, 70), torch.randint(-1, 50, (80,), dtype=torch.int32, device="cuda")
    X, state = matrix(x), torch.randn(80, 72, device="cuda")
    Q, S = held(80, 70, "int8")
    out = torch.empty_like(state)
    side = torch.cuda.Stream()

    def run(stream):
        B.pgcn_mx_quantize(format=B.PGCN_MX_INT8, dtype=B.PGCN_F32, rows=80, cols=70, src_rows=50, ld_x=X.stride(0), ld_q=Q.stride(0),
                           ld_s=S.stride(0), X=X, index=index, Q=Q, S=S, stream=stream)
        B.pgcn_mx_dequantize(format=B.PGCN_MX_INT8, dtype=B.PGCN_F32, rows=80, cols=70, ld_q=Q.stride(0), ld_s=S.stride(0), ld_out=72,
                             gamma=0.75, Q=Q, S=S, out=out, stream=stream)

    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        run(torch.cuda.current_stream())
    for k in range(4):
        xk = x * (k + 1)
        X[:, :70] = torch.from_numpy(xk.astype(np.float32)).cuda()
        out.copy_(state)
        torch.cuda.synchronize()
        run(side)
        torch.cuda.synchronize()
        want, q = out.clone(), Q.clone()
        check_held(Q, S, mx.gather(host(X, 70), index.cpu().numpy()), "int8")
        out.copy_(state)
        Q.fill_(0xA5)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(Q, q)


def test_more_rows_than_a_launch_counts_in_32_bits():
    """2^30 + 70 rows of one element, four threads each; what lies past 2^32 threads, and 2^34 bytes into Q."""
    rows, n = (1 << 30) + 70, 5
    x = np.float64([[1.0], [-3.0], [0.25], [0.0], [6.0]])
    X = matrix(x, pad=0)
    index = torch.zeros(rows, dtype=torch.int32, device="cuda")
    index[-140:] = torch.arange(140, device="cuda").remainder(n).to(torch.int32)
    Q, S = torch.empty(rows, 16, dtype=torch.uint8, device="cuda"), torch.empty(rows, 4, dtype=torch.uint8, device="cuda")
    Q[-140:], S[-140:] = 0xA5, 0xA5
    B.pgcn_mx_quantize(format=B.PGCN_MX_FP4, dtype=B.PGCN_F32, rows=rows, cols=1, src_rows=n, ld_x=X.stride(0), ld_q=16, ld_s=4, X=X,
                       index=index, Q=Q, S=S)
    torch.cuda.synchronize()
    code, s = mx.quantize(x, "fp4")
    at = np.arange(140) % n
    assert np.array_equal(Q[-140:].cpu().numpy(), mx.to_bytes(code, "fp4")[at]) and np.array_equal(S[-140:, :1].cpu().numpy(), s[at])
    del index
    out = torch.full((rows, 4), 77.0, device="cuda")
    dequantize(Q, S, rows, 1, "fp4", out=out)
    torch.cuda.synchronize()
    assert np.array_equal(out[-140:, 0].cpu().numpy(), x[at, 0]) and (out[:, 1:][-140:] == 77).all()


def test_reading_more_chunks_than_a_launch_counts_in_32_bits():
    """Three chunks a row: 2^32 and some threads in all."""
    rows = ((1 << 32) // 3) + 50
    Q, S = torch.zeros(rows, 16, dtype=torch.uint8, device="cuda"), torch.full((rows, 4), 127, dtype=torch.uint8, device="cuda")
    code = np.random.default_rng(3).integers(0, 16, (120, 32))
    Q[-120:] = torch.from_numpy(mx.to_bytes(code, "fp4")).cuda()
    out = torch.empty(rows, 24, dtype=torch.bfloat16, device="cuda")
    out[-120:] = 77.0
    dequantize(Q, S, rows, 20, "fp4", "bf16", out=out)
    torch.cuda.synchronize()
    assert np.array_equal(host(out[-120:], 20), mx.values(code, np.full((120, 1), 127), 20, "fp4"))
    assert (out[-120:, 20:] == 77).all()
