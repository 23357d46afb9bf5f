"""Layers with operands in 8 and 4 bits through the C ABI: the backward whose kept aggregate is held in 8 bits
(pgcn_layer_bwd_mx, pgcn_sage_layer_bwd_mx) and the forward in PGCN_MXFP4, against ``oracle.mx`` and against the
calls that they are made of.

Bounds, u = 2^-24.  dW: those of the weight gradient's own tests, (2 rows + 260) u sum |v J|.  H_out in MXFP4: A and W are
quantised from the fp32 A that the call returns, so the product's own bound holds, 2 (f_in + 64) u sum |a w|."""
import numpy as np
import pytest
import torch

from gpu_helpers import dev, host, random_partition_graph
from mx_helpers import U, quantize
from oracle import mx
from oracle.partition import build_partition
from paper_2203_10428_amd import binding as B
from paper_2203_10428_amd.step import ld_of

pytestmark = pytest.mark.gpu
CODE = {"f32": B.PGCN_F32, "bf16": B.PGCN_BF16}


class Layer:
    def __init__(self, sage=False, symmetric=False, empty=False, f_in=70, f_out=41, seed=3):
        n_g, rowptr, col, owner = random_partition_graph(900, 400, 3, 9, seed)
        if empty:
            owner = np.where(owner == 0, 1, owner).astype(np.int32)
        ref = build_partition(n_g, rowptr, col, owner, 0, 3, self_loop=not sage)
        self.part = B.pgcn_partition_setup(n_g, rowptr, col, owner, 3, 0, self_loop=not sage, symmetric=symmetric)
        self.sage, self.f_in, self.f_out, self.n, self.b = sage, f_in, f_out, ref.n_inner, ref.n_bd
        self.n_send = B.pgcn_partition_info(self.part)["n_send"]
        rng = np.random.default_rng(seed)
        x = np.maximum(rng.standard_normal((self.n + self.b, f_in)), 0) * np.exp(rng.standard_normal((self.n + self.b, 1)))
        self.X, self.X_bd = dev(x[:self.n], f_in), dev(x[self.n:], f_in)
        self.W = torch.from_numpy(rng.uniform(-0.3, 0.3, ((1 + sage) * f_in, f_out)).astype(np.float32)).cuda()
        self.J = dev(1e-2 * rng.standard_normal((self.n, f_out)), f_out)

    def common(self, dtype):
        need = max(B.pgcn_layer_workspace_size(self.part, self.f_in, self.f_out, dtype, B.PGCN_ORDER_AGG), 256)
        return dict(f_in=self.f_in, f_out=self.f_out, gemm_dtype=dtype, relu=True, ld_in=ld_of(self.f_in), ld_out=ld_of(self.f_out),
                    W=self.W, workspace=torch.full((need,), 255, dtype=torch.uint8, device="cuda"), workspace_bytes=need)

    def forward(self, dtype, **over):
        A, H = torch.zeros(self.n, ld_of(self.f_in), device="cuda"), torch.zeros(self.n, ld_of(self.f_out), device="cuda")
        A16 = X16 = None
        if dtype == B.PGCN_BF16:
            A16, X16 = torch.zeros_like(A, dtype=torch.bfloat16), self.X.to(torch.bfloat16)
        args = {**self.common(dtype), "A": A, "A_bf16": A16, "H_out": H, **over}
        if self.sage:
            B.pgcn_sage_layer_fwd(self.part, X_in=self.X, X_in_bf16=X16, X_bd=self.X_bd, **args)
        else:
            B.pgcn_layer_fwd(self.part, H_in=self.X, H_bd=self.X_bd, **args)
        return A, A16, X16, H

    def backward(self, dtype, A, A16, X16, H, **mx_args):
        k = 2 if self.sage else 1
        dW = torch.full((k * self.f_in, self.f_out), 3.0, device="cuda")
        J_in, J_bd = torch.zeros_like(self.X), torch.zeros_like(self.X_bd)
        args = dict(self.common(dtype), J_out=self.J, H_out=H, A=A, A_bf16=A16, dW=dW, J_in=J_in, J_bd_out=J_bd, **mx_args)
        if self.sage:
            B.pgcn_sage_layer_bwd(self.part, X_in=self.X if "X_in_mx" not in mx_args else None,
                                  X_in_bf16=X16 if "X_in_mx" not in mx_args else None, **args)
        else:
            B.pgcn_layer_bwd(self.part, **args)
        torch.cuda.synchronize()
        return dW, J_in, J_bd


def hold(X, f, source):
    return quantize(X, f, "int8", "bf16" if source.dtype == torch.bfloat16 else "f32")


def check_dw(dW, x, f, J, H, dtype):
    """dW against the oracle's, from the values that the rows of x stand for."""
    v = mx.values(*mx.quantize(x, "int8"), f, "int8")
    Jm = np.where(H > 0, J, 0.0)
    if dtype == "bf16":
        Jm = torch.from_numpy(Jm).float().to(torch.bfloat16).double().numpy()
    got = dW.cpu().numpy().astype(np.float64)
    assert (np.abs(got - mx.wgrad(v, Jm)) <= (2 * len(J) + 260) * U * (np.abs(v).T @ np.abs(Jm)) + 2.0 ** -126).all()


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("symmetric", [False, True])
def test_gcn_backward_from_8_bits(dt, symmetric):
    g = Layer(symmetric=symmetric)
    A, A16, _, H = g.forward(CODE[dt])
    held = hold(A if A16 is None else A16, g.f_in, A if A16 is None else A16)
    want = g.backward(CODE[dt], A, A16, None, H)
    got = g.backward(CODE[dt], None, None, None, H, A_mx=held)
    assert torch.equal(got[1], want[1]) and torch.equal(got[2], want[2])
    check_dw(got[0], host(A if A16 is None else A16, g.f_in), g.f_in, host(g.J, g.f_out), host(H, g.f_out), dt)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("both", [False, True])
def test_sage_backward_from_8_bits(dt, both):
    g = Layer(sage=True, f_in=33, f_out=16)
    z, z16, X16, H = g.forward(CODE[dt])
    zs = z if dt == "f32" else z16
    mx_args = dict(A_mx=hold(zs, g.f_in, zs))
    if both:
        mx_args["X_in_mx"] = hold(g.X, g.f_in, g.X)
    want = g.backward(CODE[dt], z, z16, X16, H)
    got = g.backward(CODE[dt], None, None, X16, H, **mx_args)
    assert torch.equal(got[1], want[1]) and torch.equal(got[2], want[2])
    J, Hh = host(g.J, g.f_out), host(H, g.f_out)
    check_dw(got[0][:g.f_in], host(zs, g.f_in), g.f_in, J, Hh, dt)
    if both:
        check_dw(got[0][g.f_in:], host(g.X, g.f_in), g.f_in, J, Hh, dt)
    else:
        assert torch.equal(got[0][g.f_in:], want[0][g.f_in:])


def test_backward_of_an_empty_partition():
    for sage in (False, True):
        g = Layer(sage=sage, empty=True)
        byte = lambda ld: torch.zeros(1, ld, dtype=torch.uint8, device="cuda")
        held = (byte(96), byte(4))
        dW = torch.full(((1 + sage) * g.f_in, g.f_out), 3.0, device="cuda")
        args = dict(g.common(B.PGCN_F32), J_out=None, H_out=None, A=None, A_bf16=None, dW=dW, J_in=None, J_bd_out=None, A_mx=held)
        if sage:
            B.pgcn_sage_layer_bwd(g.part, X_in=None, X_in_bf16=None, X_in_mx=held, **args)
        else:
            B.pgcn_layer_bwd(g.part, **args)
        torch.cuda.synchronize()
        assert (dW == 0).all()


def check_fp4(H, A, W, relu, n, f_in, f_out):
    a, w = mx.values(*mx.quantize(A, "fp4"), f_in, "fp4"), mx.values(*mx.quantize(np.ascontiguousarray(W.T), "fp4"), f_in, "fp4")
    tol = 2 * (f_in + 64) * U * (np.abs(a) @ np.abs(w).T) + 2.0 ** -120
    assert (np.abs(host(H, f_out) - mx.product(a, w, relu)) <= tol).all()


@pytest.mark.parametrize("symmetric", [False, True])
@pytest.mark.parametrize("relu", [False, True])
@pytest.mark.parametrize("f_in,f_out", [(70, 41), (7, 3), (256, 128)])
def test_forward_in_4_bits(f_in, f_out, relu, symmetric):
    g = Layer(symmetric=symmetric, f_in=f_in, f_out=f_out)
    A32 = g.forward(B.PGCN_F32)[0]
    send = torch.full((g.n_send + 1, ld_of(f_out)), 77.0, device="cuda")
    A, _, _, H = g.forward(B.PGCN_MXFP4, relu=relu, send_out=send)
    torch.cuda.synchronize()
    assert torch.equal(A, A32)
    check_fp4(H, host(A, f_in), g.W.cpu().numpy().astype(np.float64), relu, g.n, f_in, f_out)
    rows = torch.zeros_like(send[:g.n_send])
    B.pgcn_pack_boundary(g.part, B.PGCN_PACK_FEAT, H, rows, f_out, ld_of(f_out))
    torch.cuda.synchronize()
    assert torch.equal(send[:g.n_send, :f_out], rows[:, :f_out]) and (send[g.n_send:] == 77).all()
    given = torch.zeros_like(H)
    B.pgcn_layer_fwd(g.part, H_in=None, H_bd=None, A=A, A_bf16=None, H_out=given, a_given=True,
                     **{**g.common(B.PGCN_MXFP4), "relu": relu})
    torch.cuda.synchronize()
    assert torch.equal(given[:, :f_out], H[:, :f_out])


def test_forward_in_4_bits_without_an_allocation():
    g = Layer()
    _, _, _, H = g.forward(B.PGCN_MXFP4)
    A, again = torch.zeros(g.n, ld_of(g.f_in), device="cuda"), torch.zeros_like(H)
    args = {k: v for k, v in g.common(B.PGCN_MXFP4).items() if not k.startswith("workspace")}
    B.pgcn_layer_fwd_noalloc(g.part, H_in=g.X, H_bd=g.X_bd, A=A, A_bf16=None, H_out=again, **args)
    torch.cuda.synchronize()
    assert torch.equal(again, H)


def test_forward_in_4_bits_of_an_empty_partition():
    g = Layer(empty=True)
    B.pgcn_layer_fwd(g.part, H_in=None, H_bd=g.X_bd, A=None, A_bf16=None, H_out=None, **g.common(B.PGCN_MXFP4))
    torch.cuda.synchronize()


def test_one_workspace_serves_every_call_of_a_layer_in_a_graph():
    """Forward in 4 bits, its aggregate held in 8 bits, the backward from them: captured, replayed with eager runs between."""
    g = Layer(f_in=100, f_out=72)
    common = g.common(B.PGCN_MXFP4)
    A, H = torch.zeros(g.n, ld_of(100), device="cuda"), torch.zeros(g.n, ld_of(72), device="cuda")
    ld_q, ld_s = B.mx_strides(B.PGCN_MX_INT8, 100)
    Q, S = torch.zeros(g.n, ld_q, dtype=torch.uint8, device="cuda"), torch.zeros(g.n, ld_s, dtype=torch.uint8, device="cuda")
    dW, J_in, J_bd = torch.zeros(100, 72, device="cuda"), torch.zeros_like(g.X), torch.zeros_like(g.X_bd)

    def run(stream):
        B.pgcn_layer_fwd(g.part, H_in=g.X, H_bd=g.X_bd, A=A, A_bf16=None, H_out=H, stream=stream, **common)
        B.pgcn_mx_quantize(format=B.PGCN_MX_INT8, dtype=B.PGCN_F32, rows=g.n, cols=100, src_rows=g.n, ld_x=A.stride(0), ld_q=ld_q,
                           ld_s=ld_s, X=A, index=None, Q=Q, S=S, stream=stream)
        B.pgcn_layer_bwd(g.part, J_out=g.J, H_out=H, A=None, A_bf16=None, dW=dW, J_in=J_in, J_bd_out=J_bd, A_mx=(Q, S), stream=stream,
                         **{**common, "gemm_dtype": B.PGCN_F32})

    outs = (A, H, Q, S, dW, J_in, J_bd)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    run(side)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        run(torch.cuda.current_stream())
    for k in range(4):
        g.X.mul_(0.5)
        torch.cuda.synchronize()
        run(side)
        torch.cuda.synchronize()
        want = [o.clone() for o in outs]
        for o in outs:
            o.fill_(3)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        cols = (100, 72, ld_q, 4, 72, 100, 100)
        assert all(torch.equal(o[:, :c], w[:, :c]) for o, w, c in zip(outs, want, cols))


def refused(call, code=B.PGCN_EINVAL):
    with pytest.raises(B.PgcnError) as e:
        call()
    assert e.value.code == code and B.pgcn_last_error()


@pytest.mark.parametrize("sage", [False, True])
def test_backward_refuses_what_has_no_form_in_8_bits(sage):
    g = Layer(sage=sage)
    held = hold(g.X, g.f_in, g.X)
    H = torch.zeros(g.n, ld_of(g.f_out), device="cuda")
    args = dict(g.common(B.PGCN_F32), J_out=g.J, H_out=H, A=None, A_bf16=None, dW=torch.zeros(2 * g.f_in, g.f_out, device="cuda"),
                J_in=torch.zeros_like(g.X), J_bd_out=torch.zeros_like(g.X_bd), A_mx=held)
    call = (lambda **kw: B.pgcn_sage_layer_bwd(g.part, X_in=g.X, X_in_bf16=None, **kw)) if sage else (lambda **kw: B.pgcn_layer_bwd(g.part, **kw))
    for over in (dict(order=B.PGCN_ORDER_TRANSFORM), dict(gemm_dtype=B.PGCN_MXFP4), dict(gemm_dtype=3), dict(f_in=0), dict(ld_in=68), dict(J_out=None),
                 dict(H_out=None), dict(dW=None)):
        refused(lambda: call(**{**args, **over}))
    refused(lambda: call(**{**args, "workspace_bytes": 64}), B.PGCN_EWORKSPACE)
    if sage:                                                # X_in is read in fp32 or bf16 unless it is held in 8 bits
        refused(lambda: B.pgcn_sage_layer_bwd(g.part, X_in=None, X_in_bf16=None, **args))
        refused(lambda: B.pgcn_sage_layer_bwd(g.part, X_in=g.X, X_in_bf16=None, **{**args, "gemm_dtype": B.PGCN_BF16}))


def test_forward_in_4_bits_refuses():
    g = Layer()
    A, H = torch.zeros(g.n, ld_of(g.f_in), device="cuda"), torch.zeros(g.n * ld_of(g.f_out) + 4, device="cuda")
    args = dict(g.common(B.PGCN_MXFP4), H_in=g.X, H_bd=g.X_bd, A=A, A_bf16=None, H_out=H)
    for over in (dict(order=B.PGCN_ORDER_TRANSFORM), dict(A=None), dict(H_out=H[1:]), dict(W=g.W.view(-1)[1:]), dict(gemm_dtype=3), dict(ld_out=40)):
        refused(lambda: B.pgcn_layer_fwd(g.part, **{**args, **over}))
    refused(lambda: B.pgcn_layer_fwd(g.part, **{**args, "workspace_bytes": 256}), B.PGCN_EWORKSPACE)
    refused(lambda: B.pgcn_layer_fwd(g.part, **{**args, "workspace": args["workspace"][8:], "workspace_bytes": 1 << 40}))
    s = Layer(sage=True)
    refused(lambda: B.pgcn_sage_layer_fwd(s.part, X_in=s.X, X_in_bf16=None, X_bd=s.X_bd, A=torch.zeros_like(s.X), A_bf16=None, H_out=H,
                                          **{**s.common(B.PGCN_F32), "gemm_dtype": B.PGCN_MXFP4}))
