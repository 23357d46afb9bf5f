"""The training step with checkpoints in 8 bits, boundary rows in 8 or 4 bits and forward updates in 4 bits, on the Tiny
workload.  What an option does not touch has to be the same bits as without it; what it touches is checked against
``oracle.mx``: exact bytes, values and products within the bounds of the operators' own tests."""
import numpy as np
import pytest
import torch

from mx_helpers import U
from oracle import mx
from paper_2203_10428_amd import configs
from paper_2203_10428_amd.step import PartitionTrainer, StepOptions

pytestmark = pytest.mark.gpu


def trainer(dt="f32", model="gcn", **kw):
    w = configs.TINY
    g = configs.make_graph(w)
    d = configs.make_dense(w, g.n, model=model)
    return w, PartitionTrainer(g, d.X, d.labels, d.W, w.widths, w.loss, w.loss_scale, dt,
                               StepOptions(model=model, gamma=w.gamma, eta=w.eta, **{"copy_mode": "pipe", **kw}))


def get(t, f):
    return t[:, :f].float().cpu().numpy().astype(np.float64)


def inputs(tr, l):
    return tr.X if l == 1 else tr.H[l - 1]


def step(*trs):
    torch.cuda.synchronize()
    for tr in trs:
        tr.step()
        tr.synchronize()


def check_dw(dW, v, J, H, dt, relu):
    J = np.where(H > 0, J, 0.0) if relu else J
    if dt == "bf16":
        J = torch.from_numpy(J).float().to(torch.bfloat16).double().numpy()
    tol = (2 * len(J) + 260) * U * (np.abs(v).T @ np.abs(J)) + 2.0 ** -126
    assert (np.abs(dW.cpu().numpy().astype(np.float64) - mx.wgrad(v, J)) <= tol).all()


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("model", ["gcn", "sage"])
@pytest.mark.parametrize("dropout", [0.0, 0.3])
def test_checkpoints_in_8_bits(dt, model, dropout):
    kw = dict(dt=dt, model=model, dropout=dropout, seed=5)
    w, plain = trainer(**kw)
    _, tr = trainer(checkpoint_bits=8, **kw)
    L = w.layers
    for t in range(3):
        for a, b in zip(tr.W, plain.W):                        # the same weights, whose gradients differ
            a.copy_(b)
        step(plain, tr)
        assert torch.equal(tr.loss, plain.loss)
        for l in range(1, L + 1):
            assert torch.equal(tr.H[l], plain.H[l])
            if l > 1:
                assert torch.equal(tr.J_in[l], plain.J_in[l]) and torch.equal(tr.J_bd_out[l], plain.J_bd_out[l])
            A = plain.A[l] if plain.A[l] is not None else plain.A16[l]
            f, held = w.widths[l - 1], tr.A_mx[l]
            if model == "gcn" and dt == "bf16":                # its fp32 aggregate is what is quantised: within the rounding to bf16
                v = mx.values(mx.from_bytes(held.Q.cpu().numpy(), "int8"), held.S.cpu().numpy()[:, :mx.blocks(f)], f, "int8")
                a = get(A, f)
                top = np.abs(a).reshape(len(a), -1, min(f, 32)).max(2)
                assert (np.abs(v - a) <= np.repeat(top, min(f, 32), 1) * 1.01 * (2.0 ** -7 + 2.0 ** -8)).all()
            else:
                code, s = mx.quantize(get(A, f), "int8")
                assert np.array_equal(held.Q.cpu().numpy()[:, :code.shape[1]], mx.to_bytes(code, "int8"))
                assert np.array_equal(held.S.cpu().numpy()[:, :s.shape[1]], s)
                v = mx.values(code, s, f, "int8")
            J, H = get(plain.J_top if l == L else plain.J_in[l + 1], w.widths[l]), get(plain.H[l], w.widths[l])
            check_dw(tr.dW[l - 1][:f], v, J, H, dt, l < L)
            if model == "sage" and tr.X_mx:
                x = mx.values(*mx.quantize(get(plain.X_used[l], f), "int8"), f, "int8")
                check_dw(tr.dW[l - 1][f:], x, J, H, dt, l < L)
            elif model == "sage":
                assert torch.equal(tr.dW[l - 1][f:], plain.dW[l - 1][f:])


@pytest.mark.parametrize("dropout", [0.0, 0.3])
def test_only_layers_that_aggregate_first_are_held(dropout):
    """One layer of three narrows and transforms first: it keeps what it keeps without the options."""
    w = configs.TINY
    widths = (32, 48, 16, 8)                                  # auto: the first aggregates first
    g = configs.make_graph(w)
    d = configs.make_dense(w, g.n)
    rng = np.random.default_rng(2)
    W = [rng.uniform(-0.2, 0.2, (a, b)).astype(np.float32) for a, b in zip(widths, widths[1:])]
    make = lambda **kw: PartitionTrainer(g, d.X, d.labels, W, widths, w.loss, w.loss_scale, "f32",
                                         StepOptions(gamma=w.gamma, eta=w.eta, copy_mode="pipe", order="auto", dropout=dropout, seed=5, **kw))
    plain, tr, both = make(), make(checkpoint_bits=8), make(checkpoint_bits=8, forward_mx4=True)
    assert set(tr.A_mx) == tr.ckpt == both.mx4 == {1}
    for t in range(3):
        for a, c, b in zip(tr.W, both.W, plain.W):
            a.copy_(b)
            c.copy_(b)
        step(plain, tr, both)
        assert torch.equal(tr.loss, plain.loss) and np.isfinite(both.loss.item())
        for l in (2, 3):
            assert torch.equal(tr.dW[l - 1], plain.dW[l - 1]) and torch.equal(tr.J_in[l], plain.J_in[l])
        v = mx.values(*mx.quantize(get(plain.A[1], 32), "int8"), 32, "int8")
        check_dw(tr.dW[0], v, get(plain.J_in[2], 48), get(plain.H[1], 48), "f32", True)


def test_checkpoints_take_less_memory():
    """The aggregates that stay between forward and backward: 8 bits and a scale to 32 elements, against 32 bits."""
    w, tr = trainer(checkpoint_bits=8)
    held = sum(h.bytes.numel() for h in tr.A_mx.values())
    assert held == sum(tr.n * ((f + 31) // 32 * 32 + 4) for f in w.widths[:-1])
    assert len({t.data_ptr() for t in tr.A.values()}) == 1


def read(held):
    """The values of a message, with the row stride of a message in fp32."""
    fmt = "int8" if held.format == 0 else "fp4"
    v = mx.values(mx.from_bytes(held.Q.cpu().numpy(), fmt), held.S.cpu().numpy()[:, :mx.blocks(held.cols)], held.cols, fmt)
    return torch.from_numpy(v.astype(np.float32)).cuda()


def check_message(held, x):
    fmt = "int8" if held.format == 0 else "fp4"
    code, s = mx.quantize(x, fmt)
    b = mx.to_bytes(code, fmt)
    assert np.array_equal(held.Q.cpu().numpy()[:, :b.shape[1]], b) and np.array_equal(held.S.cpu().numpy()[:, :s.shape[1]], s)


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("mode,remote", [("pipe", "device"), ("pipe", "host"), ("serial", "device"), ("none", "device")])
@pytest.mark.parametrize("smooth", [False, True])
def test_boundary_rows_in_fewer_bits(bits, mode, remote, smooth):
    """Against a step in fp32 whose peers send what the bytes stand for: the same bits without smoothing.  With it, the two
    moving averages round differently (one product-sum or two roundings): a few u of their terms, compared at 1e-5."""
    kw = dict(smooth_f=smooth, smooth_g=smooth, copy_mode=mode)
    w, plain = trainer(**kw)
    _, tr = trainer(exchange_bits=bits, remote=remote, **kw)
    L = w.layers
    for l, held in tr.remote_fq.items():
        check_message(held, get(tr.remote_f[l], w.widths[l - 1]))
        plain.remote_f[l][:, :w.widths[l - 1]] = read(held)
    for l, held in tr.remote_gq.items():
        check_message(held, get(tr.remote_g[l], w.widths[l - 1]))
        plain.remote_g[l][:, :w.widths[l - 1]] = read(held)
    for t in range(4):
        step(plain, tr)
        same = (lambda a, b: torch.equal(a, b)) if not smooth else (lambda a, b: float((a - b).abs().max()) <= 1e-5 * float(b.abs().max()))
        assert same(tr.loss, plain.loss)
        for l in range(1, L + 1):
            f = w.widths[l - 1]
            assert same(tr.H[l], plain.H[l]) and same(tr.dW[l - 1], plain.dW[l - 1]) and same(tr.W[l - 1], plain.W[l - 1])
            check_message(tr.send_f[l], get(inputs(tr, l), f)[tr.send_idx])
            if l > 1:
                assert same(tr.J_in[l], plain.J_in[l])
                check_message(tr.send_g[l], get(tr.J_bd_out[l], f))
    copied = sum(h.bytes.numel() for h in (*tr.remote_fq.values(), *tr.remote_gq.values()))
    assert tr.refill_bytes == copied


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("cache", [False, True])
def test_forward_updates_in_4_bits(dt, cache):
    w, tr = trainer(dt=dt, forward_mx4=True, cache_layer1=cache)
    for t in range(3):
        W = [x.cpu().numpy().astype(np.float64) for x in tr.W]
        step(tr)
        assert np.isfinite(tr.loss.item())
        for l in range(1, w.layers + 1):
            f = w.widths[l - 1]
            A = get(tr.A1_used if cache and l == 1 else tr.A[l], f)
            a, b = mx.values(*mx.quantize(A, "fp4"), f, "fp4"), mx.values(*mx.quantize(np.ascontiguousarray(W[l - 1].T), "fp4"), f, "fp4")
            tol = 2 * (f + 64) * U * (np.abs(a) @ np.abs(b).T) + 2.0 ** -120
            assert (np.abs(get(tr.H[l], w.widths[l]) - mx.product(a, b, l < w.layers)) <= tol).all()
            J = get(tr.J_top if l == w.layers else tr.J_in[l + 1], w.widths[l])
            if l < w.layers:
                J = np.where(get(tr.H[l], w.widths[l]) > 0, J, 0.0)
            size = np.abs(A).T @ np.abs(J)
            # fp32 by parts or bf16 operands (2^-8 each), sums of n terms
            tol = ((2 * len(J) + 260) * U + (2 * 2.0 ** -8 + 2.0 ** -16 if dt == "bf16" else 16 * U)) * size
            assert (np.abs(tr.dW[l - 1].cpu().numpy() - A.T @ J) <= tol).all()


def test_all_three_together_with_group_norm():
    w, tr = trainer(checkpoint_bits=8, exchange_bits=8, forward_mx4=True, smooth_f=True, smooth_g=True, norm_groups=4)
    for t in range(4):
        step(tr)
        assert np.isfinite(tr.loss.item()) and all(torch.isfinite(x).all() for x in (*tr.W, *tr.dW))
        for l in range(1, w.layers + 1):
            check_message(tr.send_f[l], get(inputs(tr, l), w.widths[l - 1])[tr.send_idx])


def test_two_trainers_at_once_keep_their_own():
    """Steps of two trainers on streams of their own, interleaved, give what each gives alone."""
    kw = dict(checkpoint_bits=8, exchange_bits=4, smooth_f=True, smooth_g=True)
    alone = [trainer(**kw)[1], trainer(model="sage", dropout=0.2, **kw)[1]]
    both = [trainer(**kw)[1], trainer(model="sage", dropout=0.2, **kw)[1]]
    for tr in alone:
        for _ in range(3):
            tr.step()
        tr.synchronize()
    torch.cuda.synchronize()
    for _ in range(3):
        for tr in both:
            tr.step()
    for tr in both:
        tr.synchronize()
    for a, b in zip(alone, both):
        assert torch.equal(a.loss, b.loss) and all(torch.equal(x, y) for x, y in zip(a.W, b.W))


@pytest.mark.parametrize("kw", [dict(checkpoint_bits=4), dict(exchange_bits=16), dict(checkpoint_bits=8, order="transform"),
                                dict(forward_mx4=True, order="auto"), dict(forward_mx4=True, model="sage"),
                                dict(checkpoint_bits=8, cache_layer1=True), dict(exchange_bits=8, cache_layer1=True)])
def test_refused_options(kw):
    with pytest.raises(AssertionError):
        trainer(**kw)
