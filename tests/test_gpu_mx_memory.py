"""What a training step keeps with checkpoints in 8 bits: bytes against the plain step's, and the same results where layers
take turns in the gradients' space, with widths whose rows are padded.

Bytes a node: the plain step keeps the aggregates (4 a value in fp32, 2 in bf16), the dropped inputs (4; GraphSAGE in bf16 2
more) and the gradients J (4).  In 8 bits: whole blocks of 32 values and scales to whole dwords for each aggregate (and
GraphSAGE's dropped input), the gradients, and as much as the layers' full-precision buffers take beyond them."""
import numpy as np
import pytest
import torch

from paper_2203_10428_amd import configs
from paper_2203_10428_amd.step import HeldRows, PartitionTrainer, StepOptions, ld_of

pytestmark = pytest.mark.gpu
WIDTHS = [(32, 16, 8), (30, 20, 13, 7), (100, 128, 128, 47), (602, 256, 256, 256, 41), (300, 512, 512, 512, 100), (7, 5), (64, 64, 64)]


def trainer(widths, dt, model, dropout=0.0, **kw):
    w = configs.TINY
    g = configs.make_graph(w)
    rng = np.random.default_rng(2)
    k = 2 if model == "sage" else 1
    W = [rng.uniform(-0.2, 0.2, (k * a, b)).astype(np.float32) for a, b in zip(widths, widths[1:])]
    X = rng.standard_normal((g.n, widths[0])).astype(np.float32)
    labels = rng.integers(0, widths[-1], g.n).astype(np.int32)
    return PartitionTrainer(g, X, labels, W, widths, w.loss, w.loss_scale, dt,
                            StepOptions(model=model, gamma=w.gamma, eta=w.eta, copy_mode="pipe", dropout=dropout, seed=5, **kw))


def kept(tr):
    """Bytes of what is alive between a layer's forward and its backward, each storage once."""
    store = {}
    for group in (tr.A, tr.A16, tr.A_mx, tr.X_mx, tr.Xd_in, tr.Xd_16, tr.J_in, {0: tr.J_top}):
        for t in group.values():
            if t is not None:
                u = (t.bytes if isinstance(t, HeldRows) else t).untyped_storage()
                store[u.data_ptr()] = u.nbytes()
    return sum(store.values())


@pytest.mark.parametrize("order", ["agg", "auto"])
@pytest.mark.parametrize("dropout", [0.0, 0.3])
@pytest.mark.parametrize("model", ["gcn", "sage"])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("widths", WIDTHS, ids=str)
def test_checkpoints_in_8_bits_take_less(widths, dt, model, dropout, order):
    tr = trainer(widths, dt, model, dropout, order=order)
    if not any(o == 0 for o in tr.order.values()):
        with pytest.raises(AssertionError):                    # no layer aggregates first
            trainer(widths, dt, model, dropout, order=order, checkpoint_bits=8)
        return
    plain = kept(tr)
    tr = trainer(widths, dt, model, dropout, order=order, checkpoint_bits=8)
    held = lambda f: (f + 31) // 32 * 32 + (f + 127) // 128 * 4
    dropped = dropout > 0 or (model == "sage" and dt == "bf16")
    a = 4 if dt == "f32" else 2
    own = [l for l in tr.order if l not in tr.ckpt]            # layers that transform first keep their dropped inputs
    x = 4 * dropped + 2 * (model == "sage" and dt == "bf16")
    want = sum(held(widths[l - 1]) * (2 if model == "sage" and dropped else 1) for l in tr.ckpt) + \
        sum(x * ld_of(widths[l - 1]) for l in own) + \
        max((a + x) * max(ld_of(widths[l - 1]) for l in tr.ckpt), 4 * sum(ld_of(f) for f in widths[1:]))
    assert kept(tr) == tr.n * want
    if len(widths) > 2:                                        # of a single layer's aggregate there is nothing to share
        assert kept(tr) < plain


@pytest.mark.parametrize("dropout", [0.0, 0.3])
@pytest.mark.parametrize("model", ["gcn", "sage"])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("widths", [(30, 20, 13, 7), (7, 61, 5), (100, 12, 12, 3)], ids=str)
def test_the_same_results_from_the_shared_space(widths, dt, model, dropout):
    """dW: an element x in 8 bits is off by half a step, at most 2^-7 (1 + 2^-7) of its row's largest, and where the plain
    step has it in bf16 by 2^-9 more; so dW by the sum over the rows of that times |J|, and by the rounding of both sums."""
    plain, tr = trainer(widths, dt, model, dropout), trainer(widths, dt, model, dropout, checkpoint_bits=8)
    for t in range(3):
        for a, b in zip(tr.W, plain.W):
            a.copy_(b)
        torch.cuda.synchronize()
        for x in (plain, tr):
            x.step()
            x.synchronize()
        assert torch.equal(tr.loss, plain.loss)
        assert torch.equal(tr.J_top[:, :widths[-1]], plain.J_top[:, :widths[-1]])
        for l, f in enumerate(widths[1:], 1):
            assert torch.equal(tr.H[l][:, :f], plain.H[l][:, :f])
            k = widths[l - 1]
            J = (plain.J_top if l == len(widths) - 1 else plain.J_in[l + 1])[:, :f].double().abs()
            for half, x in enumerate([plain.A[l] if plain.A[l] is not None else plain.A16[l], plain.X_used[l]][:1 + (model == "sage")]):
                top = x[:, :k].double().abs().amax(1, keepdim=True)
                off = (top * (2.0 ** -7 * (1 + 2.0 ** -7) + 2.0 ** -9 + 4 * (plain.n + 130) * 2.0 ** -24)).t() @ J
                assert ((tr.dW[l - 1] - plain.dW[l - 1])[half * k:(half + 1) * k].double().abs() <= off + 2.0 ** -120).all()
            if l > 1:
                g = widths[l - 1]
                assert torch.equal(tr.J_in[l][:, :g], plain.J_in[l][:, :g]) and torch.equal(tr.J_bd_out[l][:, :g], plain.J_bd_out[l][:, :g])
