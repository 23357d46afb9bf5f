"""Pins of ``oracle.ops``: against torch in float64 (autograd of the loss written as a dense
KL divergence, group_norm) and against central differences."""
import numpy as np
import pytest
import torch

from oracle import ops


def dense_kl(z, values, ids, tail, label, T, soft, hard):
    """The distillation loss of one row from dense probability rows, the rest as one more bucket."""
    C = len(z)
    keep = [k for k in range(len(ids)) if ids[k] >= 0 and ids[k] not in list(ids[:k])]
    loss = torch.zeros((), dtype=torch.float64)
    if keep:
        logits = torch.tensor([values[k] / T for k in keep] + ([] if tail is None else [tail]), dtype=torch.float64)
        p = torch.softmax(logits, 0)
        q = torch.softmax(z / T, 0)
        listed = torch.zeros(C, dtype=torch.bool)
        listed[[int(ids[k]) for k in keep]] = True
        buckets = torch.stack([q[int(ids[k])] for k in keep] + ([] if tail is None else [q[~listed].sum()]))
        on = p > 0
        loss = loss + soft * (p[on] * (p[on].log() - buckets[on].log())).sum()
    if label >= 0:
        loss = loss - hard * torch.log_softmax(z, 0)[label]
    return loss


@pytest.mark.parametrize("T", [1.0, 2.5])
@pytest.mark.parametrize("use_tail", [False, True])
@pytest.mark.parametrize("label", [-1, 3])
def test_distill_row_is_the_dense_divergence(T, use_tail, label):
    rng = np.random.default_rng(int(10 * T) + label)
    for ids in ([4, 0, 7], [2, -1, -1], [-1, -1, -1], [3, 5, 3], [1, 2, 0]):
        z0 = 2.0 * rng.standard_normal(9)
        values, tail = rng.standard_normal(3), (0.3 if use_tail else None)
        z = torch.tensor(z0, dtype=torch.float64, requires_grad=True)
        ref = dense_kl(z, values, np.array(ids), tail, label, T, 0.7, 0.4)
        loss, g = ops.distill_row(z0, values, ids, tail, label, T, 0.7, 0.4)
        assert abs(loss - float(ref.detach())) <= 1e-12
        want = torch.autograd.grad(ref, z)[0].numpy() if ref.requires_grad else np.zeros(9)
        assert np.abs(g - want).max() <= 1e-12
        for c in range(9):                                            # central differences
            e = np.zeros(9)
            e[c] = 1e-5
            hi = ops.distill_row(z0 + e, values, ids, tail, label, T, 0.7, 0.4)[0]
            lo = ops.distill_row(z0 - e, values, ids, tail, label, T, 0.7, 0.4)[0]
            assert abs((hi - lo) / 2e-5 - g[c]) <= 1e-8


def test_distill_of_a_teacher_to_itself_is_zero():
    rng = np.random.default_rng(0)
    Z = rng.standard_normal((6, 12))
    v, i, tail = ops.top_logits(Z, 5, 1.7)
    loss, J = ops.distill(Z, v, i, tail, None, 1.7, 1.0, 0.0)
    assert abs(loss) <= 1e-12 and np.abs(J).max() <= 1e-12


def test_distill_masked_classes_carry_nothing():
    z = np.array([0.3, -np.inf, 1.0, -np.inf, -0.2])
    loss, g = ops.distill_row(z, [1.0, -np.inf], [2, 1], 0.1, 0, 1.0, 1.0, 1.0)
    keep = [0, 2, 4]
    ref, gr = ops.distill_row(z[keep], [1.0, -np.inf], [1, -1], 0.1, 0, 1.0, 1.0, 1.0)
    assert abs(loss - ref) <= 1e-14 and np.abs(g[keep] - gr).max() <= 1e-14 and (g[[1, 3]] == 0).all()


def test_top_logits_against_torch():
    rng = np.random.default_rng(1)
    Z = np.round(2 * rng.standard_normal((20, 17))) / 2                # many ties
    Z[3, ::2] = -np.inf
    Z[4] = -np.inf
    v, i, tail = ops.top_logits(Z, 6, 0.8)
    zt = torch.from_numpy(Z)
    order = torch.sort(zt, dim=1, descending=True, stable=True)
    rows = [r for r in range(20) if r != 4]
    assert np.array_equal(v[rows], order.values[rows, :6].numpy())
    assert np.array_equal(i[rows], order.indices[rows, :6].numpy())
    assert np.allclose(tail[rows], torch.logsumexp(order.values[rows, 6:] / 0.8, 1).numpy(), rtol=1e-13, atol=0)
    assert (i[4] == -1).all() and (v[4] == -np.inf).all() and tail[4] == -np.inf


@pytest.mark.parametrize("kind", ["none", "relu", "silu", "gelu"])
@pytest.mark.parametrize("samples,rows,f,groups", [(1, 7, 12, 3), (5, 1, 8, 1), (3, 4, 6, 6)])
def test_group_norm_against_torch(kind, samples, rows, f, groups):
    rng = np.random.default_rng(f + samples)
    X = rng.standard_normal((samples * rows, f)) + 0.3
    ga, be = 1 + 0.2 * rng.standard_normal(f), 0.2 * rng.standard_normal(f)
    J = rng.standard_normal(X.shape)
    x = torch.tensor(X, requires_grad=True)
    g, b = torch.tensor(ga, requires_grad=True), torch.tensor(be, requires_grad=True)
    t = x.reshape(samples, rows, f).permute(0, 2, 1)
    u = torch.nn.functional.group_norm(t, groups, g, b, 1e-5).permute(0, 2, 1).reshape(X.shape)
    y = {"none": lambda v: v, "relu": torch.relu, "silu": torch.nn.functional.silu,
         "gelu": torch.nn.functional.gelu}[kind](u)
    y.backward(torch.tensor(J))
    Y, mean, rstd = ops.group_norm_forward(X, ga, be, samples, groups, 1e-5, kind)
    dX, dg, db = ops.group_norm_backward(X, J, ga, be, mean, rstd, samples, groups, kind)
    for a, r in ((Y, y), (dX, x.grad), (dg, g.grad), (db, b.grad)):
        assert np.abs(a - r.detach().numpy()).max() <= 1e-11
