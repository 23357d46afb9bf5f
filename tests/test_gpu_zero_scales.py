"""A scale of 0 takes its term out of the distillation loss, also where the term itself would be infinite or
NaN: as if no list, or no label, were given.

Bounds.  By the notes of ``test_gpu_distill`` a row's log-sums are off by at most 2 EPS at these arguments, whether they are
formed of one part or of two, so two ways to the same loss differ by at most 4 EPS a row (the scales are at most 1),
and the same J by 4 EPS and, in bf16, by one rounding of a size below 1."""
import numpy as np
import pytest
import torch

from test_gpu_distill import EPS, NINF, call, logits, matrix, put, teacher

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [1.0, 2.0])
@pytest.mark.parametrize("rows,C,K", [(20, 41, 8), (9, 1500, 30), (5, 2500, 64), (2, 70000, 40)])
def test_a_scale_of_zero_takes_its_term_out(rows, C, K, T, dtype):
    rng = np.random.default_rng(C)
    z = logits(rng, rows, C)
    v, i, tail = teacher(rng, z, K, T, none=0.0)
    y = np.argmax(z, 1)
    no_list = np.full_like(i, -1)

    def run(z, i, y, soft, hard, tail=tail):
        J, loss = call(matrix(z, dtype), C, *put(v, i, tail), None if y is None else torch.from_numpy(y.astype(np.int32)).cuda(), T,
                       soft, hard, dtype)
        torch.cuda.synchronize()
        return J[:, :C], float(loss[0])

    # listed classes that the student masks: the divergence is +inf
    off = z.copy()
    for r in range(rows):
        off[r, [c for c in i[r] if c != y[r]]] = NINF
    J, l = run(off, i, y, 1.0, 0.5)
    assert l == np.inf
    J, l = run(off, i, y, 0.0, 0.5)
    J0, l0 = run(off, no_list, y, 1.0, 0.5)
    assert np.isfinite(l) and abs(l - l0) <= 4 * EPS * rows and (J - J0).abs().max() <= 4 * EPS + (2.0 ** -8) * (dtype == "bf16")
    # a label that the student masks: the label term is +inf
    lab = i[:, K - 1].copy()
    off = z.copy()
    off[np.arange(rows), lab] = NINF
    only = np.where(i == lab[:, None], -1, i)
    assert run(off, only, lab, 1.0, 0.5)[1] == np.inf
    J, l = run(off, only, lab, 1.0, 0.0)
    J0, l0 = run(off, only, None, 1.0, 0.0)
    assert np.isfinite(l) and abs(l - l0) <= 4 * EPS * rows and torch.isfinite(J).all() and (J - J0).abs().max() <= 4 * EPS + (2.0 ** -8) * (dtype == "bf16")
    # NaN among the listed values
    bad = i.copy()
    v[0, 1] = np.nan
    J, l = run(z, bad, y, 0.0, 0.5)
    J0, l0 = run(z, no_list, y, 0.0, 0.5)
    assert abs(l - l0) <= 4 * EPS * rows and torch.isfinite(J).all()
    # both terms out: nothing is left
    v[0, 1] = 0.0
    J, l = run(off, i, lab, 0.0, 0.0)
    assert l == 0.0 and (J == 0).all()
