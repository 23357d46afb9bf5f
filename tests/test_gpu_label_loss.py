"""The distillation loss's label term on rows far from zero, where the row's maximum, added to the
logarithm first, would take the logarithm's digits.

Bounds.  With u = 2^-24 and the notes of ``test_gpu_distill``: the term is (m - z_y) + log sum e^{z - m}.  Both logits
are held exactly, their difference and the sum are rounded once, u of each, and the logarithm is off by EPS and 2 u of
itself: |error| <= 2 u (m - z_y) + 4 u log + EPS a row."""
import numpy as np
import pytest
import torch

from test_gpu_distill import EPS, U, call, logits, matrix

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [1.0, 2.0])
@pytest.mark.parametrize("rows,C", [(30, 41), (7, 1500), (6, 2500), (130, 9000), (2, 70000)])
@pytest.mark.parametrize("at", [0.0, 1e3, -(2.0 ** 20), 3e6, -1e9, 1e12])
def test_label_loss_far_from_zero(at, rows, C, T, dtype):
    rng = np.random.default_rng(C)
    step = float(np.spacing(np.float32(max(abs(at), 1.0)))) * (1 if dtype == "f32" else 2 ** 16)
    z = at + step * np.round(logits(rng, rows, C) / step)          # what the type can hold, and its neighbours
    Z = matrix(z, dtype)
    z = Z[:, :C].float().cpu().numpy().astype(np.float64)
    y = rng.integers(-1, C, rows)
    v, i = torch.zeros(rows, 1, device="cuda"), torch.full((rows, 1), -1, dtype=torch.int32, device="cuda")
    hard = 0.5
    loss = call(Z, C, v, i, None, torch.from_numpy(y.astype(np.int32)).cuda(), T, 1.0, hard, dtype)[1]
    torch.cuda.synchronize()
    m = z.max(1)
    log = np.log(np.exp(z - m[:, None]).sum(1))
    far = m - np.take_along_axis(z, np.maximum(y, 0)[:, None], 1)[:, 0]
    on = y >= 0
    want, bound = hard * (far + log)[on].sum(), hard * (2 * U * far + 4 * U * log + EPS)[on].sum()
    assert abs(float(loss[0]) - want) <= bound + 2 * U * abs(want), (float(loss[0]), want, bound)
