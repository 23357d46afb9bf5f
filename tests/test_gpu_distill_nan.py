"""Where a NaN among a row's logits shows in the distillation loss and its gradient: the interface's words, kernel by kernel."""
import numpy as np
import pytest
import torch

from test_gpu_distill import NINF, call, logits, matrix, put, teacher

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [1.0, 2.0])
@pytest.mark.parametrize("rows,C,K", [(20, 41, 8), (9, 1500, 30), (8, 2500, 64), (7, 70000, 40)])
def test_nan_logits(rows, C, K, T, dtype):
    rng = np.random.default_rng(C)
    z = logits(rng, rows, C)
    v, i, tail = teacher(rng, z, K, T, none=0.0)
    masked = next(c for c in range(C - 1, 0, -1) if c not in i[0] and c not in i[1])
    z[:2, masked] = NINF
    y = np.zeros(rows)
    listed, free = i[0, 1], next(c for c in range(1, C) if c != masked and c not in i[:, :])
    # row 0: both terms; 1: a list; 2: a label; 3: neither; 4: neither, its slots hold -inf; 5: neither, NaN unlisted
    z[0, listed], z[1, free], z[2, free], z[3, i[3, 0]], z[4, i[4, 0]], z[5, free] = (np.nan,) * 6
    y[[1, 3, 4, 5]] = -1
    own = (i[3, 0], i[4, 0], free)
    i[[2, 3, 5]] = -1
    v[4] = NINF
    y = torch.from_numpy(y.astype(np.int32)).cuda()

    def run(keep):
        J, loss = call(matrix(z[keep], dtype), C, *put(v[keep], i[keep], tail[keep]), y[keep], T, 0.7, 0.5, dtype)
        torch.cuda.synchronize()
        return J[:, :C].float().cpu().numpy(), float(loss[0])

    for r in range(3):
        J, l = run([r])
        on = z[r] != NINF                                          # a NaN is not -inf
        assert np.isnan(l) and np.isnan(J[0, on]).all()
    J, l = run([3, 4, 5])
    assert l == 0.0
    for r in range(3):
        rest = np.arange(C) != own[r]
        assert (J[r, rest] == 0).all()
    J, l = run(list(range(6, rows)))
    assert np.isfinite(l)
