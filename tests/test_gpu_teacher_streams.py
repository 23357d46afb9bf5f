"""The trainer's own stream and its callers' streams around top_logits and set_teacher: one that is kept busy holds back
what has to wait for it."""
import numpy as np
import pytest
import torch

from oracle import ops
from paper_2203_10428_amd import configs
from paper_2203_10428_amd.step import PartitionTrainer, StepOptions

pytestmark = pytest.mark.gpu

BUSY = 50_000_000                                          # clock cycles: some ten milliseconds


def trainer(**kw):
    w = configs.TINY
    g = configs.make_graph(w)
    d = configs.make_dense(w, g.n)
    return w, PartitionTrainer(g, d.X, d.labels, d.W, w.widths, w.loss, w.loss_scale, "f32",
                               StepOptions(smooth_f=False, smooth_g=False, copy_mode="none", eta=0.1, **kw))


def test_top_logits_follows_the_trainers_stream():
    """Called on another stream while the trainer's still writes its output, and before it writes the next one."""
    w, tr = trainer()
    tr.step()
    tr.synchronize()
    rng = np.random.default_rng(0)
    H = tr.H[w.layers]
    new = torch.from_numpy(rng.standard_normal(tuple(H.shape)).astype(np.float32)).cuda()
    other = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(tr.stream):
        torch.cuda._sleep(BUSY)
        H.copy_(new)
    with torch.cuda.stream(other):
        v, i, tail = tr.top_logits(3, 2.0)
        seen = [x.clone() for x in (v, i, tail)]           # the caller's next work sees the lists
    with torch.cuda.stream(tr.stream):
        H.zero_()
    torch.cuda.synchronize()
    rv, ri, rt = ops.top_logits(new[:, :w.classes].cpu().numpy().astype(np.float64), 3, 2.0)
    assert np.array_equal(seen[1].cpu().numpy(), ri) and np.array_equal(seen[0].cpu().numpy(), rv)
    assert np.abs(seen[2].cpu().numpy() - rt).max() <= 1e-5
    assert all(torch.equal(a, b) for a, b in zip(seen, (v, i, tail)))
