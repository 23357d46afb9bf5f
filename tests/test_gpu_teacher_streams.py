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


def test_a_step_waits_for_the_lists_it_trains_on():
    """Lists that one stream still writes when set_teacher is called there, and a step on another stream."""
    w, tr = trainer(distill_temp=2.0)
    tr.step()
    v, i, tail = tr.top_logits(3, 2.0)
    full = (v + 0.5, i.clone(), tail.clone())
    tr.set_teacher(*full)
    loss, want = float(tr.step()), tr.dW[0].clone()
    w, tr = trainer(distill_temp=2.0)
    tr.step()
    tr.synchronize()
    lists = [torch.zeros_like(x) for x in full]
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(a):
        torch.cuda._sleep(BUSY)
        for x, y in zip(lists, full):
            x.copy_(y)
        tr.set_teacher(*lists)
    with torch.cuda.stream(b):
        got = tr.step()
    torch.cuda.synchronize()
    assert float(got) == loss and torch.equal(tr.dW[0], want)


def test_a_teacher_is_kept_until_the_step_has_read_it():
    """Another teacher takes its place, and its memory is asked for again, while a step is still to read it."""
    w, tr = trainer(distill_temp=2.0)
    tr.step()
    v, i, tail = tr.top_logits(3, 2.0)
    tr.synchronize()
    tr.set_teacher(v + 0.5, i.clone(), tail.clone())
    loss = float(tr.step())
    want = tr.dW[0].clone()
    w, tr = trainer(distill_temp=2.0)
    tr.step()
    tr.synchronize()
    side, other = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        tr.set_teacher(v + 0.5, i.clone(), tail.clone())
    with torch.cuda.stream(tr.stream):
        torch.cuda._sleep(BUSY)
    with torch.cuda.stream(other):
        got = tr.step()
    with torch.cuda.stream(side):
        tr.set_teacher(None, None)
        again = [torch.full_like(x, 7) for x in (v, i, tail) for _ in range(4)]
    torch.cuda.synchronize()
    assert float(got) == loss and torch.equal(tr.dW[0], want) and len(again) == 12
