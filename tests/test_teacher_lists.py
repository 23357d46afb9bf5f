"""What ``PartitionTrainer.set_teacher`` refuses, without a GPU: lists whose sizes do not fit the partition would
be read past their ends by the step's kernel."""
import pytest
import torch

from paper_2203_10428_amd import binding as B
from paper_2203_10428_amd.step import PartitionTrainer, StepOptions

N, CLASSES, TOP = 12, 41, 5


def trainer(**kw):
    """The fields that the checks read; nothing of a device."""
    tr = PartitionTrainer.__new__(PartitionTrainer)
    tr.dev, tr.opts, tr.n, tr.widths, tr.L = torch.device("cpu"), StepOptions(**kw), N, [7, CLASSES], 1
    tr.loss_kind, tr.ws_bytes, tr.ws, tr.teacher = B.PGCN_SOFTMAX_CE, 1 << 20, None, "before"
    return tr


def lists(rows=N, top=TOP):
    return torch.zeros(rows, top), torch.zeros(rows, top, dtype=torch.int32)


@pytest.mark.parametrize("shape", [(N - 1,), (0,), (N + 1,), (N, 2), (1,), ()])
def test_a_log_sum_for_every_node(shape):
    tr = trainer()
    with pytest.raises(ValueError, match="tail_lse"):
        tr.set_teacher(*lists(), torch.zeros(shape))
    assert tr.teacher == "before"


@pytest.mark.parametrize("values,ids", [
    (torch.zeros(N - 1, TOP), torch.zeros(N - 1, TOP, dtype=torch.int32)), (torch.zeros(N), torch.zeros(N, dtype=torch.int32)),
    (torch.zeros(N, 0), torch.zeros(N, 0, dtype=torch.int32)),
    (torch.zeros(N, CLASSES + 1), torch.zeros(N, CLASSES + 1, dtype=torch.int32)),
    (torch.zeros(N, TOP, 2), torch.zeros(N, TOP, 2, dtype=torch.int32))], ids=["rows", "1d", "empty", "wide", "3d"])
def test_lists_of_every_node(values, ids):
    tr = trainer()
    with pytest.raises(ValueError):
        tr.set_teacher(values, ids)
    assert tr.teacher == "before"


def test_values_and_ids_belong_together():
    with pytest.raises(ValueError):
        trainer().set_teacher(lists()[0], lists(top=TOP + 1)[1])


@pytest.mark.parametrize("kw", [dict(distill_temp=0.0), dict(distill_temp=2e4), dict(distill_temp=float("nan")),
                                dict(distill_soft=float("inf")), dict(distill_hard=float("nan"))], ids=str)
def test_options_that_no_step_could_run(kw):
    tr = trainer(**kw)
    with pytest.raises(ValueError, match="distill_"):
        tr.set_teacher(*lists())
    assert tr.teacher == "before"
