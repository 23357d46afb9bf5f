"""The operators beside the layers, without a GPU: structure layouts, workspace sizes, refusals (each
is a status before any device call) and the trace kinds' names."""
import ctypes as C
import os
import re
import subprocess

import pytest
import torch

from paper_2203_10428_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
A = 1 << 20                                # stands for a 16-byte aligned buffer; never dereferenced
STEP = 1 << 24                             # buffers that far apart do not overlap


def at(i):
    return A + i * STEP


TOP = dict(dtype=B.PGCN_F32, rows=10, classes=41, ld=48, top=8, ld_top=8, temperature=2.0, Z=at(0), top_values=at(1),
           top_ids=at(2), tail_lse=at(3), workspace=at(4), workspace_bytes=STEP)
DISTILL = dict(TOP, soft_scale=1.0, hard_scale=0.5, labels=at(5), J=at(6), loss_out=at(7))
NORM = dict(dtype=B.PGCN_F32, act=B.PGCN_ACT_SILU, channels=32, groups=4, samples=3, sample_rows=5, ld_x=32, X=at(0),
            gamma=at(1), beta=at(2), mean=at(3), rstd=at(4), workspace=at(5), workspace_bytes=STEP)
FWD = dict(NORM, ld_y=32, eps=1e-5, Y=at(6))
BWD = dict(NORM, ld_j_out=32, ld_j_in=32, J_out=at(6), J_in=at(7), dgamma=at(8), dbeta=at(9))

LONG = dict(rows=1, classes=100000, ld=100000, top=50, ld_top=50)          # a row that goes in parts

BAD_TOP = [dict(dtype=2), dict(rows=-1), dict(rows=1 << 31), dict(classes=0), dict(classes=B.PGCN_MAX_CLASSES + 1, ld=1 << 20),
           dict(top=0), dict(top=42), dict(classes=512, ld=512, top=257, ld_top=257), dict(ld=40), dict(ld=42),
           dict(dtype=B.PGCN_BF16, ld=44), dict(ld_top=7), dict(temperature=0.0), dict(temperature=-1.0),
           dict(temperature=float("nan")), dict(temperature=float("inf")), dict(temperature=1e-45), dict(temperature=0.9e-4), dict(temperature=1.1e4),
           dict(Z=None), dict(top_values=None), dict(top_ids=None), dict(Z=at(0) + 4), dict(top_values=at(0)),
           dict(tail_lse=at(1) + 8), dict(LONG, workspace=at(4) + 4)]
BAD_DISTILL = BAD_TOP[:-3] + [dict(J=None), dict(J=at(6) + 8), dict(J=at(0)), dict(J=at(0) + 16), dict(loss_out=None),
                              dict(loss_out=at(5) + 4), dict(J=at(2)), dict(soft_scale=float("inf")),
                              dict(hard_scale=float("nan")), dict(loss_out=at(6) + 64), dict(workspace=at(4) + 4)]
BAD_NORM = [dict(dtype=-1), dict(act=4), dict(act=-1), dict(channels=0), dict(channels=8196, groups=4, ld_x=8196), dict(groups=5),
            dict(groups=0), dict(samples=-1), dict(sample_rows=0), dict(samples=1 << 20, sample_rows=1 << 20),
            dict(samples=1 << 31), dict(ld_x=28), dict(ld_x=34), dict(dtype=B.PGCN_BF16, ld_x=36), dict(X=None),
            dict(X=at(0) + 4), dict(workspace=at(5) + 8)]


def refused(call, args, code=B.PGCN_EINVAL):
    with pytest.raises(B.PgcnError) as e:
        call(**args)
    assert e.value.code == code and B.pgcn_last_error()


@pytest.mark.parametrize("bad", BAD_TOP, ids=str)
def test_top_logits_refuses(bad):
    refused(B.pgcn_top_logits, {**TOP, **bad})


@pytest.mark.parametrize("bad", BAD_DISTILL, ids=str)
def test_distill_refuses(bad):
    refused(B.pgcn_distill_loss_fwd_bwd, {**DISTILL, **bad})


@pytest.mark.parametrize("bad", BAD_NORM + [dict(eps=0.0), dict(eps=-1e-5), dict(eps=float("nan")), dict(ld_y=30), dict(Y=None),
                                            dict(Y=at(6) + 4), dict(Y=at(0)), dict(Y=at(1)), dict(mean=at(4) + 4),
                                            dict(rstd=at(2))], ids=str)
def test_group_norm_forward_refuses(bad):
    refused(B.pgcn_group_norm_fwd, {**FWD, **bad})


@pytest.mark.parametrize("bad", BAD_NORM + [dict(J_out=None), dict(J_out=at(6) + 4), dict(mean=None), dict(rstd=None),
                                            dict(ld_j_out=30), dict(ld_j_in=30), dict(J_in=at(6)), dict(J_in=at(0)),
                                            dict(dgamma=at(9)), dict(dbeta=at(1)), dict(J_in=at(7) + 4)], ids=str)
def test_group_norm_backward_refuses(bad):
    refused(B.pgcn_group_norm_bwd, {**BWD, **bad})


def test_short_workspaces_are_refused():
    need = B.pgcn_distill_workspace_size(B.PGCN_F32, 10, 41, 8)
    assert need > 0
    for ws in (dict(workspace=None, workspace_bytes=0), dict(workspace_bytes=need - 1)):
        refused(B.pgcn_distill_loss_fwd_bwd, {**DISTILL, **ws}, B.PGCN_EWORKSPACE)
    need = B.pgcn_top_logits_workspace_size(B.PGCN_F32, 1, 100000, 50)
    assert need > 0
    for ws in (dict(workspace=None, workspace_bytes=0), dict(workspace_bytes=need - 1)):
        refused(B.pgcn_top_logits, {**TOP, **LONG, **ws}, B.PGCN_EWORKSPACE)
    need = B.pgcn_group_norm_workspace_size(B.PGCN_F32, 32, 4, 3, 5)
    assert need > 0
    for call, args in ((B.pgcn_group_norm_fwd, FWD), (B.pgcn_group_norm_bwd, BWD)):
        refused(call, {**args, "workspace": None, "workspace_bytes": 0}, B.PGCN_EWORKSPACE)
        refused(call, {**args, "workspace_bytes": need - 1}, B.PGCN_EWORKSPACE)


def test_null_args_and_empty_calls():
    for name in ("pgcn_top_logits", "pgcn_distill_loss_fwd_bwd", "pgcn_group_norm_fwd", "pgcn_group_norm_bwd"):
        assert getattr(B.lib, name)(None, None) == B.PGCN_EINVAL
    none = dict(Z=None, top_values=None, top_ids=None, tail_lse=None, workspace=None, workspace_bytes=0)
    B.pgcn_top_logits(**{**TOP, **none, "rows": 0})                    # no rows: nothing to do
    B.pgcn_group_norm_fwd(**{**FWD, "samples": 0, "X": None, "Y": None, "workspace": None, "workspace_bytes": 0})


def test_workspace_sizes_of_rejected_arguments_are_zero():
    assert B.pgcn_top_logits_workspace_size(7, 10, 41, 8) == 0
    assert B.pgcn_distill_workspace_size(B.PGCN_F32, 10, 41, 42) == 0
    assert B.pgcn_distill_workspace_size(B.PGCN_F32, -1, 41, 4) == 0
    assert B.pgcn_group_norm_workspace_size(B.PGCN_F32, 32, 5, 3, 5) == 0
    assert B.pgcn_group_norm_workspace_size(B.PGCN_F32, 32, 4, 1 << 20, 1 << 20) == 0


def test_tensors_in_host_memory_are_refused():
    z = torch.zeros(10, 48)
    with pytest.raises(ValueError, match="current device"):
        B.pgcn_top_logits(**{**TOP, "Z": z})


def test_structs_match_the_header(tmp_path):
    structs = [B.pgcn_top_logits_args, B.pgcn_distill_args, B.pgcn_group_norm_fwd_args, B.pgcn_group_norm_bwd_args]
    lines = ["#include <stdio.h>", "#include <stddef.h>", '#include "pgcn.h"', "int main(void) {"]
    for cls in structs:
        name = cls.__name__
        lines.append(f'  printf("{name} %zu\\n", sizeof({name}));')
        lines += [f'  printf("{name}.{f} %zu\\n", offsetof({name}, {f}));' for f, _ in cls._fields_]
    lines += ['  printf("kinds %d\\n", PGCN_TK_GROUP_NORM_BWD + 1);', "  return 0;", "}"]
    src = tmp_path / "layout.c"
    src.write_text("\n".join(lines) + "\n")
    exe = tmp_path / "layout"
    r = subprocess.run(["gcc", "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(ROOT, "include"), "-I", "/opt/rocm/include",
                        str(src), "-o", str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    got = dict(l.split() for l in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.splitlines())
    for cls in structs:
        assert int(got[cls.__name__]) == C.sizeof(cls)
        for f, _ in cls._fields_:
            assert int(got[f"{cls.__name__}.{f}"]) == getattr(cls, f).offset, f
    assert int(got["kinds"]) == len(B.TRACE_KINDS)


def test_limits_match_the_header():
    header = open(os.path.join(ROOT, "include", "pgcn.h")).read()
    for name in ("PGCN_MAX_TOP", "PGCN_MAX_CLASSES", "PGCN_MAX_CHANNELS"):
        assert int(re.search(rf"#define {name} (\d+)", header).group(1)) == getattr(B, name)
