"""The operators in 8 and 4 bits without a GPU: structure layouts, strides, refusals (each a status before any
device call) and the trace kinds' names."""
import ctypes as C
import os
import re
import subprocess

import pytest
import torch

from paper_2203_10428_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
STEP = 1 << 24


def at(i):                                 # stands for an aligned buffer; never dereferenced
    return (1 << 20) + i * STEP


QUANT = dict(format=B.PGCN_MX_INT8, dtype=B.PGCN_F32, rows=10, cols=70, src_rows=20, ld_x=72, ld_q=96, ld_s=4, X=at(0), index=at(1),
             Q=at(2), S=at(3))
READ = dict(format=B.PGCN_MX_FP4, dtype=B.PGCN_F32, rows=10, cols=70, ld_q=48, ld_s=4, ld_out=72, gamma=0.5, Q=at(0), S=at(1), out=at(2))
WGRAD = dict(dtype=B.PGCN_F32, rows=1000, f_in=70, f_out=30, ld_q=96, ld_s=4, ld_j=32, ld_h=32, Q=at(0), S=at(1), J=at(2), H=at(3),
             dW=at(4), workspace=at(5), workspace_bytes=STEP)
MATMUL = dict(dtype=B.PGCN_BF16, relu=True, m=10, n=30, k=70, ld_a=48, ld_a_scales=4, ld_b=48, ld_b_scales=4, ld_c=32, A=at(0),
              A_scales=at(1), B=at(2), B_scales=at(3), C=at(4), workspace=at(5), workspace_bytes=STEP)

BAD = {
    "quantize": [dict(format=2), dict(format=-1), dict(dtype=2), dict(rows=-1), dict(rows=1 << 31), dict(src_rows=-1), dict(cols=0),
                 dict(cols=B.PGCN_MAX_MX_COLS + 1, ld_x=1 << 25, ld_q=1 << 25, ld_s=1 << 20), dict(ld_x=68), dict(ld_x=74),
                 dict(dtype=B.PGCN_BF16, ld_x=76), dict(ld_q=80), dict(ld_q=104), dict(ld_s=2), dict(ld_s=6), dict(cols=129, ld_x=132, ld_q=160),
                 dict(X=None), dict(Q=None), dict(S=None), dict(X=at(0) + 8), dict(Q=at(2) + 8), dict(S=at(3) + 2), dict(index=at(1) + 2),
                 dict(index=None, rows=21), dict(transpose=True), dict(transpose=True, index=None), dict(transpose=2, index=None),
                 dict(transpose=True, index=None, rows=B.PGCN_MAX_MX_COLS + 1, src_rows=B.PGCN_MAX_MX_COLS + 1, ld_q=1 << 25, ld_s=1 << 20),
                 dict(transpose=True, index=None, rows=200, src_rows=200), dict(Q=at(0)), dict(S=at(2) + 32), dict(Q=at(1)), dict(S=at(0) + 64)],
    "dequantize": [dict(format=2), dict(dtype=-1), dict(rows=-1), dict(rows=1 << 31), dict(cols=0), dict(ld_q=32), dict(ld_q=56),
                   dict(ld_s=0), dict(ld_s=5), dict(ld_out=68), dict(ld_out=70), dict(gamma=-0.1), dict(gamma=1.1), dict(gamma=float("nan")),
                   dict(dtype=B.PGCN_BF16), dict(dtype=B.PGCN_BF16, gamma=0.0, ld_out=76), dict(Q=None), dict(S=None), dict(out=None),
                   dict(out=at(2) + 4), dict(Q=at(0) + 4), dict(S=at(1) + 1), dict(out=at(0)), dict(out=at(1))],
    "wgrad": [dict(dtype=2), dict(rows=-1), dict(rows=1 << 31), dict(f_in=0), dict(f_out=0), dict(f_in=B.PGCN_MAX_WIDTH + 1, ld_q=1 << 20, ld_s=1 << 12),
              dict(f_out=B.PGCN_MAX_WIDTH + 1, ld_j=1 << 17, ld_h=1 << 17), dict(ld_q=80), dict(ld_q=100), dict(ld_s=0), dict(ld_j=28),
              dict(ld_j=30), dict(ld_h=28), dict(ld_h=34), dict(Q=None), dict(S=None), dict(J=None), dict(dW=None), dict(Q=at(0) + 8),
              dict(J=at(2) + 8), dict(H=at(3) + 8), dict(dW=at(4) + 2), dict(dW=at(2)), dict(dW=at(0) + 16), dict(dW=at(3)), dict(dW=at(1)),
              dict(workspace=at(5) + 8), dict(workspace=at(2)), dict(dW=at(5) + 16)],
    "matmul": [dict(dtype=2), dict(relu=2), dict(m=-1), dict(m=1 << 31), dict(n=0), dict(k=0), dict(n=B.PGCN_MAX_MX_COLS + 1, ld_c=1 << 25),
               dict(k=B.PGCN_MAX_MX_COLS + 1, ld_a=1 << 24, ld_a_scales=1 << 20, ld_b=1 << 24, ld_b_scales=1 << 20), dict(ld_a=32),
               dict(ld_a=40), dict(ld_a_scales=2), dict(ld_b=32), dict(ld_b=56), dict(ld_b_scales=6), dict(ld_c=28), dict(ld_c=36),
               dict(A=None), dict(A_scales=None), dict(B=None), dict(B_scales=None), dict(C=None), dict(A=at(0) + 4), dict(B=at(2) + 8),
               dict(C=at(4) + 8), dict(A_scales=at(1) + 1), dict(B_scales=at(3) + 2), dict(C=at(0)), dict(C=at(3))],
}
CALLS = {"quantize": (B.pgcn_mx_quantize, QUANT), "dequantize": (B.pgcn_mx_dequantize, READ), "wgrad": (B.pgcn_mx_wgrad, WGRAD),
         "matmul": (B.pgcn_mx_matmul, MATMUL)}


def refused(call, args, code=B.PGCN_EINVAL):
    with pytest.raises(B.PgcnError) as e:
        call(**args)
    assert e.value.code == code and B.pgcn_last_error()


@pytest.mark.parametrize("name,bad", [(n, b) for n in BAD for b in BAD[n]], ids=str)
def test_refuses(name, bad):
    call, good = CALLS[name]
    if "relu" in bad:                                                  # the binding takes truth values: straight to the library
        a = B.pgcn_mx_matmul_args(B.PGCN_F32, bad["relu"], 10, 30, 70, 48, 4, 48, 4, 32, at(0), at(1), at(2), at(3), at(4), at(5), STEP)
        assert B.lib.pgcn_mx_matmul(C.byref(a), None) == B.PGCN_EINVAL
    else:
        refused(call, {**good, **bad})


def test_short_workspaces_are_refused():
    need = B.pgcn_mx_wgrad_workspace_size(B.PGCN_F32, 1000, 70, 30)
    assert need > 0
    for ws in (dict(workspace=None, workspace_bytes=0), dict(workspace_bytes=need - 1)):
        refused(B.pgcn_mx_wgrad, {**WGRAD, **ws}, B.PGCN_EWORKSPACE)
    assert B.pgcn_mx_wgrad_workspace_size(2, 1000, 70, 30) == 0
    assert B.pgcn_mx_wgrad_workspace_size(B.PGCN_F32, -1, 70, 30) == 0
    assert B.pgcn_mx_wgrad_workspace_size(B.PGCN_F32, 10, 0, 30) == 0
    assert B.pgcn_mx_matmul_workspace_size(B.PGCN_F32, 10, 0, 30) == 0
    assert B.pgcn_mx_matmul_workspace_size(3, 10, 10, 30) == 0


def test_null_args_and_empty_calls():
    for name in ("quantize", "dequantize", "wgrad", "matmul"):
        assert getattr(B.lib, "pgcn_mx_" + name)(None, None) == B.PGCN_EINVAL
    B.pgcn_mx_quantize(**{**QUANT, "rows": 0, "X": None, "Q": None, "S": None, "index": None})
    B.pgcn_mx_dequantize(**{**READ, "rows": 0, "Q": None, "S": None, "out": None})
    B.pgcn_mx_matmul(**{**MATMUL, "m": 0, "A": None, "A_scales": None, "C": None, "workspace": None, "workspace_bytes": 0})


def test_tensors_in_host_memory_are_refused():
    with pytest.raises(ValueError, match="current device"):
        B.pgcn_mx_quantize(**{**QUANT, "X": torch.zeros(20, 72)})


def test_strides():
    assert B.mx_strides(B.PGCN_MX_INT8, 602) == (608, 20) and B.mx_strides(B.PGCN_MX_FP4, 602) == (304, 20)
    assert B.mx_strides(B.PGCN_MX_FP4, 1) == (16, 4) and B.mx_strides(B.PGCN_MX_INT8, 128) == (128, 4)


def test_structs_and_limits_match_the_header(tmp_path):
    structs = [B.pgcn_mx_quantize_args, B.pgcn_mx_dequantize_args, B.pgcn_mx_wgrad_args, B.pgcn_mx_matmul_args, B.pgcn_mx_rows]
    lines = ["#include <stdio.h>", "#include <stddef.h>", '#include "pgcn.h"', "int main(void) {"]
    for cls in structs:
        name = cls.__name__
        lines.append(f'  printf("{name} %zu\\n", sizeof({name}));')
        lines += [f'  printf("{name}.{f} %zu\\n", offsetof({name}, {f}));' for f, _ in cls._fields_]
    lines += ['  printf("kinds %d\\n", PGCN_TK_MX_MATMUL + 1);', "  return 0;", "}"]
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
    assert int(got["kinds"]) == len(B.TRACE_KINDS) + len(B.MX_TRACE_KINDS)
    header = open(os.path.join(ROOT, "include", "pgcn.h")).read()
    for name in ("PGCN_MX_BLOCK", "PGCN_MAX_MX_COLS"):
        assert int(re.search(rf"#define {name} (\d+)", header).group(1)) == getattr(B, name)


# ---------------------------------------------------------------- in layers --

@pytest.fixture(scope="module")
def parts():
    import numpy as np
    rowptr, col = np.array([0, 2, 4, 5, 6], np.int64), np.array([1, 2, 0, 3, 0, 1], np.int32)
    owner = np.array([0, 0, 0, 1], np.int32)
    return [B.pgcn_partition_setup(4, rowptr, col, owner, 2, 0, self_loop=not sage, host_only=True) for sage in (False, True)]


LAYER = dict(f_in=70, f_out=30, gemm_dtype=B.PGCN_F32, relu=1, ld_in=72, ld_out=32)


def bwd_args(cls, **over):
    a = cls()
    for k, v in {**LAYER, "J_out": at(1), "H_out": at(2), "W": at(3), "dW": at(4), "workspace": at(5), "workspace_bytes": STEP, **over}.items():
        setattr(a, k, v)
    return a


BAD_ROWS = [dict(Q=None), dict(S=None), dict(Q=at(6) + 8), dict(S=at(7) + 2), dict(ld_q=80), dict(ld_q=104), dict(ld_s=2), dict(ld_s=6),
            dict(ld_q=(1 << 40) + 16)]


def rows_in_8_bits(**over):
    r = {**dict(Q=at(6), S=at(7), ld_q=96, ld_s=4), **over}
    return B.pgcn_mx_rows(r["Q"], r["S"], r["ld_q"], r["ld_s"])


@pytest.mark.parametrize("bad", BAD_ROWS, ids=str)
def test_layer_backwards_refuse_bad_rows(parts, bad):
    gcn, sage = parts
    good, ill = rows_in_8_bits(), rows_in_8_bits(**bad)
    a, b = bwd_args(B.pgcn_bwd_args), bwd_args(B.pgcn_sage_bwd_args)
    assert B.lib.pgcn_layer_bwd_mx(gcn.handle, C.byref(a), C.byref(ill), None) == B.PGCN_EINVAL
    assert "pgcn_layer_bwd_mx" in B.pgcn_last_error()
    for x in ((ill, None), (ill, good), (good, ill)):
        assert B.lib.pgcn_sage_layer_bwd_mx(sage.handle, C.byref(b), C.byref(x[0]), None if x[1] is None else C.byref(x[1]), None) == B.PGCN_EINVAL
        assert "pgcn_sage_layer_bwd_mx" in B.pgcn_last_error()


def test_layer_backwards_refuse_null_arguments(parts):
    gcn, sage = parts
    good, a, b = rows_in_8_bits(), bwd_args(B.pgcn_bwd_args), bwd_args(B.pgcn_sage_bwd_args)
    for args in ((None, C.byref(a), C.byref(good)), (gcn.handle, None, C.byref(good)), (gcn.handle, C.byref(a), None),
                 (gcn.handle, C.byref(a), C.byref(good))):           # the last: a partition without a device
        assert B.lib.pgcn_layer_bwd_mx(*args, None) == B.PGCN_EINVAL
    for args in ((None, C.byref(b), C.byref(good)), (sage.handle, None, C.byref(good)), (sage.handle, C.byref(b), None),
                 (sage.handle, C.byref(b), C.byref(good))):
        assert B.lib.pgcn_sage_layer_bwd_mx(*args, None, None) == B.PGCN_EINVAL


def test_workspaces_of_layers_in_4_bits(parts):
    gcn, _ = parts
    size = lambda dt, order: B.pgcn_layer_workspace_size(gcn, 70, 30, dt, order)
    assert size(B.PGCN_MXFP4, B.PGCN_ORDER_AGG) >= max(size(dt, B.PGCN_ORDER_AGG) for dt in (B.PGCN_F32, B.PGCN_BF16)) - (1 << 20)
    assert size(B.PGCN_MXFP4, B.PGCN_ORDER_TRANSFORM) == 0
