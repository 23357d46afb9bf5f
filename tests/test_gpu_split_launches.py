"""Top logits of more rows than one launch holds (2^31 threads): rows on both sides of the border, and that
there are two launches indeed."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import ops
from paper_2203_10428_amd import binding as B
from test_gpu_distill import log_error, logits

pytestmark = pytest.mark.gpu


def launches(call):
    """Kernel nodes of a captured call, which does not run."""
    g = torch.cuda.CUDAGraph(keep_graph=True)
    with torch.cuda.graph(g):
        call(torch.cuda.current_stream())
    n = ctypes.c_size_t()
    get = B.lib.hipGraphGetNodes
    get.restype, get.argtypes = ctypes.c_int, [ctypes.c_void_p, ctypes.c_void_p, ctypes.POINTER(ctypes.c_size_t)]
    assert get(g.raw_cuda_graph(), None, ctypes.byref(n)) == 0
    return n.value


# a workgroup to a row; parts of a row, three workgroups of 512 threads each, and the launch that joins them
@pytest.mark.parametrize("C,K,most,one,two,gib", [(136, 129, 2 ** 23, 1, 2, 16), (32776, 66, 2 ** 22 // 3, 2, 3, 104)],
                         ids=["workgroup", "parts"])
def test_rows_on_both_sides_of_a_launch(C, K, most, one, two, gib):
    if torch.cuda.mem_get_info()[0] < gib << 30:
        torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < gib << 30:
        pytest.skip(f"needs {gib} GiB of device memory")
    rows = most + 3
    rng = np.random.default_rng(7)
    at = torch.tensor([0, 1, most - 1, most, rows - 1], device="cuda")
    Z = torch.zeros((rows, C), dtype=torch.bfloat16, device="cuda")
    Z[at] = torch.from_numpy(logits(rng, len(at), C)).to("cuda").to(torch.bfloat16)
    v = torch.full((rows, K), 7.0, device="cuda")
    i = torch.full((rows, K), 77, dtype=torch.int32, device="cuda")
    t = torch.full((rows,), 7.0, device="cuda")
    n = B.pgcn_top_logits_workspace_size(B.PGCN_BF16, rows, C, K)
    ws = torch.empty(max(n, 16), dtype=torch.uint8, device="cuda")

    def call(stream, rows=rows):
        B.pgcn_top_logits(dtype=B.PGCN_BF16, rows=rows, classes=C, ld=C, top=K, ld_top=K, temperature=1.0, Z=Z, top_values=v,
                          top_ids=i, tail_lse=t, workspace=ws, workspace_bytes=ws.numel(), stream=stream)

    assert launches(lambda s: call(s, most)) == one and launches(call) == two
    call(torch.cuda.current_stream())
    rv, ri, rt = ops.top_logits(Z[at].float().cpu().numpy().astype(np.float64), K, 1.0)
    assert np.array_equal(i[at].cpu().numpy(), ri) and np.array_equal(v[at].cpu().numpy().astype(np.float64), rv)
    assert (np.abs(t[at].cpu().numpy() - rt) <= log_error(4 * 12.0, rt)).all()
    # all others are rows of zeros: the first K classes, the rest's logarithm
    rest = torch.ones(rows, dtype=torch.bool, device="cuda")
    rest[at] = False
    order = torch.arange(K, dtype=torch.int32, device="cuda")
    assert bool(((i == order).all(1) & (v == 0).all(1))[rest].all())
    assert float((t[rest] - float(np.log(C - K))).abs().max()) <= log_error(0.0, np.log(C - K))
    del Z, v, i, t, ws
    torch.cuda.empty_cache()
