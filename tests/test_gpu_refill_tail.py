"""Device refills whose size is no multiple of 16 bytes, as messages in 8 and 4 bits have: the copy kernel takes them too,
from 4 MiB on, and copies no byte more or less."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2203_10428_amd import binding as B
from paper_2203_10428_amd import configs, synth
from paper_2203_10428_amd.step import PartitionTrainer, StepOptions

pytestmark = pytest.mark.gpu
MIN = 4 << 20


def nodes(call):
    """Types of the nodes of a captured call, which does not run: 0 a kernel, 1 the runtime's copy."""
    g = torch.cuda.CUDAGraph(keep_graph=True)
    with torch.cuda.graph(g):
        call(torch.cuda.current_stream())
    n = ctypes.c_size_t()
    get, kind = B.lib.hipGraphGetNodes, B.lib.hipGraphNodeGetType
    get.restype, get.argtypes = ctypes.c_int, [ctypes.c_void_p, ctypes.c_void_p, ctypes.POINTER(ctypes.c_size_t)]
    kind.restype, kind.argtypes = ctypes.c_int, [ctypes.c_void_p, ctypes.POINTER(ctypes.c_int)]
    assert get(g.raw_cuda_graph(), None, ctypes.byref(n)) == 0
    at = (ctypes.c_void_p * n.value)()
    assert get(g.raw_cuda_graph(), at, ctypes.byref(n)) == 0
    out = []
    for node in at:
        t = ctypes.c_int(-1)
        assert kind(node, ctypes.byref(t)) == 0
        out.append(t.value)
    return out


@pytest.mark.parametrize("nbytes", [MIN, MIN + 1, MIN + 4, MIN + 15, MIN + 16, MIN + 16 * 1024 + 12, 3 * MIN + 7])
def test_sizes_that_are_no_multiple_of_16(nbytes):
    src = torch.randint(0, 256, (nbytes + 256,), dtype=torch.uint8, device="cuda")
    dst = torch.full_like(src, 0xA5)
    call = lambda st: B.pgcn_refill_async(dst, src, nbytes, 0, st)
    assert nodes(call) == [0]
    torch.cuda.synchronize()
    assert (dst == 0xA5).all()
    call(torch.cuda.current_stream())
    torch.cuda.synchronize()
    assert torch.equal(dst[:nbytes], src[:nbytes]) and (dst[nbytes:] == 0xA5).all()


def test_small_and_unaligned_refills_go_to_the_runtime():
    src, dst = (torch.zeros(MIN + 64, dtype=torch.uint8, device="cuda") for _ in range(2))
    for d, s, n in ((dst, src, MIN - 1), (dst[4:], src, MIN), (dst, src[8:], MIN)):
        assert nodes(lambda st: B.pgcn_refill_async(d, s, n, 0, st)) == [1]


@pytest.mark.parametrize("bits", [8, 4])
def test_large_messages_of_a_step(bits):
    """Boundary rows of an odd number, more than 4 MiB of them, arrive as they were sent."""
    w, f = configs.TINY, 10000
    g = synth.tiny_uniform(2002, 10000, 2, seed=1)
    rng = np.random.default_rng(1)
    X, labels = rng.standard_normal((g.n, f)).astype(np.float32), rng.integers(0, 8, g.n).astype(np.int32)
    W = [rng.uniform(-0.02, 0.02, s).astype(np.float32) for s in ((f, 16), (16, 8))]
    tr = PartitionTrainer(g, X, labels, W, (f, 16, 8), w.loss, w.loss_scale, "f32",
                          StepOptions(gamma=w.gamma, eta=w.eta, copy_mode="pipe", exchange_bits=bits))
    sent = tr.remote_fq[1].bytes
    assert sent.numel() > MIN and sent.numel() % 16 != 0
    assert nodes(lambda st: tr._refill_features(1, tr.feat[1][0], st)) == [0]
    for _ in range(3):
        tr.step()
    tr.synchronize()
    assert torch.isfinite(tr.loss).all()
    for buf in tr.feat[1]:
        assert torch.equal(buf.bytes, sent)
