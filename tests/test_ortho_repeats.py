"""Orthogonal updates give the same bits every time: nothing in them depends on which of two things ends first."""
import pytest

from paper_2305_11624_b200 import convbn as C

pytestmark = pytest.mark.gpu


def same_bits(shape, dtype, steps=5, times=20):
    import torch
    t = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[dtype]
    gen = torch.Generator(device="cuda").manual_seed(3)
    g = (1e-3 * torch.randn(*shape, generator=gen, device="cuda")).to(t)
    ws = torch.empty(C.convbn_orthogonalise_workspace_bytes(*shape[1:], shape[0]), dtype=torch.uint8, device="cuda")
    outs = []
    for k in range(times):
        ws.fill_(255 * (k % 2))
        out = torch.empty_like(g)
        C.convbn_orthogonalise(g, out, steps, 1e-7, ws)
        outs.append(out)
    C.convbn_check()
    assert bool(torch.isfinite(outs[0].float()).all())
    return [int((o != outs[0]).sum()) for o in outs[1:]]


@pytest.mark.parametrize("shape,dtype", [((2, 2048, 8192), "bf16"), ((1, 4096, 1000), "f16"), ((1, 512, 4608), "f32"), ((1, 700, 900), "bf16"),
                                         ((3, 300, 1030), "f32"), ((1, 1500, 1400), "f16")], ids=str)
def test_large_matrices(shape, dtype):
    assert not any(same_bits(shape, dtype))


# (clusters of 2, 4, 8 and 16 blocks; all of A's rows in one block's share, or in some; tall ones; more matrices than run at a time)
CLUSTERS = [(1, 128, 1152), (1, 1152, 128), (1, 64, 300), (1, 16, 2268), (3, 100, 4000), (2, 4096, 128), (1, 33, 1025), (20, 128, 600)]


@pytest.mark.parametrize("shape", CLUSTERS, ids=str)
def test_clusters(shape):
    """Blocks of a cluster send one another rows of A by copies that nothing in the sending block waits for, and write P where A was."""
    assert not any(same_bits(shape, "f32", times=100))


@pytest.mark.parametrize("kind", ["noise", "few"])
@pytest.mark.parametrize("shape", CLUSTERS, ids=str)
def test_clusters_are_as_near_as_the_formula_in_fp32(shape, kind):
    """Tolerance, 2-norm.  X, A and P are rounded to 22 bits where the fp32 formula rounds these and what lies between them to 24: at most four
    times its error.  An MMA cuts its sum below 2^-23, by half of that in the mean; 16 of them on an accumulator, of at most 256 columns, are
    2^-20 of A, which moves X by at most 0.9 as much of itself, in each of five steps.  A row whose low halves were lost would be off by 2^-12."""
    import numpy as np
    from oracle import muon_oracle as M
    from test_muon import matrices, orthogonalise
    g = matrices(kind, *shape, seed=6)
    got = orthogonalise(g).double().cpu().numpy()
    a, b, c = (np.float32(v) for v in M.COEFFICIENTS)
    for i in {0, shape[0] - 1}:
        ref = M.orthogonalise(g[i].double().numpy(), 5, 1e-7)
        x = g[i].numpy() / np.float32(np.linalg.norm(g[i].double().numpy()))
        for _ in range(5):
            s = x @ x.T if shape[1] <= shape[2] else x.T @ x
            p = b * s + c * (s @ s)
            x = a * x + (p @ x if shape[1] <= shape[2] else x @ p)
        allowed = 4 * np.linalg.norm(x - ref) + 5 * 2.0 ** -20 * np.linalg.norm(ref)
        assert np.linalg.norm(got[i] - ref) <= allowed, np.linalg.norm(got[i] - ref) / allowed


def test_threads_that_ask_at_once():
    """The first calls of a process, made by four threads on streams of their own, choose the same kernel and give the same bits."""
    import subprocess
    import sys
    import os
    code = '''
import threading, torch
from paper_2305_11624_b200 import convbn as C
g = torch.randn(100, 2000, device="cuda")
out, ws = [torch.empty_like(g) for _ in range(5)], [torch.empty(C.convbn_orthogonalise_workspace_bytes(100, 2000), dtype=torch.uint8, device="cuda") for _ in range(5)]
streams, gate = [torch.cuda.Stream() for _ in range(4)], threading.Barrier(4)
torch.cuda.synchronize()
def one(k):
    gate.wait()
    C.convbn_orthogonalise(g, out[k], 5, 1e-7, ws[k], stream=streams[k])
threads = [threading.Thread(target=one, args=(k,)) for k in range(4)]
for t in threads: t.start()
for t in threads: t.join()
torch.cuda.synchronize()
C.convbn_orthogonalise(g, out[4], 5, 1e-7, ws[4])
C.convbn_check()
assert all(torch.equal(o, out[4]) for o in out[:4])
'''
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", code], cwd=root, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]
