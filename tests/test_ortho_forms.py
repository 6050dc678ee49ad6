"""The large kernel's forms: direct steps, stages of several steps over m x m matrices, each storage type (GPU).

Tolerance (2-norm): the formula in fp32, run here, shows what the steps make of roundings.  Pairs of halves have 22 bits for 24: four times its
error at most; stages form A again only every two or three steps: four times that.  The tensor core's sums of up to 1024 terms lose 2^-17 of the
result in five steps, and a fifth of that more for each further one.  Storing adds half a step of the type."""
import numpy as np
import pytest

from oracle import muon_oracle as M
from paper_2305_11624_b200 import convbn as C
from test_muon import HALF_STEP, matrices, orthogonalise

pytestmark = pytest.mark.gpu


def plain(g, steps):
    """The formula in fp32."""
    x = g.astype(np.float32) / np.float32(np.linalg.norm(g.astype(np.float64)))
    a, b, c = (np.float32(v) for v in M.COEFFICIENTS)
    wide = g.shape[0] <= g.shape[1]
    for _ in range(steps):
        s = x @ x.T if wide else x.T @ x
        p = b * s + c * (s @ s)
        x = a * x + (p @ x if wide else x @ p)
    return x


def check(got, g, steps, half, staged):
    ref = M.orthogonalise(g.astype(np.float64), steps, 1e-7)
    size = np.linalg.norm(ref)
    allowed = (16 if staged else 4) * np.linalg.norm(plain(g, steps) - ref) + (2.0 ** -17 * max(1.0, steps / 5) + half) * size
    off = np.linalg.norm(got.astype(np.float64) - ref)
    assert off <= allowed, off / allowed


@pytest.mark.parametrize("steps", [1, 2, 4, 5, 7])
@pytest.mark.parametrize("dtype,shape,staged", [("bf16", (300, 1030), True), ("f16", (1030, 300), True), ("bf16", (701, 905), False),
                                                ("f16", (3, 257, 333), False), ("f16", (2, 1100, 2601), True), ("f32", (1030, 300), False)], ids=str)
def test_types(dtype, shape, staged, steps):
    import torch
    t = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[dtype]
    stack = matrices("noise", *(shape if len(shape) == 3 else (1, *shape)), seed=8).to(t)
    got = orthogonalise(stack.view(shape), steps).view(stack.shape)
    for i in {0, len(stack) - 1}:
        check(got[i].float().cpu().numpy(), stack[i].float().numpy(), steps, HALF_STEP[dtype], staged)


@pytest.mark.parametrize("kind", ["noise", "few"])
@pytest.mark.parametrize("steps", [1, 2, 3, 4, 5, 7])
def test_stages_in_fp32(steps, kind):
    """A Muon step from nothing, lr 1, leaves the update itself in the fp32 weights, which is formed in stages where the heaviest layer is long."""
    import torch
    shapes = [(300, 1030), (2304, 256), (400, 330)]
    grads = [matrices(kind, 1, *s, seed=k)[0] for k, s in enumerate(shapes)]
    dev = [(g.cuda(), torch.zeros_like(g, device="cuda"), torch.zeros_like(g, device="cuda"), None) for g in grads]
    layers = C.MuonLayers(dev)
    ws = torch.empty(C.convbn_muon_workspace_bytes(layers), dtype=torch.uint8, device="cuda")
    C.convbn_muon_step(layers, C.MuonParams.make(lr=1.0, momentum=0.0, steps=steps), ws)
    C.convbn_check()
    for g, (_, _, master, _) in zip(grads, dev):
        scale = max(1.0, g.shape[0] / g.shape[1]) ** 0.5
        # (the scale is a rounded fp32 number too)
        check(master.cpu().numpy() / -scale, g.numpy(), steps, 2 * HALF_STEP["f32"], True)


def test_many_steps_stay_in_their_bounds():
    """64 steps, direct and in stages: singular values stay where the steps keep them, whichever they have come to."""
    import torch
    for dtype, shape in (("f32", (200, 260)), ("bf16", (150, 1000))):
        g = matrices("noise", 1, *shape, seed=2)[0].to({"f32": torch.float32, "bf16": torch.bfloat16}[dtype])
        s = torch.linalg.svdvals(orthogonalise(g, 64).double().cpu())
        assert bool((s > 0.3).all()) and bool((s < 1.25).all())
