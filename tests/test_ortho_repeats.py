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
