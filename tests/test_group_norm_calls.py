"""Group norm's calls: what they refuse on the way to the kernels, and sums over many samples (GPU)."""
import pytest

from paper_2305_11624_b200 import convbn as C

pytestmark = pytest.mark.gpu


def tensors(n, h, w, c, groups, dtype):
    import torch
    x = torch.randn(n, h, w, c, device="cuda", dtype=dtype)
    v = lambda: torch.ones(c, device="cuda")
    return x, torch.empty_like(x), v(), v(), torch.empty(2, n, groups, device="cuda")


def status(call, *args, **kw):
    with pytest.raises(C.ConvBNError) as e:
        call(*args, **kw)
    return e.value.status


def test_four_dimensions_in_another_order():
    """As many elements, channels and rows, but samples and columns change places."""
    import torch
    d = C.NormDesc.make(2, 32, 4, 6, 8, dtype=C.BF16)
    x, z, gamma, beta, saved = tensors(2, 4, 6, 32, 8, torch.bfloat16)
    ws = torch.empty(C.convbn_group_norm_workspace_bytes(d), dtype=torch.uint8, device="cuda")
    other = lambda t: t.view(6, 4, 2, 32)
    for x_, z_ in ((other(x), z), (x, other(z)), (x.view(1, 4, 12, 32), z)):
        assert status(C.convbn_group_norm_fwd, d, x_, gamma, beta, z_, saved, ws) == C.EINVAL
    C.convbn_group_norm_fwd(d, x, gamma, beta, z, saved, ws)
    # without four dimensions, as rows, or as a permuted view: the same memory
    again = torch.empty_like(z)
    C.convbn_group_norm_fwd(d, x.view(-1, 32), gamma, beta, again.view(-1), saved, ws)
    assert torch.equal(again, z)
    C.convbn_group_norm_fwd(d, x.permute(0, 3, 1, 2), gamma, beta, again.zero_().permute(0, 3, 1, 2), saved, ws)
    assert torch.equal(again, z)
    dx, dg, db = torch.empty_like(x), torch.empty_like(gamma), torch.empty_like(beta)
    assert status(C.convbn_group_norm_bwd, d, z, x, gamma, beta, saved, other(dx), dg, db, ws) == C.EINVAL
    C.convbn_check()


@pytest.mark.parametrize("c", [4, 6])                        # on chip; two passes
def test_gradients_of_vectors_over_many_samples(c):
    """Sums that fp32 additions one after the other lose: 32 large gradients, one for each warp, and many small ones.  Pairs of channels
    hold (1, -1): xhat is that.  Tolerance: a value takes part in 15 fp32 additions at most, each off by half a step, 2^-24, of the
    large ones' sum; then the result's own half step."""
    import torch
    n, groups = 65536 + 32, c // 2
    d = C.NormDesc.make(n, c, 1, 1, groups, dtype=C.F32, eps=0.0)
    sign = torch.tensor([1.0, -1.0], device="cuda").repeat(groups)
    x, dx = sign.expand(n, 1, 1, c).contiguous(), torch.empty(n, 1, 1, c, device="cuda")
    dz = torch.ones(n, 1, 1, c, device="cuda")
    dz[:32] = 2.0 ** 24
    gamma, beta, dgamma, dbeta = (torch.ones(c, device="cuda") for _ in range(4))
    saved = torch.cat((torch.zeros(1, n, groups), torch.ones(1, n, groups))).cuda()
    ws = torch.empty(C.convbn_group_norm_workspace_bytes(d), dtype=torch.uint8, device="cuda")
    C.convbn_group_norm_bwd(d, dz, x, gamma, beta, saved, dx, dgamma, dbeta, ws)
    C.convbn_check()
    exact, allowed = 2.0 ** 29 + 65536, 15 * 2.0 ** -24 * 2.0 ** 29 + 32
    assert bool(((dbeta - exact).abs() <= allowed).all()) and bool(((dgamma - exact * sign).abs() <= allowed).all())
    assert allowed < 65536 / 16
