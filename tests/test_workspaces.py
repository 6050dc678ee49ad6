"""Workspaces of the group norm and of the optimiser's calls: memory of another device, or in several pieces, is refused before an address is taken.
(CPU: tensors that say they are on GPU 0; GPU: the calls themselves.)"""
import pytest
import torch

from paper_2305_11624_b200 import convbn as C


class OnGpu:
    """A CPU tensor that says it is on GPU 0."""
    is_cuda = True

    def __init__(self, t):
        self._t = t

    def get_device(self):
        return 0

    def __getattr__(self, name):
        return getattr(self._t, name)


def status(call, *args, **kw):
    with pytest.raises(C.ConvBNError) as e:
        call(*args, **kw)
    return e.value.status


def calls(place):
    """(call of a workspace, bytes it needs) of every entry point"""
    zeros = lambda *shape: place(torch.zeros(*shape))
    g, out = zeros(40, 50), zeros(40, 50)
    yield lambda ws: C.convbn_orthogonalise(g, out, 5, 1e-7, ws), C.convbn_orthogonalise_workspace_bytes(40, 50)
    layers = C.MuonLayers([tuple(zeros(40, 50) for _ in range(3)) + (None,)])
    yield lambda ws: C.convbn_muon_step(layers, C.MuonParams.make(), ws), C.convbn_muon_workspace_bytes(layers)
    d = C.NormDesc.make(2, 32, 4, 4, 8, dtype=C.F32)
    x, z, gamma, beta, saved, dgamma, dbeta = zeros(2, 4, 4, 32), zeros(2, 4, 4, 32), *(zeros(n) for n in (32, 32, 32, 32, 32))
    need = C.convbn_group_norm_workspace_bytes(d)
    yield lambda ws: C.convbn_group_norm_fwd(d, x, gamma, beta, z, saved, ws), need
    yield lambda ws: C.convbn_group_norm_bwd(d, x, x, gamma, beta, saved, z, dgamma, dbeta, ws), need


def look(place, expand):
    for call, need in calls(place):
        assert status(call, torch.zeros(need, dtype=torch.uint8)) == C.EINVAL                                  # host memory
        again = expand(place(torch.zeros(64, dtype=torch.uint8)), need // 64 + 1, 64)                          # (64 bytes that say they are more)
        assert status(call, again) == C.EINVAL


@pytest.mark.skipif(torch.cuda.is_available(), reason="tensors that are not where they say they are")
def test_looked_at_on_the_host(monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    look(OnGpu, lambda t, *shape: OnGpu(t._t.expand(*shape)))


@pytest.mark.gpu
def test_refused_on_the_way_to_a_gpu():
    look(lambda t: t.cuda(), lambda t, *shape: t.expand(*shape))
    for call, _ in calls(lambda t: t.cuda()):
        assert status(call, None) == C.EWORKSPACE
    C.convbn_check()
