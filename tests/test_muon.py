"""Orthogonal updates: the oracle, refusals (CPU), the kernels against the oracle (GPU).

Tolerance (2-norm of a whole matrix).  Every step rounds X to a pair of halves and leaves out the smallest of four products: 2^-22 of X each, as
often for P: four of them.  What is left of the steps lifts an error by as much as a small singular value, 3.4445 a step, and X itself
grows no more than that, so each step adds at most 4 * 2^-22 * 3.4445^steps to an X that began with norm 1.  The tensor core's sums of 1024 terms
lose up to 64 * 2^-24 of A, against which X does not grow: 2^-17 of the result.  Storing adds half a step of the type."""
import ctypes
import math

import numpy as np
import pytest

from oracle import muon_oracle as M
from paper_2305_11624_b200 import convbn as C

HALF_STEP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
EPS = 1e-7


def status(call, *args, **kw):
    with pytest.raises(C.ConvBNError) as e:
        call(*args, **kw)
    return e.value.status


# ---- the oracle ----------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("shape", [(5, 5), (3, 9), (9, 3), (1, 4), (4, 1)])
def test_oracle_acts_on_singular_values(shape):
    g = np.random.default_rng(1).standard_normal(shape)
    assert np.allclose(M.orthogonalise(g, 5, EPS), M.orthogonalise_by_svd(g, 5, EPS), atol=1e-9)
    s = np.linalg.svd(M.orthogonalise(g, 5, EPS), compute_uv=False)
    assert (s > 0.3).all() and (s < 1.21).all()


def test_oracle_step_by_hand():
    v, w = M.muon_step([[2.0]], [[1.0]], [[10.0]], 0.1, 0.5, 0.2, 0.0, True, 1)
    # v = 0.5 + 2, u = 2 + 1.25 -> 1; one step: 3.4445 - 4.775 + 2.0315 = 0.701
    assert np.allclose(v, 2.5) and np.allclose(w, 0.98 * 10 - 0.1 * 0.701)


# ---- refusals ------------------------------------------------------------------------------------------------------
def test_orthogonalise_refusals():
    at, need = 4096, C.convbn_orthogonalise_workspace_bytes(100, 300, 2)
    assert need > 0 and need % 256 == 0
    raw = C.lib().convbn_orthogonalise
    good = dict(dtype=C.F32, g=at, out=at, rows=100, cols=300, count=2, steps=5, eps=EPS, ws=at, bytes_=need)
    go = lambda **kw: raw(*{**good, **kw}.values(), 0)
    for kw in (dict(dtype=3), dict(rows=0), dict(cols=-1), dict(count=-1), dict(steps=0), dict(steps=65), dict(eps=-1.0), dict(eps=math.nan),
               dict(g=None), dict(out=None), dict(rows=1 << 20, cols=(1 << 11) + 1), dict(rows=1, cols=1 << 20, count=1 << 20)):
        assert go(**kw) == C.EINVAL, kw
    assert go(g=at + 2) == C.EALIGN and go(out=at + 1) == C.EALIGN and go(ws=at + 128) == C.EALIGN
    assert go(ws=None) == C.EWORKSPACE and go(bytes_=need - 1) == C.EWORKSPACE
    assert go(count=0, g=None, out=None, ws=None, bytes_=0) == C.OK
    assert C.convbn_orthogonalise_workspace_bytes(0, 4) == 0 and C.convbn_orthogonalise_workspace_bytes(4, 4, -1) == 0


def test_orthogonalise_tensors():
    import torch
    g = torch.zeros(4, 6)
    call = lambda g, out: status(C.convbn_orthogonalise, g, out, 5, EPS, 4096, 1 << 30, stream=0)
    assert call(g, torch.zeros(4, 6)) == C.EINVAL                       # not on a GPU
    assert call(g, torch.zeros(6, 4)) == C.EINVAL and call(g, g.half()) == C.EINVAL
    assert call(g.t(), g.t()) == C.EINVAL and call(torch.zeros(3), torch.zeros(3)) == C.EINVAL
    with pytest.raises(TypeError):
        C.convbn_orthogonalise(g.double(), g.double(), 5, EPS, 4096, 1 << 30, stream=0)


def _layer(rows=4, cols=6, grad=4096, momentum=8192, master=12288, weight=16384):
    return C._MuonLayer(rows, cols, grad, momentum, master, weight)


def test_muon_refusals():
    raw, size = C.lib().convbn_muon_step, C.lib().convbn_muon_workspace_bytes

    def go(layers=None, count=None, dtype=C.BF16, ws=4096, bytes_=1 << 40, params=None, **kw):
        layers = [_layer(**kw)] if layers is None else layers
        array = (C._MuonLayer * len(layers))(*layers)
        return raw(ctypes.addressof(array), len(layers) if count is None else count, dtype, params or C.MuonParams.make(), ws, bytes_, 0)
    P = C.MuonParams.make
    for kw in (dict(rows=0), dict(cols=-3), dict(rows=1 << 20, cols=1 << 12), dict(grad=None), dict(momentum=None), dict(master=None), dict(dtype=5),
               dict(count=-1), dict(params=P(steps=0)), dict(params=P(steps=65)), dict(params=P(eps=-1)), dict(params=P(lr=math.nan)),
               dict(params=P(momentum=math.inf)), dict(params=P(weight_decay=math.nan))):
        assert go(**kw) == C.EINVAL, kw
    assert go(grad=4098) == C.EALIGN and go(weight=16385) == C.EALIGN and go(weight=16386, dtype=C.F32) == C.EALIGN
    assert go(ws=None) == C.EWORKSPACE and go(bytes_=1024) == C.EWORKSPACE and go(ws=4100) == C.EALIGN
    assert raw(None, 0, C.BF16, P(), None, 0, 0) == C.OK and raw(None, 1, C.BF16, P(), None, 0, 0) == C.EINVAL
    assert raw(None, 0, C.BF16, None, None, 0, 0) == C.EINVAL
    # a launch takes 64 layers: the workspace is that of the largest launch
    many = (C._MuonLayer * 130)(*[_layer() for _ in range(130)])
    assert size(ctypes.addressof(many), 130) == size(ctypes.addressof(many), 64) <= 64 * size(ctypes.addressof(many), 1)


def test_muon_layers_are_looked_at():
    import torch
    t = lambda *s, dtype=torch.float32: torch.zeros(*s, dtype=dtype)
    bad = lambda *layer: status(C.MuonLayers, [layer])
    assert bad(t(4, 6), t(4, 6), t(4, 6), None) == C.EINVAL                                  # not on a GPU
    assert bad(t(4, 6).half(), t(4, 6), t(4, 6), None) == C.EINVAL and bad(None, t(4, 6), t(4, 6), None) == C.EINVAL
    assert bad(t(4, 6), t(4, 5), t(4, 6), None) == C.EINVAL and bad(t(6, 4).t(), t(4, 6), t(4, 6), None) == C.EINVAL
    assert bad(t(()), t(()), t(()), None) == C.EINVAL


# ---- the kernels ----------------------------------------------------------------------------------------------------
def matrices(kind, count, rows, cols, seed=0):
    """[count][rows][cols] fp32"""
    import torch
    gen = torch.Generator().manual_seed(seed)
    g = torch.randn(count, rows, cols, generator=gen)
    if kind == "few":                          # few strong directions and noise
        k = max(1, min(rows, cols) // 8)
        g = torch.randn(count, rows, k, generator=gen) @ torch.randn(count, k, cols, generator=gen) + 0.01 * g
    return 1e-3 * g


def allowed(ref, dtype, steps):
    return steps * 4 * 2.0 ** -22 * 3.4445 ** steps + (2.0 ** -17 + HALF_STEP[dtype]) * np.linalg.norm(ref)


def orthogonalise(g, steps=5, eps=EPS, in_place=False, stream=None):
    import torch
    g = g.cuda()
    out = g if in_place else torch.full_like(g, float("nan"))
    count = g.shape[0] if g.dim() == 3 else 1
    ws = torch.full((C.convbn_orthogonalise_workspace_bytes(*g.shape[-2:], count),), 255, dtype=torch.uint8, device="cuda")
    C.convbn_orthogonalise(g, out, steps, eps, ws, stream=stream)
    C.convbn_check(stream)
    return out


SHAPES = [(1, 1), (1, 7), (7, 1), (64, 64), (64, 147), (147, 64), (100, 33), (96, 9), (128, 128), (129, 257), (257, 129), (384, 128), (130, 2100),
          (2100, 130), (513, 70), (300, 1030), (128, 2048), (2048, 127), (17, 1025), (3, 4000), (33, 300), (129, 129)]


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["noise", "few"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_orthogonalise(shape, kind):
    g = matrices(kind, 1, *shape)[0]
    got = orthogonalise(g).double().cpu().numpy()
    ref = M.orthogonalise(g.double().numpy(), 5, EPS)
    off = np.linalg.norm(got - ref)
    assert off <= allowed(ref, "f32", 5), off / allowed(ref, "f32", 5)


@pytest.mark.gpu
@pytest.mark.parametrize("count,rows,cols", [(1, 16, 2268), (2, 4096, 128), (1, 3001, 30), (9, 64, 2052), (1, 40, 4097), (16, 128, 1500), (40, 36, 1030), (300, 8, 12)])
def test_lengths_and_stacks_on_either_side_of_the_choices(count, rows, cols):
    """One matrix on chip in a cluster, as many as run at a time, and more; elements by fours, and one off where fours could lie."""
    import torch
    g = matrices("noise", count, rows, cols)
    got = orthogonalise(g)
    for i in {0, count // 2, count - 1}:
        ref = M.orthogonalise(g[i].double().numpy(), 5, EPS)
        assert np.linalg.norm(got[i].double().cpu().numpy() - ref) <= allowed(ref, "f32", 5)
    room = torch.full((2, count * rows * cols + 2), 7.0, device="cuda")
    room[0, 1:-1] = g.flatten().cuda()
    views = [r[1:-1].view(count, rows, cols) for r in room]
    ws = torch.empty(C.convbn_orthogonalise_workspace_bytes(rows, cols, count), dtype=torch.uint8, device="cuda")
    C.convbn_orthogonalise(views[0], views[1], 5, EPS, ws)
    C.convbn_check()
    close = [np.linalg.norm((a - b).double().cpu().numpy()) for a, b in zip(views[1], got)]
    # (the norm's squares are added up in another order, in 64 bits: at most a rounding of the scale)
    assert max(close) <= 2 * allowed(M.orthogonalise(g[0].double().numpy(), 5, EPS), "f32", 5)
    assert room[1, 0] == 7 and room[1, -1] == 7


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [(64, 64), (256, 1152), (1152, 256), (512, 2048)], ids=str)
def test_as_near_as_documented(shape):
    """As near as the formula in fp32 comes.  That is 1e-5 for these matrices, whose noise, 2^-8 of the whole, becomes most of the result:
    in exact arithmetic, X rounded to 24 bits once a step moves it by 2.7e-6 to 4.5e-6, and each step of the fp32 formula rounds three
    products and two sums (64 x 64: 1.27e-5).  Pairs of halves have two bits less and half as many roundings: twice that error."""
    g = matrices("few", 1, *shape, seed=4)[0]
    ref = M.orthogonalise(g.double().numpy(), 5, EPS)
    x = g.numpy() / np.float32(np.linalg.norm(g.double().numpy()))
    a, b, c = (np.float32(v) for v in M.COEFFICIENTS)
    for _ in range(5):
        s = x @ x.T if shape[0] <= shape[1] else x.T @ x
        p = b * s + c * (s @ s)
        x = a * x + (p @ x if shape[0] <= shape[1] else x @ p)
    assert np.linalg.norm(orthogonalise(g).double().cpu().numpy() - ref) <= 2 * np.linalg.norm(x - ref)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("steps", [1, 2, 7])
def test_stacks_and_types(dtype, steps):
    import torch
    g = matrices("noise", 3, 90, 201).to({"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}[dtype])
    got = orthogonalise(g, steps).double().cpu().numpy()
    for i in range(3):
        ref = M.orthogonalise(g[i].double().numpy(), steps, EPS)
        assert np.linalg.norm(got[i] - ref) <= allowed(ref, dtype, steps)
    assert torch.equal(orthogonalise(g, steps, in_place=True).cpu().double(), torch.from_numpy(got))


@pytest.mark.gpu
@pytest.mark.parametrize("scale", [1e-30, 1e-18, 1e18, 1e30])
def test_range_of_the_norm(scale):
    """The squares leave fp32's range."""
    g = (matrices("noise", 1, 70, 90)[0].double() * 1e3 * scale).float()
    ref = M.orthogonalise(g.double().numpy(), 5, 0.0)
    assert np.linalg.norm(orthogonalise(g, eps=0.0).double().cpu().numpy() - ref) <= allowed(ref, "f32", 5)


@pytest.mark.gpu
def test_zeros_and_what_is_no_number():
    import torch
    g = matrices("noise", 4, 130, 200)
    clean = orthogonalise(g)
    g[1] = 0.0
    g[2, 3, 4] = float("nan")
    g[3, 129, 199] = float("inf")
    got = orthogonalise(g)
    assert torch.equal(got[0], clean[0]) and bool((got[1] == 0).all()) and bool(torch.isnan(got[2:]).all())


def muon(layers, dtype, params, repeat=1, graph=False):
    """layers: (grad, momentum, master) fp32 on the CPU -> (momentum, master, weight) after `repeat` steps"""
    import torch
    t = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": None}[dtype]
    dev = [(g.cuda(), v.cuda().clone(), m.cuda().clone(), torch.full_like(m, float("nan"), dtype=t, device="cuda") if t else None)
           for g, v, m in layers]
    table = C.MuonLayers(dev)
    ws = torch.full((C.convbn_muon_workspace_bytes(table),), 255, dtype=torch.uint8, device="cuda")
    for _ in range(repeat):
        C.convbn_muon_step(table, params, ws)
    C.convbn_check()
    return [d[1:] for d in dev]


def check_muon(layers, got, dtype, p):
    for (g, v, m), (v1, m1, w1) in zip(layers, got):
        flat = lambda t: t.reshape(t.shape[0], -1).double().cpu().numpy()
        V, W = M.muon_step(flat(g), flat(v), flat(m), p.lr, p.momentum, p.weight_decay, p.eps, bool(p.nesterov), p.steps)
        # coefficients are fp32 too: three half steps
        assert (np.abs(flat(v1) - V) <= 3 * 2.0 ** -24 * (np.abs(flat(g)) + np.abs(p.momentum * flat(v)))).all()
        rows, cols = W.shape
        scale = p.lr * math.sqrt(max(1.0, rows / cols))
        X = (flat(m) * (1 - p.lr * p.weight_decay) - W) / scale
        off = np.linalg.norm(flat(m1) - W)
        # the update's input is rounded too: 2^-22 more of it a step
        assert off <= 2 * scale * allowed(X, "f32", p.steps) + 3 * 2.0 ** -24 * np.linalg.norm(flat(m)), off
        if w1 is not None:
            import torch
            assert torch.equal(w1, m1.to(w1.dtype))


def some_layers(shapes, seed=0):
    import torch
    gen = torch.Generator().manual_seed(seed)
    rn = lambda *s: torch.randn(*s, generator=gen)
    return [(1e-3 * rn(*s), 5e-3 * rn(*s), 0.1 * rn(*s)) for s in shapes]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,nesterov", [("bf16", True), ("f16", False), ("f32", True)])
def test_muon_step(dtype, nesterov):
    layers = some_layers([(64, 7, 7, 3), (64, 64), (256, 3, 3, 64), (130, 1, 1, 70), (96, 3, 3, 1), (10, 500), (5,), (1, 1)])
    p = C.MuonParams.make(lr=0.02, momentum=0.95, weight_decay=0.1, nesterov=nesterov)
    check_muon(layers, muon(layers, dtype, p), dtype, p)


@pytest.mark.gpu
def test_muon_more_layers_than_a_launch_takes():
    layers = some_layers([(8 + i % 5, 20 + i) for i in range(150)])
    p = C.MuonParams.make(lr=0.1, momentum=0.9)
    check_muon(layers, muon(layers, "bf16", p), "bf16", p)


@pytest.mark.gpu
def test_muon_repeats_itself():
    """The same bits from the same list; a layer by itself is right too (what else is in the list decides the kernel and how sums are cut); a
    captured step is the eager one."""
    import torch
    layers = some_layers([(64, 147), (130, 300), (512, 128)])
    p = C.MuonParams.make(lr=0.02, weight_decay=0.01)
    both = muon(layers, "bf16", p)
    assert all(torch.equal(a, b) for x, y in zip(muon(layers, "bf16", p), both) for a, b in zip(x, y))
    for layer in layers:
        check_muon([layer], muon([layer], "bf16", p), "bf16", p)
    twice = muon(layers, "bf16", p, repeat=2)
    dev = [(g.cuda(), v.cuda().clone(), m.cuda().clone(), m.cuda().to(torch.bfloat16)) for g, v, m in layers]
    table = C.MuonLayers(dev)
    ws = torch.empty(C.convbn_muon_workspace_bytes(table), dtype=torch.uint8, device="cuda")
    C.convbn_muon_step(table, p, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        C.convbn_muon_step(table, p, ws)
    graph.replay()
    C.convbn_check()
    for a, b in zip(twice, dev):
        assert all(torch.equal(x, y) for x, y in zip(a, b[1:]))


@pytest.mark.gpu
def test_two_streams_with_workspaces_of_their_own():
    import torch
    g = [matrices("noise", 1, 300, 400, seed=i)[0].cuda() for i in range(2)]
    ref = [orthogonalise(t) for t in g]
    streams = [torch.cuda.Stream() for _ in range(2)]
    ws = [torch.empty(C.convbn_orthogonalise_workspace_bytes(300, 400), dtype=torch.uint8, device="cuda") for _ in range(2)]
    out = [torch.empty_like(t) for t in g]
    torch.cuda.synchronize()
    for _ in range(10):
        for k in range(2):
            C.convbn_orthogonalise(g[k], out[k], 5, EPS, ws[k], stream=streams[k])
    torch.cuda.synchronize()
    C.convbn_check()
    assert all(torch.equal(a, b) for a, b in zip(ref, out))


@pytest.mark.gpu
@pytest.mark.parametrize("eps", [0.0, 1e-300, 1e-7])
@pytest.mark.parametrize("rows,cols", [(20, 30), (64, 700), (130, 200)])
def test_a_zero_matrix_whatever_eps_is(rows, cols, eps):
    """Zeros on chip, in a cluster and in tiles; beside it what is no number still is none, and the smallest numbers are as good as any."""
    import torch
    g = torch.zeros(4, rows, cols)
    g[1] = matrices("noise", 1, rows, cols)[0] * 1e3
    g[2] = (g[1].double() * 2.0 ** -126).float()
    g[3, 1, 2] = float("nan")
    got = orthogonalise(g, eps=eps)
    assert bool((got[0] == 0).all()) and bool(torch.isnan(got[3]).all())
    for i in (1, 2) if eps < 1e-7 else (1,):
        ref = M.orthogonalise(g[i].double().numpy(), 5, eps)
        assert np.linalg.norm(got[i].double().cpu().numpy() - ref) <= allowed(ref, "f32", 5)


@pytest.mark.gpu
@pytest.mark.parametrize("rows,cols", [(20, 30), (130, 200)])
def test_muon_step_of_nothing(rows, cols):
    """A layer that had no gradient yet: its weights decay and stay numbers, also without eps."""
    import torch
    zero, master = torch.zeros(rows, cols), torch.randn(rows, cols, generator=torch.Generator().manual_seed(1))
    p = C.MuonParams.make(lr=0.5, momentum=0.9, weight_decay=0.25, eps=0.0)
    (v, m, w), = muon([(zero, zero, master)], "bf16", p)
    assert bool((v == 0).all()) and torch.equal(m.cpu(), master * 0.875) and torch.equal(w, m.to(w.dtype))


def test_a_small_long_layer_does_not_choose_for_the_list():
    """Steps over m x m matrices have two more of them in the workspace (three places each): 6 x 9 tile pairs of 32 KB for sides of 300."""
    def size(*shapes):
        array = (C._MuonLayer * len(shapes))(*[_layer(*s) for s in shapes])
        bytes_ = C.lib().convbn_muon_workspace_bytes(ctypes.addressof(array), len(shapes))
        assert bytes_ > 0
        return bytes_
    direct, staged = size((300, 310)), size((300, 2000))
    assert size((300, 310), (5, 1)) - direct < 6 * 9 * 32768 and size((5, 1), (300, 310)) - direct < 6 * 9 * 32768
    # but a long layer that is most of the work does
    assert size((300, 2000), (5, 5)) >= staged and size((300, 2000), (5, 5)) - staged < 6 * 9 * 32768
