"""Group norm with an activation, channels last: the oracle against differences, refusals (CPU), the kernels against the oracle (GPU).

Tolerances.  A stored value is off by half a step of its type, relative to it (fp32 2^-24, bf16 2^-8, half 2^-11; below half's normal range 2^-25).
Behind it stand fp32 sums: a thread adds up to a few hundred values one after the other, then trees: 2^-16 (256 half steps) of the sum of
magnitudes is allowed, and the same of what a mean is subtracted from, since mean and x are both rounded."""
import ctypes

import numpy as np
import pytest

from oracle import norm_oracle as N
from paper_2305_11624_b200 import convbn as C

ACTS = {"none": C.ACT_NONE, "relu": C.ACT_RELU, "silu": C.ACT_SILU}
KINDS = {"f32": C.F32, "bf16": C.BF16, "f16": C.F16}
HALF_STEP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
SUM = 2.0 ** -16
EPS = 1e-5


# ---- the oracle ----------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("act", ["none", "relu", "silu"])
def test_oracle_gradients_are_differences(act):
    rng = np.random.default_rng(3)
    n, h, w, c, g = 2, 2, 3, 6, 2
    x, dz = rng.standard_normal((n, h, w, c)), rng.standard_normal((n, h, w, c))
    gamma, beta = rng.uniform(0.5, 1.5, c), 0.3 * rng.standard_normal(c)
    z, mean, rstd = N.forward(x, g, gamma, beta, EPS, act)
    got = N.backward(dz, x, g, gamma, beta, mean, rstd, act)
    f = lambda x, gamma, beta: (N.forward(x, g, gamma, beta, EPS, act)[0] * dz).sum()
    step = 1e-6
    for name, args in (("dx", 0), ("dgamma", 1), ("dbeta", 2)):
        base = [x, gamma, beta]
        flat = base[args].reshape(-1)
        for i in range(flat.size):
            up, down = [a.copy() for a in base], [a.copy() for a in base]
            up[args].reshape(-1)[i] += step
            down[args].reshape(-1)[i] -= step
            assert abs((f(*up) - f(*down)) / (2 * step) - got[name].reshape(-1)[i]) < 1e-7, (name, i)


def test_oracle_by_hand():
    x = np.array([1.0, 3.0, 10.0, 10.0]).reshape(1, 1, 2, 2)          # pixels (1, 3), (10, 10); groups are channels
    z, mean, rstd = N.forward(x, 2, np.array([2.0, 1.0]), np.array([0.0, 5.0]), 0.0, "none")
    assert np.allclose(mean, [[5.5, 6.5]]) and np.allclose(rstd, [[1 / 4.5, 1 / 3.5]])
    assert np.allclose(z.reshape(-1), [-2.0, 4.0, 2.0, 6.0])


# ---- refusals ------------------------------------------------------------------------------------------------------
def desc(**kw):
    base = dict(n=2, c=32, h=4, w=4, groups=8, act=C.ACT_RELU, dtype=C.BF16)
    base.update(kw)
    return C.NormDesc.make(**base)


def status(call, *args, **kw):
    with pytest.raises(C.ConvBNError) as e:
        call(*args, **kw)
    return e.value.status


@pytest.mark.parametrize("kw", [dict(n=0), dict(c=0), dict(h=-1), dict(w=0), dict(groups=0), dict(groups=5), dict(act=3), dict(act=-1),
                                dict(dtype=3), dict(layout=2), dict(eps=-1e-5), dict(eps=float("nan")), dict(c=1 << 21, groups=1),
                                dict(n=1 << 30, h=1 << 10, w=1 << 10), dict(h=(1 << 31) - 1, w=(1 << 31) - 1), dict(c=65536, groups=65536)])
def test_bad_descriptors(kw):
    d = desc(**kw)
    assert C.convbn_group_norm_workspace_bytes(d) == 0 and C.convbn_group_norm_saved_bytes(d) == 0
    at = 4096
    assert status(C.convbn_group_norm_fwd, d, at, at, at, at, at, at, 1 << 40, stream=0) == C.EINVAL
    assert status(C.convbn_group_norm_bwd, d, at, at, at, at, at, at, at, at, at, 1 << 40, stream=0) == C.EINVAL


def test_other_refusals():
    at, d = 4096, desc()
    assert status(C.convbn_group_norm_fwd, desc(layout=C.NCHW), at, at, at, at, at, at, 1 << 40, stream=0) == C.EUNSUPPORTED
    assert C.convbn_group_norm_workspace_bytes(desc(layout=C.NCHW)) == 0
    need = C.convbn_group_norm_workspace_bytes(d)
    assert need > 0 and need % 256 == 0 and C.convbn_group_norm_saved_bytes(d) == 2 * 2 * 8 * 4
    good = [at] * 5
    for i in range(5):
        args = list(good)
        args[i] = None
        assert status(C.convbn_group_norm_fwd, d, *args, at, need, stream=0) == C.EINVAL
        args[i] = at + 2
        assert status(C.convbn_group_norm_fwd, d, *args, at, need, stream=0) == C.EALIGN
    assert status(C.convbn_group_norm_fwd, d, *good, at, need - 1, stream=0) == C.EWORKSPACE
    assert status(C.convbn_group_norm_fwd, d, *good, None, None, stream=0) == C.EWORKSPACE
    assert status(C.convbn_group_norm_fwd, d, *good, at + 128, need, stream=0) == C.EALIGN
    good = [at] * 8
    for i in range(8):
        args = list(good)
        args[i] = None
        assert status(C.convbn_group_norm_bwd, d, *args, at, need, stream=0) == C.EINVAL
        args[i] = at + 2
        assert status(C.convbn_group_norm_bwd, d, *args, at, need, stream=0) == C.EALIGN
    assert status(C.convbn_group_norm_bwd, d, *good, at, need - 1, stream=0) == C.EWORKSPACE
    assert status(C.convbn_group_norm_bwd, d, *good, at + 16, need, stream=0) == C.EALIGN
    lib = C.lib()
    assert lib.convbn_group_norm_fwd(None, at, at, at, at, at, at, need, 0) == C.EINVAL
    with pytest.raises(TypeError):
        C.convbn_group_norm_fwd(C.Desc.make(1, 8, 1, 1, 8, 1, 1), at, at, at, at, at, at, need, stream=0)


def test_tensors_that_are_not_what_the_descriptor_says():
    import torch
    d, v = desc(), torch.zeros(32)
    x, saved = torch.zeros(2, 4, 4, 32, dtype=torch.bfloat16), torch.zeros(2, 2, 8)
    call = lambda x=x, gamma=v, z=x, saved=saved: status(C.convbn_group_norm_fwd, d, x, gamma, v, z, saved, 4096, 1 << 20, stream=0)
    assert call() == C.EINVAL                                                            # not on a GPU
    assert call(x=x.float()) == C.EINVAL and call(z=x.half()) == C.EINVAL                # another type
    assert call(x=torch.zeros(2, 32, 4, 4, dtype=torch.bfloat16)) == C.EINVAL            # channels first
    assert call(x=torch.zeros(2, 4, 4, 64, dtype=torch.bfloat16)[..., ::2]) == C.EINVAL
    assert call(gamma=torch.zeros(16)) == C.EINVAL and call(gamma=torch.zeros(64)[::2]) == C.EINVAL
    assert call(saved=torch.zeros(2, 8)) == C.EINVAL and call(saved=saved.double() if False else torch.zeros(2, 2, 8, dtype=torch.float16)) == C.EINVAL


def test_shapes_that_plan_nothing_empty():
    """Every sample, channel and pixel belongs to a block: sizes stay positive for awkward channel and group counts."""
    for c, g in ((1, 1), (635, 127), (4099, 1), (8008, 2), (257, 257), (65535, 65535), (1 << 20, 1), (96, 32), (30, 3)):
        for dtype in KINDS.values():
            d = desc(n=3, c=c, groups=g, h=7, w=5, dtype=dtype)
            assert C.convbn_group_norm_workspace_bytes(d) > 0


# ---- the kernels ----------------------------------------------------------------------------------------------------
def make(n, h, w, c, dtype, seed=0, offset=0.5, spread=0.3):
    import torch
    t = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[dtype]
    gen = torch.Generator().manual_seed(seed)
    rn = lambda *s: torch.randn(*s, generator=gen)
    x = (rn(n, h, w, c) * torch.exp(spread * rn(c)) + offset * rn(c)).to(t)
    return x, rn(n, h, w, c).to(t), torch.rand(c, generator=gen) + 0.5, 0.1 * rn(c)


def call(x, dz, gamma, beta, groups, act, dtype, eps=EPS, in_place=False, saved=None, stream=None):
    """(z, mean, rstd, dx, dgamma, dbeta) by the library"""
    import torch
    n, h, w, c = x.shape
    d = C.NormDesc.make(n, c, h, w, groups, act=ACTS[act], dtype=KINDS[dtype], eps=eps)
    dev = lambda t: t.cuda() if not t.is_cuda else t
    x, dz, gamma, beta = dev(x), dev(dz), dev(gamma), dev(beta)
    ws = torch.full((C.convbn_group_norm_workspace_bytes(d),), 255, dtype=torch.uint8, device="cuda")     # (all NaN)
    kept = torch.full((2, n, groups), float("nan"), device="cuda")
    z = x.clone() if in_place else torch.full_like(x, float("nan"))
    C.convbn_group_norm_fwd(d, z if in_place else x, gamma, beta, z, kept, ws, stream=stream)
    dx = dz.clone() if in_place else torch.full_like(x, float("nan"))
    ws.fill_(255)
    dgamma, dbeta = torch.full_like(gamma, float("nan")), torch.full_like(beta, float("nan"))
    C.convbn_group_norm_bwd(d, dx if in_place else dz, x, gamma, beta, kept if saved is None else saved, dx, dgamma, dbeta, ws, stream=stream)
    C.convbn_check(stream)
    return z, kept, dx, dgamma, dbeta


def far(t):
    return t.double().cpu().numpy()


def check(x, dz, gamma, beta, groups, act, dtype, got, eps=EPS):
    z, kept, dx, dgamma, dbeta = got
    X, DZ, G, B = far(x), far(dz), far(gamma), far(beta)
    n, h, w, c = X.shape
    Z, mean, rstd = N.forward(X, groups, G, B, eps, act)
    wide = lambda t: np.broadcast_to(t[:, None, None, :, None], (n, h, w, groups, c // groups)).reshape(X.shape)
    top = np.abs(X.reshape(n, h * w, groups, -1)).max(axis=(1, 3))
    half, tiny = HALF_STEP[dtype], 2.0 ** -25 if dtype == "f16" else 0.0
    m, r = far(kept)
    assert (np.abs(m - mean) <= SUM * top).all()
    # of the variance: 2^-16 of itself and of eps, and what the mean's and x's rounding brings in
    assert (np.abs(r / rstd - 1) <= SUM * (1 + top * rstd)).all()
    xhat = (X - wide(mean)) * wide(rstd)
    allowed = half * np.abs(Z) + tiny + 1.1 * SUM * ((np.abs(xhat) * (1 + wide(top * rstd)) + wide(top * rstd)) * np.abs(G) + np.abs(B))
    off = np.abs(far(z) - Z)
    assert (off <= allowed).all(), (off / allowed).max()
    # the backward pass is given the forward call's own statistics
    ref = N.backward(DZ, X, groups, G, B, m, r, act)
    more = 1 + wide(top * r)
    allowed = half * np.abs(ref["dx"]) + tiny + SUM * ref["dx_size"] * more
    off = np.abs(far(dx) - ref["dx"])
    assert (off <= allowed).all(), (off / allowed).max()
    for name, v in (("dgamma", dgamma), ("dbeta", dbeta)):
        allowed = SUM * ref[name + "_size"] * (1 + (top * r).max()) + 2.0 ** -140
        off = np.abs(far(v) - ref[name])
        assert (off <= allowed).all(), (name, (off / allowed).max())


SHAPES = [(1, 1, 1, 1, 1),            # one value: its variance is zero
          (2, 16, 16, 32, 8),
          (3, 5, 7, 30, 3),           # rows that allow accesses of two elements
          (2, 9, 11, 96, 32),         # three channels a group
          (5, 1, 1, 36, 4),           # a matrix
          (1, 1, 1, 2048, 1),
          (2, 3, 3, 4099, 1),         # odd, wider than a block
          (1, 3, 3, 8008, 2),
          (2, 5, 3, 8192, 1),
          (2, 33, 65, 64, 1),
          (1, 4, 9, 635, 127),        # a prime number of groups of five channels
          (2, 3, 2, 257, 257),        # instance norm
          (4, 7, 7, 2048, 32),
          (1, 211, 137, 64, 4),
          (64, 14, 14, 24, 8),
          (3, 1, 129, 520, 65)]


@pytest.mark.gpu
@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("dtype,act", [("f32", "relu"), ("bf16", "silu"), ("f16", "relu"), ("bf16", "none"), ("f32", "silu")])
def test_against_the_oracle(shape, dtype, act):
    n, h, w, c, groups = shape
    args = make(n, h, w, c, dtype)
    check(*args, groups, act, dtype, call(*args, groups, act, dtype))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_large_offset(dtype):
    """A mean a thousand times the spread: the variance is a sum of squared distances, not a difference."""
    x, dz, gamma, beta = make(2, 40, 40, 64, dtype, offset=0.0, spread=0.0)
    x = (x.float() + 1000.0).to(x.dtype)
    check(x, dz, gamma, beta, 8, "none", dtype, call(x, dz, gamma, beta, 8, "none", dtype))


@pytest.mark.gpu
def test_one_value_far_away():
    """A first pixel far from the others, as a padded border has it."""
    x, dz, gamma, beta = make(2, 40, 40, 64, "f32", offset=0.0, spread=0.0)
    x += 100.0
    x[:, 0, 0] = 0.0
    check(x, dz, gamma, beta, 8, "relu", "f32", call(x, dz, gamma, beta, 8, "relu", "f32"))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "f16"])
def test_constant_input(dtype):
    x, dz, gamma, beta = make(2, 6, 6, 32, dtype)
    x.fill_(3.25)
    z, kept, dx, _, _ = call(x, dz, gamma, beta, 4, "none", dtype)
    assert (far(kept)[0] == 3.25).all() and np.allclose(far(kept)[1], EPS ** -0.5, rtol=1e-6)
    assert (z == beta.cuda().to(z.dtype)).all()
    check(x, dz, gamma, beta, 4, "none", dtype, call(x, dz, gamma, beta, 4, "none", dtype))


@pytest.mark.gpu
def test_not_a_number_stays_in_its_group():
    import torch
    x, dz, gamma, beta = make(2, 5, 6, 64, "bf16")
    clean = call(x, dz, gamma, beta, 8, "silu", "bf16")
    x[1, 2, 3, 17] = float("nan")
    x[0, 4, 5, 63] = float("inf")
    z, kept, dx, _, _ = call(x, dz, gamma, beta, 8, "silu", "bf16")
    for i, g in ((1, 2), (0, 7)):
        assert torch.isnan(z[i, :, :, 8 * g:8 * g + 8]).all() and torch.isnan(dx[i, :, :, 8 * g:8 * g + 8]).all()
        for got, had in ((z, clean[0]), (dx, clean[2])):
            got[i, :, :, 8 * g:8 * g + 8] = had[i, :, :, 8 * g:8 * g + 8]
    assert torch.equal(z, clean[0]) and torch.equal(dx, clean[2])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_relu_gradient_next_to_zero(dtype):
    """beta is set so that one pixel of every channel has y within fp32's rounding of zero: the sign is the exact one."""
    x, dz, gamma, beta = make(2, 8, 8, 256, dtype, offset=1.0)
    kept = call(x, dz, gamma, beta, 16, "none", dtype)[1]
    X, G = far(x), far(gamma)
    m, r = (np.repeat(far(kept)[k], 16, axis=1) for k in (0, 1))
    pixel = np.arange(256) % 64
    at = X[0].reshape(64, 256)[pixel, np.arange(256)]
    import torch
    beta = torch.tensor(-(G * (at - m[0]) * r[0])).float()
    y = G * (at - m[0]) * r[0] + far(beta)
    assert (np.abs(y) <= 2.0 ** -24 * np.abs(far(beta))).all() and (y > 0).any() and (y < 0).any()
    got = call(x, dz, gamma, beta, 16, "relu", dtype)
    ref = N.backward(far(dz), X, 16, G, far(beta), far(kept)[0], far(kept)[1], "relu")
    allowed = SUM * ref["dbeta_size"]
    assert (np.abs(far(got[4]) - ref["dbeta"]) <= allowed).all()       # (a wrong sign moves dbeta by a whole dz)
    check(x, dz, gamma, beta, 16, "relu", dtype, got)


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [(2, 16, 16, 32, 8), (3, 5, 7, 30, 3), (2, 100, 100, 256, 32)], ids=str)
def test_in_place_repeated_and_on_a_stream(shape):
    import torch
    n, h, w, c, groups = shape
    args = make(n, h, w, c, "bf16")
    first = call(*args, groups, "relu", "bf16")
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        again = call(*args, groups, "relu", "bf16", in_place=True)
    torch.cuda.synchronize()
    for a, b in zip(first, again):
        assert torch.equal(a, b)


@pytest.mark.gpu
def test_captured_and_replayed():
    """Two captured chains that share a workspace, replayed one after the other on new inputs."""
    import torch
    cases = []
    d = [C.NormDesc.make(4, 64, 30, 31, 8, act=C.ACT_SILU, dtype=C.BF16), C.NormDesc.make(2, 96, 20, 20, 32, act=C.ACT_RELU, dtype=C.BF16)]
    ws = torch.empty(max(C.convbn_group_norm_workspace_bytes(k) for k in d), dtype=torch.uint8, device="cuda")
    for k in d:
        x, dz, gamma, beta = (t.cuda() for t in make(k.n, k.h, k.w, k.c, "bf16"))
        z, dx, kept = torch.empty_like(x), torch.empty_like(x), torch.empty(2, k.n, k.groups, device="cuda")
        dg, db = torch.empty_like(gamma), torch.empty_like(beta)

        def step(k=k, x=x, dz=dz, gamma=gamma, beta=beta, z=z, dx=dx, kept=kept, dg=dg, db=db):
            C.convbn_group_norm_fwd(k, x, gamma, beta, z, kept, ws)
            C.convbn_group_norm_bwd(k, dz, x, gamma, beta, kept, dx, dg, db, ws)
        step()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        cases.append((k, graph, x, dz, gamma, beta, z, kept, dx, dg, db))
    for k, graph, x, dz, *_ in cases:
        x2, dz2, _, _ = make(k.n, k.h, k.w, k.c, "bf16", seed=9)
        x.copy_(x2)
        dz.copy_(dz2)
    for _ in range(2):
        for case in cases:
            case[1].replay()
    torch.cuda.synchronize()
    for k, graph, x, dz, gamma, beta, z, kept, dx, dg, db in cases:
        check(x, dz, gamma, beta, k.groups, "silu" if k.act == C.ACT_SILU else "relu", "bf16", (z, kept, dx, dg, db))


@pytest.mark.gpu
def test_many_samples():
    """More samples than a launch takes."""
    args = make(40000, 1, 1, 8, "f32")
    check(*args, 2, "relu", "f32", call(*args, 2, "relu", "f32"))


@pytest.mark.gpu
def test_beyond_2_31_elements():
    import torch
    n, h, w, c, groups = 33, 1024, 1024, 64, 8
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(n, h, w, c, generator=gen, device="cuda", dtype=torch.bfloat16)
    dz = torch.randn(n, h, w, c, generator=gen, device="cuda", dtype=torch.bfloat16)
    gamma, beta = torch.rand(c, device="cuda") + 0.5, torch.randn(c, device="cuda")
    z, kept, dx, dgamma, dbeta = call(x, dz, gamma, beta, groups, "silu", "bf16")
    alone = call(x[-1:], dz[-1:], gamma, beta, groups, "silu", "bf16")
    # one sample by itself is cut into other runs: statistics agree to rounding, values to a step
    assert torch.allclose(kept[:, -1:], alone[1], rtol=1e-5, atol=1e-5)
    for whole, part in ((z, alone[0]), (dx, alone[2])):
        d = (whole[-1:].float() - part.float()).abs()
        assert bool((d <= 2.0 ** -7 * part.float().abs() + 2.0 ** -14).all())
    parts = [call(x[i:i + 11], dz[i:i + 11], gamma, beta, groups, "silu", "bf16") for i in (0, 11, 22)]
    for k in (3, 4):
        total = sum(p[k].double() for p in parts)
        assert torch.allclose((dgamma, dbeta)[k - 3].double(), total, rtol=0.0, atol=SUM * n * h * w * 0.4)      # E|dy| is about 0.4
