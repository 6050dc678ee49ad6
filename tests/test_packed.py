"""X in 8 bits from forward to backward: convbn_pack, convbn_unpack, convbn_tune_bwd_packed."""
import numpy as np
import pytest

import parity
from oracle import packed_oracle as P
from paper_2305_11624_b200 import convbn as C
from paper_2305_11624_b200 import inputs as I

ROUND = {"bf16": I.round_bf16, "f16": lambda a: np.asarray(a, np.float16).astype(np.float32), "f32": lambda a: np.asarray(a, np.float32)}


# ---- the definition itself ------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_the_definition_keeps_signs_and_half_a_step(dtype):
    rng = np.random.default_rng(3)
    x = ROUND[dtype]((rng.standard_normal(6400) * np.repeat(10.0 ** rng.uniform(-3, 3, 200), 32)).astype(np.float32)).astype(np.float64)
    x[::7] = 0.0
    q, s = P.pack(x, dtype)
    back, step = P.unpack(q, s), np.repeat(2.0 ** (s.astype(float) - 127), 32)
    assert np.array_equal(np.sign(back), np.sign(x))
    large = np.abs(x) >= step / 2
    assert np.all(np.abs(back - x)[large] <= step[large] / 2) and np.all(np.abs(back - x) <= step)
    top = np.abs(x).reshape(-1, 32).max(1)
    assert np.all((np.abs(q.astype(int)).reshape(-1, 32).max(1) >= 64) | (s == P.BOUNDS[dtype][0] + 127))
    assert np.all(top <= 127.5 * 2.0 ** (s.astype(float) - 127))
    np.testing.assert_array_equal(ROUND[dtype](back), back)              # exact in the storage type


@pytest.mark.parametrize("dtype,largest,step", [("bf16", 255 * 2.0 ** 120, 2.0 ** 121), ("f32", float(np.float32(3.4028235e38)), 2.0 ** 121),
                                                ("f16", 65504.0, 512.0)])
def test_the_definition_at_the_largest_values(dtype, largest, step):
    """Steps are held at their upper bound there: what is above 127.5 of them stands for 127, less than one step away."""
    rng = np.random.default_rng(5)
    for top in (largest, 127.5 * step, 127.4 * step, 64 * step, 63.75 * step):
        x = ROUND[dtype]((rng.uniform(-1, 1, 32) * top).astype(np.float32)).astype(np.float64)
        x[7] = ROUND[dtype](np.float32(top)) * (-1) ** int(rng.integers(2))
        q, s = P.pack(x, dtype)
        assert 2.0 ** (int(s[0]) - 127) == step and np.abs(q.astype(int)).max() <= 127
        err = np.abs(P.unpack(q, s) - x)
        cut, small = np.abs(x) > 127.5 * step, np.abs(x) < step / 2
        assert np.all(err[cut] < step) and np.all(err[small] < step) and np.all(err[~cut & ~small] <= step / 2)
        assert dtype != "bf16" or not cut.any()


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_half_a_step_against_the_largest_magnitude(dtype):
    """Between 1/255 and 1/127.5 of it, and as near to both as the type has values."""
    tops = np.unique(ROUND[dtype](np.append(np.linspace(60, 128, 20000), 63.75).astype(np.float32))).astype(np.float64)
    x = np.zeros((tops.size, 32))
    x[:, 3] = tops
    _, s = P.pack(x.ravel(), dtype)
    share = 2.0 ** (s.astype(float) - 128) / tops
    assert share.min() > 1 / 255 and share.max() == 1 / 127.5 and share.min() < 1.01 / 255


# ---- refusals (host) -------------------------------------------------------------------------------------------------
def test_pack_refusals():
    lib, ok = C.lib(), 4096
    for f in (lib.convbn_pack, lib.convbn_unpack):
        assert f(C.BF16, 0, 0, 0, 0, 0) == C.OK                         # nothing to do
        assert f(C.BF16, ok, ok, ok, -1, 0) == C.EINVAL
        assert f(C.BF16, ok, ok, ok, (1 << 40) + 1, 0) == C.EINVAL
        assert f(3, ok, ok, ok, 5, 0) == C.EINVAL
        for i in range(3):
            p = [ok] * 3
            p[i] = 0
            assert f(C.F32, *p, 5, 0) == C.EINVAL
            p[i] = ok + 8
            assert f(C.F16, *p, 5, 0) == C.EALIGN


def test_packed_backward_refusals():
    d = C.Desc.make(2, 64, 8, 8, 64, 1, 1)
    size = C.convbn_workspace_bytes(d, C.PHASE_TUNE_BWD_PACKED)
    assert size >= C.convbn_workspace_bytes(d, C.PHASE_TUNE_BWD) > 0 and size % 256 == 0
    names = ("dz", "codes", "steps", "w", "b", "run_mean", "saved", "dx", "dw", "db", "dgamma", "dbeta", "add")

    def status(desc=d, ws=4096, bytes_=size, **over):
        a = {n: (None if n in ("b", "db", "add") else 4096) for n in names}
        a.update(over)
        with pytest.raises(C.ConvBNError) as e:
            C.convbn_tune_bwd_packed(desc, *[a[n] for n in names], True, False, ws, bytes_, stream=0)
        return e.value.status

    for n in names:
        if n not in ("b", "db", "add"):
            assert status(**{n: None}) == C.EINVAL, n
        off = 2 if n in ("b", "run_mean", "db", "dgamma", "dbeta") else 8
        pair = {"b": dict(db=4096), "db": dict(b=4096)}.get(n, {})
        assert status(**{n: 4096 + off}, **pair) == C.EALIGN, n
    assert status(b=4096) == C.EINVAL and status(db=4096) == C.EINVAL
    assert status(ws=None) == C.EWORKSPACE and status(bytes_=size - 1) == C.EWORKSPACE and status(ws=4096 + 16) == C.EALIGN
    assert status(desc=C.Desc.make(2, 64, 8, 8, 64, 1, 1, dtype=C.BF16, layout=C.NCHW)) == C.EUNSUPPORTED
    assert status(desc=C.Desc.make(2, 64, 8, 8, 64, 1, 1, dtype=C.F16, layout=C.NCHW)) == C.EUNSUPPORTED
    assert status(desc=C.Desc.make(0, 64, 8, 8, 64, 1, 1)) == C.EINVAL


def test_tensors_that_do_not_hold_what_is_read_or_written_are_refused():
    """The library takes addresses and a count, so what is too short, of another width, or has gaps is refused before the call."""
    import torch
    x = torch.zeros(100, 64, dtype=torch.bfloat16)
    codes, steps = torch.zeros(6400, dtype=torch.int8), torch.zeros(200, dtype=torch.uint8)

    def refused(what, x=x, codes=codes, steps=steps):
        for call in (lambda: C.convbn_pack(x, codes, steps, stream=0), lambda: C.convbn_unpack(codes, steps, x, stream=0)):
            with pytest.raises(C.ConvBNError, match=what) as e:
                call()
            assert e.value.status == C.EINVAL

    refused("codes", codes=codes[:6399])
    refused("steps", steps=steps[:199])
    refused("codes", codes=codes.view(100, 64)[:, :32])
    refused("codes", codes=torch.zeros(128, 64, dtype=torch.int8).t())
    refused("codes", codes=torch.zeros(6400, dtype=torch.int32))
    refused("steps", steps=torch.zeros(400, dtype=torch.uint8)[::2])
    refused("steps", steps=torch.zeros(200, dtype=torch.float32))
    refused("one piece", x=x[:, ::2])
    refused("one piece", x=x.t())
    refused("one piece", x=torch.zeros(64, dtype=torch.bfloat16).expand(100, 64))
    refused("one GPU")                                                   # (nothing else is wrong, in any of the three)
    refused("one GPU", x=torch.zeros(2, 8, 20, 20, dtype=torch.bfloat16).to(memory_format=torch.channels_last))
    refused("codes", codes=codes[:2 * 64 * 8 * 8 - 1], x=torch.zeros(2, 8, 8, 64, dtype=torch.float32))

    d = C.Desc.make(2, 64, 8, 8, 64, 1, 1)
    for c, s in ((codes, torch.zeros(256, dtype=torch.uint8)), (torch.zeros(8191, dtype=torch.int8), torch.zeros(256, dtype=torch.uint8)),
                 (torch.zeros(8192, dtype=torch.int8), torch.zeros(255, dtype=torch.uint8)),
                 (torch.zeros(8192, dtype=torch.int8), torch.zeros(512, dtype=torch.uint8)[::2])):
        with pytest.raises(C.ConvBNError, match="codes|steps") as e:
            C.convbn_tune_bwd_packed(d, 4096, c, s, 4096, None, 4096, 4096, 4096, 4096, None, 4096, 4096, None, True, False, 4096, 1 << 30,
                                     stream=0)
        assert e.value.status == C.EINVAL


def test_room_for_slices_that_keep_sums_short():
    """A weight gradient's fp32 accumulators add up 6144 pixels at most: a partial tensor for each slice of so many."""
    size = lambda rows, ci, co: C.convbn_workspace_bytes(C.convbn_linear_desc(rows, ci, co), C.PHASE_TUNE_BWD_PACKED)
    for rows, ci, co in ((100000, 1024, 512), (144900, 1024, 512), (1560000, 64, 128), (1200000, 256, 64)):
        assert size(rows, ci, co) >= -(-rows // 6144) * ci * co * 4, (rows, ci, co)


def test_room_for_the_short_sums_of_stems_and_groups_of_eight():
    """The same for the kernels whose accumulators stay with a block: a stem's read straight from X (3 -> 64, two accumulators a block,
    224 pixels a row: 14400 rows and more), groups of eight channels."""
    def partials(d, elements):
        return (C.convbn_workspace_bytes(d, C.PHASE_TUNE_BWD_PACKED) - elements * 2 - C.convbn_workspace_bytes(d, C.PHASE_TUNE_BWD_DATA))
    for kind in (C.BF16, C.F16):
        for n in (256, 1024):
            d = C.Desc.make(n, 3, 224, 224, 64, 7, 7, 2, 2, 3, 3, dtype=kind)
            assert partials(d, n * 224 * 224 * 3) >= n * 112 * 112 // (2 * 6144) * 147 * 64 * 4
        d = C.Desc.make(256, 2048, 28, 28, 2048, 3, 3, 1, 1, 1, 1, groups=256, dtype=kind)
        assert partials(d, 256 * 28 * 28 * 2048) >= 256 * 28 * 28 // 6144 * 2048 * 72 * 4


def test_half_values_need_no_more_room_than_the_other_call():
    """Their accumulators are emptied on the way, so the slices, and the partial tensors, are those of convbn_tune_bwd: beside those, X
    restored where the weight gradient does not do that itself."""
    for args in ((100000, 2048, 1, 1, 2048, 1), (100000, 2048, 1, 1, 1024, 1), (23, 1024, 63, 100, 512, 1), (240, 64, 100, 65, 128, 1),
                 (64, 2048, 7, 7, 512, 1), (256, 64, 56, 56, 64, 3), (128, 512, 28, 28, 512, 3), (17, 256, 15, 14, 512, 1)):
        n, ci, h, w, co, k = args
        d = C.Desc.make(n, ci, h, w, co, k, k, 1, 1, k // 2, k // 2, dtype=C.F16)
        packed, plain = (C.convbn_workspace_bytes(d, p) for p in (C.PHASE_TUNE_BWD_PACKED, C.PHASE_TUNE_BWD))
        assert plain <= packed <= plain + n * h * w * ci * 2 + 256, args


def test_layers_of_several_taps_need_no_more_room_than_the_other_call():
    """The same in bf16, whose 1x1 layers alone have slices instead."""
    for n, c, hw, groups in ((256, 64, 56, 1), (128, 512, 28, 1), (256, 128, 56, 4), (64, 256, 14, 1)):
        d = C.Desc.make(n, c, hw, hw, c, 3, 3, 1, 1, 1, 1, groups=groups, dtype=C.BF16)
        packed, plain = (C.convbn_workspace_bytes(d, p) for p in (C.PHASE_TUNE_BWD_PACKED, C.PHASE_TUNE_BWD))
        assert plain <= packed <= plain + n * hw * hw * c * 2 + 256, (n, c, hw, groups)


# ---- packing on the device ------------------------------------------------------------------------------------------
def _values(count, dtype, seed):
    """Every kind of group: ordinary, all zero, one value, values at a tie, the type's largest and smallest, infinities, NaN."""
    rng = np.random.default_rng(seed)
    groups = -(-count // 32)
    v = rng.standard_normal((groups, 32)) * 2.0 ** rng.integers(-20, 20, groups)[:, None]
    for g in range(groups):
        kind = (g + seed) % 12
        if kind == 1:
            v[g] = 0.0
        elif kind == 2:
            v[g] = 0.0
            v[g, rng.integers(32)] = -3.25
        elif kind == 3:
            v[g] = (rng.integers(-127, 127, 32) + 0.5) * 0.25           # ties, and 127.5 steps
            v[g, 0] = 127.5 * 0.25
        elif kind == 4:
            v[g, 5] = {"bf16": 3.3895314e38, "f32": 3.4028235e38, "f16": 65504.0}[dtype]
        elif kind == 5:
            v[g] = rng.integers(-3, 4, 32) * {"bf16": 2.0 ** -133, "f32": 2.0 ** -149, "f16": 2.0 ** -24}[dtype]
        elif kind == 6:
            v[g, 31] = np.inf * (-1) ** g
        elif kind == 7:
            v[g, 0] = np.nan
        elif kind == 8:
            v[g] = np.abs(v[g]) * (rng.random(32) < 0.5)                # a ReLU's output
        elif kind == 9:
            v[g] *= 2.0 ** rng.integers(-30, 1, 32)                     # far below half a step
    with np.errstate(over="ignore"):
        return ROUND[dtype](v.astype(np.float32).ravel()[:count])


def _torch(dtype):
    import torch
    return {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}[dtype]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("count", [1, 15, 16, 17, 31, 32, 33, 511, 513, 4099, 148 * 16 * 4096 + 77])
def test_pack_and_unpack_are_exact(dtype, count):
    import torch
    host = _values(count, dtype, count % 5)
    groups = -(-count // 32)
    x = torch.from_numpy(host).cuda().to(_torch(dtype))
    codes = torch.full((count + 48,), 99, dtype=torch.int8, device="cuda")
    steps = torch.full((groups + 48,), 99, dtype=torch.uint8, device="cuda")
    out = torch.full((count + 24,), 7.0, dtype=_torch(dtype), device="cuda")
    C.convbn_pack(x, codes, steps)
    C.convbn_unpack(codes, steps, out[:count])
    C.convbn_check()
    q, s = P.pack(host, dtype)
    assert np.array_equal(steps[:groups].cpu().numpy(), s)
    assert np.array_equal(codes[:count].cpu().numpy(), q)
    np.testing.assert_array_equal(out[:count].float().cpu().numpy().astype(np.float64), P.unpack(q, s))
    assert bool((codes[count:] == 99).all()) and bool((steps[groups:] == 99).all()) and bool((out[count:] == 7.0).all())


@pytest.mark.gpu
def test_packing_takes_channels_last_tensors_and_addresses():
    """In the order of memory: an NCHW tensor stored as NHWC is packed as NHWC."""
    import torch
    x = torch.randn(2, 24, 7, 9, device="cuda").to(torch.bfloat16).to(memory_format=torch.channels_last)
    codes, steps = torch.full((x.numel(),), 99, dtype=torch.int8, device="cuda"), torch.full((95,), 99, dtype=torch.uint8, device="cuda")
    q, s = P.pack(x.permute(0, 2, 3, 1).float().cpu().numpy().ravel(), "bf16")
    for c, t in ((codes, steps), (codes.data_ptr(), steps.data_ptr()), (codes.view(torch.uint8), steps.data_ptr())):
        codes.fill_(99)
        C.convbn_pack(x, c, t)
        C.convbn_check()
        assert np.array_equal(codes.cpu().numpy(), q) and np.array_equal(steps.cpu().numpy(), s)
        out = torch.empty_like(x)
        C.convbn_unpack(c, t, out)
        C.convbn_check()
        np.testing.assert_array_equal(out.permute(0, 2, 3, 1).float().cpu().numpy().ravel().astype(np.float64), P.unpack(q, s))
    with pytest.raises(C.ConvBNError):
        C.convbn_pack(x, codes.cpu(), steps)
    with pytest.raises(C.ConvBNError):
        C.convbn_unpack(codes, steps, x.cpu())


@pytest.mark.gpu
def test_a_type_that_is_not_a_storage_type_is_refused():
    import torch
    x = torch.zeros(64, dtype=torch.float64, device="cuda")
    codes, steps = torch.zeros(64, dtype=torch.int8, device="cuda"), torch.zeros(2, dtype=torch.uint8, device="cuda")
    with pytest.raises(TypeError):
        C.convbn_pack(x, codes, steps)
    with pytest.raises(TypeError):
        C.convbn_unpack(codes, steps, codes)


# ---- the backward pass -----------------------------------------------------------------------------------------------
LAYERS = [
    I.LayerSpec("wide_in", 2, 256, 20, 15, 64, 1, 1),                    # one kernel reads dZ once
    I.LayerSpec("wide_in_128", 3, 128, 14, 13, 64, 1, 1),
    I.LayerSpec("wide_out", 2, 64, 17, 19, 256, 1, 1),
    I.LayerSpec("wide_out_128", 5, 64, 11, 13, 128, 1, 1),
    I.LayerSpec("wide_in_many_tiles", 13, 256, 56, 55, 64, 1, 1),        # several tiles a CTA, the last one short
    I.LayerSpec("wide_out_many_tiles", 13, 64, 56, 55, 128, 1, 1),
    I.LayerSpec("wide_few_pixels", 1, 256, 3, 5, 64, 1, 1),
    I.LayerSpec("one_pixel", 1, 64, 1, 1, 64, 1, 1),
    I.LayerSpec("rows", 777, 256, 1, 1, 192, 1, 1),                      # Linear-BN
    I.LayerSpec("rows_wide", 130, 2048, 1, 1, 512, 1, 1),
    I.LayerSpec("odd_slices", 3, 192, 9, 7, 320, 1, 1),
    I.LayerSpec("reduce", 4, 1024, 7, 7, 256, 1, 1),
    I.LayerSpec("shortcut", 2, 256, 15, 14, 512, 1, 1, stride=2),
    I.LayerSpec("conv3", 2, 64, 13, 17, 64, 3, 3, pad=1),
    I.LayerSpec("conv3_stride2", 2, 128, 16, 18, 128, 3, 3, stride=2, pad=1),
    I.LayerSpec("conv3_dilated", 1, 64, 16, 18, 64, 3, 3, pad=2, dil=2),
    I.LayerSpec("stem", 1, 3, 33, 40, 64, 7, 7, stride=2, pad=3),
    I.LayerSpec("depthwise", 2, 96, 12, 11, 96, 3, 3, pad=1, groups=96),
    I.LayerSpec("grouped8", 2, 64, 10, 12, 64, 3, 3, pad=1, groups=8),
    I.LayerSpec("grouped32", 2, 128, 10, 12, 128, 3, 3, pad=1, groups=4),
    I.LayerSpec("odd_channels", 2, 10, 9, 8, 20, 3, 3, pad=1),
    I.LayerSpec("f32", 2, 16, 9, 11, 24, 3, 3, pad=1, dtype="f32", layout="nchw"),
    I.LayerSpec("f32_rows", 37, 24, 1, 1, 10, 1, 1, dtype="f32", layout="nchw"),
]


def _restored(spec, x):
    """x [N, C, H, W] as the packed form holds it, and its codes and steps in memory order."""
    flat = I.act_to_layout(x, spec.layout).ravel()
    q, s = P.pack(flat, spec.dtype)
    return I.act_from_layout(P.unpack(q, s), spec.layout, x.shape), q, s


def _packed_pass(spec, t, add, mask, begin=False, stream=None, expect=None):
    """The calls of a training step whose X is kept packed; outputs as float64 in logical order."""
    import torch
    from paper_2305_11624_b200.harness import Block
    blk = Block(spec, modes=("tune",))
    blk.load(t)
    codes = torch.empty(blk.x.numel(), dtype=torch.int8, device="cuda")
    steps = torch.empty(-(-blk.x.numel() // 32), dtype=torch.uint8, device="cuda")
    more = None
    if add is not None:
        more = torch.empty_like(blk.x)
        blk._up(more, I.act_to_layout(add, spec.layout))
    for name in ("dx", "dw", "dgamma", "dbeta"):
        getattr(blk, name).fill_(float("nan"))
    blk.tune_fwd()
    C.convbn_pack(blk.x, codes, steps)
    _, q, s = _restored(spec, t["x"])
    assert np.array_equal(codes.cpu().numpy(), q) and np.array_equal(steps.cpu().numpy(), s)
    blk.x.fill_(float("nan"))                                            # X itself is gone
    size = C.convbn_workspace_bytes(blk.desc, C.PHASE_TUNE_BWD_PACKED)
    room = torch.full((size + 256,), 0xFF, dtype=torch.uint8, device="cuda")
    C.convbn_tune_bwd_packed(blk.desc, blk.dz, codes, steps, blk.w, blk.b, blk.mu_hat, blk.saved, blk.dx, blk.dw, blk.db, blk.dgamma,
                             blk.dbeta, more, mask, begin, room[:size] if size else None)
    if begin:
        C.convbn_tune_bwd_join()
    C.convbn_check()
    assert bool((room[size:] == 0xFF).all())
    if expect is not None:
        assert C.convbn_last_kernel(C.PHASE_TUNE_BWD_PACKED) == expect
    names = ["dx", "dw", "dgamma", "dbeta"] + (["db"] if spec.bias else [])
    return dict({n: blk.fetch(n) for n in names}, **({} if spec.bias else {"db": None}))


def _reference(spec, t, add, mask):
    back, _, _ = _restored(spec, t["x"])
    ref = parity.oracle_tune(spec, dict(t, x=back))
    if add is not None:
        ref["dx"] = ref["dx"] + add
    if mask:
        ref["dx"] = ref["dx"] * (t["x"] > 0)                             # (the mask is the true one)
    return ref


HALF_STEP = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": 2.0 ** -24}


def _compare(spec, t, got, ref, add, mask):
    """Norms and the parameter gradients as parity.py bounds them.  dX element by element, proven: with S = sum |dZ| |omega'| over
    an element's products, the rounding of omega' costs u S (2^-25 |dZ| a product where half has no smaller steps), s and the fp32
    sum of K products (8 + K) 2^-24 S, the store u |dX|, the addend's sum another u |dX + add|.  (parity.py measures an element
    against the rms of its channel instead, which 15 pixels, half of them masked, do not give: a layer with 15 pixels, its dX
    right, came to 1.26 of that bound.)"""
    parity.compare(got, ref, parity.TOL[spec.dtype], ("dw", "db", "dgamma", "dbeta"), spec.name, dtype=spec.dtype)
    assert parity.O.rel_l2(got["dx"], ref["dx"]) <= parity.TOL[spec.dtype]
    plain = parity.oracle_tune(spec, t)
    shape = parity.oracle_shape(spec)
    size = parity.O.tune_backward(shape, np.abs(t["dz"]), t["x"], t["w"], np.abs(plain["w_f"]), t["b"], t["gamma"], t["mu_hat"],
                                  t["var_hat"])["dx"]
    products = spec.c_out // spec.groups * spec.kh * spec.kw
    u = HALF_STEP[spec.dtype] * (1 + 2.0 ** -6)
    bound = (u + (8 + products) * 2.0 ** -24) * size + u * np.abs(plain["dx"])
    bound += 2.0 ** -25 * (1 + products * np.abs(t["dz"]).max())
    if add is not None:
        bound += u * (np.abs(plain["dx"] + add) + bound)
    if mask:
        assert not got["dx"][t["x"] <= 0].any()
        bound = bound * (t["x"] > 0)
    err = np.abs(got["dx"] - ref["dx"])
    assert np.all(err <= bound), float((err / np.maximum(bound, 1e-30)).max())


def _relu_inputs(spec, seed):
    t = parity.make_inputs(spec, seed)
    t["x"] = np.maximum(t["x"], 0.0)
    return t


@pytest.mark.gpu
@pytest.mark.parametrize("mask,with_add", [(False, False), (True, False), (True, True)])
@pytest.mark.parametrize("spec", LAYERS, ids=lambda s: s.name)
def test_packed_backward_against_the_oracle(spec, mask, with_add):
    """X enters the gradients as the value that its code stands for, exactly, so the bounds are those of the same layer with that
    X."""
    t = _relu_inputs(spec, 5) if mask else parity.make_inputs(spec, 5)
    add = ROUND[spec.dtype](np.random.default_rng(1).standard_normal(t["x"].shape).astype(np.float32)) if with_add else None
    got = _packed_pass(spec, t, add, mask)
    _compare(spec, t, got, _reference(spec, t, add, mask), add, mask)


# which kernels take X as it is packed (the single kernel from 512 pixels on); the others restore it first
PATHS = dict({s.name: "umma-fused-bwd" for s in LAYERS[:6]}, wide_few_pixels="umma", one_pixel="umma", rows="umma", rows_wide="umma", reduce="umma")


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("spec", LAYERS, ids=lambda s: s.name)
def test_which_kernels_a_layer_takes(spec, dtype):
    import dataclasses
    if spec.dtype == "bf16":
        spec = dataclasses.replace(spec, dtype=dtype)
    _packed_pass(spec, parity.make_inputs(spec, 2), None, False, expect=PATHS.get(spec.name, "unpack"))


# few taps, borders and dilations in the weight gradient that restores X on its way
FEW_TAPS = [I.LayerSpec("pair", 2, 64, 9, 11, 64, 1, 2), I.LayerSpec("column", 2, 1024, 9, 7, 64, 3, 1),
            I.LayerSpec("dilated_row", 3, 1024, 6, 10, 128, 1, 3, dil=2), I.LayerSpec("four", 1, 1024, 8, 7, 128, 2, 2),
            I.LayerSpec("four_with_border", 2, 1024, 6, 5, 64, 2, 2, pad=1), I.LayerSpec("border_1x1", 2, 64, 6, 9, 128, 1, 1, pad=1)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("spec", FEW_TAPS, ids=lambda s: s.name)
def test_few_taps_against_the_oracle(spec, dtype):
    import dataclasses
    spec = dataclasses.replace(spec, dtype=dtype, bias=True)
    t = _relu_inputs(spec, 3)
    add = ROUND[dtype](np.random.default_rng(1).standard_normal(t["x"].shape).astype(np.float32))
    got = _packed_pass(spec, t, add, True, expect="umma")
    _compare(spec, t, got, _reference(spec, t, add, True), add, True)


@pytest.mark.gpu
@pytest.mark.parametrize("spec", [s for s in LAYERS if s.name in ("wide_in", "wide_out", "rows", "reduce", "conv3", "shortcut")], ids=lambda s: s.name)
def test_packed_backward_in_half_with_bias_deferred(spec):
    import dataclasses
    spec = dataclasses.replace(spec, dtype="f16", bias=True)
    t = _relu_inputs(spec, 9)
    add = ROUND["f16"](np.random.default_rng(1).standard_normal(t["x"].shape).astype(np.float32))
    got = _packed_pass(spec, t, add, True, begin=True)
    _compare(spec, t, got, _reference(spec, t, add, True), add, True)


# ---- together, as a training iteration uses them -----------------------------------------------------------------------
@pytest.mark.gpu
@pytest.mark.parametrize("deferred", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_a_backbone_that_keeps_its_inputs_packed(dtype, deferred):
    """The forward pass is the same, bit for bit; input gradients do not depend on what is kept (a ReLU's decision is the sign of
    the code), within the rounding of the layers' other kernels; the parameter gradients of the last block are those of the
    restored input."""
    import torch
    from oracle import oracle as O
    from paper_2305_11624_b200.backbone import BackboneReplay, Bottleneck
    plan = [Bottleneck(64, 64, 256, 1, (12, 12)), Bottleneck(256, 64, 256, 1, (12, 12)), Bottleneck(256, 128, 512, 2, (12, 12))]
    runs = []
    for packed in (False, True):
        rp = BackboneReplay(4, plan, "tune", seed=3, dtype=dtype, async_param_grads=deferred, packed=packed)
        ins = rp.make_inputs(5)
        keep = {}
        rp.forward_backward(ins, keep)
        torch.cuda.synchronize()
        C.convbn_check()
        runs.append((rp, ins, keep))
    (_, _, plain), (rp, ins, keep) = runs
    assert torch.equal(plain["out"], keep["out"])
    f = lambda t: t.float().cpu().numpy().astype(np.float64)
    assert O.rel_l2(f(keep["dx"]), f(plain["dx"])) <= parity.TOL[dtype] * 3
    # the last 1x1 convolution: dZ = g where the output is above zero, X = the restored ReLU output in front of it
    c3 = rp.blocks[-1][2].blk
    spec = c3.spec
    shape = (4, 512, 6, 6)
    dz = I.act_from_layout(f(ins["g"]) * (f(keep["out"]) > 0), "nhwc", shape)
    q, s = P.pack(f(keep["relu_outputs"][-1][1]).ravel(), dtype)
    x = I.act_from_layout(P.unpack(q, s), "nhwc", (4, 128, 6, 6))
    t = {k: c3.fetch(k) for k in ("w", "gamma", "beta", "mu_hat", "var_hat")}
    ref = parity.oracle_tune(spec, dict(t, x=x, dz=dz, b=None))
    got = {k: c3.fetch(k) for k in ("dw", "dgamma", "dbeta")}
    parity.compare(got, ref, parity.TOL["f32"], ("dw", "dgamma", "dbeta"), "c3", dtype="f32")


@pytest.mark.gpu
def test_a_packed_backbone_needs_less_memory():
    """Of what an iteration holds, the kept inputs shrink from 2 bytes an element to 33 / 32, gradients and scratch do not: over
    six identical bottlenecks of 256 channels at 56 x 56 the inputs (384 elements a pixel and bottleneck) are most of it."""
    from paper_2305_11624_b200.backbone import BackboneReplay, Bottleneck
    plan = [Bottleneck(256, 64, 256, 1, (56, 56))] * 6
    peaks = [BackboneReplay(8, plan, "tune", seed=1, packed=packed).measure(iters=1, warmup=1)[1] for packed in (False, True)]
    assert peaks[1] < 0.75 * peaks[0], peaks


@pytest.mark.gpu
def test_packed_calls_are_captured_and_replayed_on_other_inputs():
    import torch
    from paper_2305_11624_b200.harness import Block
    spec = I.LayerSpec("captured", 3, 256, 14, 13, 64, 1, 1)
    blk = Block(spec, modes=("tune", "packed"))
    for seed in (1, 2):
        t = _relu_inputs(spec, seed)
        if seed == 1:
            blk.load(t)
            blk.tune_fwd(); blk.pack_x(); blk.tune_bwd_packed(relu_mask=True, defer_join=True); C.convbn_tune_bwd_join()
            torch.cuda.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                blk.tune_fwd()
                blk.pack_x()
                blk.tune_bwd_packed(relu_mask=True, defer_join=True)
                C.convbn_tune_bwd_join()
        blk.load(t)
        graph.replay()
        C.convbn_check()
        got = dict({n: blk.fetch(n) for n in ("dx", "dw", "dgamma", "dbeta")}, db=None)
        _compare(spec, t, got, _reference(spec, t, None, True), None, True)


@pytest.mark.gpu
def test_a_group_that_is_no_number_shows_in_the_gradients():
    """An infinity in X: its group is restored as NaN, so every gradient of its channels' weights is, and dX is masked there."""
    spec = I.LayerSpec("inf", 1, 256, 6, 5, 64, 1, 1)
    t = parity.make_inputs(spec, 4)
    t["x"][0, 40, 2, 3] = np.inf
    got = _packed_pass(spec, t, None, True)
    assert np.isnan(got["dw"][:, 32:64]).all() and np.isfinite(np.delete(got["dw"], np.s_[32:64], 1)).all()
    assert not got["dx"][0, 32:64, 2, 3].any() and np.isfinite(got["dx"]).all() and np.isfinite(got["dbeta"]).all()


@pytest.mark.gpu
def test_more_than_two_to_the_31_elements():
    import torch
    count, tail = (1 << 31) + 32 * 1001 + 5, 32 * 4000 + 5
    x = torch.empty(count, dtype=torch.bfloat16, device="cuda")
    for at in range(0, count, 1 << 28):
        x[at:at + (1 << 28)].normal_(generator=torch.Generator("cuda").manual_seed(at & 1023))
    codes, steps = torch.empty(count, dtype=torch.int8, device="cuda"), torch.empty(-(-count // 32), dtype=torch.uint8, device="cuda")
    C.convbn_pack(x, codes, steps)
    q, s = P.pack(x[count - tail:].float().cpu().numpy(), "bf16")
    assert np.array_equal(codes[count - tail:].cpu().numpy(), q) and np.array_equal(steps[(count - tail) // 32:].cpu().numpy(), s)
    x.zero_()
    C.convbn_unpack(codes, steps, x)
    C.convbn_check()
    np.testing.assert_array_equal(x[count - tail:].float().cpu().numpy().astype(np.float64), P.unpack(q, s))


@pytest.mark.gpu
def test_a_packed_backward_pass_of_more_than_two_to_the_31_elements():
    """dX of the last rows by themselves: the same bits.  dbeta: the sum over all rows of dZ = 1 and 0."""
    import torch
    rows, ci, co, tail = 8_500_000, 256, 64, 128 * 1000
    g = torch.Generator("cuda").manual_seed(1)
    codes = torch.empty(rows, ci, dtype=torch.int8, device="cuda")
    for at in range(0, rows, 1_000_000):
        codes[at:at + 1_000_000].random_(-127, 128, generator=g)
    steps = torch.full((rows, ci // 32), 121, dtype=torch.uint8, device="cuda")
    dz = (torch.arange(rows, device="cuda") % 2).to(torch.bfloat16)[:, None].expand(rows, co).contiguous()
    w = torch.randn(co, ci, device="cuda", generator=g).to(torch.bfloat16)
    mean, saved = torch.zeros(co, device="cuda"), torch.ones(3 * co, device="cuda")
    out = []
    for first in (0, rows - tail):
        n = rows - first
        d = C.convbn_linear_desc(n, ci, co)
        dx = torch.empty(n, ci, dtype=torch.bfloat16, device="cuda")
        dw, dgamma, dbeta = torch.empty(co, ci, device="cuda"), torch.empty(co, device="cuda"), torch.empty(co, device="cuda")
        ws = torch.empty(max(256, C.convbn_workspace_bytes(d, C.PHASE_TUNE_BWD_PACKED)), dtype=torch.uint8, device="cuda")
        C.convbn_tune_bwd_packed(d, dz[first:], codes[first:], steps[first:], w, None, mean, saved, dx, dw, None, dgamma, dbeta, None, True,
                                 False, ws)
        C.convbn_check()
        assert bool((dbeta == n // 2).all())
        out.append(dx[n - tail:].clone())
    assert torch.equal(out[0], out[1]) and bool((out[0][codes[rows - tail:] <= 0] == 0).all())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("rows,ci,co", [(144900, 1024, 512), (100000, 512, 1024), (1560000, 64, 128)])
def test_sums_over_many_pixels(rows, ci, co, dtype):
    """Against 64 bits.  An fp32 accumulator adds up 6144 pixels at most (half values: 1024), 384 (64) additions of 16 products.  An addition
    that cuts what does not fit is off by half a last place on average, 2^-24 of the sum so far or less, always towards zero; sums of random
    signs have 2/3 of their last size on average, which gives 384 2/3 2^-24 = 1.5e-5 (2.5e-6) of a sum.  The sums of these are rounded to
    nearest, each by 2^-25 in the mean and either way: 2^-20 for the 512 that there are at most.  Products are exact (8 or 11 bits by 7)."""
    import torch
    kind, td = (C.BF16, torch.bfloat16) if dtype == "bf16" else (C.F16, torch.float16)
    g = torch.Generator("cuda").manual_seed(3)
    x = torch.randn(rows, ci, device="cuda", generator=g).to(td)
    codes, steps = torch.empty(rows, ci, dtype=torch.int8, device="cuda"), torch.empty(rows, ci // 32, dtype=torch.uint8, device="cuda")
    C.convbn_pack(x, codes, steps)
    dz, w = torch.randn(rows, co, device="cuda", generator=g).to(td), torch.randn(co, ci, device="cuda", generator=g).to(td)
    d = C.Desc.make(rows, ci, 1, 1, co, 1, 1, dtype=kind, layout=C.NHWC)
    mean, saved = torch.zeros(co, device="cuda"), torch.ones(3 * co, device="cuda")
    dw, dgamma, dbeta = torch.empty(co, ci, device="cuda"), torch.empty(co, device="cuda"), torch.empty(co, device="cuda")
    ws = torch.empty(C.convbn_workspace_bytes(d, C.PHASE_TUNE_BWD_PACKED), dtype=torch.uint8, device="cuda")
    C.convbn_tune_bwd_packed(d, dz, codes, steps, w, None, mean, saved, x, dw, None, dgamma, dbeta, None, False, False, ws)
    C.convbn_check()
    exact, total = torch.zeros(co, ci, dtype=torch.float64, device="cuda"), torch.zeros(co, dtype=torch.float64, device="cuda")
    for at in range(0, rows, 1 << 17):
        part = slice(at, at + (1 << 17))
        step = torch.exp2(steps[part].double() - 127.0).repeat_interleave(32, 1)
        exact += dz[part].double().t() @ (codes[part].double() * step)
        total += dz[part].double().sum(0)
    rel = lambda a, b: float((a.double() - b).norm() / b.norm())
    bound = (384 if dtype == "bf16" else 64) * 2 / 3 * 2.0 ** -24 + 2.0 ** -20
    assert rel(dw, exact) <= bound and rel(dbeta, total) <= bound
    assert rel(dgamma, (exact * w.double()).sum(1)) <= bound * 2


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("n,ci,hw,co,stride,mask", [(3, 128, 15, 256, 2, True), (2, 512, 9, 192, 2, False), (3, 64, 14, 64, 3, True),
                                                     (4, 512, 12, 128, 1, True), (2, 256, 17, 64, 1, True)])
def test_an_addend_is_rounded_with_the_sum(n, ci, hw, co, stride, mask, dtype):
    """Whole numbers whose products add up without rounding in fp32, to more bits than the storage type has: dX is the sum with the
    addend, rounded, bit for bit."""
    import torch
    kind, td = (C.BF16, torch.bfloat16) if dtype == "bf16" else (C.F16, torch.float16)
    g = torch.Generator("cuda").manual_seed(n + ci)
    whole = lambda most, *shape: torch.randint(-most, most + 1, shape, device="cuda", generator=g).float()
    ho = (hw - 1) // stride + 1
    x, dz, w = whole(7, n, hw, hw, ci), whole(9, n, ho, ho, co), whole(9, co, ci)
    add = (whole(4000, n, hw, hw, ci) / 3).to(td)
    codes, steps = torch.empty(x.numel(), dtype=torch.int8, device="cuda"), torch.empty(x.numel() // 32, dtype=torch.uint8, device="cuda")
    C.convbn_pack(x.to(td), codes, steps)
    d = C.Desc.make(n, ci, hw, hw, co, 1, 1, stride, stride, dtype=kind, layout=C.NHWC)
    dx = torch.empty(n, hw, hw, ci, dtype=td, device="cuda")
    dw, dgamma, dbeta = torch.empty(co, ci, device="cuda"), torch.empty(co, device="cuda"), torch.empty(co, device="cuda")
    ws = torch.empty(max(256, C.convbn_workspace_bytes(d, C.PHASE_TUNE_BWD_PACKED)), dtype=torch.uint8, device="cuda")
    C.convbn_tune_bwd_packed(d, dz.to(td), codes, steps, w.to(td), None, torch.zeros(co, device="cuda"), torch.ones(3 * co, device="cuda"),
                             dx, dw, None, dgamma, dbeta, add, mask, False, ws)
    C.convbn_check()
    conv = torch.zeros(n, hw, hw, ci, dtype=torch.float64, device="cuda")
    conv[:, ::stride, ::stride] = dz.double() @ w.double()
    want = (conv + add.double()).float().to(td)                       # (to fp32 first, as an fp32 sum is)
    want = torch.where(x > 0, want, torch.zeros_like(want)).float() if mask else want.float()
    assert int((dx.float() != want).sum()) == 0


def _exact_weight_gradient(x, dz, k, stride, pad, groups):
    """domega' [C_out, k, k, C_in / groups] of NHWC tensors in 64 bits, some images at a time."""
    import torch
    n, h, w, ci = x.shape
    ho, wo, co = dz.shape[1:]
    cg = ci // groups
    exact = torch.zeros(co, k, k, cg, dtype=torch.float64, device="cuda")
    some = max(1, int(2e8 // (h * w * ci + ho * wo * co)))
    for at in range(0, n, some):
        xp = torch.nn.functional.pad(x[at:at + some].double(), (0, 0, pad, pad, pad, pad))
        z = dz[at:at + some].double().reshape(-1, groups, co // groups).permute(1, 2, 0)
        for r in range(k):
            for q in range(k):
                v = xp[:, r:r + (ho - 1) * stride + 1:stride, q:q + (wo - 1) * stride + 1:stride]
                exact[:, r, q] += torch.bmm(z, v.reshape(-1, groups, cg).permute(1, 0, 2)).reshape(co, cg)
    return exact


# name, n, C_in, h, w, C_out, k, stride, groups, kernel, whether the accumulators are emptied every 1024 pixels: half, bf16
LONG_SUMS = [("stem_window", 512, 3, 224, 224, 64, 7, 2, 1, "umma-stem", (False, False)),
             ("stem_packed", 256, 3, 225, 225, 64, 7, 2, 1, "umma-stem", (True, True)),
             ("stem_packed_wide", 256, 3, 64, 64, 256, 5, 2, 1, "umma-stem", (True, True)),
             ("groups_of_8", 256, 2048, 28, 28, 2048, 3, 1, 256, "grouped-mma", (False, False)),
             ("groups_of_32", 128, 64, 56, 56, 64, 3, 1, 2, "grouped-umma", (True, False)),
             ("four_taps", 16, 1024, 80, 80, 64, 2, 1, 1, "umma", (True, True)),
             ("conv3", 64, 128, 56, 56, 128, 3, 1, 1, "umma", (True, False))]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("layer", LONG_SUMS, ids=lambda l: l[0])
def test_sums_over_many_pixels_of_other_layers(layer, dtype):
    """As test_sums_over_many_pixels, with its bounds: 6144 pixels (384 additions of 16 products) where an accumulator is not emptied, 1024
    (64) where it is; partial sums of a CTA and of the CTAs after that, fewer than 512 roundings one after the other."""
    import torch
    name, n, ci, h, w, co, k, stride, groups, kernel, emptied = layer
    kind, td = (C.BF16, torch.bfloat16) if dtype == "bf16" else (C.F16, torch.float16)
    d = C.Desc.make(n, ci, h, w, co, k, k, stride, stride, k // 2, k // 2, groups=groups, dtype=kind, layout=C.NHWC)
    ho, wo = C.convbn_out_shape(d)
    g = torch.Generator("cuda").manual_seed(7)
    rand = lambda *shape: torch.randn(shape, device="cuda", generator=g).to(td)
    x, dz, wt = rand(n, h, w, ci), rand(n, ho, wo, co), rand(co, k, k, ci // groups)
    codes, steps = torch.empty(x.numel(), dtype=torch.int8, device="cuda"), torch.empty(-(-x.numel() // 32), dtype=torch.uint8, device="cuda")
    C.convbn_pack(x, codes, steps)
    mean, saved = torch.zeros(co, device="cuda"), torch.ones(3 * co, device="cuda")
    dx = torch.empty_like(x)
    dw, dgamma, dbeta = torch.empty(co, k, k, ci // groups, device="cuda"), torch.empty(co, device="cuda"), torch.empty(co, device="cuda")
    ws = torch.empty(C.convbn_workspace_bytes(d, C.PHASE_TUNE_BWD_PACKED), dtype=torch.uint8, device="cuda")
    C.convbn_tune_bwd_packed(d, dz, codes, steps, wt, None, mean, saved, dx, dw, None, dgamma, dbeta, None, False, False, ws)
    C.convbn_check()
    assert C.convbn_last_kernel(C.PHASE_TUNE_BWD_WEIGHT) == kernel
    C.convbn_unpack(codes, steps, x)
    exact, total = _exact_weight_gradient(x, dz, k, stride, k // 2, groups), dz.double().sum((0, 1, 2))
    rel = lambda a, b: float((a.double() - b).norm() / b.norm())
    bound = (64 if emptied[0 if dtype == "f16" else 1] else 384) * 2 / 3 * 2.0 ** -24 + 2.0 ** -20
    assert rel(dw, exact) <= bound and rel(dbeta, total) <= bound, (rel(dw, exact), rel(dbeta, total), bound)
    assert rel(dgamma, (exact * wt.double()).sum((1, 2, 3))) <= bound * 2


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("ci,co", [(256, 64), (64, 256)])
def test_no_number_in_the_single_kernel(ci, co, dtype):
    """test_a_group_that_is_no_number_shows_in_the_gradients with pixels enough for the kernel that reads dZ once."""
    spec = I.LayerSpec("inf", 3, ci, 30, 20, co, 1, 1, dtype=dtype)
    t = parity.make_inputs(spec, 4)
    t["x"][2, 40, 29, 18], t["x"][1, 5, 2, 3] = -np.inf, np.nan
    got = _packed_pass(spec, t, None, True, expect="umma-fused-bwd")
    assert np.isnan(got["dw"][:, :64]).all() and np.isfinite(got["dw"][:, 64:]).all()
    assert not got["dx"][2, 32:64, 29, 18].any() and not got["dx"][1, :32, 2, 3].any()
    assert np.isfinite(got["dx"]).all() and np.isfinite(got["dbeta"]).all()


@pytest.mark.gpu
def test_a_weight_gradient_that_restores_more_than_two_to_the_31_elements():
    """Only rows beyond the 2^31st element have a dZ that is not zero; whole numbers, so the sums are exact in fp32 in any order."""
    import torch
    rows, ci, co, tail = 2_200_000, 1024, 64, 100_000
    g = torch.Generator("cuda").manual_seed(1)
    codes = torch.empty(rows, ci, dtype=torch.int8, device="cuda")
    for at in range(0, rows, 500_000):
        codes[at:at + 500_000].random_(-3, 4, generator=g)
    steps = torch.full((rows, ci // 32), 127, dtype=torch.uint8, device="cuda")
    assert (rows - tail) * ci > 1 << 31
    dz = torch.zeros(rows, co, dtype=torch.bfloat16, device="cuda")
    dz[rows - tail:] = torch.randint(-2, 3, (tail, co), device="cuda", generator=g).to(torch.bfloat16)
    w = torch.randint(-2, 3, (co, ci), device="cuda", generator=g).to(torch.bfloat16)
    d = C.convbn_linear_desc(rows, ci, co)
    mean, saved = torch.zeros(co, device="cuda"), torch.ones(3 * co, device="cuda")
    dx = torch.full((rows, ci), 7.0, dtype=torch.bfloat16, device="cuda")
    dw, dgamma, dbeta = torch.empty(co, ci, device="cuda"), torch.empty(co, device="cuda"), torch.empty(co, device="cuda")
    ws = torch.empty(C.convbn_workspace_bytes(d, C.PHASE_TUNE_BWD_PACKED), dtype=torch.uint8, device="cuda")
    C.convbn_tune_bwd_packed(d, dz, codes, steps, w, None, mean, saved, dx, dw, None, dgamma, dbeta, None, True, False, ws)
    C.convbn_check()
    assert C.convbn_last_kernel(C.PHASE_TUNE_BWD_PACKED) == "umma"
    last, q = dz[rows - tail:].double(), codes[rows - tail:]
    assert torch.equal(dw.double(), last.t() @ q.double()) and torch.equal(dbeta.double(), last.sum(0))
    want = (last @ w.double()).to(torch.bfloat16) * (q > 0)
    assert torch.equal(dx[rows - tail:], want) and not bool(dx[:rows - tail].any())


def _call(spec, seed):
    """A packed backward call on tensors of its own: (call, outputs)."""
    import torch
    from paper_2305_11624_b200.harness import Block
    blk = Block(spec, modes=("tune", "packed"))
    blk.randomize(seed)
    blk.tune_fwd()
    blk.pack_x()
    outputs = [o for o in (blk.dx, blk.dw, blk.db, blk.dgamma, blk.dbeta) if o is not None]
    return lambda defer=False: blk.tune_bwd_packed(relu_mask=True, defer_join=defer), outputs


AT_ONCE = [("wide_in", 8, 256, 40, 41, 64, 1, 1), ("restoring", 8, 512, 28, 28, 128, 1, 1), ("shortcut", 4, 256, 28, 28, 512, 1, 2),
           ("conv3", 9, 64, 56, 56, 64, 3, 1)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_the_same_call_gives_the_same_bits(dtype):
    import torch
    more = [("many_rows", 150000, 64, 1, 1, 128, 1, 1), ("wide_rows", 60000, 1024, 1, 1, 64, 1, 1), ("conv3_long", 64, 64, 112, 112, 64, 3, 1)]
    for name, n, ci, h, w, co, k, stride in AT_ONCE + more:
        call, outputs = _call(I.LayerSpec(name, n, ci, h, w, co, k, k, stride=stride, pad=k // 2, dtype=dtype), 3)
        call()
        first = [o.clone() for o in outputs]
        for o in outputs:
            o.fill_(float("nan"))
        call()
        C.convbn_check()
        assert all(torch.equal(a, b) for a, b in zip(first, outputs)), name


@pytest.mark.gpu
def test_packed_calls_of_two_threads_on_streams_of_their_own():
    """Backward passes, some with a deferred join, beside packing and restoring on another thread and stream: the bits of the calls
    made one after the other."""
    import threading
    import torch
    work, expected = [], []
    for i, (name, n, ci, h, w, co, k, stride) in enumerate(AT_ONCE):
        call, outputs = _call(I.LayerSpec(name, n, ci, h, w, co, k, k, stride=stride, pad=k // 2, dtype="f16" if i % 2 else "bf16"), i)
        call()
        work.append((call, outputs))
        expected.append([o.clone() for o in outputs])
    x = torch.randn(3_000_001, device="cuda", generator=torch.Generator("cuda").manual_seed(3)).to(torch.bfloat16)
    codes, steps, back = torch.empty(x.numel(), dtype=torch.int8, device="cuda"), torch.empty(-(-x.numel() // 32), dtype=torch.uint8, device="cuda"), torch.empty_like(x)
    C.convbn_pack(x, codes, steps)
    C.convbn_unpack(codes, steps, back)
    packed = (codes.clone(), steps.clone(), back.clone())
    for _, outputs in work:
        for o in outputs:
            o.fill_(float("nan"))
    C.convbn_check()
    torch.cuda.synchronize()
    failed = []

    def run(mine):
        try:
            stream = torch.cuda.Stream()
            with torch.cuda.stream(stream):
                for turn in range(12):
                    for i in mine:
                        work[i][0](turn % 2 == 1)
                        if turn % 2:
                            C.convbn_tune_bwd_join()
                    if 0 in mine:
                        C.convbn_pack(x, codes, steps)
                        C.convbn_unpack(codes, steps, back)
            stream.synchronize()
        except Exception as e:                                           # (shown by the main thread)
            failed.append(e)

    threads = [threading.Thread(target=run, args=(mine,)) for mine in ((0, 1), (2, 3))]
    for th in threads:
        th.start()
    for th in threads:
        th.join()
    assert not failed, failed
    C.convbn_check()
    for (_, outputs), want in zip(work, expected):
        assert all(torch.equal(a, b) for a, b in zip(outputs, want))
    assert all(torch.equal(a, b) for a, b in zip((codes, steps, back), packed))


@pytest.mark.gpu
@pytest.mark.parametrize("what", ["umma-fused-bwd", "umma", "unpack", "tune_fwd", "tune_bwd", "strip", "stem", "grouped", "depthwise", "conv_transposed",
                                  "quant-mma", "quant-umma", "quant-umma-fused", "deploy"])
def test_the_first_cuda_call_of_a_thread(what):
    """A thread that has made no CUDA call has no context: the library's first call there makes the device's current."""
    import threading
    import torch
    from paper_2305_11624_b200.harness import Block
    sizes = {"umma-fused-bwd": (3, 256, 20, 15, 64, 1, 1), "umma": (3, 512, 9, 8, 128, 1, 1), "unpack": (3, 128, 9, 8, 512, 1, 1),
             "tune_fwd": (3, 512, 9, 8, 128, 1, 1), "tune_bwd": (3, 256, 20, 15, 64, 1, 1), "strip": (2, 64, 20, 24, 64, 3, 1),
             "stem": (2, 3, 64, 64, 64, 7, 2), "grouped": (2, 64, 10, 12, 64, 3, 1), "depthwise": (2, 96, 12, 11, 96, 3, 1),
             "conv_transposed": (2, 128, 14, 14, 64, 3, 2), "quant-mma": (7, 64, 1, 1, 64, 1, 1), "quant-umma": (64, 2048, 1, 1, 64, 1, 1),
             "quant-umma-fused": (20000, 64, 1, 1, 64, 1, 1), "deploy": (3, 512, 9, 8, 128, 1, 1)}
    n, ci, h, w, co, k, stride = sizes[what]
    groups = {"grouped": 8, "depthwise": 96}.get(what, 1)
    mode = ("quant",) if what.startswith("quant") else ("deploy",) if what == "deploy" else ("tune", "packed")
    blk = Block(I.LayerSpec("first", n, ci, h, w, co, k, k, stride=stride, pad=k // 2, groups=groups), modes=mode)
    blk.randomize(1)
    stream = torch.cuda.Stream()
    if mode == ("quant",):
        call, outputs = lambda: blk.deploy_fwd_quant(stream=stream.cuda_stream), ("z",)
        blk.deploy_prepare_quant()
    elif mode == ("deploy",):
        call, outputs = lambda: blk.deploy_fwd(stream=stream.cuda_stream), ("z",)
        blk.deploy_prepare()
    else:
        blk.tune_fwd()
        blk.pack_x()
        if what in ("umma-fused-bwd", "umma", "unpack"):
            call = lambda: blk.tune_bwd_packed(stream=stream.cuda_stream)
        elif what in ("tune_fwd", "strip", "stem", "grouped", "depthwise"):
            call = lambda: blk.tune_fwd(stream=stream.cuda_stream)
        else:
            call = lambda: blk.tune_bwd(stream=stream.cuda_stream)
        outputs = ("z",) if what in ("tune_fwd", "strip", "stem", "grouped", "depthwise") else ("dx", "dw", "dgamma", "dbeta")
    torch.cuda.synchronize()
    call()                                                               # (set-up that is made once a process is done)
    stream.synchronize()
    want = [getattr(blk, o).clone() for o in outputs]
    for o in outputs:
        getattr(blk, o).fill_(float("nan"))
    torch.cuda.synchronize()
    failed = []

    def run():
        try:
            call()
        except Exception as e:
            failed.append(e)

    thread = threading.Thread(target=run)
    thread.start()
    thread.join()
    assert not failed, failed
    stream.synchronize()
    C.convbn_check()
    assert all(torch.equal(getattr(blk, o), e) for o, e in zip(outputs, want))
