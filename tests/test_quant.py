"""Deploy mode in 8-bit integers: convbn_deploy_prepare_quant, convbn_deploy_fwd_quant."""
import numpy as np
import pytest

from oracle import packed_oracle as P
from paper_2305_11624_b200 import convbn as C
from paper_2305_11624_b200 import inputs as I

KIND = {"bf16": C.BF16, "f16": C.F16, "f32": C.F32}
HALF_STEP = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": 2.0 ** -24}
ROUND = {"bf16": I.round_bf16, "f16": lambda a: np.asarray(a, np.float16).astype(np.float32), "f32": lambda a: np.asarray(a, np.float32)}


def _desc(n, ci, h, w, co, dtype="bf16", stride=1, **kw):
    return C.Desc.make(n, ci, h, w, co, 1, 1, stride, stride, dtype=KIND[dtype], layout=C.NCHW if dtype == "f32" else C.NHWC, **kw)


# ---- host ------------------------------------------------------------------------------------------------------------
def test_which_layers_are_taken():
    size = lambda d: C.convbn_workspace_bytes(d, C.PHASE_DEPLOY_FWD_QUANT)
    refused = [C.Desc.make(2, 64, 8, 8, 64, 3, 3, 1, 1, 1, 1), C.Desc.make(2, 64, 8, 8, 64, 1, 1, 1, 1, 1, 0),
               C.Desc.make(2, 64, 8, 8, 64, 1, 1, groups=2), _desc(2, 64, 8, 8, 64, "f32"), _desc(1, 131073, 1, 1, 64)]
    for d in refused:
        assert size(d) == 0
        for call in (lambda: C.convbn_deploy_fwd_quant(d, 4096, 4096, 4096, 4096, 4096, None, False, 4096, 1 << 30, stream=0),
                     lambda: C.convbn_deploy_prepare_quant(d, 4096, None, 4096, 4096, 4096, 4096, 4096, 4096, 4096, stream=0)):
            with pytest.raises(C.ConvBNError) as e:
                call()
            assert e.value.status == C.EUNSUPPORTED


def test_refusals():
    d = _desc(2, 64, 8, 8, 64)
    size = C.convbn_workspace_bytes(d, C.PHASE_DEPLOY_FWD_QUANT)
    names = ("x", "w_codes", "w_scale", "b_fused", "z", "add")

    def forward(desc=d, ws=4096, bytes_=size, **over):
        a = {n: None if n == "add" else 4096 for n in names}
        a.update(over)
        with pytest.raises(C.ConvBNError) as e:
            C.convbn_deploy_fwd_quant(desc, *[a[n] for n in names], False, ws, bytes_, stream=0)
        return e.value.status

    for n in names:
        if n != "add":
            assert forward(**{n: None}) == C.EINVAL, n
        assert forward(**{n: 4096 + (2 if n in ("w_scale", "b_fused") else 8)}) == C.EALIGN, n
    if size:
        assert forward(ws=None) == C.EWORKSPACE and forward(bytes_=size - 1) == C.EWORKSPACE and forward(ws=4096 + 16) == C.EALIGN
    assert forward(desc=_desc(0, 64, 8, 8, 64)) == C.EINVAL
    assert forward(desc=C.Desc.make(2, 64, 8, 8, 64, 1, 1, dtype=C.F16, layout=C.NCHW)) == C.EUNSUPPORTED
    named = ("w", "b", "gamma", "beta", "run_mean", "run_var", "w_codes", "w_scale", "b_fused")

    def prepare(**over):
        a = {n: None if n == "b" else 4096 for n in named}
        a.update(over)
        with pytest.raises(C.ConvBNError) as e:
            C.convbn_deploy_prepare_quant(d, *[a[n] for n in named], stream=0)
        return e.value.status

    for n in named:
        if n != "b":
            assert prepare(**{n: None}) == C.EINVAL, n
        assert prepare(**{n: 4096 + (8 if n in ("w", "w_codes") else 2)}) == C.EALIGN, n


def test_the_definition_is_within_its_rounding_of_the_plain_block():
    """Against the unrounded product: an operand is off by half a step of its row, so a sum of K products is off by at most
    (a_x / 254) sum |w| + (a_w / 254) sum |xhat|, both ends worst."""
    rng = np.random.default_rng(2)
    x, w = rng.standard_normal((17, 40)), rng.standard_normal((9, 40))
    one, zero = np.ones(9), np.zeros(9)
    got = P.deploy_forward(x, w, None, one, zero, zero, one, 0.0)
    ax, aw = np.abs(x).max(1), np.abs(w).max(1)
    bound = ax[:, None] / 254 * np.abs(w).sum(1) + aw[None, :] / 254 * (np.abs(x).sum(1)[:, None] + 40 * ax[:, None] / 254)
    assert np.all(np.abs(got["z"] - x @ w.T) <= bound * (1 + 1e-5))


# ---- device ----------------------------------------------------------------------------------------------------------
def _draw(n, ci, h, w, co, dtype, stride, bias, with_add, seed=0):
    rng = np.random.default_rng(seed + n + ci + co)
    r = lambda a: ROUND[dtype](a.astype(np.float32)).astype(np.float64)
    ho, wo = (h - 1) // stride + 1, (w - 1) // stride + 1
    f32 = lambda a: a.astype(np.float32).astype(np.float64)
    t = dict(x=r(rng.standard_normal((n, h, w, ci)) * np.exp(rng.standard_normal(ci))), w=r(rng.standard_normal((co, ci)) * np.sqrt(2.0 / ci)),
             b=f32(rng.standard_normal(co)) if bias else None, gamma=f32(rng.uniform(0.5, 1.5, co) * np.sign(rng.standard_normal(co))),
             beta=f32(rng.standard_normal(co) * 0.1), mu_hat=f32(rng.standard_normal(co) * 0.1), var_hat=f32(rng.uniform(0.5, 2.0, co)))
    t["add"] = r(rng.standard_normal((n * ho * wo, co))) if with_add else None
    return t


def _run(t, desc, dtype, relu, ws_fill=0xFF):
    import torch
    td = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}[dtype]
    dev = lambda a, d=torch.float32: None if a is None else torch.from_numpy(np.ascontiguousarray(a, np.float32)).cuda().to(d)
    co, ci = t["w"].shape
    ho, wo = C.convbn_out_shape(desc)
    rows, pitch = desc.n * ho * wo, -(-ci // 16) * 16
    codes = torch.full((co * pitch + 64,), 99, dtype=torch.int8, device="cuda")
    scale, shift = torch.full((co + 4,), 5.0, device="cuda"), torch.full((co + 4,), 5.0, device="cuda")
    C.convbn_deploy_prepare_quant(desc, dev(t["w"], td), dev(t["b"]), dev(t["gamma"]), dev(t["beta"]), dev(t["mu_hat"]), dev(t["var_hat"]),
                                  codes, scale, shift)
    z = torch.full((rows * co + 64,), 9.0, dtype=td, device="cuda")
    size = C.convbn_workspace_bytes(desc, C.PHASE_DEPLOY_FWD_QUANT)
    room = torch.full((size + 256,), ws_fill, dtype=torch.uint8, device="cuda")
    C.convbn_deploy_fwd_quant(desc, dev(t["x"], td), codes, scale, shift, z, dev(t["add"], td), relu, room, size)
    C.convbn_check()
    assert bool((room[size:] == ws_fill).all()) and bool((z[rows * co:] == 9.0).all())
    assert bool((codes[co * pitch:] == 99).all()) and bool((scale[co:] == 5.0).all()) and bool((shift[co:] == 5.0).all())
    f = lambda a: a.float().cpu().numpy().astype(np.float64)
    return {"z": f(z[:rows * co]).reshape(rows, co), "w_codes": codes[:co * pitch].cpu().numpy().reshape(co, pitch),
            "w_scale": f(scale[:co]), "b_fused": f(shift[:co])}


def _check(got, t, dtype, stride, relu):
    x = t["x"][:, ::stride, ::stride].reshape(-1, t["w"].shape[1])
    ref = P.deploy_forward(x, t["w"], t["b"], t["gamma"], t["beta"], t["mu_hat"], t["var_hat"], 1e-5, t["add"], relu)
    ci = t["w"].shape[1]
    assert np.array_equal(got["w_codes"][:, :ci], ref["w_codes"]) and not got["w_codes"][:, ci:].any()
    # var + eps, root, reciprocal, gamma r, 1 / 127, a times it, their product: seven roundings
    tiny = 2.0 ** -24
    assert np.all(np.abs(got["w_scale"] - ref["w_scale"]) <= 7 * tiny * np.abs(ref["w_scale"]))
    parts = np.abs((0 if t["b"] is None else t["b"])) + np.abs(t["mu_hat"])
    s = np.abs(t["gamma"]) / np.sqrt(t["var_hat"] + 1e-5)
    assert np.all(np.abs(got["b_fused"] - ref["b_fused"]) <= 8 * tiny * (parts * s + np.abs(t["beta"])))
    # the sum as a float, a / 127 of the row (two), the channel's scale (seven), two products and the shift (eight of its own), the
    # addend; then one rounding to the storage type (2^-25: half of half precision's smallest number)
    arithmetic = 12 * tiny * np.abs(ref["product"]) + 8 * tiny * (parts * s + np.abs(t["beta"])) + tiny * np.abs(ref["before_add"])
    u = HALF_STEP[dtype] * (1 + 2.0 ** -6)
    total = ref["before_add"] if t["add"] is None else ref["before_add"] + t["add"]
    bound = arithmetic + (u + tiny) * np.abs(total) + 2.0 ** -25
    err = np.abs(got["z"] - ref["z"])
    assert np.all(err <= bound), float((err / bound).max())


SIZES = [(1, 1, 1, 1, 1), (1, 64, 1, 1, 64), (1, 2048, 1, 1, 1000), (2, 500, 1, 1, 10), (7, 256, 1, 1, 129), (16, 24, 1, 1, 2048),
         (17, 130, 1, 1, 40), (33, 1024, 1, 1, 256), (100, 512, 1, 1, 130), (128, 64, 1, 1, 64), (129, 96, 1, 1, 200), (300, 2000, 1, 1, 72),
         (1000, 256, 1, 1, 64), (2, 64, 13, 11, 256), (3, 256, 9, 15, 64), (1, 1024, 14, 14, 512), (2, 2048, 7, 7, 512), (5, 8, 3, 7, 8),
         (40, 512, 7, 7, 2048), (6, 192, 21, 19, 320), (9500, 520, 1, 1, 1032), (1700, 1032, 1, 1, 1500), (300, 4104, 1, 1, 2056),
         # rows enough for the kernel that makes codes on its way (148 units of 128)
         (19000, 256, 1, 1, 64), (20001, 64, 1, 1, 256), (19500, 128, 1, 1, 200), (25000, 192, 1, 1, 320), (19001, 40, 1, 1, 129),
         (40000, 16, 1, 1, 8), (19200, 256, 1, 1, 1032), (31, 64, 27, 28, 640)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
def test_forward_against_the_definition(size, dtype):
    n, ci, h, w, co = size
    if dtype == "f32" and h * w > 1:
        n, h, w = n * h * w, 1, 1
    for bias, with_add, relu in ((False, False, False), (True, True, True)):
        t = _draw(n, ci, h, w, co, dtype, 1, bias, with_add)
        _check(_run(t, _desc(n, ci, h, w, co, dtype), dtype, relu), t, dtype, 1, relu)


# rows to codes on the way to the product; codes in the workspace first (the others: few rows, one launch)
FUSED = [(19000, 256, 1, 1, 64), (20001, 64, 1, 1, 256), (19500, 128, 1, 1, 200), (25000, 192, 1, 1, 320), (19001, 40, 1, 1, 129),
         (40000, 16, 1, 1, 8), (31, 64, 27, 28, 640)]
TWO_KERNELS = [(300, 2000, 1, 1, 72), (2, 2048, 7, 7, 512), (40, 512, 7, 7, 2048), (6, 192, 21, 19, 320), (9500, 520, 1, 1, 1032),
               (1700, 1032, 1, 1, 1500), (300, 4104, 1, 1, 2056), (19200, 256, 1, 1, 1032)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_which_kernels_a_size_takes(dtype):
    import torch
    units = 128 * torch.cuda.get_device_properties(0).multi_processor_count      # rows that give every SM a unit
    td = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}[dtype]
    zeros = lambda count, t=torch.float32: torch.zeros(count, dtype=t, device="cuda")

    def taken(n, ci, h, w, co, stride=1):
        d = _desc(n, ci, h, w, co, dtype, stride)
        ho, wo = C.convbn_out_shape(d)
        size = C.convbn_workspace_bytes(d, C.PHASE_DEPLOY_FWD_QUANT)
        C.convbn_deploy_fwd_quant(d, zeros(n * h * w * ci, td), zeros(co * (-(-ci // 16) * 16), torch.int8), zeros(co), zeros(co),
                                  zeros(n * ho * wo * co, td), None, False, zeros(max(256, size), torch.uint8))
        C.convbn_check()
        name = C.convbn_last_kernel(C.PHASE_DEPLOY_FWD_QUANT)
        assert (size > 0) == (name == "umma")
        return name, n * ho * wo

    for size in SIZES:
        n, ci, h, w, co = size
        if dtype == "f32" and h * w > 1:
            n, h, w = n * h * w, 1, 1
        name, rows = taken(n, ci, h, w, co)
        if size in FUSED:
            assert rows < units or name == "umma-fused", (size, name)
        else:
            assert name == ("umma" if size in TWO_KERNELS else "mma"), (size, name)
    if dtype == "f32":
        return
    for size, fused in (((14, 256, 111, 114, 64), True), ((7, 96, 160, 161, 40), False)):
        name, rows = taken(*size, stride=2)
        assert rows >= units and name == ("umma-fused" if fused else "umma"), (size, name)


@pytest.mark.gpu
@pytest.mark.parametrize("size", [(2, 256, 15, 14, 512), (1, 40, 7, 9, 24), (3, 512, 28, 28, 128), (14, 256, 111, 114, 64), (7, 96, 160, 161, 40)], ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("stride", [2, 3])
def test_strided_shortcuts(size, stride):
    n, ci, h, w, co = size
    t = _draw(n, ci, h, w, co, "bf16", stride, True, True)
    _check(_run(t, _desc(n, ci, h, w, co, "bf16", stride), "bf16", True), t, "bf16", stride, True)


@pytest.mark.gpu
@pytest.mark.parametrize("size,stride,kernel", [((14, 256, 111, 114, 64), 2, "umma-fused"), ((7, 96, 160, 161, 40), 2, "umma"),
                                                ((2, 256, 15, 14, 512), 3, "mma")], ids=lambda s: "x".join(map(str, s)) if type(s) is tuple else s)
def test_strided_shortcuts_in_half(size, stride, kernel):
    n, ci, h, w, co = size
    t = _draw(n, ci, h, w, co, "f16", stride, True, True)
    got = _run(t, _desc(n, ci, h, w, co, "f16", stride), "f16", True)
    assert C.convbn_last_kernel(C.PHASE_DEPLOY_FWD_QUANT) == kernel
    _check(got, t, "f16", stride, True)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,ci", [(40, 64), (20000, 64), (20000, 256), (3000, 512)])
def test_strides_that_leave_no_pixel_out(rows, ci, dtype):
    """One pixel per image, or one line of them and a stride across lines: the rows of X are side by side all the same."""
    t = _draw(rows, ci, 1, 1, 64, dtype, 1, True, True)
    _check(_run(t, _desc(rows, ci, 1, 1, 64, dtype, 2), dtype, True), t, dtype, 1, True)
    if dtype != "f32":
        t["x"] = t["x"].reshape(rows // 20, 1, 20, ci)
        desc = C.Desc.make(rows // 20, ci, 1, 20, 64, 1, 1, 9, 1, dtype=C.BF16, layout=C.NHWC)
        _check(_run(t, desc, dtype, True), t, dtype, 1, True)


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [3, 200])
def test_rows_and_channels_that_are_zero_tiny_infinite_or_not_numbers(rows):
    t = _draw(rows, 128, 1, 1, 64, "bf16", 1, True, False)
    t["x"][0] = 0.0
    t["x"][1] = ROUND["bf16"](np.full((1, 1, 128), 1e-35, np.float32))
    t["w"][5] = 0.0
    t["w"][6] = ROUND["bf16"](np.full(128, 1e-33, np.float32))
    t["gamma"][7] = 0.0
    _check(_run(t, _desc(rows, 128, 1, 1, 64), "bf16", False), t, "bf16", 1, False)
    t["x"][2, 0, 0, 77] = np.inf
    t["x"][rows - 1, 0, 0, 0] = np.nan
    t["w"][9, 3] = -np.inf
    got = _run(t, _desc(rows, 128, 1, 1, 64), "bf16", False)["z"]
    bad = np.zeros((rows, 64), bool)
    bad[[2, rows - 1]] = True
    bad[:, 9] = True
    assert np.array_equal(np.isnan(got), bad) and np.isfinite(got[~bad]).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,largest", [("bf16", 255 * 2.0 ** 120), ("f32", 1.9 * 2.0 ** 127), ("f16", 65504.0)])
@pytest.mark.parametrize("rows,ci,kernel", [(5, 128, "mma"), (64, 2048, "umma"), (19008, 128, "umma-fused")])
def test_rows_and_channels_near_the_largest_value(rows, ci, kernel, dtype, largest):
    """Reciprocals of maxima above 2^126 are subnormal.  Channel c has its largest weight where rows are zero and code 1 at one other
    place, so z is a row's code there, one after the other, times the scales: no sum passes the range."""
    rng = np.random.default_rng(9)
    t = _draw(rows, ci, 1, 1, 64, dtype, 1, False, False)
    t["beta"], t["mu_hat"] = t["beta"] * 0, t["mu_hat"] * 0
    t["w"] = np.zeros((64, ci))
    t["w"][:, 1] = ROUND[dtype](rng.uniform(0.5, 1.0, 64).astype(np.float32))
    t["w"][np.arange(64), 2 + np.arange(64)] = ROUND[dtype]((t["w"][:, 1] * 0.0082).astype(np.float32))
    t["x"][..., 1] = 0.0
    plain = t["x"].copy()
    for r, top in enumerate((largest, largest / 2, largest / 1.9, 1.01 * largest / 2)):
        t["x"][r] = ROUND[dtype]((rng.uniform(-1, 1, ci) * top).astype(np.float32))
        t["x"][r, 0, 0, :2] = float(ROUND[dtype](np.float32(-top))), 0.0
    got = _run(t, _desc(rows, ci, 1, 1, 64, dtype), dtype, False)
    assert C.convbn_last_kernel(C.PHASE_DEPLOY_FWD_QUANT) == kernel and np.isfinite(got["z"]).all()
    assert set(np.unique(got["w_codes"])) == {0, 1, 127}
    _check(got, t, dtype, 1, False)
    # channels of such weights
    t["x"] = plain
    scale = largest / t["w"][:4, 1] / np.array([1.0, 2.0, 1.9, 1.98])
    t["w"][:4] = ROUND[dtype]((t["w"][:4] * scale[:, None]).astype(np.float32))
    got = _run(t, _desc(rows, ci, 1, 1, 64, dtype), dtype, False)
    assert np.isfinite(got["w_scale"]).all()
    _check(got, t, dtype, 1, False)


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [1, 300])
@pytest.mark.parametrize("ci", [131072, 131071])
def test_the_longest_sums(rows, ci):
    """All codes 127: 127^2 131072 is below 2^31 by 1.6 %.  x = 1 and omega = -1, then 1 in every other channel."""
    import torch
    co = 72
    d = _desc(rows, ci, 1, 1, co)
    x, w = torch.ones(rows, ci, dtype=torch.bfloat16, device="cuda"), torch.ones(co, ci, dtype=torch.bfloat16, device="cuda")
    w[::2] = -1
    one, zero = torch.ones(co, device="cuda"), torch.zeros(co, device="cuda")
    codes = torch.empty(co * 131072, dtype=torch.int8, device="cuda")
    scale, shift = torch.empty(co, device="cuda"), torch.empty(co, device="cuda")
    C.convbn_deploy_prepare_quant(d, w, None, one, zero, zero, one - 1e-5, codes, scale, shift)
    z = torch.empty(rows, co, dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(max(256, C.convbn_workspace_bytes(d, C.PHASE_DEPLOY_FWD_QUANT)), dtype=torch.uint8, device="cuda")
    C.convbn_deploy_fwd_quant(d, x, codes, scale, shift, z, None, False, ws)
    C.convbn_check()
    sign = torch.ones(co, device="cuda")
    sign[::2] = -1
    assert bool((z.float() == sign * 131072.0).all())              # (131071 too, rounded to bf16)


# ---- together, as a deployed network uses them ---------------------------------------------------------------------------
@pytest.mark.gpu
def test_a_deployed_bottleneck_of_three_calls_captured_and_replayed():
    """A reducing layer, a wide one and one row after the other on a stream of their own, in one captured graph, replayed on other
    inputs: every result is that of the definition for the stored result of the layer before."""
    import torch
    from paper_2305_11624_b200.harness import Block
    specs = [I.LayerSpec("q1", 7, 256, 28, 28, 64, 1, 1), I.LayerSpec("q2", 7, 64, 28, 28, 640, 1, 1), I.LayerSpec("q3", 7, 640, 28, 28, 72, 1, 1)]
    blocks = [Block(s, modes=("quant",)) for s in specs]
    for k, b in enumerate(blocks):
        b.randomize(k)
        b.deploy_prepare_quant()
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()

    def chain():
        for k, b in enumerate(blocks):
            if k:
                b.x = blocks[k - 1].z
            b.deploy_fwd_quant(relu=k < 2)

    with torch.cuda.stream(stream):
        chain()
    stream.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        chain()
    for seed in (5, 6):
        blocks[0].x.copy_(torch.randn(blocks[0].x.numel(), generator=torch.Generator("cuda").manual_seed(seed), device="cuda").to(torch.bfloat16))
        graph.replay()
        C.convbn_check()
        for k, b in enumerate(blocks):
            f = lambda t: t.float().cpu().numpy().astype(np.float64)
            t = dict(x=f(b.x).reshape(7, 28, 28, -1), w=f(b.w).reshape(b.spec.c_out, -1), b=None, gamma=f(b.gamma), beta=f(b.beta), mu_hat=f(b.mu_hat),
                     var_hat=f(b.var_hat), add=None)
            got = {"z": f(b.z).reshape(-1, b.spec.c_out), "w_codes": b.w_codes.cpu().numpy().reshape(b.spec.c_out, -1), "w_scale": f(b.w_scale),
                   "b_fused": f(b.b_fused)}
            _check(got, t, "bf16", 1, k < 2)


@pytest.mark.gpu
@pytest.mark.parametrize("rows,ci,co", [(9_000_000, 256, 64), (1_100_000, 2048, 64)])
def test_inputs_of_more_than_two_to_the_31_elements(rows, ci, co):
    """The last rows by themselves give the same bits: they are the same rows, by the same kernel."""
    import torch
    g = torch.Generator("cuda").manual_seed(1)
    x = torch.empty(rows, ci, dtype=torch.bfloat16, device="cuda")
    for at in range(0, rows, 500_000):
        x[at:at + 500_000].normal_(generator=g)
    pitch, tail = -(-ci // 16) * 16, 150_000
    codes = torch.randint(-127, 128, (co, pitch), dtype=torch.int8, device="cuda", generator=g)
    scale, shift = torch.rand(co, device="cuda", generator=g), torch.rand(co, device="cuda", generator=g)
    out = []
    for part in (x, x[rows - tail:]):
        d = C.convbn_linear_desc(part.shape[0], ci, co)
        z = torch.empty(part.shape[0], co, dtype=torch.bfloat16, device="cuda")
        ws = torch.empty(max(256, C.convbn_workspace_bytes(d, C.PHASE_DEPLOY_FWD_QUANT)), dtype=torch.uint8, device="cuda")
        C.convbn_deploy_fwd_quant(d, part, codes, scale, shift, z, None, False, ws)
        C.convbn_check()
        out.append(z[part.shape[0] - tail:].clone())
    assert torch.equal(out[0], out[1]) and bool(out[0].float().abs().sum() > 0)


@pytest.mark.gpu
def test_calls_of_two_threads_on_streams_of_their_own():
    """Each kernel beside each other one, with workspaces of their own: the bits of the calls made one after the other."""
    import threading
    import torch
    from paper_2305_11624_b200.harness import Block
    blocks = [Block(I.LayerSpec("t%d" % i, *s, 1, 1), modes=("quant",)) for i, s in
              enumerate([(60, 256, 28, 28, 64), (40, 512, 20, 20, 640), (40, 64, 28, 28, 256), (1, 2048, 1, 1, 1000)])]
    expected = []
    for k, b in enumerate(blocks):
        b.randomize(k)
        b.deploy_prepare_quant()
        b.deploy_fwd_quant(relu=True)
        expected.append((b.z.clone(), b.w_codes.clone(), b.w_scale.clone(), b.b_fused.clone()))
        b.z.fill_(float("nan"))
    C.convbn_check()
    torch.cuda.synchronize()
    failed = []

    def run(mine):
        try:
            stream = torch.cuda.Stream()
            with torch.cuda.stream(stream):
                for _ in range(30):
                    for b in mine:
                        b.deploy_prepare_quant()
                        b.deploy_fwd_quant(relu=True)
            stream.synchronize()
        except Exception as e:                                           # (shown by the main thread)
            failed.append(e)

    threads = [threading.Thread(target=run, args=(mine,)) for mine in (blocks[:2], blocks[2:])]
    for th in threads:
        th.start()
    for th in threads:
        th.join()
    assert not failed, failed
    C.convbn_check()
    for b, want in zip(blocks, expected):
        assert all(torch.equal(a, e) for a, e in zip((b.z, b.w_codes, b.w_scale, b.b_fused), want))
