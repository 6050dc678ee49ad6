"""What trains a block whose statistics are not frozen, as measurable cases: the batch-independent normalisation and the update.

- "norm_fwd", "norm_bwd": group norm with its activation over channels-last activations, forward and backward.
- "ortho": an update made orthogonal by five Newton-Schulz products, one matrix or a stack of them.
- "muon": the optimiser's whole step over a list of layers: momentum, orthogonal update, weights in fp32 and in storage type.

A case is one pass.  Layer shapes are those of the benchmark configurations and of a ResNet-50, or generic.
"""
import math

import torch

own = False

DEVICE = "cuda:0"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
ELEMENT_BYTES = {"f32": 4, "bf16": 2, "f16": 2}
EPS = 1e-5
COEFFICIENTS = (3.4445, -4.7750, 2.0315)         # of X, (X X^T) X and (X X^T)^2 X in one Newton-Schulz step
STEPS = 5
NORM_EPS = 1e-7                                  # added to the norm an update is divided by
LR, MOMENTUM, DECAY = 0.02, 0.95, 0.01


# ---- cases -------------------------------------------------------------------------------------------------------
def _norm(kind, n, c, h, w, groups, act="relu", dtype="bf16"):
    return dict(kind=kind, n=n, c=c, h=h, w=w, groups=groups, act=act, dtype=dtype)


def _ortho(rows, cols, count=1, dtype="f32"):
    return dict(kind="ortho", rows=rows, cols=cols, count=count, dtype=dtype)


def _muon(layers, dtype="bf16"):
    """layers: "rowsxcols" of every layer, C_out and the weights per output channel, with "*k" for k alike."""
    return dict(kind="muon", layers=layers, dtype=dtype)


RESNET50 = " ".join((
    "64x147", "64x64", "64x576*3", "256x64*4", "64x256*2", "128x256", "128x1152*4", "512x128*4", "512x256", "128x512*3",
    "256x512", "256x2304*6", "1024x256*6", "1024x512", "256x1024*5", "512x1024", "512x4608*3", "2048x512*3", "2048x1024",
    "512x2048*2"))


def listed():
    named = lambda name, case: dict(case, name=name)
    return [
        # a small fp32 block: launches count
        named("norm_fwd_small_f32", _norm("norm_fwd", 2, 32, 16, 16, 8, dtype="f32")),
        # the widest activation of a stage-2 bottleneck at an ordinary batch
        named("norm_fwd_stage2", _norm("norm_fwd", 32, 256, 56, 56, 32)),
        # a detection backbone: two images, large odd maps
        named("norm_fwd_detection", _norm("norm_fwd", 2, 256, 200, 334, 32)),
        # a mobile network's expanded map in half precision, three channels a group: the largest activation
        named("norm_fwd_expanded_f16", _norm("norm_fwd", 64, 96, 112, 112, 32, "silu", "f16")),
        # the last stage: few pixels, many channels
        named("norm_bwd_stage5", _norm("norm_bwd", 64, 2048, 7, 7, 32)),
        # the detection map's backward pass
        named("norm_bwd_detection", _norm("norm_bwd", 2, 256, 200, 334, 32)),
        # the expanded map's backward pass
        named("norm_bwd_expanded_f16", _norm("norm_bwd", 64, 96, 112, 112, 32, "silu", "f16")),
        # the first 1x1 layer of a ResNet: latency counts
        named("ortho_small", _ortho(64, 64)),
        # one 3x3 layer of the last stage
        named("ortho_3x3_stage5", _ortho(512, 4608)),
        # a stack of wide projections whose update is kept in the storage type
        named("ortho_wide_stack_bf16", _ortho(2048, 8192, 2, "bf16")),
        # a classifier: an odd number of rows
        named("muon_classifier", _muon("1000x2048", "f16")),
        # all convolutions of a ResNet-50
        named("muon_resnet50", _muon(RESNET50)),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case: the kinds of the listed ones at sizes spread over their logarithm, odd ones among them."""
    kind = rng.choice(("norm_fwd", "norm_fwd", "norm_bwd", "norm_bwd", "ortho", "ortho", "muon"))
    if kind.startswith("norm"):
        dtype = rng.choice(("f32", "bf16", "bf16", "f16"))
        most = 64 * 112 * 112 * 96 * 2 // ELEMENT_BYTES[dtype]
        while True:
            groups = rng.choice((1, 4, 8, 16, 32, 32, 32))
            c = groups * _log_int(rng, 1, max(1, 2048 // groups))
            h = _log_int(rng, 1, 256)
            w = max(1, min(334, int(h * rng.uniform(0.75, 1.7))))
            n = _log_int(rng, 1, 64)
            if 1000 <= n * c * h * w <= most:
                return _norm(kind, n, c, h, w, groups, rng.choice(("none", "relu", "silu")), dtype)
    if kind == "ortho":
        largest = work(_ortho(2048, 8192, 2))["flops"]
        while True:
            case = _ortho(_log_int(rng, 16, 4096), _log_int(rng, 16, 8192), rng.choice((1, 1, 1, 2, 3, 8)), rng.choice(("f32", "bf16", "f16")))
            if work(case)["flops"] <= largest:
                return case
    names = set()
    for _ in range(rng.randint(1, 12)):
        taps = rng.choice((1, 1, 9))
        names.add("%dx%d" % (_log_int(rng, 16, 1024), taps * _log_int(rng, 16, 2048 // taps)))
    return _muon(" ".join(sorted(names)), rng.choice(("f32", "bf16", "f16")))


def _layers(case):
    """[(rows, cols)] of a muon case."""
    out = []
    for item in case["layers"].split():
        shape, _, times = item.partition("*")
        out += [tuple(int(v) for v in shape.split("x"))] * int(times or 1)
    return out


def work(case):
    """Each input read once, each output written once; products with the symmetric ones (X X^T and its square) counted half."""
    if case["kind"].startswith("norm"):
        n, c, g, pixels, es = case["n"], case["c"], case["groups"], case["h"] * case["w"], ELEMENT_BYTES[case["dtype"]]
        tensors = 2 if case["kind"] == "norm_fwd" else 3
        vectors = 2 * c if case["kind"] == "norm_fwd" else 4 * c
        return dict(bytes=tensors * n * c * pixels * es + 4 * vectors + 8 * n * g, flops=(8 if tensors == 2 else 16) * n * c * pixels)
    if case["kind"] == "ortho":
        shapes = [(case["rows"], case["cols"])] * case["count"]
        per = 2 * ELEMENT_BYTES[case["dtype"]]
    else:
        shapes = _layers(case)
        per = 4 + 8 + 8 + (ELEMENT_BYTES[case["dtype"]] if case["dtype"] != "f32" else 0)      # gradient, momentum, weights
    size, products = 0, 0
    for rows, cols in shapes:
        m, n = min(rows, cols), max(rows, cols)
        size += rows * cols
        products += STEPS * (3 * m * m * n + m * m * m)
    return dict(bytes=per * size, flops=products)


# ---- what a program has in hand ----------------------------------------------------------------------------------
def _gradient(randn, rows, cols, count):
    """Sums of outer products over fewer directions than the matrix has, and noise: what a weight gradient looks like."""
    inner = max(1, min(rows, cols) // 4)
    fall = torch.exp(-4.0 * torch.arange(inner, device=DEVICE) / inner)
    g = torch.bmm(randn(count, rows, inner) * fall, randn(count, inner, cols)) / math.sqrt(inner)
    return g.add_(randn(count, rows, cols), alpha=0.05).mul_(1e-3)


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(seed)
    t, kind = DTYPES[case["dtype"]], case["kind"]
    randn = lambda *shape: torch.randn(*shape, generator=gen, device=DEVICE)
    if kind == "ortho":
        g = _gradient(randn, case["rows"], case["cols"], case["count"]).to(t)
        return dict(case=case, g=g, out=torch.empty_like(g))
    if kind == "muon":
        # the layers' tensors are parts of one buffer each, as a bucket of gradients has them
        shapes, at, total = _layers(case), [], 0
        for rows, cols in shapes:
            at.append(total)
            total += -(-rows * cols // 64) * 64
        grad, momentum, master = (torch.zeros(total, device=DEVICE) for _ in range(3))
        parts = lambda flat: [flat[o:o + r * k].view(r, k) for o, (r, k) in zip(at, shapes)]
        for g, v, m in zip(parts(grad), parts(momentum), parts(master)):
            g.copy_(_gradient(randn, *g.shape, 1)[0])
            v.copy_(_gradient(randn, *g.shape, 1)[0] * 5.0)
            m.copy_(randn(*g.shape) * math.sqrt(2.0 / g.shape[1]))
        weight = master.to(t) if t != torch.float32 else None
        return dict(case=case, flat=[f for f in (momentum, master, weight) if f is not None], grad=parts(grad), momentum=parts(momentum),
                    master=parts(master), weight=parts(weight) if weight is not None else [None] * len(shapes))
    n, c, h, w, groups = (case[k] for k in ("n", "c", "h", "w", "groups"))
    # a convolution's outputs: channels of their own offset and spread
    x = (randn(n, h, w, c) * torch.exp(0.3 * randn(c)) + 0.5 * randn(c)).to(t)
    gamma, beta = torch.rand(c, generator=gen, device=DEVICE) + 0.5, randn(c) * 0.1
    s = dict(case=case, x=x, gamma=gamma, beta=beta)
    if kind == "norm_fwd":
        return dict(s, z=torch.empty_like(x), saved=torch.empty(2, n, groups, device=DEVICE))
    part = x.view(n, h * w, groups, c // groups).double()
    mean = part.mean((1, 3))
    var = (part - mean[:, None, :, None]).square().mean((1, 3))
    del part
    empty = lambda: torch.empty(c, device=DEVICE)
    return dict(s, saved=torch.stack((mean, torch.rsqrt(var + EPS))).float(), dz=randn(n, h, w, c).to(t), dx=torch.empty_like(x),
                dgamma=empty(), dbeta=empty())


# ---- one pass ----------------------------------------------------------------------------------------------------
def run(state):
    return (_own if own else _plain)[state["case"]["kind"]](state)


# The plain forms.
def _grouped(s, t):
    """[n, pixels, groups, channels of a group]"""
    n, h, w, c = t.shape
    return t.view(n, h * w, s["case"]["groups"], -1)


def _plain_norm_fwd(s):
    c = s["case"]
    x = _grouped(s, s["x"]).float()
    mean = x.mean((1, 3), keepdim=True)
    centred = x - mean
    rstd = torch.rsqrt(centred.square().mean((1, 3), keepdim=True) + EPS)
    y = centred * rstd * s["gamma"].view(c["groups"], -1) + s["beta"].view(c["groups"], -1)
    if c["act"] == "relu":
        y = torch.where(y > 0, y, 0.0)
    elif c["act"] == "silu":
        y = y / (1.0 + torch.exp(-y))
    return [y.view(s["x"].shape).to(s["x"].dtype), torch.stack((mean.view(c["n"], -1), rstd.view(c["n"], -1)))]


def _plain_norm_bwd(s):
    c = s["case"]
    gamma, beta = s["gamma"].view(c["groups"], -1), s["beta"].view(c["groups"], -1)
    mean, rstd = s["saved"][0][:, None, :, None], s["saved"][1][:, None, :, None]
    x, dy = _grouped(s, s["x"]), _grouped(s, s["dz"]).float()
    xhat = (x.float() - mean) * rstd
    if c["act"] == "relu":           # the sign of a value next to zero decides a gradient
        dy = torch.where((x.double() - mean) * rstd * gamma.double() + beta > 0, dy, 0.0)
    elif c["act"] == "silu":
        y = xhat * gamma + beta
        gate = 1.0 / (1.0 + torch.exp(-y))
        dy = dy * gate * (1.0 + y * (1.0 - gate))
    weighted = dy * gamma
    first = weighted.mean((1, 3), keepdim=True)
    second = (weighted * xhat).mean((1, 3), keepdim=True)
    dx = (weighted - first - xhat * second) * rstd
    # sums over all pixels: in 64 bits
    dgamma = (dy * xhat).sum((0, 1), dtype=torch.float64)
    dbeta = dy.sum((0, 1), dtype=torch.float64)
    return [dx.view(s["x"].shape).to(s["x"].dtype), dgamma.view(-1).float(), dbeta.view(-1).float()]


def _newton_schulz(g):
    """[count, rows, cols] in fp32"""
    tall = g.shape[1] > g.shape[2]
    x = g.transpose(1, 2) if tall else g
    top = x.abs().amax((1, 2), keepdim=True).clamp(min=1e-30)              # (squares of small updates leave fp32's range)
    norm = (x / top).square().sum((1, 2), keepdim=True).sqrt() * top
    x = x / (norm + NORM_EPS)
    a, b, c = COEFFICIENTS
    for _ in range(STEPS):
        gram = torch.bmm(x, x.transpose(1, 2))
        x = a * x + torch.bmm(b * gram + c * torch.bmm(gram, gram), x)
    return x.transpose(1, 2) if tall else x


def _plain_ortho(s):
    return [_newton_schulz(s["g"].float()).to(s["g"].dtype).contiguous()]


def _plain_muon(s):
    for grad, momentum, master, weight in zip(s["grad"], s["momentum"], s["master"], s["weight"]):
        momentum.mul_(MOMENTUM).add_(grad)
        update = _newton_schulz((grad + MOMENTUM * momentum)[None])[0]
        rows, cols = update.shape
        master.mul_(1.0 - LR * DECAY).sub_(update, alpha=LR * math.sqrt(max(1.0, rows / cols)))
        if weight is not None:
            weight.copy_(master)
    return s["flat"]


_plain = {"norm_fwd": _plain_norm_fwd, "norm_bwd": _plain_norm_bwd, "ortho": _plain_ortho, "muon": _plain_muon}


# The framework's calls.  Descriptor, list of layers and workspace are made at the first pass and kept with the other buffers.
def _call(s, make):
    if "call" not in s:
        s["call"] = make()
    return s["call"]


def _norm_call(s):
    from paper_2305_11624_b200 import convbn as C
    c = s["case"]
    desc = C.NormDesc.make(c["n"], c["c"], c["h"], c["w"], c["groups"], act={"none": C.ACT_NONE, "relu": C.ACT_RELU, "silu": C.ACT_SILU}[c["act"]],
                           dtype={"f32": C.F32, "bf16": C.BF16, "f16": C.F16}[c["dtype"]], eps=EPS)
    return C, desc, torch.empty(C.convbn_group_norm_workspace_bytes(desc), dtype=torch.uint8, device=DEVICE)


def _own_norm_fwd(s):
    C, desc, workspace = _call(s, lambda: _norm_call(s))
    C.convbn_group_norm_fwd(desc, s["x"], s["gamma"], s["beta"], s["z"], s["saved"], workspace)
    return [s["z"], s["saved"]]


def _own_norm_bwd(s):
    C, desc, workspace = _call(s, lambda: _norm_call(s))
    C.convbn_group_norm_bwd(desc, s["dz"], s["x"], s["gamma"], s["beta"], s["saved"], s["dx"], s["dgamma"], s["dbeta"], workspace)
    return [s["dx"], s["dgamma"], s["dbeta"]]


def _ortho_call(s):
    from paper_2305_11624_b200 import convbn as C
    c = s["case"]
    bytes_ = C.convbn_orthogonalise_workspace_bytes(c["rows"], c["cols"], c["count"])
    return C, torch.empty(bytes_, dtype=torch.uint8, device=DEVICE)


def _own_ortho(s):
    C, workspace = _call(s, lambda: _ortho_call(s))
    C.convbn_orthogonalise(s["g"], s["out"], STEPS, NORM_EPS, workspace)
    return [s["out"]]


def _muon_call(s):
    from paper_2305_11624_b200 import convbn as C
    layers = C.MuonLayers(zip(s["grad"], s["momentum"], s["master"], s["weight"]))
    params = C.MuonParams.make(lr=LR, momentum=MOMENTUM, weight_decay=DECAY, eps=NORM_EPS, nesterov=True, steps=STEPS)
    return C, layers, params, torch.empty(C.convbn_muon_workspace_bytes(layers), dtype=torch.uint8, device=DEVICE)


def _own_muon(s):
    C, layers, params, workspace = _call(s, lambda: _muon_call(s))
    C.convbn_muon_step(layers, params, workspace)
    return s["flat"]


_own = {"norm_fwd": _own_norm_fwd, "norm_bwd": _own_norm_bwd, "ortho": _own_ortho, "muon": _own_muon}


# ---- the definitions in 64 bits ----------------------------------------------------------------------------------
def exact(case, seed):
    with torch.no_grad():
        return _exact[case["kind"]](prepare(case, seed))


def _exact_norm_fwd(s):
    c, (n, h, w, ch) = s["case"], s["x"].shape
    g, size = c["groups"], ch // c["groups"]
    z, mean, rstd = torch.empty(n, h, w, ch, dtype=torch.float64, device=DEVICE), [], []
    for i in range(n):                                                # image by image, groups first
        v = s["x"][i].double().reshape(h * w, g, size).permute(1, 0, 2).reshape(g, -1)
        var, m = torch.var_mean(v, 1, correction=0)
        r = 1.0 / torch.sqrt(var + EPS)
        y = ((v - m[:, None]) * r[:, None]).view(g, h * w, size).permute(1, 0, 2).reshape(h, w, ch)
        y = y * s["gamma"].double() + s["beta"].double()
        z[i] = y.clamp(min=0.0) if c["act"] == "relu" else y * torch.sigmoid(y) if c["act"] == "silu" else y
        mean.append(m)
        rstd.append(r)
    return [z, torch.stack((torch.stack(mean), torch.stack(rstd)))]


def _exact_norm_bwd(s):
    c, (n, h, w, ch) = s["case"], s["x"].shape
    g, size = c["groups"], ch // c["groups"]
    gamma, beta = s["gamma"].double(), s["beta"].double()
    dx = torch.empty(n, h, w, ch, dtype=torch.float64, device=DEVICE)
    dgamma, dbeta = torch.zeros_like(gamma), torch.zeros_like(beta)
    spread = lambda v: v.double().repeat_interleave(size)
    for i in range(n):
        mean, rstd = spread(s["saved"][0, i]), spread(s["saved"][1, i])
        xhat = (s["x"][i].double().view(h * w, ch) - mean) * rstd
        y, dy = xhat * gamma + beta, s["dz"][i].double().view(h * w, ch)
        if c["act"] == "relu":
            dy = dy * (y > 0)
        elif c["act"] == "silu":
            gate = torch.sigmoid(y)
            dy = dy * (gate + y * gate * (1.0 - gate))
        into_beta, into_gamma = dy.sum(0), (dy * xhat).sum(0)
        dbeta += into_beta
        dgamma += into_gamma
        mean_of = lambda v: ((v * gamma).view(g, size).sum(1) / (h * w * size)).repeat_interleave(size)
        dx[i] = ((dy * gamma - mean_of(into_beta) - xhat * mean_of(into_gamma)) * rstd).view(h, w, ch)
    return [dx, dgamma, dbeta]


def _exact_update(g):
    """[rows, cols] in 64 bits: the shorter side's Gram matrix, on either side of X."""
    x = g / (torch.linalg.matrix_norm(g) + NORM_EPS)
    a, b, c = COEFFICIENTS
    for _ in range(STEPS):
        if x.shape[0] <= x.shape[1]:
            once = x @ x.t() @ x
            x = a * x + b * once + c * (x @ x.t() @ once)
        else:
            gram = x.t() @ x
            x = x @ (a * torch.eye(len(gram), dtype=x.dtype, device=x.device) + b * gram + c * gram @ gram)
    return x


def _exact_ortho(s):
    return [torch.stack([_exact_update(g.double()) for g in s["g"]])]


def _exact_muon(s):
    out = [f.double() for f in s["flat"]]
    for i, grad in enumerate(s["grad"]):
        momentum = MOMENTUM * s["momentum"][i].double() + grad.double()
        update = _exact_update(grad.double() + MOMENTUM * momentum)
        scale = max(1.0, update.shape[0] / update.shape[1]) ** 0.5
        master = s["master"][i].double() * (1.0 - LR * DECAY) - LR * scale * update
        at = s["master"][i].storage_offset()
        for flat, value in zip(out, (momentum, master, master)):
            flat[at:at + value.numel()] = value.reshape(-1)
    return out


_exact = {"norm_fwd": _exact_norm_fwd, "norm_bwd": _exact_norm_bwd, "ortho": _exact_ortho, "muon": _exact_muon}
