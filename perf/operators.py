"""The 8-bit forms of a block's input, as measurable cases: what training keeps of it and what a deployed block multiplies.

- "pack": an activation is packed into 8-bit codes with a power-of-two step for every 32 elements, and restored.
- "backward": the Tune-mode backward pass of a ConvBN or Linear-BN block whose input was kept packed.
- "deploy": the forward pass of a deployed 1x1 or Linear-BN block as a product of 8-bit integers, with a scale for every row
  of X (a pixel, a token) and every output channel.

A case is one pass.  Layer shapes are those of the benchmark configurations and of a ResNet-50, or generic.
"""
import functools
import math

import torch

own = False

DEVICE = "cuda:0"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
ELEMENT_BYTES = {"f32": 4, "bf16": 2, "f16": 2}
GROUP = 32                                       # consecutive elements that share a step
EXPONENTS = {"f32": (-126, 121), "bf16": (-126, 121), "f16": (-24, 9)}
EPS = 1e-5


# ---- cases -------------------------------------------------------------------------------------------------------
def _pack(count, dtype="bf16"):
    return dict(kind="pack", count=count, dtype=dtype)


def _backward(n, c_in, h, w, c_out, k, stride=1, dtype="bf16", bias=False, add=False, mask=True):
    """h = w = 1: a Linear-BN block on n rows.  add: a gradient arrives over the skip connection.  mask: the block's input
    is the output of a ReLU."""
    return dict(kind="backward", n=n, c_in=c_in, h=h, w=w, c_out=c_out, k=k, stride=stride, dtype=dtype, bias=bias, add=add,
                mask=mask)


def _deploy(n, c_in, h, w, c_out, dtype="bf16", add=False, relu=True):
    return dict(kind="deploy", n=n, c_in=c_in, h=h, w=w, c_out=c_out, dtype=dtype, add=add, relu=relu)


def listed():
    named = lambda name, case: dict(case, name=name)
    return [
        # the input of a small fp32 block: launches count
        named("pack_small_f32", _pack(2 * 16 * 16 * 16, "f32")),
        # the input of a depthwise block under half-precision training
        named("pack_depthwise_f16", _pack(64 * 112 * 112 * 96, "f16")),
        # the residual stream of stage 2 at a large training batch: the largest activation that is kept
        named("pack_stage2_large", _pack(256 * 56 * 56 * 256)),
        # a Linear-BN head on one batch of features
        named("backward_linear_head", _backward(1000, 256, 1, 1, 64, 1)),
        # the 3x3 convolution of a stage-2 bottleneck at an ordinary batch
        named("backward_3x3_stage2", _backward(32, 64, 56, 56, 64, 3)),
        # the first 1x1 convolution of the last stage under half-precision training, few pixels, where the two branches meet
        named("backward_reduce_stage5_f16", _backward(64, 2048, 7, 7, 512, 1, dtype="f16", add=True)),
        # the first 1x1 convolution of a stage-2 bottleneck at a large batch, where the two branches meet
        named("backward_reduce_large", _backward(256, 256, 56, 56, 64, 1, add=True)),
        # the classifier-sized layer of a deployed network on one image: one row, an odd width
        named("deploy_one_row", _deploy(1, 2048, 1, 1, 1000, relu=False)),
        # the Linear-BN head on one batch of features, in half precision
        named("deploy_linear_head_f16", _deploy(1000, 256, 1, 1, 64, "f16")),
        # the last 1x1 convolution of a stage-2 bottleneck, deployed, with the skip connection's sum and ReLU
        named("deploy_expand_stage2", _deploy(32, 64, 56, 56, 256, add=True)),
        # the first 1x1 convolution of a stage-2 bottleneck at a large batch: the largest activations
        named("deploy_reduce_large", _deploy(256, 256, 56, 56, 64)),
        # a wide projection of many tokens: the product itself counts
        named("deploy_wide_projection", _deploy(65536, 2048, 1, 1, 2048)),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case: the kinds of the listed ones at sizes spread over their logarithm, odd ones among them."""
    wide = (64, 128, 256, 512, 1024, 2048)
    dtype = rng.choice(("bf16", "bf16", "f16"))
    kind = rng.choice(("pack", "conv1", "conv1", "conv3", "linear", "deploy", "deploy", "deploy_linear"))
    if kind == "pack":
        dtype = rng.choice(("f32", "bf16", "bf16", "f16"))
        return _pack(_log_int(rng, 100, 100_000_000 if dtype == "f32" else 200_000_000), dtype)
    while True:
        h = _log_int(rng, 7, 112)
        w = max(7, min(168, int(h * rng.uniform(0.75, 1.7))))
        n = _log_int(rng, 1, 256)
        mask = rng.random() < 0.75
        add = rng.random() < 0.4
        if kind == "conv1":
            stride = rng.choice((1, 1, 1, 2))
            case = _backward(n, rng.choice(wide), h, w, rng.choice(wide), 1, stride, dtype, add=add, mask=mask)
        elif kind == "conv3":
            c = rng.choice(wide[:4])
            case = _backward(n, c, h, w, c, 3, rng.choice((1, 1, 2)), dtype, bias=rng.random() < 0.2, add=False, mask=mask)
        elif kind == "linear":
            case = _backward(_log_int(rng, 128, 100_000), rng.choice(wide), 1, 1, rng.choice(wide), 1, 1, dtype,
                             bias=rng.random() < 0.5, add=False, mask=mask)
        elif kind == "deploy":
            case = _deploy(n, rng.choice(wide), h, w, rng.choice(wide), dtype, add, mask)
        else:
            odd = lambda: rng.choice((rng.choice(wide), _log_int(rng, 24, 2048)))
            case = _deploy(_log_int(rng, 1, 65536), odd(), 1, 1, odd(), rng.choice((dtype, dtype, "f32")), False, mask)
        x, z = _sizes(case)
        if kind == "conv3" and x > 3e7:
            continue
        if max(x, z) <= 2.0e8 and work(case)["flops"] <= 5e11:
            return case


def _out(case, extent):
    return (extent + 2 * (case["k"] // 2) - case["k"]) // case["stride"] + 1


def _sizes(case):
    """Elements of X and of Z."""
    n, h, w = case["n"], case["h"], case["w"]
    ho, wo = (_out(case, h), _out(case, w)) if case["kind"] == "backward" else (h, w)
    return n * h * w * case["c_in"], n * ho * wo * case["c_out"]


# ---- what a program has in hand ----------------------------------------------------------------------------------
def _packed(x, dtype):
    """(codes, step bytes) of x, flat: what a forward pass left behind."""
    lo, hi = EXPONENTS[dtype]
    count = x.numel()
    v = torch.nn.functional.pad(x.reshape(-1).float(), (0, -count % GROUP)).view(-1, GROUP)
    e = ((v.abs().amax(1).view(torch.int32) + 0x10000 >> 23) - 133).clamp(lo, hi)
    q = torch.round(v * torch.exp2(-e.float())[:, None]).clamp(-127, 127)
    q = torch.where(q == 0, torch.sign(v), q)
    bad = ~torch.isfinite(v).all(1)
    codes = torch.where(bad[:, None], 0, q).to(torch.int8).view(-1)[:count].contiguous()
    return codes, torch.where(bad, 255, e + 127).to(torch.uint8)


def prepare(case, seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    t, kind = DTYPES[case["dtype"]], case["kind"]
    randn = lambda *shape: torch.randn(*shape, generator=g, device=DEVICE)
    uniform = lambda n, lo, hi: torch.rand(n, generator=g, device=DEVICE) * (hi - lo) + lo
    if kind == "pack":
        # ReLU outputs: half zeros, magnitudes that differ from region to region
        count = case["count"]
        x = randn(count).relu_().mul_(torch.exp(randn(-(-count // 4096))).repeat_interleave(4096)[:count]).to(t)
        return dict(case=case, x=x, out=torch.empty_like(x), codes=torch.empty(count, dtype=torch.int8, device=DEVICE),
                    steps=torch.empty(-(-count // GROUP), dtype=torch.uint8, device=DEVICE))
    n, ci, h, w, co = (case[key] for key in ("n", "c_in", "h", "w", "c_out"))
    k = case.get("k", 1)
    weight = (randn(co, k, k, ci) * math.sqrt(2.0 / (ci * k * k))).to(t)
    gamma, var = uniform(co, 0.5, 1.5), uniform(co, 0.5, 2.0)
    beta, mean = randn(co) * 0.1, randn(co) * 0.1
    b = randn(co) * 0.01 if case.get("bias") else None
    r = torch.rsqrt(var + EPS)
    shift = ((b if b is not None else 0.0) - mean) * gamma * r + beta
    x = randn(n, h, w, ci)
    if kind == "backward":
        x = (x.relu_() if case["mask"] else x).to(t)
        codes, steps = _packed(x, case["dtype"])
        ho, wo = _out(case, h), _out(case, w)
        empty = lambda *shape: torch.empty(*shape, device=DEVICE)
        return dict(case=case, codes=codes, steps=steps, w=weight, b=b, mean=mean, saved=torch.cat([gamma * r, shift, r]),
                    dz=randn(n, ho, wo, co).to(t), add=randn(n, h, w, ci).to(t) if case["add"] else None,
                    dx=torch.empty_like(x), dw=empty(co, k, k, ci), db=empty(co) if b is not None else None, dgamma=empty(co),
                    dbeta=empty(co))
    # a few channels that stand out, as activations have them
    x = x.relu_().mul_(torch.exp(0.5 * randn(ci))).to(t)
    wide = weight.view(co, ci).float()
    peak = wide.abs().amax(1)
    codes = torch.round(wide.double() * (127.0 / peak).double()[:, None]).to(torch.int8)
    return dict(case=case, x=x, w_codes=torch.nn.functional.pad(codes, (0, -ci % 16)).contiguous(),
                w_scale=gamma * r * (peak / 127.0), b_fused=shift, add=randn(n, h, w, co).to(t) if case["add"] else None,
                z=torch.empty(n, h, w, co, dtype=t, device=DEVICE))


# ---- one pass ----------------------------------------------------------------------------------------------------
def run(state):
    return (_own if own else _plain)[state["case"]["kind"]](state)


# The plain forms.
def _plain_pack(s):
    dtype = s["case"]["dtype"]
    codes, steps = _packed(s["x"], dtype)
    return [_restored(codes, steps).to(DTYPES[dtype])]


def _restored(codes, steps):
    step = torch.where(steps == 255, torch.nan, torch.exp2(steps.float() - 127.0))
    return codes.float() * step.repeat_interleave(GROUP)[:codes.numel()]


def _windows(t, k):
    """[N, H, W, C] -> [N, H - k + 1, W - k + 1, k k C]."""
    if k == 1:
        return t
    v = t.unfold(1, k, 1).unfold(2, k, 1).permute(0, 1, 2, 4, 5, 3)
    return v.reshape(*v.shape[:3], -1)


def _plain_backward(s):
    c, (n, ho, wo, co) = s["case"], s["dz"].shape
    h, w, ci, k, st = (c[key] for key in ("h", "w", "c_in", "k", "stride"))
    pad, t = k // 2, DTYPES[c["dtype"]]
    scale, _, r = s["saved"].view(3, co)
    x = _restored(s["codes"], s["steps"]).view(n, h, w, ci)
    dz, weight = s["dz"].float(), s["w"].float()
    xp = torch.nn.functional.pad(x, (0, 0, pad, pad, pad, pad))
    cols = _windows(xp, k)[:, ::st, ::st].reshape(n, ho * wo, k * k * ci)
    rows = dz.view(n, ho * wo, co)
    # long sums over pixels: image by image (rows in 64 parts for a Linear-BN block), those added in 64 bits
    if ho * wo == 1:
        parts = max(1, n // 256)
        first = n // parts * parts
        cut = lambda a: a.view(n, -1)[:first].view(parts, n // parts, -1)
        raw = torch.bmm(cut(rows).transpose(1, 2), cut(cols)).double().sum(0)
        raw = raw + rows.view(n, co)[first:].double().t() @ cols.view(n, -1)[first:].double()
    else:
        raw = torch.bmm(rows.transpose(1, 2), cols).double().sum(0)
    dbeta = rows.double().sum((0, 1))
    centred = (s["b"] if s["b"] is not None else 0.0) - s["mean"]
    dgamma = r * ((raw * weight.view(co, -1)).sum(1) + dbeta * centred)
    dw = (raw * scale[:, None]).float().view(co, k, k, ci)
    # dX: the rotated, scaled weights over dZ, which stands `stride` apart
    spread = dz
    if st > 1:
        spread = dz.new_zeros(n, h + 2 * pad - k + 1, w + 2 * pad - k + 1, co)
        spread[:, ::st, ::st] = dz
    edge = k - 1 - pad
    spread = torch.nn.functional.pad(spread, (0, 0, edge, edge, edge, edge))
    turned = (weight * scale[:, None, None, None]).flip(1, 2).permute(1, 2, 0, 3).reshape(k * k * co, ci)
    dx = (_windows(spread, k).reshape(-1, k * k * co) @ turned).view(n, h, w, ci)
    if s["add"] is not None:
        dx = dx + s["add"].float()
    if c["mask"]:
        dx = torch.where(x > 0, dx, 0.0)
    out = [dx.to(t), dw, dgamma.float(), dbeta.float()]
    return out + [(scale * dbeta).float()] if s["b"] is not None else out


def _plain_deploy(s):
    c = s["case"]
    x = s["x"].float().view(-1, c["c_in"])
    peak = x.abs().amax(1, keepdim=True)
    inverse = torch.where(peak > 0, 127.0 / peak, 0.0)
    codes = torch.round(x.double() * inverse.double()).float()       # a product next to a half decides a code
    acc = codes @ s["w_codes"][:, :c["c_in"]].float().t()
    z = acc * (peak / 127.0) * s["w_scale"] + s["b_fused"]
    z = z.view(s["z"].shape)
    if s["add"] is not None:
        z = z + s["add"].float()
    return [(z.relu() if c["relu"] else z).to(s["z"].dtype)]


_plain = {"pack": _plain_pack, "backward": _plain_backward, "deploy": _plain_deploy}


# The framework's calls.  A layer's descriptor is a function of its sizes; its workspace is kept with its other buffers.
@functools.lru_cache(maxsize=None)
def _layer(n, c_in, h, w, c_out, k, stride, dtype):
    from paper_2305_11624_b200 import convbn as C
    kind = {"f32": C.F32, "bf16": C.BF16, "f16": C.F16}[dtype]
    return C, C.Desc.make(n, c_in, h, w, c_out, k, k, stride, stride, k // 2, k // 2, dtype=kind,
                          layout=C.NCHW if dtype == "f32" else C.NHWC, eps=EPS)


def _kept(s, phase):
    if "layer" not in s:
        c = s["case"]
        C, desc = _layer(c["n"], c["c_in"], c["h"], c["w"], c["c_out"], c.get("k", 1), c.get("stride", 1), c["dtype"])
        size = C.convbn_workspace_bytes(desc, getattr(C, phase))
        s["layer"] = C, desc, torch.empty(max(256, size), dtype=torch.uint8, device=DEVICE)
    return s["layer"]


def _own_pack(s):
    from paper_2305_11624_b200 import convbn as C
    C.convbn_pack(s["x"], s["codes"], s["steps"])
    C.convbn_unpack(s["codes"], s["steps"], s["out"])
    return [s["out"]]


def _own_backward(s):
    C, desc, workspace = _kept(s, "PHASE_TUNE_BWD_PACKED")
    C.convbn_tune_bwd_packed(desc, s["dz"], s["codes"], s["steps"], s["w"], s["b"], s["mean"], s["saved"], s["dx"], s["dw"],
                             s["db"], s["dgamma"], s["dbeta"], s["add"], s["case"]["mask"], False, workspace)
    out = [s["dx"], s["dw"], s["dgamma"], s["dbeta"]]
    return out + [s["db"]] if s["b"] is not None else out


def _own_deploy(s):
    C, desc, workspace = _kept(s, "PHASE_DEPLOY_FWD_QUANT")
    C.convbn_deploy_fwd_quant(desc, s["x"], s["w_codes"], s["w_scale"], s["b_fused"], s["z"], s["add"], s["case"]["relu"],
                              workspace)
    return [s["z"]]


_own = {"pack": _own_pack, "backward": _own_backward, "deploy": _own_deploy}


# ---- what a pass cannot do without --------------------------------------------------------------------------------
def work(case):
    es = ELEMENT_BYTES[case["dtype"]]
    packed = lambda count: count + -(-count // GROUP)
    if case["kind"] == "pack":
        count = case["count"]
        return {"bytes": 2.0 * es * count + 2.0 * packed(count), "flops": 8.0 * count}
    x, z = _sizes(case)
    ci, co, k = case["c_in"], case["c_out"], case.get("k", 1)
    if case["kind"] == "deploy":
        return {"bytes": float(es * (x + z * (2 if case["add"] else 1)) + co * ci + 8 * co), "flops": 2.0 * x * co}
    weights = co * ci * k * k
    return {"bytes": float(es * (z + x * (2 if case["add"] else 1)) + packed(x) + (es + 4) * weights + 40 * co),
            "flops": 4.0 * (z // co) * weights}


# ---- the operators' definitions in 64 bits -------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "pack":
        return [_exact_pack(s["x"], case["dtype"])]
    return _exact_backward(s) if case["kind"] == "backward" else _exact_deploy(s)


def _exact_pack(x, dtype):
    """The smallest step 2^e, e within its bounds, at which the group's largest magnitude rounds to 127 at most; every value
    to the nearest multiple of it (the even one of two), never to zero unless it is zero."""
    lo, hi = EXPONENTS[dtype]
    out = torch.empty(x.numel(), dtype=torch.float64, device=x.device)
    for at in range(0, x.numel(), 1 << 25):                          # whole groups, a part at a time
        v = x[at:at + (1 << 25)].double()
        count = v.numel()
        v = torch.cat([v, v.new_zeros(-count % GROUP)]).view(-1, GROUP)
        top = v.abs().max(dim=1, keepdim=True).values
        e = torch.frexp(top)[1].double() - 7.0                       # top 2^-e in [64, 128), or 0
        e = torch.where(torch.round(torch.ldexp(top, -e)) > 127.0, e + 1.0, e).clamp(lo, hi)
        q = torch.round(torch.ldexp(v, -e)).clamp(-127.0, 127.0)
        q = q + torch.sign(v) * (q == 0)
        out[at:at + count] = torch.ldexp(q, e).view(-1)[:count]
    return out


def _exact_backward(s):
    c, (n, ho, wo, co) = s["case"], s["dz"].shape
    h, w, ci, k, st = (c[key] for key in ("h", "w", "c_in", "k", "stride"))
    pad = k // 2
    scale, r = s["saved"][:co].double(), s["saved"][2 * co:].double()
    exponent = (s["steps"].int() - 127).repeat_interleave(GROUP)[:s["codes"].numel()]
    x = torch.ldexp(s["codes"].double(), exponent).view(n, h, w, ci)
    weight, dz = s["w"].double(), s["dz"].double()
    flat = dz.reshape(-1, co)
    bordered = x.new_zeros(n, h + 2 * pad, w + 2 * pad, ci)
    bordered[:, pad:pad + h, pad:pad + w] = x
    into = torch.zeros_like(bordered)
    raw = torch.empty(co, k, k, ci, dtype=torch.float64, device=x.device)
    for i in range(k):                                               # tap by tap
        for j in range(k):
            at = (slice(None), slice(i, i + (ho - 1) * st + 1, st), slice(j, j + (wo - 1) * st + 1, st))
            raw[:, i, j] = flat.t() @ bordered[at].reshape(-1, ci)
            into[at] += (flat @ (weight[:, i, j] * scale[:, None])).view(n, ho, wo, ci)
    dx = into[:, pad:pad + h, pad:pad + w].clone()
    if s["add"] is not None:
        dx += s["add"].double()
    if c["mask"]:
        dx *= x > 0
    dbeta = flat.sum(0)
    shift = -s["mean"].double() + (s["b"].double() if s["b"] is not None else 0.0)
    dgamma = r * (torch.einsum("oijc,oijc->o", raw, weight) + dbeta * shift)
    out = [dx, raw * scale[:, None, None, None], dgamma, dbeta]
    return out + [scale * dbeta] if s["b"] is not None else out


def _exact_deploy(s):
    c, shape = s["case"], s["z"].shape
    rows, weights = s["x"].reshape(-1, c["c_in"]), s["w_codes"][:, :c["c_in"]].double()
    z = torch.empty(rows.shape[0], shape[-1], dtype=torch.float64, device=rows.device)
    for at in range(0, rows.shape[0], 1 << 17):
        v = rows[at:at + (1 << 17)].double()
        top = v.abs().max(dim=1, keepdim=True).values
        # the factor is the 32-bit one: it belongs to the definition
        factor = (127.0 / top.float()).double().masked_fill(top == 0, 0.0)
        z[at:at + (1 << 17)] = (torch.round(v * factor) @ weights.t()) * (top / 127.0)
    z = (z * s["w_scale"].double() + s["b_fused"].double()).view(shape)
    if s["add"] is not None:
        z += s["add"].double()
    return [z.clamp(min=0.0) if c["relu"] else z]
