"""A chain of bottlenecks with group norms, forward and backward, and the optimiser's step on its gradients: what a user runs one after the
other, against the fp64 oracles chained the same way."""
import numpy as np
import pytest
import torch

import parity
from oracle import muon_oracle as M
from oracle import norm_oracle as N
from oracle import oracle as O
from paper_2305_11624_b200 import convbn as C
from paper_2305_11624_b200 import inputs as I
from paper_2305_11624_b200.backbone import BackboneReplay, Bottleneck
from paper_2305_11624_b200.muon import Muon

pytestmark = pytest.mark.gpu

PLAN = [Bottleneck(64, 64, 256, 1, (12, 12)), Bottleneck(256, 64, 256, 1, (12, 12)), Bottleneck(256, 128, 512, 2, (12, 12))]
GROUPS = 32
nhwc, nchw = (lambda a: a.transpose(0, 2, 3, 1)), (lambda a: a.transpose(0, 3, 1, 2))


class Layer:
    """One convolution, norm and perhaps ReLU in fp64, from a replay's parameters."""

    def __init__(self, layer):
        b = layer.blk
        self.w, self.gamma, self.beta = (b.fetch(k) for k in ("w", "gamma", "beta"))
        self.shape, self.eps = parity.oracle_shape(b.spec), b.spec.eps

    def forward(self, x, relu):
        self.x, self.act = x, "relu" if relu else "none"
        self.y = nhwc(O.conv(self.shape, x, self.w))
        z, self.mean, self.rstd = N.forward(self.y, GROUPS, self.gamma, self.beta, self.eps, self.act)
        return nchw(z)

    def backward(self, dz, mask=None):
        """mask: the decisions of this layer's ReLU"""
        g = N.backward(nhwc(dz if mask is None else dz * mask), self.y, GROUPS, self.gamma, self.beta, self.mean, self.rstd, "none")
        dy = nchw(g["dx"])
        self.dgamma, self.dbeta, self.dw = g["dgamma"], g["dbeta"], O.conv_grad_weight(self.shape, dy, self.x)
        return O.conv_grad_input(self.shape, dy, self.w)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_a_training_step(dtype):
    rp = BackboneReplay(2, PLAN, "group", seed=3, dtype=dtype)
    opt = rp.optimiser(lr=0.05, momentum=0.9, weight_decay=0.01)
    ins, keep = rp.make_inputs(5), {}
    tape = [[Layer(l) if l is not None else None for l in blk] for blk in rp.blocks]
    weights = [l.blk.fetch("w") for l in rp.layers]
    rp.forward_backward(ins, keep)
    C.convbn_check()
    logical = lambda t, c, hw: I.act_from_layout(t.float().cpu().numpy().astype(np.float64), "nhwc", (2, c, hw[0], hw[1]))
    x = logical(ins["x"], 64, (12, 12))
    outs = []
    for c1, c2, c3, ds in tape:
        a = c1.forward(x, True)
        b = c2.forward(a, True)
        out = np.maximum(c3.forward(b, False) + (ds.forward(x, False) if ds else x), 0.0)
        outs.append((a, b, out))
        x = out
    # the sign of a value within rounding of zero is decided by the arithmetic that formed it: both sides take the kernels' decisions, which may
    # differ from the oracle's only there: a stored value is off by 1.7e-3 of itself (bf16; half 2.1e-4) in the mean square; up to the last output there
    # are two such roundings for each of nine convolutions and one for each of three sums, sqrt(21) of one; gamma makes a channel's values up to 1.5 of
    # the mean; 4.5 sigma covers the 4e4 values of a tensor; before the ReLU the mean square is twice what it is behind it
    near = 4.5 * {"bf16": 1.7e-3, "f16": 2.1e-4}[dtype] * 21 ** 0.5 * 1.5 * 2 ** 0.5
    masks = []
    for kernels, oracle in zip(keep["relu_outputs"], outs):
        masks.append([logical(k, o.shape[1], o.shape[2:]) > 0 for k, o in zip(kernels, oracle)])
        for m, o in zip(masks[-1], oracle):
            assert np.abs(o[m != (o > 0)]).max(initial=0.0) <= near * np.sqrt((o * o).mean())
    g = logical(ins["g"], 512, (6, 6))
    for (c1, c2, c3, ds), (ma, mb, mo), i in zip(reversed(tape), reversed(masks), range(2, -1, -1)):
        g = g * mo
        ga = c2.backward(c3.backward(g), mb)
        g = c1.backward(ga, ma) + (ds.backward(g) if ds else g)
    # per layer two roundings of an activation, as in Tune mode; errors of successive layers add in quadrature
    tol = parity.TOL[dtype] * np.sqrt(3 * len(PLAN))
    errs = {"out": O.rel_l2(logical(keep["out"], 512, (6, 6)), x), "dx": O.rel_l2(logical(keep["dx"], 64, (12, 12)), g)}
    flat = [l for blk in tape for l in blk if l is not None]
    for k, (layer, ref) in enumerate(zip(rp.layers, flat)):
        for name in ("dw", "dgamma", "dbeta"):
            errs["%s%d" % (name, k)] = O.rel_l2(layer.blk.fetch(name), getattr(ref, name).reshape(layer.blk.fetch(name).shape))
    assert all(v <= tol for v in errs.values()), errs
    # the step on these gradients, twice: weights in storage type are the masters', rounded
    state = [(np.zeros_like(w.reshape(w.shape[0], -1)), m.double().cpu().numpy()) for w, m in zip(weights, opt.master)]
    for _ in range(2):
        grads = [l.blk.dw.view(l.blk.spec.c_out, -1).double().cpu().numpy() for l in rp.layers]
        opt.step()
        state = [M.muon_step(g, v, m, 0.05, 0.9, 0.01, 1e-7, True, 5) for g, (v, m) in zip(grads, state)]
    C.convbn_check()
    for layer, got, (v, m) in zip(rp.layers, opt.master, state):
        # (two updates of lr sqrt(max(1, rows / cols)) X, each off by 1e-4 of X at most, and fp32 weights)
        scale = 0.05 * max(1.0, m.shape[0] / m.shape[1]) ** 0.5
        assert np.linalg.norm(got.double().cpu().numpy() - m) <= 2e-4 * scale * np.sqrt(min(m.shape)) + 2.0 ** -22 * np.linalg.norm(m)
        assert torch.equal(layer.blk.w.view_as(got), got.to(layer.blk.w.dtype))
    # and another pass with the new weights
    keep2 = {}
    rp.forward_backward(ins, keep2)
    C.convbn_check()
    assert not torch.equal(keep2["out"], keep["out"]) and bool(torch.isfinite(keep2["dx"].float()).all())


def test_a_captured_iteration():
    """Pass and step in one graph: the same weights as pass and step one after the other."""
    results = []
    for captured in (False, True):
        rp = BackboneReplay(2, PLAN, "group", seed=3)
        opt, ins = rp.optimiser(lr=0.02), rp.make_inputs(5)

        def iteration():
            rp.forward_backward(ins)
            opt.step()
        iteration()
        torch.cuda.synchronize()
        if captured:
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                iteration()
            iteration = graph.replay
        for _ in range(2):
            iteration()
        C.convbn_check()
        results.append([m.clone() for m in opt.master])
    assert all(torch.equal(a, b) for a, b in zip(*results))


def test_tune_mode_and_a_bucket_of_gradients():
    from paper_2305_11624_b200.dataparallel import GradientBucket
    rp = BackboneReplay(2, PLAN, "tune", seed=3)
    bucket = GradientBucket({"%d" % i: l.blk.dw.numel() for i, l in enumerate(rp.layers)})
    for i, l in enumerate(rp.layers):
        l.blk.dw = bucket.views["%d" % i]
    rp.forward_backward(rp.make_inputs(5))
    bucket.all_reduce()
    before = [l.blk.w.clone() for l in rp.layers]
    opt = Muon([(l.blk.w.view(l.blk.spec.c_out, -1), l.blk.dw) for l in rp.layers], lr=0.02)
    opt.lr = 0.1
    opt.step()
    C.convbn_check()
    for l, w in zip(rp.layers, before):
        step = (l.blk.w.float() - w.float()).view(l.blk.spec.c_out, -1)
        # singular values of the update near lr sqrt(max(1, rows / cols))
        scale = 0.1 * max(1.0, step.shape[0] / step.shape[1]) ** 0.5
        top = float(torch.linalg.matrix_norm(step, 2))
        assert 0.5 * scale < top < 1.5 * scale
