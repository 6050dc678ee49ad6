"""The optimiser over the convolutions' and linear layers' weights: momentum, an update made orthogonal by Newton-Schulz products, weights kept
in fp32 and in their storage type.  One call of the library for all layers (``convbn_muon_step``); this module only owns the buffers.

The per-channel vectors (biases, gamma, beta) are no matrices and are left to the caller.
"""
from typing import Iterable, Tuple

import torch

from . import convbn as C


class Muon:
    """layers: (weight, gradient) pairs; weight: [C_out, ...] in its storage type, one piece, updated in place; gradient: fp32, as many
    elements in the same order (a block's dw, a view of a GradientBucket).  The very tensors given are read at every step: a gradient that is formed
    anew elsewhere has to be copied into its own."""

    def __init__(self, layers: Iterable[Tuple[torch.Tensor, torch.Tensor]], lr=0.02, momentum=0.95, weight_decay=0.0, nesterov=True, steps=5, eps=1e-7):
        layers = [(w.detach(), g.detach()) for w, g in layers]
        self.params = C.MuonParams.make(lr, momentum, weight_decay, eps, nesterov, steps)
        self.momentum = [torch.zeros_like(w, dtype=torch.float32) for w, _ in layers]
        self.master = [w if w.dtype == torch.float32 else w.float() for w, _ in layers]
        stored = [None if w.dtype == torch.float32 else w for w, _ in layers]
        self.layers = C.MuonLayers(zip([g for _, g in layers], self.momentum, self.master, stored))
        self.workspace = None

    @property
    def lr(self) -> float:
        return self.params.lr

    @lr.setter
    def lr(self, value: float):
        self.params.lr = float(value)

    def step(self, stream=None):
        """New weights of every layer from the gradients as they are now."""
        if self.workspace is None and len(self.layers):
            self.workspace = torch.empty(C.convbn_muon_workspace_bytes(self.layers), dtype=torch.uint8, device=self.layers.device)
        C.convbn_muon_step(self.layers, self.params, self.workspace, stream=stream)
