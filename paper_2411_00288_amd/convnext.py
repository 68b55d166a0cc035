"""A ConvNeXt-T stage at the 4-bit precision point, as a chain of library calls.

A block is: depthwise 7x7 (dense, 16-bit) -> LayerNorm, written as MXFP4 -> pointwise expansion on those codes with GELU -> pointwise contraction
(its 16-bit input quantised on the way) -> layer scale, a stochastic-depth gate per image, and the residual sum.  Both pointwise matrices carry a 2:4
mask and are kept in MXFP4.  The stage ends in the LayerNorm in front of the downsample, fused with the last block's tail; ``tail_gradient`` is that
call's gradient for a forward pass, which is where learning the layer scale and the norms of a network with frozen 4-bit layers begins.  Weights are random
(``workloads.make_weights``), as everywhere in this package.
"""
from __future__ import annotations

import numpy as np
import torch

import paper_2411_00288_amd as ss
from . import workloads as wl

EPS = 1e-6


class StageOutput(tuple):
    """(the stream behind the last block, its LayerNorm) of one forward pass; `tail` is what the gradient of its last call takes."""

    def __new__(cls, x: torch.Tensor, y: torch.Tensor, h: torch.Tensor, gate: torch.Tensor | None):
        self = super().__new__(cls, (x, y))
        self.tail = (x, h, gate)
        return self


class Stage4bit:
    """`blocks` blocks of `channels` channels; activations are NHWC of `dtype` (``wl.F16`` or ``wl.BF16``)."""

    def __init__(self, blocks: int = 3, channels: int = 96, dtype: int = wl.BF16, seed: int = 0, device="cuda"):
        self.channels, self.tdt = channels, ss.torch_dtype(dtype)
        self.expand = ss.make_desc(4 * channels, channels, 1, 1, dtype)
        self.contract = ss.make_desc(channels, 4 * channels, 1, 1, dtype)
        self.norm = ss.make_norm_desc(channels, dtype, ss.SS_NORM_LAYER, EPS)
        self.sum = ss.make_norm_desc(channels, dtype, ss.SS_NORM_NONE)
        rng = np.random.Generator(np.random.PCG64(seed))
        vector = lambda around, spread: torch.from_numpy((around + spread * rng.standard_normal(channels)).astype(np.float32)).to(device)
        self.blocks = []
        for i in range(blocks):
            block = {"dw": torch.from_numpy((rng.standard_normal((7, 7, channels)) / 7).astype(np.float32)).to(device, self.tdt), "dw_bias": vector(0, 0.1),
                     "w": vector(1, 0.1), "b": vector(0, 0.1), "scale": vector(0.3, 0.05)}
            for name, desc in (("expand", self.expand), ("contract", self.contract)):
                layer = wl.Layer(f"{name}{i}", N=1, H=1, W=1, cin=desc.cin, cout=desc.cout, kh=1, kw=1, dtype=dtype, mask="top2", seed=seed + 10 * i + len(name))
                d = wl.make_weights(layer)
                block[name + "_W"] = torch.from_numpy(d["W"].view(np.int16)).to(device).view(self.tdt)
                block[name + "_M"] = torch.from_numpy(d["M"]).to(device)
                block[name + "_bias"] = torch.from_numpy(d["bias"]).to(device)
                block[name] = ss.ss_mx4_pack(desc, block[name + "_W"], block[name + "_M"])
            self.blocks.append(block)
        self.w, self.b = vector(1, 0.1), vector(0, 0.1)
        self._last, self._passes = None, 0      # the last forward pass, and how many there were since the last gradient

    def branch(self, block: dict, x: torch.Tensor) -> torch.Tensor:
        """A block without its tail: x NHWC -> h of the same shape."""
        t = ss.ss_dwconv2d_fwd(x, block["dw"], block["dw_bias"], (3, 3))
        codes, scales = ss.ss_norm_mx4_fwd(self.norm, t, block["w"], block["b"])
        wide = ss.ss_pw_mx4_q_fwd(self.expand, codes, scales, block["expand"], block["expand_bias"], None, ss.SS_ACT_GELU)
        return ss.ss_pw_mx4_fwd(self.contract, wide, block["contract"], block["contract_bias"])

    def forward(self, x: torch.Tensor, gates=None) -> StageOutput:
        """x [N, H, W, channels] -> (the stream behind the last block, its LayerNorm).  gates: one [N, 1] of x's type, or None, for each block; or None."""
        gates = [None] * len(self.blocks) if gates is None else list(gates)
        if len(gates) != len(self.blocks):
            raise ValueError(f"{len(gates)} gates for {len(self.blocks)} blocks")
        for block, gate in zip(self.blocks[:-1], gates):
            x = ss.ss_norm_fwd(self.sum, x, None, None, self.branch(block, x), block["scale"], gate)
        last = self.blocks[-1]
        h = self.branch(last, x)
        x, y = ss.ss_norm_fwd(self.norm, x, self.w, self.b, h, last["scale"], gates[-1])
        self._last = StageOutput(x, y, h, gates[-1])
        self._passes += 1
        return self._last

    def tail_gradient(self, dy: torch.Tensor, dx_out: torch.Tensor | None = None, of: StageOutput | None = None) -> "ss.NormGrads":
        """Gradients at a forward pass's closing norm: of the stream before the last block, of its branch, its gate, the norm's vectors and the layer
        scale, for a gradient dy of the norm's output and dx_out of the stream.  of: what that pass returned (its tensors as they were); it may be left out
        where there was one pass only since the last gradient."""
        if of is None:
            if self._passes > 1:
                raise ValueError(f"{self._passes} forward passes since the last gradient: which one's is wanted (of=)?")
            if self._last is None:
                raise ValueError("no forward pass to take the gradient of")
            of = self._last
        self._passes = 0
        x, h, gate = of.tail
        return ss.ss_norm_bwd(self.norm, dy, x, self.w, self.b, h, self.blocks[-1]["scale"], gate, dx_out=dx_out)
