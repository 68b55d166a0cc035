"""A ConvNeXt stage at 4 bits through the public calls: every step of a block against the 64-bit definition of that step on the step's own input, and the stage's
tail with its gradient."""
import numpy as np
import pytest
import torch

import oracle
import rows_reference as ref
from paper_2411_00288_amd import workloads as wl
from helpers import check_close, host_bits

pytestmark = pytest.mark.gpu


def _wide(t):
    return t.double().cpu().numpy().reshape(-1, t.shape[-1])


@pytest.mark.parametrize("dtype", [wl.F16, wl.BF16])
@pytest.mark.parametrize("N,H,W,C", [(2, 7, 7, 96), (1, 9, 5, 64)])
def test_stage_step_by_step(ss, dtype, N, H, W, C):
    from paper_2411_00288_amd.convnext import EPS, Stage4bit
    stage = Stage4bit(2, C, dtype, seed=5)
    g = torch.Generator(device="cuda").manual_seed(1)
    x0 = torch.randn((N, H, W, C), generator=g, device="cuda").to(stage.tdt)
    gates = [torch.tensor([[1.25]] * N, device="cuda").to(stage.tdt), torch.tensor([[0.0 if n else 1.25] for n in range(N)], device="cuda").to(stage.tdt)]
    x = x0
    for i, block in enumerate(stage.blocks):
        t = ss.ss_dwconv2d_fwd(x, block["dw"], block["dw_bias"], (3, 3))
        want = oracle.dwconv2d(host_bits(x), host_bits(block["dw"]), dtype=dtype, bias=block["dw_bias"].cpu().numpy(), pad=(3, 3), act=0)
        check_close(t, want, "depthwise")
        codes, scales = ss.ss_norm_mx4_fwd(stage.norm, t, block["w"], block["b"])
        xq = ref.dequantize(codes.cpu().numpy().reshape(-1, codes.shape[-1]), scales.cpu().numpy().reshape(-1, scales.shape[-1]), C)
        exact = ref.norm(_wide(t), 1, _wide(block["w"][None])[0], _wide(block["b"][None])[0], EPS)
        # (half a step of the elements is at most an eighth of a block's largest; a value between 6 and 8 times its scale loses up to a quarter)
        blocks = np.abs(exact).reshape(-1, C // 32, 32).max(axis=-1).repeat(32, axis=1)
        assert (np.abs(xq - exact) <= 0.25 * blocks + 1e-5).all()
        wq1, wq2 = (ref.through_mx4(_wide(block[n + "_W"]) * _wide(block[n + "_M"])) for n in ("expand", "contract"))
        wide = ss.ss_pw_mx4_q_fwd(stage.expand, codes, scales, block["expand"], block["expand_bias"], None, ss.SS_ACT_GELU)
        want, bound = ref.pointwise(xq, wq1, block["expand_bias"].double().cpu().numpy(), None, 2)
        ref.close(wide.view(-1, 4 * C), want, bound, stage.tdt, "expansion")
        h = ss.ss_pw_mx4_fwd(stage.contract, wide, block["contract"], block["contract_bias"])
        want, bound = ref.pointwise(ref.through_mx4(_wide(wide)), wq2, block["contract_bias"].double().cpu().numpy(), None, 0)
        ref.close(h.view(-1, C), want, bound, stage.tdt, "contraction")
        assert torch.equal(h, stage.branch(block, x))
        if i == 0:
            x = ss.ss_norm_fwd(stage.sum, x, None, None, h, block["scale"], gates[0])
    out, y = stage.forward(x0, gates)
    p = {"x": _wide(x), "h": _wide(h), "w": _wide(stage.w[None])[0], "b": _wide(stage.b[None])[0], "scale": _wide(stage.blocks[-1]["scale"][None])[0],
         "gate": _wide(gates[1]), "post_w": None, "post_b": None}
    want_x, want_y = ref.block_forward(p, (1, 0))
    check_close(out.reshape(-1, C), want_x, "stream")
    check_close(y.reshape(-1, C), want_y, "norm")
    dy, dx_out = (torch.randn(x0.shape, generator=g, device="cuda").to(stage.tdt) for _ in range(2))
    grads = stage.tail_gradient(dy, dx_out)
    want = ref.block_backward(dict(p, x=_wide(out)), (1, 0), _wide(dy), _wide(dx_out))
    for name in ("dx", "dh", "dw", "db", "dscale"):
        got = getattr(grads, name)
        check_close(got.reshape(want[name].shape), want[name], name)
    # (one value to the image, of the activations' type: a relative norm over so few would be smaller than the type's own rounding, 2^-8 in bfloat16)
    terms = np.abs(want["dx"] * p["scale"] * p["h"]).reshape(N, -1).sum(axis=1, keepdims=True)
    ref.close(grads.dgate, want["dgate"], (H * W * C + 300) * ref.U32 * terms, stage.tdt, "dgate")
    if N > 1:
        assert (grads.dh[1] == 0).all()                       # a dropped branch learns nothing


def test_stage_graph(ss):
    """The whole chain captured once and replayed between eager work, on new inputs every time."""
    from paper_2411_00288_amd.convnext import Stage4bit
    stage = Stage4bit(2, 96, wl.BF16, seed=9)
    x = torch.randn((2, 14, 14, 96), device="cuda").bfloat16()
    stage.forward(x)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = stage.forward(x)
    for turn in range(4):
        x.mul_(-0.75)
        eager = stage.forward(x)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, eager)), turn
