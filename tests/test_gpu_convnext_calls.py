"""How the ConvNeXt stage is called: a gate to the block, a gradient to the forward pass."""
import pytest
import torch

from paper_2411_00288_amd import workloads as wl

pytestmark = pytest.mark.gpu


@pytest.fixture
def stage(ss):
    from paper_2411_00288_amd.convnext import Stage4bit
    return Stage4bit(3, 64, wl.BF16, seed=3)


def _x(n=2, seed=0):
    return torch.randn((n, 5, 5, 64), generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").bfloat16()


@pytest.mark.parametrize("count", [0, 1, 2, 4])
def test_as_many_gates_as_blocks(stage, count):
    """Fewer gates would leave blocks out, more would give the last block the wrong one."""
    gate = torch.full((2, 1), 0.5, device="cuda").bfloat16()
    with pytest.raises(ValueError, match="gates"):
        stage.forward(_x(), [gate] * count)
    with pytest.raises(ValueError, match="gates"):
        stage.forward(_x(), (gate for _ in range(count)))


def test_gates_of_one_are_no_gates(stage):
    one = torch.ones((2, 1), device="cuda").bfloat16()
    plain = stage.forward(_x())
    for gates in ([one] * 3, [None, one, None], (one for _ in range(3))):
        assert all(torch.equal(a, b) for a, b in zip(plain, stage.forward(_x(), gates)))


def _same(a, b):
    return all((u is None) == (v is None) and (u is None or torch.equal(u, v)) for u, v in zip(a, b))


def test_gradient_without_a_forward_pass(stage):
    with pytest.raises(ValueError, match="no forward"):
        stage.tail_gradient(_x())


@pytest.mark.parametrize("gated", [False, True])
def test_gradients_of_several_forward_passes(stage, gated):
    """Two batches before their gradients: each takes its own activations and gate, and the stage does not guess which."""
    gates = [[None, None, torch.full((2, 1), v, device="cuda").bfloat16()] if gated else None for v in (0.5, 2.0)]
    dy, dx_out = _x(seed=8), _x(seed=9)
    alone = []
    for i in range(2):
        stage.forward(_x(seed=i), gates[i])
        alone.append(stage.tail_gradient(dy, dx_out))
        assert _same(alone[i], stage.tail_gradient(dy, dx_out))                   # (again, of the same pass)
    passes = [stage.forward(_x(seed=i), gates[i]) for i in range(2)]
    with pytest.raises(ValueError, match="2 forward passes"):
        stage.tail_gradient(dy, dx_out)
    assert not _same(*alone)
    for i in range(2):
        assert _same(alone[i], stage.tail_gradient(dy, dx_out, of=passes[i]))
        x, y = passes[i]
        assert x is passes[i].tail[0] and y.shape == x.shape
    stage.forward(_x(seed=0), gates[0])
    assert _same(alone[0], stage.tail_gradient(dy, dx_out))


def test_gradient_captured_between_other_passes(stage):
    """Forward pass and gradient in a graph; eager passes of another batch between its replays change nothing."""
    x, other, dy = _x(seed=1), _x(n=4, seed=2), _x(seed=3)
    stage.tail_gradient(dy, of=stage.forward(x))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = stage.forward(x)
        grads = stage.tail_gradient(dy, of=out)
    for turn in range(4):
        x.mul_(-0.75)
        want = stage.tail_gradient(dy, of=stage.forward(x))
        stage.forward(other)
        graph.replay()
        stage.forward(other)
        torch.cuda.synchronize()
        assert _same(grads, want), turn
