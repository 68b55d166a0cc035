"""How the ConvNeXt stage is called: a gate to the block."""
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
