"""groupNorm and groupNormGradient of tensors of other ranks, and with a scale or a shift alone."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def both(x, dy, scale, shift, groups, activation="silu"):
    from paper_1511_05950_amd import binding
    y, dx = torch.full_like(x, 3.0), torch.full_like(x, 3.0)
    stats = torch.zeros(x.shape[0], groups, 2, device="cuda")
    dscale, dshift = (torch.full((x.shape[-1],), 3.0, device="cuda") for _ in range(2))
    binding.groupNorm(x, scale, shift, groups, y, stats, activation=activation, workspace=torch.empty(max(16, binding.groupNormWorkspace(x, groups)), dtype=torch.uint8, device="cuda"))
    binding.groupNormGradient(x, scale, shift, groups, stats, dy, dx, dscale, dshift, activation=activation,
                              workspace=torch.empty(max(16, binding.groupNormWorkspace(x, groups, True)), dtype=torch.uint8, device="cuda"))
    return y, stats, dx, dscale, dshift


@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("shape", [(70, 48), (5, 13, 48), (3, 4, 5, 6, 48), (2, 1, 3, 1, 2, 1, 7, 48), (1, 61, 50, 2, 48), (2, 1, 1, 48)])
def test_other_ranks(shape, kind):
    """The same bits as the four-dimensional tensor of as many positions."""
    x, dy = (torch.randn(*shape, device="cuda").to(kind) for _ in range(2))
    scale, shift = torch.randn(48, device="cuda"), torch.randn(48, device="cuda")
    flat = (shape[0], 1, -1, 48)
    for a, b in zip(both(x, dy, scale, shift, 3), both(x.view(flat), dy.view(flat), scale, shift, 3)):
        assert torch.equal(a.flatten(), b.flatten())


@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("shape", [(3, 10, 12, 48), (2, 61, 50, 48), (2, 7, 5, 45)])
@pytest.mark.parametrize("activation", ["none", "relu", "silu"])
def test_scale_or_shift_alone(shape, kind, activation):
    """What is not given is ones and zeros, bit for bit, and its gradient is the same."""
    c = shape[-1]
    x, dy = (torch.randn(*shape, device="cuda").to(kind) for _ in range(2))
    scale, shift, ones, zeros = torch.randn(c, device="cuda"), torch.randn(c, device="cuda"), torch.ones(c, device="cuda"), torch.zeros(c, device="cuda")
    for given, same in (((scale, None), (scale, zeros)), ((None, shift), (ones, shift)), ((None, None), (ones, zeros))):
        for a, b in zip(both(x, dy, *given, 3, activation), both(x, dy, *same, 3, activation)):
            assert torch.equal(a, b)
