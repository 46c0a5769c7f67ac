"""groupNorm and groupNormGradient agree about which outputs a ReLU passes."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("h, w, c, groups", [(4, 4, 2048, 2), (3, 5, 1000, 40), (3, 5, 999, 3), (24, 24, 2048, 2), (70, 61, 1000, 1)])
def test_outputs_a_rounding_from_zero(h, w, c, groups, kind):
    """Shifts that take one value of every channel to 0 or a rounding beside it: dy reaches dx, dscale and dshift where y is positive, and nowhere else."""
    from paper_1511_05950_amd import binding
    gen = torch.Generator(device="cuda")
    gen.manual_seed(h * w)
    x = torch.randn(1, h, w, c, device="cuda", generator=gen).to(kind)
    scale = 1 + 0.3 * torch.randn(c, device="cuda", generator=gen)
    stats, y = torch.zeros(1, groups, 2, device="cuda"), torch.empty_like(x)
    work = torch.empty(max(16, binding.groupNormWorkspace(x, groups), binding.groupNormWorkspace(x, groups, True)), dtype=torch.uint8, device="cuda")
    binding.groupNorm(x, scale, None, groups, y, stats, workspace=work)          # (a shift does not move the statistics)
    mean, r = (stats[0, :, k].repeat_interleave(c // groups) for k in range(2))
    values = x.view(h * w, c).float()
    some = values[torch.randint(h * w, (c,), device="cuda", generator=gen), torch.arange(c, device="cuda")]
    shift = -((some - mean) * r * scale)
    binding.groupNorm(x, scale, shift, groups, y, stats, activation="relu", workspace=work)
    dscale, dshift, dx = torch.empty(c, device="cuda"), torch.empty(c, device="cuda"), torch.empty_like(x)
    binding.groupNormGradient(x, scale, shift, groups, stats, torch.ones_like(x), dx, dscale, dshift, activation="relu", workspace=work)
    on = (y.view(h * w, c) > 0)
    assert torch.equal(dshift, on.sum(0).float())                                # counts: exact in any order
    # dx from what passed: off by some roundings, where one more or less moves it by scale r
    dz = on.double()
    hat = ((values - mean) * r).double()
    q = (dz * scale.double()).view(h * w, groups, -1)
    hat = hat.view(h * w, groups, -1)
    want = stats[0, :, 1].double()[None, :, None] * (q - q.mean((0, 2), keepdim=True) - hat * (q * hat).mean((0, 2), keepdim=True))
    got = dx.double().view(h * w, groups, -1)
    half = 2.0 ** -8 if kind == torch.bfloat16 else 2.0 ** -24
    # (sums of up to 4 270 000 values of a group, lane by lane: 1e-4 of their mean magnitudes)
    assert bool(((got - want).abs() <= half * want.abs() + 1e-3 * float(r.max())).all())
