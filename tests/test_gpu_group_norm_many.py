"""Group normalisation of more images than one launch takes."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("images, positions, kind", [((1 << 24) + 5, 1, torch.float32), ((1 << 24) - 8, 1, torch.bfloat16), ((3 << 24) + 100, 2, torch.bfloat16)])
def test_more_images_than_a_launch_takes(images, positions, kind):
    """Groups of two and four values, whose formulas are short; every image of y, dx and the statistics, and the sums over all of them."""
    from paper_1511_05950_amd import binding
    gen = torch.Generator(device="cuda")
    gen.manual_seed(7)
    x = torch.randn(images, positions, 2, device="cuda", generator=gen).to(kind)
    dy = torch.randn(images, positions, 2, device="cuda", generator=gen).to(kind)
    scale, shift = torch.tensor([1.5, 0.5], device="cuda"), torch.tensor([0.25, -0.5], device="cuda")
    y, dx, stats = torch.full_like(x, 7.0), torch.full_like(x, 7.0), torch.full((images, 1, 2), 7.0, device="cuda")
    dscale, dshift = torch.empty(2, device="cuda"), torch.empty(2, device="cuda")
    binding.groupNorm(x, scale, shift, 1, y, stats, eps=0.1)
    work = torch.empty(binding.groupNormWorkspace(x, 1, True), dtype=torch.uint8, device="cuda")
    binding.groupNormGradient(x, scale, shift, 1, stats, dy, dx, dscale, dshift, workspace=work)
    u, half = 2.0 ** -24, 2.0 ** -8 if kind == torch.bfloat16 else 2.0 ** -24
    total = {k: torch.zeros(2, dtype=torch.float64, device="cuda") for k in ("scale", "shift", "scale size", "shift size")}
    for at in range(0, images, 1 << 22):
        part = slice(at, at + (1 << 22))
        v, d = x[part].double(), dy[part].double()
        mean = v.mean((1, 2), keepdim=True)
        r = ((v - mean).square().mean((1, 2), keepdim=True) + 0.1).rsqrt()
        assert bool(((stats[part, 0, :1].double() - mean[:, 0]).abs() <= 16 * u * v.abs().amax((1, 2))[:, None]).all())
        assert bool(((stats[part, 0, 1:].double() / r[:, 0] - 1).abs() <= 64 * u).all())
        hat = (v - mean) * r
        # roundings of values of up to 5, divided by a deviation of 0.3 or more: below 64 u of 16; then the output's own
        want = hat * scale + shift
        assert bool(((y[part].double() - want).abs() <= half * want.abs() + 1024 * u).all())
        q = d * scale
        want = r * (q - q.mean((1, 2), keepdim=True) - hat * (q * hat).mean((1, 2), keepdim=True))
        assert bool(((dx[part].double() - want).abs() <= half * want.abs() + 4096 * u).all())
        for name, t in (("scale", d * hat), ("shift", d)):
            total[name] += t.sum((0, 1))
            total[name + " size"] += t.abs().sum((0, 1))
    # rows of images are added 512 at a time, 32 of them by a lane each: fewer than 16384 steps one behind the other
    for name, got in (("scale", dscale), ("shift", dshift)):
        assert bool(((got.double() - total[name]).abs() <= 16384 * u * total[name + " size"]).all()), name
