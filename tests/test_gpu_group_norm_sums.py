"""groupNorm's statistics of long runs of values whose first ones are far from the rest, and of long constant runs.

Tolerance: u = 2^-24 is half an fp32 step.  A lane's sums are kept in 64 bits and rounded once, so how many values a lane adds does not count.  Lanes are then
added in at most 16 steps, units of a group in at most 8 more and chunks in at most 64, three roundings each with the products around them, so that
a mean is off by less than 128 u of the mean magnitude.  Distances of means enter the variance twice, over the deviation; its own terms are added in as many steps:
r, half the variance's, is off by less than (128 mean |x| / deviation + 256) u, bf16 pairs by the dot product 256 u more (32 steps at a time, an eighth of their sum)."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

u = 2.0 ** -24


def image(h, w, c, kind, base, every, seed):
    """Positions of which the first 256 of every `every` are random and the others `base`: where a lane's walk begins, its first value is far from the rest."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    x = torch.full((h * w, c), base, device="cuda")
    head = torch.arange(h * w, device="cuda") % every < 256
    x[head] = torch.randn(int(head.sum()), c, device="cuda", generator=gen)
    return x.to(kind).view(1, h, w, c)


def check(x, groups):
    from paper_1511_05950_amd import binding
    _, h, w, c = x.shape
    y, stats = torch.empty_like(x), torch.zeros(1, groups, 2, device="cuda")
    size = binding.groupNormWorkspace(x, groups)
    binding.groupNorm(x, None, None, groups, y, stats, workspace=torch.empty(max(size, 16), dtype=torch.uint8, device="cuda"))
    v = x.view(h * w, groups, c // groups)
    for g in range(groups):
        one = v[:, g].double()
        mean, size = one.mean(), one.abs().mean()
        var = (one - mean).square().mean()
        r = (var + 1e-5).rsqrt()
        off, rel = float((stats[0, g, 0].double() - mean).abs()), float((stats[0, g, 1].double() / r - 1).abs())
        assert off <= 128 * u * float(size), (g, off / u, float(size))
        bound = 128 * float(size) / float((var + 1e-5).sqrt()) + 256 + 256 * (x.dtype == torch.bfloat16)
        assert rel <= bound * u, (g, rel / u, bound)


@pytest.mark.parametrize("base", [0.0, 0.37])
@pytest.mark.parametrize("h, w, c, groups, kind", [
    (4096, 4096, 4, 1, torch.float32), (4096, 4096, 4, 4, torch.float32), (8192, 4096, 1, 1, torch.float32), (4096, 2048, 3, 3, torch.float32),
    (4096, 2048, 8, 8, torch.bfloat16), (4096, 2048, 8, 4, torch.bfloat16), (4096, 2048, 8, 1, torch.bfloat16), (4096, 4096, 1, 1, torch.bfloat16),
    (1024, 512, 128, 8, torch.float32), (700, 611, 40, 5, torch.float32)])
def test_first_values_far_from_the_rest_in_chunks(h, w, c, groups, kind, base):
    check(image(h, w, c, kind, base, -(-h * w // 64), h + c), groups)


@pytest.mark.parametrize("base", [0.0, 0.37])
@pytest.mark.parametrize("h, w, c, groups, kind", [
    (96, 96, 4, 1, torch.float32), (96, 96, 4, 4, torch.float32), (96, 90, 8, 8, torch.bfloat16), (96, 96, 8, 1, torch.bfloat16), (100, 61, 3, 3, torch.float32)])
def test_first_values_far_from_the_rest_held(h, w, c, groups, kind, base):
    check(image(h, w, c, kind, base, h * w, h + c), groups)


@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16])
def test_alternating_values_of_one_size(kind):
    """Squares that are all alike: their running sum is rounded the same way again and again."""
    x = torch.full((4096 * 2048, 8), 1.7, device="cuda")
    x[1::2] = -1.7
    check(x.to(kind).view(1, 4096, 2048, 8), 2)


def test_squares_beyond_32_bits():
    """Distances whose squares pass the largest fp32 value: the variance is infinite, not nothing."""
    from paper_1511_05950_amd import binding
    x = torch.randn(1, 8, 8, 4, device="cuda") * 1e25
    stats = torch.zeros(1, 1, 2, device="cuda")
    y = torch.empty_like(x)
    binding.groupNorm(x, None, None, 1, y, stats)
    assert float(stats[0, 0, 1]) == 0.0 and not y.any()
