"""gradientNorm with bounds at the ends of fp32."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bound, least, most", [(1e-50, 0.0, 2.0 ** -149), (2.0 ** -149, 0.0, 2.0 ** -149), (1e-38, 0.99e-39, 1.01e-39), (1e39, 1.0, 1.0), (float("inf"), 1.0, 1.0), (0.0, 1.0, 1.0)])
def test_a_bound_below_the_smallest_number_is_not_none(bound, least, most):
    """Of a gradient of norm 10: a bound above 0 bounds it, also where it is 0 in 32 bits (1e-39 is a multiple of 2^-149, 1.4e-45)."""
    from paper_1511_05950_amd import binding
    out, work = torch.zeros(2, device="cuda"), torch.zeros(binding.NORM_WORKSPACE, dtype=torch.uint8, device="cuda")
    binding.gradientNorm([torch.full((100,), 1.0, device="cuda")], out, max_norm=bound, workspace=work)
    norm, factor = out.double().cpu().tolist()
    assert norm == 10.0 and least <= factor <= most, (norm, factor)
