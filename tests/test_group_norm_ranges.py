"""Numbers of images and strides at the ends of what groupNorm takes (host code only)."""
import pytest

from paper_1511_05950_amd import binding as b
from test_group_norm_arguments import call


@pytest.mark.parametrize("gradient", [False, True])
@pytest.mark.parametrize("kw", [dict(yi=1 << 33, yp=2), dict(xi=1 << 33), dict(yi=1 << 18, yp=1 << 20), dict(xi=1 << 40)])
def test_images_that_reach_beyond_all_addresses_are_refused(kw, gradient):
    """2^31 images so far apart that their extent passes 64 bits, or 2^48 elements."""
    rc, msg = call(gradient, images=1 << 31, positions=2, channels=2, groups=1, **kw)
    assert rc == b.EINVAL and "stride" in msg, msg


@pytest.mark.parametrize("gradient", [False, True])
def test_one_image_may_lie_anywhere(gradient):
    """An image's distance to the next one is not used where there is none (the call then fails only for want of a workspace)."""
    rc, msg = call(gradient, images=1, positions=1 << 20, yi=1 << 40, xi=1 << 40, work=None)
    assert rc == b.EINVAL and "workspace" in msg, msg


@pytest.mark.parametrize("kw", [dict(xp=40), dict(yi=4096), dict(xi=32, xp=128)])
def test_no_images_are_not_in_place(kw):
    """Empty tensors have no address: x and y of different strides are both at 0, which is not one tensor."""
    assert call(False, images=0, x=None, y=None, stats=None, work=None, **kw)[0] == b.OK
