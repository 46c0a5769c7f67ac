"""What groupNorm and its gradient refuse before anything is enqueued, and how calls are cut into workgroups (host code only)."""
import ctypes

import pytest

from paper_1511_05950_amd import binding as b

A = 0x100000                     # stands for a device address


def call(gradient, **kw):
    s = b.SasgdNormShape(kw.get("images", 4), kw.get("positions", 64), kw.get("channels", 32), kw.get("groups", 4), kw.get("type", 0), kw.get("ptype", 0),
                         kw.get("act", 0), kw.get("eps", 1e-5), kw.get("xi", 0), kw.get("xp", 0), kw.get("yi", 0), kw.get("yp", 0))
    err = ctypes.create_string_buffer(200)
    shape = None if kw.get("no_shape") else ctypes.byref(s)
    x, y, st, scale, work = kw.get("x", A), kw.get("y", A), kw.get("stats", A), kw.get("scale", A), kw.get("work", A)
    if gradient:
        rc = b.load().sasgd_groupNormGradient(shape, x, scale, None, st, y, kw.get("dx", A), kw.get("ds", A), None, work, kw.get("bytes", 1 << 30), None, err, 200)
    else:
        rc = b.load().sasgd_groupNorm(shape, x, scale, None, y, st, work, kw.get("bytes", 1 << 30), None, err, 200)
    return rc, err.value.decode()


BOTH = [
    (dict(no_shape=1), "shape"), (dict(images=-1), "images"), (dict(positions=0), "positions"), (dict(positions=(1 << 26) + 1), "positions"),
    (dict(channels=0), "channels"), (dict(channels=4100), "channels"), (dict(groups=0), "groups"), (dict(groups=5), "groups"), (dict(groups=64), "groups"),
    (dict(type=2), "type"), (dict(ptype=-1), "type"), (dict(act=3), "activation"), (dict(eps=0.0), "eps"), (dict(eps=float("nan")), "eps"),
    (dict(eps=float("inf")), "eps"), (dict(xp=31), "overlap"), (dict(yp=31), "overlap"), (dict(xi=-1), "stride"), (dict(yi=31), "overlap"), (dict(yi=2047), "overlap"), (dict(yi=1 << 41), "stride"),
    (dict(x=None), "null"), (dict(y=None), "null"), (dict(x=A + 2), "aligned"), (dict(y=A + 2), "aligned"), (dict(scale=A + 2), "scale"),
    (dict(stats=A + 4), "stats"), (dict(channels=2048, groups=1, x=A + 4), "1024"), (dict(channels=1026, groups=1), "1024"),
    (dict(images=1 << 40), "too many images"), (dict(yi=32, yp=127), "overlap"), (dict(yi=31, yp=1 << 20), "overlap"),
    (dict(positions=1 << 20, work=None), "workspace"), (dict(positions=1 << 20, work=A + 8), "workspace"), (dict(positions=1 << 20, bytes=15), "workspace"),
]


@pytest.mark.parametrize("gradient", [False, True])
@pytest.mark.parametrize("kw, word", BOTH)
def test_refused(kw, word, gradient):
    rc, msg = call(gradient, **kw)
    assert rc == b.EINVAL and msg.startswith("groupNormGradient: " if gradient else "groupNorm: ") and word in msg, (rc, msg)


@pytest.mark.parametrize("kw, word", [(dict(stats=None), "stats"), (dict(dx=A + 2), "aligned"), (dict(ds=A + 2), "dscale"), (dict(work=None), "workspace")])
def test_gradient_refused(kw, word):
    rc, msg = call(True, **kw)
    assert rc == b.EINVAL and word in msg


@pytest.mark.parametrize("kw", [dict(yp=40), dict(xp=40), dict(yi=4096), dict(xi=32, xp=128)])
def test_in_place_with_other_strides_is_refused(kw):
    rc, msg = call(False, x=A, y=A, **kw)
    assert rc == b.EINVAL and "same strides" in msg


def test_no_images_is_no_error():
    assert call(False, images=0, x=None, y=None, stats=None, work=None)[0] == b.OK
    assert call(True, images=0, x=None, y=None, stats=None, dx=None, ds=None, work=None)[0] == b.OK


def test_workspace():
    s = b.SasgdNormShape(4, 64, 32, 4, 0, 0, 0, 1e-5, 0, 0, 0, 0)
    out = ctypes.c_size_t(1)
    assert b.load().sasgd_groupNormWorkspace(ctypes.byref(s), 0, ctypes.byref(out)) == b.OK and out.value == 0
    assert b.load().sasgd_groupNormWorkspace(ctypes.byref(s), 1, ctypes.byref(out)) == b.OK and out.value >= 4 * 32 * 8
    assert b.load().sasgd_groupNormWorkspace(ctypes.byref(s), 0, None) == b.EINVAL
    # the largest shape does not overflow; one image more is refused
    big = b.SasgdNormShape(1 << 31, 1 << 26, 4096, 1, 0, 0, 0, 1e-5, 0, 0, 0, 0)
    assert b.load().sasgd_groupNormWorkspace(ctypes.byref(big), 1, ctypes.byref(out)) == b.OK and out.value >= (1 << 31) * 4096 * 8
    big.images += 1
    assert b.load().sasgd_groupNormWorkspace(ctypes.byref(big), 1, ctypes.byref(out)) == b.EINVAL
    s.groups = 3
    assert b.load().sasgd_groupNormWorkspace(ctypes.byref(s), 0, ctypes.byref(out)) == b.EINVAL
