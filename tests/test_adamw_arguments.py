"""What gradientNorm, momentElements and applyAdamW refuse, before anything is enqueued (host code only: the addresses are never read)."""
import ctypes

import pytest

from paper_1511_05950_amd import binding as b

A = 0x10000                      # stands for a device address


def call(**kw):
    """applyAdamW on two tensors with one argument changed: (code, message)."""
    lib = b.load()
    rule = b.SasgdAdamw(kw.get("lr_mode", 0), kw.get("moments", 0), kw.get("grad_type", 0), 0, kw.get("alpha0", 1e-3), kw.get("beta1", 0.9),
                        kw.get("beta2", 0.99), kw.get("eps", 1e-8), kw.get("wd", 0.0))
    ts = (b.SasgdTensor * 2)()
    ts[0] = b.SasgdTensor(kw.get("numel", 10), kw.get("theta", A), kw.get("out", A), kw.get("shadow", None))
    ts[1] = b.SasgdTensor(0, None, None, None)
    c = kw.get("c", 1)
    n = max(c, 1)
    grads = (ctypes.c_void_p * (2 * n))(*[kw.get("grad", A)] * (2 * n))
    stale = (ctypes.c_int32 * n)(*[kw.get("tau", 0)] * n)
    mom = b.SasgdMoments(kw.get("m", A), kw.get("v", A), kw.get("ms", A), kw.get("vs", A))
    err = ctypes.create_string_buffer(200)
    rc = lib.sasgd_applyAdamW(ctypes.byref(rule), kw.get("tensors", ts), kw.get("count", 2), kw.get("grads", grads), c, kw.get("stale", stale),
                              ctypes.byref(mom), kw.get("step", 1), kw.get("step_dev", None), kw.get("factor", None), None, err, 200)
    return rc, err.value.decode()


@pytest.mark.parametrize("kw, word", [
    (dict(lr_mode=3), "lr_mode"), (dict(moments=2), "moments"), (dict(grad_type=5), "gradients"), (dict(alpha0=-1.0), "alpha0"),
    (dict(alpha0=float("nan")), "alpha0"), (dict(alpha0=float("inf")), "alpha0"), (dict(wd=-0.1), "weight_decay"), (dict(beta1=1.0), "beta1"),
    (dict(beta2=-0.1), "beta"), (dict(beta2=float("nan")), "beta"), (dict(eps=0.0), "epsilon"), (dict(eps=float("inf")), "epsilon"), (dict(c=0), "1..64"),
    (dict(c=65), "1..64"), (dict(step=0), "steps count from 1"), (dict(step_dev=A + 4), "step_dev"), (dict(factor=A + 2), "factor"), (dict(tau=-1), "staleness"),
    (dict(numel=-1), "length"), (dict(numel=(1 << 38) + 1), "length"), (dict(theta=None), "weights"), (dict(out=None), "weights"), (dict(theta=A + 2), "weights"),
    (dict(shadow=A + 1), "weights"), (dict(grad=None), "gradient"), (dict(grad=A + 2), "gradient"), (dict(grad=A + 1, grad_type=1), "gradient"),
    (dict(m=None), "moments"), (dict(v=A + 8), "moments"), (dict(moments=1, ms=None), "scales"), (dict(moments=1, vs=A + 1), "scales"),
    (dict(count=-1), "negative"), (dict(tensors=None), "null"), (dict(grads=None), "null"), (dict(stale=None), "null"),
])
def test_refused(kw, word):
    rc, msg = call(**kw)
    assert rc == b.EINVAL and msg.startswith("applyAdamW: ") and word in msg, (rc, msg)


def test_nothing_to_do_is_no_error():
    assert call(numel=0, theta=None, out=None, grad=None, m=None, v=None) == (b.OK, "")
    assert call(count=0, tensors=None, grads=None) == (b.OK, "")


@pytest.mark.parametrize("kw, word", [
    (dict(count=-1), "negative"), (dict(grads=None), "null"), (dict(numel=None), "null"), (dict(type=2), "type"), (dict(bound=-1.0), "max_norm"),
    (dict(bound=float("nan")), "max_norm"), (dict(out=None), "out_dev"), (dict(out=A + 2), "out_dev"), (dict(work=None), "workspace"), (dict(work=A + 4), "workspace"),
    (dict(n=-1), "tensor 0"), (dict(n=(1 << 38) + 1), "tensor 0"), (dict(grad=None), "tensor 0"), (dict(grad=A + 2), "tensor 0"), (dict(grad=A + 1, type=1), "tensor 0"),
])
def test_norm_refused(kw, word):
    err = ctypes.create_string_buffer(200)
    grads, numel = (ctypes.c_void_p * 1)(kw.get("grad", A)), (ctypes.c_int64 * 1)(kw.get("n", 5))
    rc = b.load().sasgd_gradientNorm(kw.get("grads", grads), kw.get("numel", numel), kw.get("count", 1), kw.get("type", 0), kw.get("bound", 0.0),
                                     kw.get("out", A), kw.get("work", A), None, err, 200)
    assert rc == b.EINVAL and err.value.decode().startswith("gradientNorm: ") and word in err.value.decode()


def test_message_buffer_is_optional():
    assert b.load().sasgd_gradientNorm(None, None, 1, 0, 0.0, A, A, None, None, 0) == b.EINVAL


def test_moment_elements():
    out = ctypes.c_int64(-5)
    sizes = (ctypes.c_int64 * 6)(0, 1, 255, 256, 257, 1 << 33)
    assert b.load().sasgd_momentElements(sizes, 6, ctypes.byref(out)) == b.OK
    assert out.value == 256 * (0 + 1 + 1 + 1 + 2) + (1 << 33)
    assert b.load().sasgd_momentElements(None, 0, ctypes.byref(out)) == b.OK and out.value == 0
    assert b.load().sasgd_momentElements(None, 1, ctypes.byref(out)) == b.EINVAL
    assert b.load().sasgd_momentElements((ctypes.c_int64 * 1)(-1), 1, ctypes.byref(out)) == b.EINVAL
