"""The oracle's group normalisation against PyTorch's in float64 and against differences; mistakes planted in a copy of it are noticed."""
import numpy as np
import pytest

import workloads as wl
from oracle import cnn
from test_oracle_mutations import SRC, load_mutant

torch = pytest.importorskip("torch")
F = torch.nn.functional

NETS = {
    "behind_conv": {"input": (2, 6, 5), "classes": 3, "layers": [("conv", 6, 3, 1, 1), ("groupnorm", 2), ("relu",), ("avgpool", 3, 2), ("fc", 3)]},
    "first": {"input": (4, 5, 5), "classes": 3, "layers": [("groupnorm", 2), ("conv", 4, 3, 1, 0), ("groupnorm", 1), ("fc", 3)]},
    "behind_fc": {"input": (2, 4, 4), "classes": 4, "layers": [("fc", 12), ("groupnorm", 3), ("relu",), ("fc", 4), ("groupnorm", 1)]},
    "behind_relu": {"input": (2, 6, 6), "classes": 3, "layers": [("conv", 4, 3, 1, 1), ("relu",), ("groupnorm", 2), ("maxpool", 3, 2), ("fc", 3)]},
}


def torch_loss(net, theta, x, y):
    t = torch.tensor(theta, requires_grad=True)
    a, at, shapes = torch.tensor(x), 0, iter(wl.param_shapes(net))
    for L in net["layers"]:
        if L[0] in ("conv", "fc", "groupnorm"):
            ws, b = next(shapes)
            n = int(np.prod(ws))
            w, bias = t[at:at + n].reshape(ws), t[at + n:at + n + b]
            at += n + b
        if L[0] == "conv":
            a = F.conv2d(a, w, bias, stride=L[3], padding=L[4])
        elif L[0] == "fc":
            a = F.linear(a.reshape(a.shape[0], -1), w, bias)
        elif L[0] == "groupnorm":
            a = F.group_norm(a, L[1], w, bias, 1e-5)
        elif L[0] == "relu":
            a = F.relu(a)
        elif L[0] == "maxpool":
            a = F.max_pool2d(a, L[1], L[2], ceil_mode=True)
        else:
            a = F.avg_pool2d(a, L[1], L[2], ceil_mode=True, count_include_pad=False)
    loss = F.cross_entropy(a.reshape(a.shape[0], -1), torch.tensor(y, dtype=torch.long))
    loss.backward()
    return float(loss.detach()), t.grad.numpy()


def draw(net, n=3, seed=0):
    rng = np.random.default_rng(seed)
    return rng.standard_normal(wl.num_params(net)) * 0.5, rng.standard_normal((n,) + net["input"]), rng.integers(0, net["classes"], n).astype(np.int32)


@pytest.mark.parametrize("name", sorted(NETS))
def test_against_torch(name):
    net = NETS[name]
    theta, x, y = draw(net)
    assert cnn.num_params(net) == wl.num_params(net)
    loss, grad = cnn.loss_and_gradient(net, theta, x, y)
    want, tg = torch_loss(net, theta, x, y)
    assert abs(loss - want) < 1e-12 and np.abs(grad - tg).max() < 1e-11


@pytest.mark.parametrize("name", sorted(NETS))
def test_against_differences(name):
    net = NETS[name]
    theta, x, y = draw(net, seed=1)
    _, grad = cnn.loss_and_gradient(net, theta, x, y)
    for k in range(0, theta.size, max(1, theta.size // 40)):
        step = np.zeros_like(theta)
        step[k] = 1e-6
        up, down = (cnn.loss_and_gradient(net, theta + s * step, x, y, want_grad=False)[0] for s in (1, -1))
        assert abs((up - down) / 2e-6 - grad[k]) < 1e-7


@pytest.mark.parametrize("old, new", [
    ("var += (x[first + i] - mean) * (x[first + i] - mean);\n      var /= count;\n      double dev", "var += x[first + i] * x[first + i];\n      var /= count;\n      double dev"),
    ("dscale[c] += dy[first + i] * d / dev;", "dscale[c] += dy[first + i] * d;"), ("dshift[c] += dy[first + i];", "dshift[c] = dy[first + i];"),
    ("dmean += -dh / dev;", ""), ("dvar += dh * d * -0.5", "dvar += dh * d * 0.5"), ("sqrt(var + 1e-5) * scale[c] + shift[c];", "sqrt(var + 1e-3) * scale[c] + shift[c];"),
    ("int c = g * per + (int)(i / HW);\n        y[", "int c = (int)(i / HW);\n        y["),
])
def test_planted_mistakes_are_noticed(old, new, tmp_path):
    text = open(SRC).read()
    assert text.count(old) >= 1
    lib = load_mutant(text.replace(old, new, 1), str(tmp_path))
    good, worst = cnn._lib, 0.0
    try:
        for name in sorted(NETS):
            net = NETS[name]
            theta, x, y = draw(net)
            want, tg = torch_loss(net, theta, x, y)
            cnn._lib = lib
            loss, grad = cnn.loss_and_gradient(net, theta, x, y)
            worst = max(worst, abs(loss - want), np.abs(grad - tg).max())
    finally:
        cnn._lib = good
    assert worst > 1e-6


def test_margin_counts_what_the_normalisation_subtracts():
    """One image of one channel, 1 x 2 pixels a and b through a unit convolution: v = (x - mean) r, its terms |x| r and the group's mean |x| r."""
    net = {"input": (1, 1, 2), "classes": 2, "layers": [("conv", 1, 1, 1, 0), ("groupnorm", 1), ("relu",), ("fc", 2)]}
    theta = np.array([1.0, 0.0, 1.0, 0.0] + [0.1] * 6)
    a, b = 3.0, 2.0
    got = cnn.min_relu_margin(net, theta, np.array([a, b]).reshape(1, 1, 1, 2))
    assert abs(got - min(0.5 / (3 + 2.5), 0.5 / (2 + 2.5))) < 1e-4
