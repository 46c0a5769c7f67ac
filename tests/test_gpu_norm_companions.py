"""Networks with group normalisation: what a learner gets does not depend on who else is in the call.

How a normalisation is cut into workgroups goes by the number of learners, so between calls of the same number every bit is the same, and between calls of
different numbers fp32 gradients differ by the order of their sums: 2^-24 each, of at most some 170 values a lane and 64 chunks, 1e-5."""
import pytest

from test_gpu_net import draw_case, rel
from test_gpu_norm_nets import NETS

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def gradients(nt, lam, mu, compute, theta, X, Y, calls):
    """{(call, learner): (gradient, loss)}, all calls on one context."""
    from paper_1511_05950_amd import binding
    Xd, Yd = torch.from_numpy(X).cuda(), torch.from_numpy(Y).cuda()
    ctx = binding.Sasgd(lam, mu, lam, 2, net=nt, compute=compute, init_weights=theta)
    out = {}
    for call in calls:
        loss = torch.full((len(call),), -1.0, device="cuda")
        for k in call:
            ctx.getMinibatch(k, Xd[k * mu:(k + 1) * mu], Yd[k * mu:(k + 1) * mu])
            ctx.pullWeights(k, 0)
        ctx.calcGradient(list(call), loss)
        for at, k in enumerate(call):
            out[call, k] = ctx.copyGradient(k), float(loss[at])
    ctx.destroy()
    return out


@pytest.mark.parametrize("name", ["conv_norm_relu_pool", "in_chunks", "behind_fc", "odd"])
@pytest.mark.parametrize("compute", ["fp32", "bf16"])
def test_other_companions_same_bits(name, compute):
    nt, lam, mu = NETS[name], 6, 3
    theta, X, Y = draw_case(nt, lam, mu, 3, 0.3)
    calls = [(0, 1), (0, 5), (2, 0), (0, 1, 2), (4, 0, 3), (5, 4, 0)]
    got = gradients(nt, lam, mu, compute, theta, X, Y, calls)
    for count in (2, 3):
        same = [got[c, 0] for c in calls if len(c) == count]
        for g, loss in same[1:]:
            assert (g == same[0][0]).all() and loss == same[0][1], (name, compute, count)


@pytest.mark.parametrize("name", ["conv_norm_relu_pool", "in_chunks", "behind_fc", "odd"])
def test_other_numbers_of_companions_fp32(name):
    nt, lam, mu = NETS[name], 9, 3
    theta, X, Y = draw_case(nt, lam, mu, 3, 0.3)
    calls = [(0,), (0, 1), tuple(range(9))]
    got = gradients(nt, lam, mu, "fp32", theta, X, Y, calls)
    for c in calls[1:]:
        assert rel(got[c, 0][0], got[calls[0], 0][0]) < 1e-5 and abs(got[c, 0][1] / got[calls[0], 0][1] - 1) < 1e-5, (name, c)
