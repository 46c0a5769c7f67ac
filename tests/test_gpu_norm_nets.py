"""Networks with group normalisation layers against the CPU oracle, and training with AdamW as the server's rule."""
import numpy as np
import pytest

import adamw_reference as ref
import workloads as wl
from oracle import cnn
from test_gpu_net import SPREAD_FACTOR, TOL, check_gradient, decided_seed, draw_case, layer_errors, one_gradient, rel

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def net(c, h, w, classes, *layers):
    return {"name": "norm", "input": (c, h, w), "classes": classes, "layers": list(layers)}


N, R = (lambda g: ("groupnorm", g)), ("relu",)
NETS = {
    "conv_norm_relu_pool": net(3, 13, 11, 8, ("conv", 16, 3, 1, 1), N(4), R, ("maxpool", 3, 2), ("conv", 24, 3, 1, 1), N(3), R, ("avgpool", 3, 2), ("fc", 8)),
    "no_activation": net(3, 9, 8, 5, ("conv", 32, 3, 1, 1), N(8), ("conv", 32, 3, 1, 1), N(2), ("fc", 5)),
    "first": net(4, 9, 8, 5, N(2), ("conv", 8, 3, 1, 1), N(2), R, ("fc", 5)),
    "behind_relu": net(3, 10, 9, 8, ("conv", 16, 5, 1, 2), R, N(4), ("conv", 16, 3, 1, 1), R, N(1), ("fc", 8)),
    "behind_pool": net(3, 12, 11, 8, ("conv", 16, 3, 1, 1), R, ("maxpool", 3, 2), N(2), R, ("fc", 8)),
    "behind_fc": net(3, 8, 8, 8, ("conv", 8, 3, 1, 1), R, ("fc", 72), N(3), R, ("fc", 40), N(5), ("fc", 8)),
    "scores": net(3, 8, 8, 8, ("conv", 8, 3, 1, 1), R, ("fc", 8), N(2)),
    "odd": net(3, 11, 9, 5, ("conv", 13, 3, 1, 1), N(1), R, ("conv", 7, 3, 2, 0), N(1), ("fc", 5)),
    # (average pooling: of the 174 517 windows of 6 such images two have their largest values within 1e-6 of each other, the nearest 3.5e-7, where the
    # winner depends on the order of an fp32 sum and moves the filter gradient by one of its terms, 4e-3 of its norm)
    "in_chunks": net(3, 70, 61, 4, ("conv", 32, 3, 1, 1), N(1), R, ("avgpool", 3, 2), ("fc", 4)),
    "strided_first": net(3, 29, 27, 8, ("conv", 16, 7, 2, 0), N(4), R, ("maxpool", 3, 2), ("conv", 64, 3, 1, 1), N(8), R, ("fc", 40), R, ("fc", 8)),
}


@pytest.mark.parametrize("name, lam, mu", [(n, lam, mu) for n in sorted(NETS) for lam, mu in ((2, 3), (9, 5)) if n != "in_chunks" or lam == 2])
def test_gradient_fp32(name, lam, mu):
    nt = NETS[name]
    seed = decided_seed(nt, lam, mu, 7 + mu, 0.3)
    for (g, rg, loss, rl) in one_gradient(nt, mu, "fp32", seed=seed, lam=lam, learners=[0, lam - 1]):
        check_gradient(nt, "fp32", g, rg, loss, rl, name)


@pytest.mark.parametrize("name", sorted(set(NETS) - {"scores"}))
def test_gradient_bf16(name):
    """Every tensor within the bound, or, where ReLU signs and pooling winners are undecided at bf16 precision, within 1.5 times the distance between the
    oracle's own two evaluations of it.  (Scores behind a normalisation are kept in bf16, which the oracle's reduced mode does not round to.)"""
    nt, lam, mu = NETS[name], 6, 4
    for (g, rg, loss, rl, eg) in one_gradient(nt, mu, "bf16", seed=5, lam=lam, both=True, learners=[0, 3]):
        errs, spread = layer_errors(nt, g, rg)[1], layer_errors(nt, rg, eg)[1]
        assert all(e <= max(TOL["bf16"], SPREAD_FACTOR * s) for e, s in zip(errs, spread)), (name, errs, spread)
        assert max(errs) < 0.2 and abs(loss - rl) < 2e-2 * max(1.0, abs(rl))


@pytest.mark.parametrize("name", ["conv_norm_relu_pool", "in_chunks"])
@pytest.mark.parametrize("compute", ["fp32", "bf16"])
def test_learners_and_evaluation_agree(name, compute):
    """A learner's gradient and loss are the same bits whoever else is in the call, and evaluate has the same losses."""
    from paper_1511_05950_amd import binding, driver
    nt, lam, mu = NETS[name], 5, 3
    theta, X, Y = draw_case(nt, lam, mu, 3, 0.3)
    Xd, Yd = torch.from_numpy(X).cuda(), torch.from_numpy(Y).cuda()
    ctx = binding.Sasgd(lam, mu, lam, 2, net=nt, compute=compute, init_weights=theta)
    loss = torch.zeros(lam, device="cuda")
    for k in range(lam):
        ctx.getMinibatch(k, Xd[k * mu:(k + 1) * mu], Yd[k * mu:(k + 1) * mu])
        ctx.pullWeights(k, 0)
    ctx.calcGradient(list(range(lam)), loss)
    grads = [ctx.copyGradient(k) for k in range(lam)]
    again = torch.zeros(1, device="cuda")
    for k in range(lam):
        ctx.getMinibatch(k, Xd[k * mu:(k + 1) * mu], Yd[k * mu:(k + 1) * mu])
        ctx.pullWeights(k, 0)
        ctx.calcGradient([k], again)
        assert rel(ctx.copyGradient(k), grads[k]) < 2e-3 and abs(float(again) - float(loss[k])) < 1e-3 * abs(float(loss[k]))    # (cut differently)
    got, rank = torch.zeros(lam, device="cuda"), torch.zeros(lam * mu, dtype=torch.int32, device="cuda")
    driver.evaluate(ctx, Xd, Yd, lam, mu, got, rank)
    assert torch.allclose(got, loss, rtol=1e-3)
    scores = [cnn.class_scores(nt, theta, X[k * mu:(k + 1) * mu], Y[k * mu:(k + 1) * mu], round_bf16=compute == "bf16")[0] for k in range(lam)]
    assert np.allclose(got.cpu().numpy(), scores, rtol=2e-2 if compute == "bf16" else 1e-4)
    ctx.destroy()


@pytest.mark.parametrize("layers, word", [([("groupnorm", 3)], "divide"), ([("groupnorm", 0)], "divide"), ([("relu",), ("groupnorm", 2), ("relu",), ("relu",)], "relu")])
def test_refused_networks(layers, word, capfd):
    from paper_1511_05950_amd import binding
    nt = net(3, 6, 6, 4, ("conv", 8, 3, 1, 1), *layers, ("fc", 4))
    with pytest.raises(binding.SasgdError):
        binding.Sasgd(1, 2, 1, 1, net=nt, init_weights=np.zeros(5000, np.float32))
    assert word in capfd.readouterr().err


# ------------------------------------------------------------------------------------------------ AdamW as the server's rule
def moments(P, states):
    n = (P + 255) // 256 * 256
    if states == "fp32":
        return torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda"), None, None
    m, v = (torch.zeros(n, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn) for _ in range(2))
    return m, v, torch.zeros(n // 256, device="cuda"), torch.zeros(n // 256, device="cuda")


@pytest.mark.parametrize("mode", ["per_gradient", "mean_staleness", "constant"])
@pytest.mark.parametrize("states", ["fp32", "e4m3"])
@pytest.mark.parametrize("ring", [1, 3])
def test_server_takes_the_steps_of_adamw(ring, states, mode):
    """Gradients from outside: the context's weights and moments are those of AdamW.apply, bit for bit."""
    from paper_1511_05950_amd import binding
    P, lam, n = 5003, 6, 2
    gen = torch.Generator(device="cuda")
    gen.manual_seed(4)
    theta = torch.randn(P, device="cuda", generator=gen) * 0.1
    ctx = binding.Sasgd(lam, 0, n, ring, num_params=P, alpha0=0.01, momentum=0.5, weight_decay=0.1, lr_mode=mode, init_weights=theta)
    mine, theirs = moments(P, states), moments(P, states)
    opt = binding.AdamW([theta], *theirs, alpha0=float(np.float32(0.01)), weight_decay=float(np.float32(0.1)), beta2=0.99, lr_mode=mode, seed=9)
    first = 0
    for i in range(6):
        grads = [torch.randn(P, device="cuda", generator=gen) for _ in range(3)]
        stale = [min(k, i) for k in range(3)]
        if i == 1:                                           # one momentum step before: its gradient leaves the moments alone
            ctx.useAdamW(*mine, beta2=0.99, seed=9)
            theta.copy_(torch.from_numpy(ctx.copyWeights()))
            first = i
        if i == 4:
            ctx.setBaseRate(0.002)
            opt.setBaseRate(float(np.float32(0.002)))
        for g, tau in zip(grads, stale):
            assert ctx.pushGradientExternal(g, i - tau) == tau
        ctx.sumGradients()
        if i >= 1:
            with pytest.raises(binding.SasgdError) as e:
                ctx.useAdamW(*mine)
            assert e.value.code == binding.ESTATE
        assert ctx.applyUpdate() == i + 1
        if i >= 1:
            opt.apply([[g] for g in grads], i - first + 1, staleness=stale)
            assert np.array_equal(ctx.copyWeights(), theta.cpu().numpy())
            assert torch.equal(mine[0].view(torch.uint8), theirs[0].view(torch.uint8)) and torch.equal(mine[1].view(torch.uint8), theirs[1].view(torch.uint8))
    with pytest.raises(binding.SasgdError) as e:
        ctx.copyMomentum()
    assert e.value.code == binding.ESTATE
    ctx.useAdamW(None, None)
    assert ctx.copyMomentum().any()
    ctx.destroy()


def test_refused_rules():
    from paper_1511_05950_amd import binding
    ctx = binding.Sasgd(2, 0, 1, 1, num_params=1000, init_weights=np.zeros(1000, np.float32))
    m, v, _, _ = moments(1000, "fp32")
    with pytest.raises(ValueError):
        ctx.useAdamW(m[:1000], v)
    for kw in (dict(beta1=1.0), dict(beta2=-1.0), dict(eps=0.0)):
        with pytest.raises(binding.SasgdError) as e:
            ctx.useAdamW(m, v, **kw)
        assert e.value.code == binding.EINVAL
    with pytest.raises(binding.SasgdError):
        binding.load().sasgd_useAdamW.argtypes and ctx._check(binding.load().sasgd_useAdamW(ctx._h, binding.ctypes.byref(binding.SasgdAdamw(0, 1, 0, 0, 0, .9, .9, 1e-8, 0)),
                                                                                           binding.ctypes.byref(binding.SasgdMoments(0x1000, 0x1000, None, None))))
    ctx.destroy()


TRAIN = net(3, 12, 12, 6, ("conv", 16, 3, 1, 1), N(4), R, ("avgpool", 3, 2), ("conv", 32, 3, 1, 1), N(4), R, ("fc", 64), R, ("fc", 6))


@pytest.mark.parametrize("flat", [True, False])
@pytest.mark.parametrize("compute", ["fp32", "bf16"])
def test_training_with_normalisation_and_adamw(compute, flat):
    """Stale learners of a normalised network, AdamW at the server, against the oracle's gradients and the rule in 64 bits.  epsilon is of the
    gradients' size: a weight's move is then off by no more than its gradient, relative to the gradients' size (1e-4 in fp32, 2e-2 in bf16 compute per
    gradient; four updates of a share 1 each of the way)."""
    from paper_1511_05950_amd import binding, driver
    lam, mu, n, K = 4, 4, 2, 4
    theta0 = wl.init_weights(TRAIN, 11, std=0.2)
    X, Y = wl.images(TRAIN, 8 * mu, 12), wl.labels(TRAIN, 8 * mu, 13)
    Xd, Yd = torch.from_numpy(X).cuda(), torch.from_numpy(Y).cuda()
    schedule = [[0, 1], [1, 0], [2, 1], [0, 2]]
    ctx = binding.Sasgd(lam, mu, n, 4, net=TRAIN, compute=compute, alpha0=0.01, weight_decay=0.01, init_weights=theta0,
                        flags=binding.FLAG_FLAT_FC_GRADIENT if flat else 0)
    keep = moments(ctx.P, "fp32")
    ctx.useAdamW(*keep, beta1=0.8, beta2=0.9, eps=0.02)
    where = lambda i, l: slice((2 * i + l) * mu, (2 * i + l + 1) * mu)  # noqa: E731
    log = driver.run_softsync(ctx, schedule, lambda i, l: (Xd[where(i, l)], Yd[where(i, l)]), lam)
    versions = [theta0.astype(np.float64)]
    m, v = np.zeros(ctx.P), np.zeros(ctx.P)
    for i in range(K):
        taus = [min(t, i) for t in schedule[i]]
        grads = [cnn.loss_and_gradient(TRAIN, versions[i - tau], X[where(i, l)], Y[where(i, l)], round_bf16=compute == "bf16")[1] for l, tau in enumerate(taus)]
        assert [e[4] for e in log if e[0] == i] == taus
        th, m, v = ref.step(versions[i], grads, m, v, i + 1, taus, "per_gradient", 0.01, 0.8, 0.9, 0.02, 0.01)
        versions.append(th)
    got = ctx.copyWeights()
    bound = 1e-3 if compute == "fp32" else 0.1
    assert rel(got - theta0, versions[-1] - theta0) < bound
    assert rel(keep[0][:ctx.P].cpu().numpy(), m) < bound
    if compute == "fp32":
        for i in range(1, K + 1):
            assert rel(ctx.copyWeights(i) - theta0, versions[i] - theta0) < bound
    ctx.destroy()


def test_gradients_bounded_outside_the_server():
    """calcGradient of a normalised network, norm, factor and AdamW on the caller's own weights."""
    from paper_1511_05950_amd import binding
    mu = 6
    theta0 = wl.init_weights(TRAIN, 21, std=0.2)
    X, Y = wl.images(TRAIN, mu, 22), wl.labels(TRAIN, mu, 23)
    ctx = binding.Sasgd(1, mu, 1, 1, net=TRAIN, compute="fp32", init_weights=theta0)
    ctx.getMinibatch(0, torch.from_numpy(X).cuda(), torch.from_numpy(Y).cuda())
    ctx.pullWeights(0, 0)
    ctx.calcGradient([0])
    flat = torch.from_numpy(ctx.copyGradient(0)).cuda()
    theta, at, weights, grads = torch.from_numpy(theta0.copy()).cuda(), 0, [], []
    for ws, b in wl.param_shapes(TRAIN):                     # tensor by tensor, as they lie in the flat vectors
        for k in (int(np.prod(ws)), b):
            weights.append(theta[at:at + k])
            grads.append(flat[at:at + k])
            at += k
    n = binding.momentElements(weights)
    opt = binding.AdamW(weights, torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda"), alpha0=0.01, beta1=0.0, beta2=0.0, eps=1.0, lr_mode="constant")
    out, work = torch.zeros(2, device="cuda"), torch.zeros(binding.NORM_WORKSPACE, dtype=torch.uint8, device="cuda")
    _, g = cnn.loss_and_gradient(TRAIN, theta0, X, Y)
    bound = float(np.linalg.norm(g)) / 3
    binding.gradientNorm(grads, out, max_norm=bound, workspace=work)
    opt.apply([grads], 1, scale=out[1:])
    assert abs(float(out[0]) / np.linalg.norm(g) - 1) < 1e-4 and abs(float(out[1]) * 3 - 1) < 1e-4
    want = -0.01 * (g / 3) / (np.abs(g / 3) + 1)
    assert rel(theta.cpu().numpy().astype(np.float64) - theta0, want) < 1e-3
    ctx.destroy()
