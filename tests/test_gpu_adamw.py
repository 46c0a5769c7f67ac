"""gradientNorm and applyAdamW against their formulas in 64 bits.

Tolerances: u = 2^-24 is half an fp32 step.  The combined gradient is a sum of c products: off by (c + 2) u of the sum of magnitudes
`G`, one product with the factor included; m and v are two products and a sum each; the weight's move is m's product (1 u), a root
of 1 ulp (2 u) times a rounded constant (2 u more), a sum (1 u), a reciprocal of 1 ulp (2 u) and a product (1 u): 9 u; theta_out has two more.  Steps are checked one by one from the state the kernel has left."""
import numpy as np
import pytest

import adamw_reference as ref

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

u = 2.0 ** -24
SIZES = [0, 1, 255, 256, 257, 1024, 1027, 5000, 0, 64]


def place(sizes, kind, gen, std=1.0, shift=0, guard=64):
    """Tensors of the given sizes in one buffer, each `shift` elements behind a multiple of 64, and the buffer."""
    starts, at = [], guard
    for n in sizes:
        starts.append(at + shift)
        at += (n + shift + 63) // 64 * 64 + guard
    flat = (torch.randn(at + guard, device="cuda", generator=gen) * std).to(kind)
    return [flat[s:s + n] for s, n in zip(starts, sizes)], flat


def generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def f64(t):
    return t.detach().double().cpu().numpy()


# ------------------------------------------------------------------------------------------------ norm
@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("sizes, shift", [([0, 1], 0), (SIZES, 0), (SIZES, 1), ([3, 300] * 130, 3), ([700_001], 0), ([3_000_000, 5], 2)])
def test_norm(kind, sizes, shift):
    from paper_1511_05950_amd import binding
    grads, _ = place(sizes, kind, generator(len(sizes) + shift), 1e-2, shift)
    want = np.sqrt(sum((f64(g) ** 2).sum() for g in grads))
    out, work = torch.full((2,), -1.0, device="cuda"), torch.full((binding.NORM_WORKSPACE,), 0xFF, dtype=torch.uint8, device="cuda")
    for bound in (0.0, float(want) * 0.25, float(want) * 4):
        binding.gradientNorm(grads, out, max_norm=bound, workspace=work)
        got = f64(out)
        assert abs(got[0] - want) <= 2 * u * want                     # 64-bit sums, rounded once
        factor = 1.0 if bound == 0 or want <= np.float32(bound) else np.float32(bound) / want
        assert abs(got[1] - factor) <= 2 * u * factor


@pytest.mark.parametrize("size", [1e-30, 1e25, 3e38])
def test_norm_of_tiny_and_huge_values(size):
    from paper_1511_05950_amd import binding
    g = torch.full((1000,), size, device="cuda")
    out, work = torch.zeros(2, device="cuda"), torch.zeros(binding.NORM_WORKSPACE // 8, dtype=torch.float64, device="cuda")
    binding.gradientNorm([g[:500], g[500:]], out, max_norm=1.0, workspace=work)
    want = np.sqrt(1000) * f64(g)[0]
    if size > 1e38:                                                   # finite in 64 bits, not in 32: the factor still bounds it
        assert np.isinf(f64(out)[0])
    else:
        assert abs(f64(out)[0] / want - 1) <= 2 * u
    assert abs(f64(out)[1] / min(1.0, 1 / want) - 1) <= 2 * u + (1e-2 if 1 / want < 1e-37 else 0)     # (denormals below 2^-126)


@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
def test_norm_that_is_not_finite(bad):
    from paper_1511_05950_amd import binding
    g = torch.ones(5000, device="cuda")
    g[4321] = bad
    out, work = torch.zeros(2, device="cuda"), torch.zeros(binding.NORM_WORKSPACE, dtype=torch.uint8, device="cuda")
    for bound in (0.0, 1.0):
        binding.gradientNorm([g], out, max_norm=bound, workspace=work)
        assert not np.isfinite(f64(out)[0]) and np.isnan(f64(out)[1])


def test_norm_of_nothing():
    from paper_1511_05950_amd import binding
    out, work = torch.full((2,), 7.0, device="cuda"), torch.full((binding.NORM_WORKSPACE,), 0xFF, dtype=torch.uint8, device="cuda")
    binding.gradientNorm([], out, max_norm=1.0, workspace=work)
    assert f64(out).tolist() == [0, 1]


# ------------------------------------------------------------------------------------------------ AdamW
def bytes_of(t):
    return t.view(torch.uint8).cpu().numpy()


class Run:
    """Weights, moments and gradients of a case, and what one step of the kernel is to give."""

    def __init__(self, sizes, kind=torch.float32, states="fp32", c=1, mode="per_gradient", shift=0, copies=True, outs=False, seed=5, beta1=0.9, beta2=0.99,
                 eps=1e-6, wd=0.1, alpha0=0.01, std=1e-2):
        from paper_1511_05950_amd import binding
        gen = generator(seed)
        self.sizes, self.c, self.mode, self.states = sizes, c, mode, states
        self.hyper = (alpha0, beta1, beta2, eps, wd)
        self.seed = 1000 + seed
        self.theta, self.flat = place(sizes, torch.float32, gen, 0.1, shift)
        self.out, self.out_flat = place(sizes, torch.float32, gen, 0.1, shift) if outs else (self.theta, self.flat)
        self.copies, self.copy_flat = place(sizes, torch.bfloat16, gen, 1.0, shift) if copies else ([None] * len(sizes), None)
        if copies:
            self.copies = [x if k % 3 else None for k, x in enumerate(self.copies)]
        self.lists = [place(sizes, kind, gen, std, shift)[0] for _ in range(c)]
        self.stale = [int(x) for x in np.random.default_rng(seed).integers(0, 6, c)]
        n = self.elements = binding.momentElements(self.theta)
        assert n == sum((s + 255) // 256 * 256 for s in sizes)
        self.ms = self.vs = None
        if states == "fp32":
            self.m, self.v = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
        else:
            self.m, self.v = (torch.zeros(n, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn) for _ in range(2))
            self.ms, self.vs = torch.zeros(n // 256, device="cuda"), torch.zeros(n // 256, device="cuda")
        self.opt = binding.AdamW(self.theta, self.m, self.v, self.ms, self.vs, copies=self.copies if copies else None, outs=self.out if outs else None,
                                 alpha0=alpha0, beta1=beta1, beta2=beta2, eps=eps, weight_decay=wd, lr_mode=mode, seed=self.seed)

    def moments(self):
        """m and v in 64 bits, padded."""
        if self.states == "fp32":
            return f64(self.m), f64(self.v)
        m = ref.e4m3(bytes_of(self.m)).reshape(-1, 256) * f64(self.ms)[:, None]
        root = ref.e4m3(bytes_of(self.v)).reshape(-1, 256) * f64(self.vs)[:, None]
        return m.flatten(), root.flatten() ** 2

    def step(self, t, factor=None, run=None):
        """One step, and every output against the formulas."""
        alpha0, beta1, beta2, eps, wd = self.hyper
        m0, v0 = self.moments()
        theta0 = [f64(x) for x in self.theta]
        grads = [[f64(x) for x in one] for one in self.lists]
        around = self.flat.clone(), self.copy_flat.clone() if self.copy_flat is not None else None, self.out_flat.clone()
        scale = None if factor is None else torch.tensor([factor], device="cuda")
        f = 1.0 if factor is None else float(np.float32(factor))
        if run is None:
            self.opt.apply(self.lists, t, staleness=self.stale, scale=scale)
        else:
            run()
        torch.cuda.synchronize()
        mean, share = ref.alphas(self.mode, self.stale)
        M, V, Mt, Vt = (np.zeros(self.elements) for _ in range(4))
        at = 0
        for k, n in enumerate(self.sizes):
            want, m, v = ref.step(theta0[k], [one[k] for one in grads], m0[at:at + n], v0[at:at + n], t, self.stale, self.mode, alpha0, beta1, beta2, eps, wd, f)
            G = abs(f) * sum(s * np.abs(one[k]) for s, one in zip(share, grads))
            dg = (self.c + 3) * u * G
            dm = (1 - beta1) * dg + 4 * u * (beta1 * np.abs(m0[at:at + n]) + (1 - beta1) * G)
            dv = (1 - beta2) * 2 * G * dg + 5 * u * (beta2 * v0[at:at + n] + (1 - beta2) * G * G)
            if self.states == "e4m3":                                  # decoded: a product, squared
                dm = dm + u * np.abs(m0[at:at + n])
                dv = dv + 3 * u * v0[at:at + n]
            rate = alpha0 * mean
            root = np.sqrt(v / (1 - beta2 ** t)) + eps
            move = rate / (1 - beta1 ** t) * np.abs(m) / root
            tol = rate / (1 - beta1 ** t) * dm / root + move * (0.5 * dv / np.maximum(v, 1e-300) * (root - eps) / root + 9 * u) + 3 * u * np.abs(theta0[k])
            got = f64(self.out[k])
            assert np.all(np.abs(got - want) <= tol + 1e-38), (k, n, np.max(np.abs(got - want) - tol))
            if self.copies[k] is not None:
                assert torch.equal(self.copies[k], self.out[k].bfloat16())
            M[at:at + n], V[at:at + n], Mt[at:at + n], Vt[at:at + n] = m, v, dm, dv
            at += (n + 255) // 256 * 256
        if self.states == "fp32":
            gm, gv = f64(self.m), f64(self.v)
            assert np.all(np.abs(gm - M) <= Mt + 1e-44) and np.all(np.abs(gv - V) <= Vt + 1e-44)
        else:
            bits = ref.chance(0, self.elements, self.seed, t)
            self.check8(self.m, self.ms, M, Mt, bits >> np.uint64(16), False)
            R = np.sqrt(V)
            self.check8(self.v, self.vs, R, np.divide(Vt, 2 * R, out=np.zeros_like(R), where=R > 0) + u * R, bits & np.uint64(0xFFFF), True)
        # nothing else was written
        for flat, before, mine in ((self.flat, around[0], self.theta if self.out is self.theta else []), (self.copy_flat, around[1], self.copies),
                                   (self.out_flat, around[2], self.out)):
            if flat is None:
                continue
            inside = torch.zeros(flat.numel(), dtype=torch.bool, device="cuda")
            for x in mine:
                if x is not None and x.numel():
                    at0 = (x.data_ptr() - flat.data_ptr()) // flat.element_size()
                    inside[at0:at0 + x.numel()] = True
            assert torch.equal(flat[~inside], before[~inside])

    @staticmethod
    def check8(codes, scales, want, tol, bits, floor):
        q, scale, y = ref.stored(want, bits, floor)
        got, gs = ref.e4m3(bytes_of(codes)).reshape(-1, 256), f64(scales)
        t = tol.reshape(-1, 256)
        most = np.abs(want).reshape(-1, 256).max(1)
        assert np.all(np.abs(gs - scale) <= t.max(1) / 448 + 3 * u * scale + 1e-38)
        # y is off by its value's and the largest's error (relative) and three roundings; the value stored may then be the other neighbour
        # where what is cut off lies that near to where the bits carry
        rel = np.divide(t, np.abs(want).reshape(-1, 256), out=np.zeros_like(t), where=want.reshape(-1, 256) != 0)
        off = y * (rel + np.divide(t.max(1), most, out=np.zeros_like(most), where=most > 0)[:, None] + 4 * u) + 4 * u * 2.0 ** -6
        low, gap = ref.grid_below(np.minimum(y, 448))
        carry = (y - low) / gap + bits.reshape(-1, 256) / 65536
        edge = np.minimum(np.abs(carry - 1), np.minimum(carry % 1, 1 - carry % 1)) <= off / gap
        edge |= (y - low <= off) | (low + gap - y <= off)
        wrong = got != q
        assert not np.any(wrong & ~edge), (np.sum(wrong & ~edge), got[wrong & ~edge][:3], q[wrong & ~edge][:3])
        assert np.all(np.abs(got - q)[wrong] <= gap[wrong] * 1.01) and wrong.mean() < 1e-3


@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("states", ["fp32", "e4m3"])
@pytest.mark.parametrize("c, mode", [(1, "constant"), (3, "per_gradient"), (64, "mean_staleness")])
@pytest.mark.parametrize("shift", [0, 1])
def test_steps(kind, states, c, mode, shift):
    r = Run(SIZES, kind, states, c, mode, shift, outs=False, seed=c + shift)
    for t in (1, 2, 3):
        r.step(t)


@pytest.mark.parametrize("states", ["fp32", "e4m3"])
def test_weights_go_elsewhere_and_the_factor_scales(states):
    r = Run(SIZES, torch.bfloat16, states, 2, outs=True)
    r.step(1, factor=0.3)
    r.step(2, factor=1.0)


@pytest.mark.parametrize("states", ["fp32", "e4m3"])
def test_more_tensors_than_a_launch_takes(states):
    r = Run([7, 300, 0, 1025] * 80, torch.float32, states, 2, copies=False)
    r.step(1)
    r.step(2)


@pytest.mark.parametrize("states", ["fp32", "e4m3"])
@pytest.mark.parametrize("c", [2, 7])
def test_gradients_that_are_flat_vectors(c, states):
    """Gradients cut alike out of flat vectors, at any distance from each other: the same bits as gradients that lie anywhere."""
    a, b = (Run([7, 300, 0, 1025, 64] * 60, torch.float32, states, c, copies=False, seed=3) for _ in range(2))
    total = sum(a.sizes)
    buffers = [torch.zeros(total + 3 * l, device="cuda") for l in range(c)]
    for l, flat in enumerate(buffers):
        at, lists = 2 * l, []
        for n, g in zip(b.sizes, b.lists[l]):
            flat[at:at + n] = g
            lists.append(flat[at:at + n])
            at += n
        b.lists[l] = lists
    for t in (1, 2):
        a.step(t)
        b.step(t)
    assert torch.equal(a.flat, b.flat) and torch.equal(a.m.view(torch.uint8), b.m.view(torch.uint8)) and torch.equal(a.v.view(torch.uint8), b.v.view(torch.uint8))


@pytest.mark.parametrize("states", ["fp32", "e4m3"])
@pytest.mark.parametrize("pad", [0, 1])
def test_flat_vectors_of_bf16_in_the_longest_window(pad, states):
    """64 flat bf16 vectors, the last the first once more, with copies and weights that go elsewhere."""
    a, b = (Run([1025, 0, 64, 300] * 30, torch.bfloat16, states, 64, "constant", outs=True, seed=6) for _ in range(2))
    a.lists[63] = a.lists[0]
    buffers = []
    for l in range(63):
        flat, at, lists = torch.zeros(sum(b.sizes) + 64, device="cuda", dtype=torch.bfloat16), pad, []
        for n, g in zip(b.sizes, b.lists[l]):
            flat[at:at + n] = g
            lists.append(flat[at:at + n])
            at += n
        b.lists[l] = lists
        buffers.append(flat)
    b.lists[63] = b.lists[0]
    for t in (1, 2):
        a.step(t)
        b.step(t)
    for x, y in ((a.out_flat, b.out_flat), (a.copy_flat, b.copy_flat), (a.m.view(torch.uint8), b.m.view(torch.uint8)), (a.v.view(torch.uint8), b.v.view(torch.uint8))):
        assert torch.equal(x, y)


@pytest.mark.parametrize("kw", [dict(beta1=0.0), dict(beta2=0.0), dict(beta1=0.0, beta2=0.0, eps=1.0), dict(wd=0.0, alpha0=0.0), dict(std=1e-12), dict(std=1e8)])
@pytest.mark.parametrize("states", ["fp32", "e4m3"])
def test_extreme_rules_and_gradients(states, kw):
    r = Run([700, 256], states=states, **kw)
    r.step(1)
    r.step(2)


@pytest.mark.parametrize("states", ["fp32", "e4m3"])
def test_zero_gradients_leave_zero_moments(states):
    r = Run([700, 256], states=states)
    for x in r.lists[0]:
        x.zero_()
    r.step(1)
    assert not r.moments()[0].any() and not r.moments()[1].any()


@pytest.mark.parametrize("outs", [False, True])
@pytest.mark.parametrize("states", ["fp32", "e4m3"])
def test_factor_that_is_nan_leaves_the_step_out(states, outs):
    r = Run(SIZES, states=states, outs=outs)
    r.step(1)
    before = [x.clone() for x in (r.m.view(torch.uint8), r.v.view(torch.uint8), *r.theta)]
    for x in r.lists[0]:
        x.fill_(float("inf"))
    r.opt.apply(r.lists, 2, scale=torch.tensor([float("nan")], device="cuda"))
    after = [r.m.view(torch.uint8), r.v.view(torch.uint8), *r.theta]
    assert all(torch.equal(a, b) for a, b in zip(before, after))
    assert all(torch.equal(a, b) for a, b in zip(r.theta, r.out))
    assert all(s is None or torch.equal(s, x.bfloat16()) for s, x in zip(r.copies, r.out))


@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
@pytest.mark.parametrize("shift", [0, 1])
def test_gradient_that_is_not_finite_stays_in_its_block(bad, shift):
    r = Run([2000], states="e4m3", shift=shift, copies=False)
    r.step(1)
    r.lists[0][0][700] = bad
    r.opt.apply(r.lists, 2)
    hit = np.arange(8) == 2
    assert np.array_equal(np.isnan(f64(r.ms)), hit) and np.array_equal(np.isnan(f64(r.vs)), hit)
    assert np.array_equal(~np.isfinite(f64(r.theta[0])), np.arange(2000) == 700) or (bad == float("inf") and np.isfinite(f64(r.theta[0])).sum() >= 1999)


@pytest.mark.parametrize("states", ["fp32", "e4m3"])
def test_captured_with_its_bound_and_replayed(states):
    """norm, factor and step in a graph; the step's number lies on the device; eager work between the replays."""
    from paper_1511_05950_amd import binding
    runs = [Run([3000, 70_001, 9], torch.bfloat16, states, 1, "constant", seed=9) for _ in range(2)]
    out = [torch.zeros(2, device="cuda") for _ in runs]
    work = [torch.zeros(binding.NORM_WORKSPACE, dtype=torch.uint8, device="cuda") for _ in runs]
    count = torch.ones(1, dtype=torch.int64, device="cuda")
    r = runs[0]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        binding.gradientNorm(r.lists[0], out[0], max_norm=0.5, workspace=work[0])
        r.opt.apply(r.lists, 1, staleness=[0], scale=out[0][1:], step_dev=count)
    for t in range(1, 6):
        count.fill_(t)
        for a, b in zip(runs[0].lists[0], runs[1].lists[0]):
            a.copy_(torch.randn(a.numel(), device="cuda") * (10.0 ** -t))
            b.copy_(a)
        graph.replay()
        binding.gradientNorm(runs[1].lists[0], out[1], max_norm=0.5, workspace=work[1])
        runs[1].opt.apply(runs[1].lists, t, staleness=[0], scale=out[1][1:])
        torch.cuda.synchronize()
        assert torch.equal(out[0], out[1]) and torch.equal(runs[0].flat, runs[1].flat)
        assert torch.equal(runs[0].m.view(torch.uint8), runs[1].m.view(torch.uint8)) and torch.equal(runs[0].v.view(torch.uint8), runs[1].v.view(torch.uint8))


def test_on_another_stream():
    from paper_1511_05950_amd import binding
    r = Run([3000, 1], c=2)
    other = torch.cuda.Stream()

    def run():
        other.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(other):
            r.opt.apply(r.lists, 1, staleness=r.stale)
        torch.cuda.current_stream().wait_stream(other)
    r.step(1, run=run)
    r.step(2, run=lambda: r.opt.apply(r.lists, 2, staleness=r.stale, stream=torch.cuda.current_stream().cuda_stream))
    assert binding.gradientNorm


def test_offsets_beyond_32_bits():
    from paper_1511_05950_amd import binding
    n = (1 << 32) + 300
    theta, g = torch.zeros(n, device="cuda"), torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    m, v = (torch.zeros(binding.momentElements([theta]), dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn) for _ in range(2))
    ms, vs = torch.zeros(m.numel() // 256, device="cuda"), torch.zeros(m.numel() // 256, device="cuda")
    ends = [0, 255, 1 << 31, (1 << 32) - 1, 1 << 32, n - 1]
    for k, e in enumerate(ends):
        g[e] = 0.5 * (k + 1)
    out, work = torch.zeros(2, device="cuda"), torch.zeros(binding.NORM_WORKSPACE, dtype=torch.uint8, device="cuda")
    binding.gradientNorm([g], out, workspace=work)
    assert abs(f64(out)[0] - 0.5 * np.sqrt(91)) < 1e-6
    binding.AdamW([theta], m, v, ms, vs, alpha0=0.25, beta1=0.0, beta2=0.0, eps=1e-20).apply([[g]], 1)
    # without memory of earlier steps every weight moves by alpha0, whatever its gradient's size
    assert int((theta != 0).sum()) == len(ends) and all(abs(float(theta[e]) + 0.25) < 1e-6 for e in ends)
    assert int((m.view(torch.uint8) != 0).sum()) == len(ends) and int((v.view(torch.uint8) != 0).sum()) == len(ends)


def test_what_the_binding_refuses():
    from paper_1511_05950_amd import binding
    w, g = [torch.zeros(300, device="cuda")], torch.zeros(300, device="cuda")
    m, v = torch.zeros(512, device="cuda"), torch.zeros(512, device="cuda")
    opt = binding.AdamW(w, m, v)
    for grads, error in (([[g[:299]]], ValueError), ([[g, g]], ValueError), ([[g.cpu()]], ValueError), ([[g.double()]], TypeError), ([[torch.zeros(600, device="cuda")[::2]]], ValueError),
                         ([[g], [g.bfloat16()]], TypeError), ([], binding.SasgdError), ([[g]] * 65, binding.SasgdError)):
        with pytest.raises(error):
            opt.apply(grads, 1)
    with pytest.raises(binding.SasgdError):
        opt.apply([[g]], 0)
    with pytest.raises(binding.SasgdError):
        opt.apply([[g]], 1, staleness=[0, 1])
    with pytest.raises(TypeError):
        opt.apply([[g]], 1, scale=torch.ones(1, dtype=torch.float64, device="cuda"))
    for args, kw in (((w, m[:511], v), {}), ((w, m, v[:511]), {}), ((w, m.bfloat16(), v), {}), (([x.bfloat16() for x in w], m, v), {}),
                     ((w, m, v), dict(copies=[g])), ((w, m, v), dict(outs=[g[:5]])), ((w, m.to(torch.float8_e4m3fn), v.to(torch.float8_e4m3fn)), {})):
        with pytest.raises((TypeError, ValueError)):
            binding.AdamW(*args, **kw)
    out = torch.zeros(2, device="cuda")
    for bad in (None, torch.zeros(100, device="cuda"), torch.zeros(binding.NORM_WORKSPACE)):
        with pytest.raises(ValueError):
            binding.gradientNorm([g], out, workspace=bad)


def test_tensors_of_other_classes():
    """Parameters (a class of their own) are read like plain tensors, with the same refusals."""
    from paper_1511_05950_amd import binding
    g = torch.randn(1000, device="cuda")
    out, work = torch.zeros(2, 2, device="cuda"), torch.zeros(binding.NORM_WORKSPACE, dtype=torch.uint8, device="cuda")
    p = torch.nn.Parameter(g.clone())
    binding.gradientNorm([g, g[:300]], out[0], workspace=work)
    binding.gradientNorm([p, p.data[:300]], out[1], workspace=work)
    assert torch.equal(out[0], out[1]) and float(out[0][0]) > 1
    for bad, error in ((torch.nn.Parameter(g.double()), TypeError), (torch.nn.Parameter(g.cpu()), ValueError),
                       (torch.nn.Parameter(g.view(20, 50).t()), ValueError), (torch.nn.Parameter(g.bfloat16()), TypeError)):
        with pytest.raises(error):
            binding.gradientNorm([g, bad], out[0], workspace=work)
