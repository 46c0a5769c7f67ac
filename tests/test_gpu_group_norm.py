"""groupNorm and groupNormGradient against their formulas in 64 bits.

Tolerances: u = 2^-24 is half an fp32 step, ub = 2^-8 half a bf16 one relative to the value.  A sum of n values in the kernels' fixed order (a
lane's own, then rows, then channels) is off by less than (n / 64 + 64) u of the sum of magnitudes; mean, r, xhat and z follow with the bound
below, computed from the case's own magnitudes.  expf is good to 2 ulp at an argument good to |z| u."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

u = 2.0 ** -24


def f64(t):
    return t.detach().double().cpu().numpy()


def act(z, kind):
    if kind == "relu":
        return np.where(z > 0, z, 0.0)
    if kind == "silu":
        with np.errstate(over="ignore"):
            return z / (1 + np.exp(-z))
    return z


def slope(z, kind):
    if kind == "relu":
        return (z > 0).astype(float)
    if kind == "silu":
        with np.errstate(over="ignore"):
            s = 1 / (1 + np.exp(-z))
        return s * (1 + z * (1 - s))
    return np.ones_like(z)


class Case:
    def __init__(self, n, h, w, c, g, kind, activation, xpad=0, ypad=0, shift=0, params="fp32", seed=0, mean=1.0):
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)
        randn = lambda *s: torch.randn(*s, device="cuda", generator=gen)  # noqa: E731
        self.dims, self.kind, self.activation = (n, h, w, c, g), kind, activation

        def tensor(values, pad):
            """Channels of a wider tensor, `shift` elements behind an aligned start; returns it and all of its memory."""
            flat = torch.full((n * h * w * (c + pad) + shift + 64,), 3.0, device="cuda").to(kind)
            view = flat[shift:shift + n * h * w * (c + pad)].view(n, h, w, c + pad)[..., :c]
            if values is not None:
                view.copy_(values)
            return view, flat
        self.x, _ = tensor((randn(n, h, w, c) * (0.5 + randn(c).abs()) + mean * randn(c)), xpad)
        self.y, self.y_flat = tensor(None, ypad)
        self.dy, _ = tensor(randn(n, h, w, c) * 0.1, ypad)
        self.dx, self.dx_flat = tensor(None, ypad)
        ptype = torch.float32 if params == "fp32" else torch.bfloat16
        self.scale, self.shift = ((1 + 0.3 * randn(c)).to(ptype), (0.3 * randn(c)).to(ptype)) if params else (None, None)
        self.stats = torch.zeros(n, g, 2, device="cuda")
        self.dscale, self.dshift = torch.full((c,), 7.0, device="cuda"), torch.full((c,), 7.0, device="cuda")

    def work(self, gradient):
        from paper_1511_05950_amd import binding
        size = binding.groupNormWorkspace(self.x, self.dims[4], gradient)
        return torch.full((size,), 0xFF, dtype=torch.uint8, device="cuda") if size else None

    def run(self, y=None, dx=None):
        from paper_1511_05950_amd import binding
        g = self.dims[4]
        binding.groupNorm(self.x, self.scale, self.shift, g, self.y if y is None else y, self.stats, activation=self.activation, workspace=self.work(False))
        binding.groupNormGradient(self.x, self.scale, self.shift, g, self.stats, self.dy, self.dx if dx is None else dx, self.dscale, self.dshift,
                                  activation=self.activation, workspace=self.work(True))

    def check(self):
        n, h, w, c, g = self.dims
        m = h * w * c // g
        x = f64(self.x).reshape(n, h * w, g, c // g)
        e = lambda t: t[:, None, :, None]  # noqa: E731
        # ---- statistics
        mean = x.mean((1, 3))
        var = ((x - e(mean)) ** 2).mean((1, 3))
        r = 1 / np.sqrt(var + 1e-5)
        k = (m / 64 + 64) * u
        tmean = k * np.abs(x).mean((1, 3)) + 2 * u * np.abs(mean)
        tvar = (2 * k + 8 * u) * var + tmean ** 2 + 4 * u * np.abs(x).max((1, 3)) * np.sqrt(var)
        tr = 0.5 * tvar / (var + 1e-5) + 4 * u                          # relative
        st = f64(self.stats)
        assert np.all(np.abs(st[..., 0] - mean) <= tmean) and np.all(np.abs(st[..., 1] - r) <= tr * r)
        # ---- forward, from the kernel's statistics' tolerances
        sc, sh = (np.ones(c), np.zeros(c)) if self.scale is None else (f64(self.scale), f64(self.shift))
        sc, sh = sc.reshape(g, c // g), sh.reshape(g, c // g)
        hat = (x - e(mean)) * e(r)
        that = e(r) * (e(tmean) + u * np.abs(x - e(mean))) + np.abs(hat) * (e(tr) + 2 * u)
        z = hat * sc + sh
        tz = that * np.abs(sc) + 2 * u * (np.abs(hat * sc) + np.abs(sh))
        want = act(z, self.activation)
        half = 2.0 ** -8 if self.kind == torch.bfloat16 else u
        ty = 1.1 * tz + np.abs(want) * (np.abs(z) + 8) * u * (self.activation == "silu")
        ty = ty + half * (np.abs(want) + ty)
        y = f64(self.y).reshape(x.shape)
        assert np.all(np.abs(y - want) <= ty + 1e-37), np.max(np.abs(y - want) - ty)
        # ---- backward: the formula with the statistics that the kernel was given
        mean, r = st[..., 0], st[..., 1]
        hat = (x - e(mean)) * e(r)
        z = hat * sc + sh
        tz = 6 * u * (np.abs(hat * sc) + np.abs(sh)) + u * e(r) * np.abs(x) * np.abs(sc)
        d = f64(self.dy).reshape(x.shape)
        dz = d * slope(z, self.activation)
        # the slope: silu's moves by at most 0.5 per unit of z, relu's jumps: where |z| is within its error dz may be 0 or dy
        tdz = 2 * u * np.abs(dz) + np.abs(d) * (0.6 * tz + (np.abs(z) + 12) * 1.2 * u) * (self.activation == "silu")
        if self.activation == "relu":
            tdz = tdz + np.abs(d) * (np.abs(z) <= tz)
        th = 4 * u * np.abs(hat) + u * e(r) * np.abs(x)
        total = n * h * w
        ks = (total / 64 + 128) * u
        for got, want, terms, tterms in ((self.dshift, dz, np.abs(dz), tdz), (self.dscale, dz * hat, np.abs(dz * hat), tdz * np.abs(hat) + np.abs(dz) * th + u * np.abs(dz * hat))):
            tol = ks * terms.sum((0, 1)) + tterms.sum((0, 1))
            assert np.all(np.abs(f64(got).reshape(g, c // g) - want.sum((0, 1))) <= tol + 1e-37)
        q = dz * sc
        s1, s2 = q.mean((1, 3)), (q * hat).mean((1, 3))
        want = e(r) * (q - e(s1) - hat * e(s2))
        tq = tdz * np.abs(sc) + u * np.abs(q)
        ts1 = tq.mean((1, 3)) + k * np.abs(q).mean((1, 3)) + 2 * u * np.abs(s1)
        ts2 = (tq * np.abs(hat) + np.abs(q) * th).mean((1, 3)) + k * np.abs(q * hat).mean((1, 3)) + 2 * u * np.abs(s2)
        tol = e(r) * (tq + e(ts1) + np.abs(hat) * e(ts2) + th * np.abs(e(s2)) + 4 * u * (np.abs(q) + np.abs(e(s1)) + np.abs(hat * e(s2)))) + 2 * u * np.abs(want)
        tol = tol + half * (np.abs(want) + tol)
        dx = f64(self.dx).reshape(x.shape)
        assert np.all(np.abs(dx - want) <= tol + 1e-37), np.max(np.abs(dx - want) - tol)

    def outside(self):
        """The memory around y and dx is as it was."""
        for view, flat in ((self.y, self.y_flat), (self.dx, self.dx_flat)):
            keep = view.clone()
            view.fill_(3.0)
            assert bool((flat == 3.0).all())
            view.copy_(keep)


SHAPES = [  # n, h, w, c, g
    (1, 1, 1, 8, 2), (3, 1, 1, 4096, 1), (2, 1, 1, 7, 7), (5, 1, 3, 24, 8), (4, 32, 32, 32, 8), (3, 9, 7, 43, 1), (2, 5, 5, 30, 10), (300, 6, 5, 16, 4),
    (2, 54, 54, 96, 8), (2, 40, 44, 320, 32), (1, 128, 100, 64, 1), (2, 27, 27, 256, 32), (2, 3, 300, 48, 16), (1, 33, 31, 1000, 5), (2, 61, 59, 43, 1),
    (1, 24, 24, 2048, 2),
]


@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("dims", SHAPES)
@pytest.mark.parametrize("activation", ["none", "relu", "silu"])
def test_shapes(dims, kind, activation):
    c = Case(*dims, kind, activation, seed=sum(dims))
    c.run()
    c.check()
    c.outside()


@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("xpad, ypad, shift", [(8, 0, 0), (0, 16, 0), (3, 5, 0), (0, 0, 1), (8, 8, 3)])
@pytest.mark.parametrize("dims", [(3, 10, 12, 32, 4), (2, 61, 50, 48, 3)])
def test_strides_and_alignment(dims, kind, xpad, ypad, shift):
    c = Case(*dims, kind, "silu", xpad, ypad, shift, seed=xpad + ypad + shift)
    c.run()
    c.check()
    c.outside()


@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("dims", [
    (40, 20, 20, 320, 32), (70, 7, 7, 480, 32), (1100, 7, 7, 64, 4),          # workgroups that share lines; larger slabs of many small images
    (2, 48, 50, 256, 256), (1, 48, 50, 4096, 4096), (1, 10, 260, 4096, 1),    # as many groups as channels, and one of all, in chunks
    (2, 70, 71, 24, 8), (1, 300, 200, 8, 8), (3, 90, 91, 1, 1), (2, 2, 5000, 6, 2),
    (17, 64, 65, 128, 8), (530, 1, 2, 40, 5)])
def test_how_calls_are_cut(dims, kind):
    c = Case(*dims, kind, "silu" if dims[0] % 2 else "relu", seed=sum(dims) + 1)
    c.run()
    c.check()
    c.outside()


@pytest.mark.parametrize("dims", [(5, 10, 12, 32, 4), (2, 61, 50, 48, 3), (3, 9, 7, 43, 1)])
def test_positions_first(dims):
    """Images side by side in every position: as with dense images."""
    from paper_1511_05950_amd import binding
    a, b = (Case(*dims, torch.bfloat16, "silu", seed=9) for _ in range(2))
    for name in ("x", "y", "dy", "dx"):
        t = getattr(b, name)
        to = t.new_empty(t.shape[1], t.shape[2], t.shape[0], t.shape[3]).permute(2, 0, 1, 3)
        to.copy_(t)
        setattr(b, name, to)
    a.run()
    b.run()
    for name in ("y", "stats", "dx", "dscale", "dshift"):
        assert torch.equal(getattr(a, name), getattr(b, name)), name
    with pytest.raises(binding.SasgdError):           # images of y that overlap
        binding.groupNorm(a.x, None, None, dims[4], a.y.as_strided(a.y.shape, (1,) + a.y.stride()[1:]), workspace=a.work(False))


def test_offsets_beyond_32_bits():
    """Images 2^32 + 64 elements apart."""
    a, b = (Case(2, 30, 31, 32, 4, torch.bfloat16, "relu", seed=5) for _ in range(2))
    for name in ("x", "y", "dy", "dx"):
        t = getattr(b, name)
        apart = (1 << 32) + 64
        to = t.new_empty(apart + t[0].numel()).as_strided(t.shape, (apart,) + t.stride()[1:])
        to.copy_(t)
        setattr(b, name, to)
    a.run()
    b.run()
    for name in ("y", "stats", "dx", "dscale", "dshift"):
        assert torch.equal(getattr(a, name), getattr(b, name)), name


@pytest.mark.parametrize("params", [None, "fp32", "bf16"])
def test_types_of_parameters(params):
    c = Case(3, 11, 8, 40, 5, torch.bfloat16, "none", params=params)
    c.run()
    c.check()


@pytest.mark.parametrize("dims", [(3, 10, 12, 32, 4), (2, 61, 50, 48, 3)])
def test_in_place(dims):
    a, b = (Case(*dims, torch.bfloat16, "relu", seed=4) for _ in range(2))
    a.run()
    b.run(y=b.x.clone(), dx=b.dy)                     # the gradient into dy
    assert torch.equal(a.dx, b.dy) and torch.equal(a.dscale, b.dscale)
    x = b.x
    b.y = x
    from paper_1511_05950_amd import binding
    binding.groupNorm(x, b.scale, b.shift, dims[4], x, activation="relu", workspace=b.work(False))
    assert torch.equal(a.y, x)


@pytest.mark.parametrize("dims", [(3, 10, 12, 32, 4), (2, 61, 50, 48, 3)])
def test_large_means(dims):
    """Channels far from zero and from each other: the variance is no difference of large numbers."""
    c = Case(*dims, torch.float32, "none", mean=1000.0, seed=2)
    c.run()
    c.check()


def test_constant_channels():
    """No spread at all: r is 1 / sqrt(eps), y the shift."""
    c = Case(2, 8, 8, 16, 4, torch.float32, "none")
    c.x.fill_(3.25)
    c.run()
    assert np.allclose(f64(c.stats)[..., 1], 1e5 ** 0.5, rtol=1e-6) and np.array_equal(f64(c.y), np.broadcast_to(f64(c.shift), c.y.shape))


@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
def test_what_is_not_finite_stays_in_its_group(bad):
    c = Case(2, 8, 8, 16, 4, torch.float32, "relu")
    c.x[1, 3, 3, 5] = bad
    c.run()
    hit = np.zeros((2, 8, 8, 16), bool)
    hit[1, :, :, 4:8] = True
    assert np.array_equal(np.isnan(f64(c.y)), hit) and np.all(np.isfinite(f64(c.dx)[~hit]))


@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16])
def test_what_is_not_finite_stays_in_its_group_in_chunks(bad, kind):
    c = Case(2, 61, 50, 48, 3, kind, "silu")
    c.x[1, 33, 3, 20] = bad
    c.run()
    hit = np.zeros((2, 61, 50, 48), bool)
    hit[1, :, :, 16:32] = True
    assert np.array_equal(np.isnan(f64(c.y)), hit) and np.all(np.isfinite(f64(c.dx)[~hit])) and np.all(np.isnan(f64(c.dx)[hit]))
    st = f64(c.stats)
    assert np.all(np.isnan(st[1, 1, 1])) and np.all(np.isfinite(np.delete(st.reshape(6, 2), 4, 0)))


@pytest.mark.parametrize("which", ["dx", "dscale", "dshift"])
@pytest.mark.parametrize("dims", [(3, 10, 12, 32, 4), (2, 61, 50, 48, 3)])
def test_each_gradient_alone(dims, which):
    from paper_1511_05950_amd import binding
    c = Case(*dims, torch.float32, "silu", seed=3)
    c.run()
    want = {k: getattr(c, k).clone() for k in ("dx", "dscale", "dshift")}
    for k in want:
        getattr(c, k).fill_(3.0)
    binding.groupNormGradient(c.x, c.scale, c.shift, dims[4], c.stats, c.dy, activation="silu", workspace=c.work(True), **{which: getattr(c, which)})
    for k in want:
        assert torch.equal(getattr(c, k), want[k]) if k == which else bool((getattr(c, k) == 3.0).all())


@pytest.mark.parametrize("dims", [(2, 4, 3, 8, 2), (2, 41, 40, 24, 3)])
@pytest.mark.parametrize("activation", ["none", "silu"])
def test_gradient_against_differences(dims, activation):
    """Central differences of L = sum dy y in the direction of one random change of x, scale and shift at a time (64-bit sums of fp32 outputs)."""
    from paper_1511_05950_amd import binding
    c = Case(*dims, torch.float32, activation, seed=6)
    c.run()
    y = torch.empty_like(c.y)

    def L():
        binding.groupNorm(c.x, c.scale, c.shift, dims[4], y, activation=activation, workspace=c.work(False))
        return float((y.double() * c.dy.double()).sum())
    for t, grad in ((c.x, c.dx), (c.scale, c.dscale), (c.shift, c.dshift)):
        step = torch.randn_like(t).abs() * 1e-2 * grad.sign()              # uphill: every term adds to the slope
        t.add_(step)
        up = L()
        t.sub_(2 * step)
        down = L()
        t.add_(step)
        want = float((grad.double() * step.double()).sum())
        # the third-order term is some 1e-4 of the slope (steps of 1e-2 of values of 1); outputs are rounded by some u of random signs
        noise = 32 * u * float((y.double() * c.dy.double()).square().sum().sqrt())
        assert abs((up - down) / 2 - want) <= 5e-3 * want + noise


def test_no_images():
    from paper_1511_05950_amd import binding
    x = torch.zeros(0, 4, 4, 8, device="cuda")
    ds, db = torch.ones(8, device="cuda"), torch.ones(8, device="cuda")
    binding.groupNorm(x, None, None, 2, x.clone(), torch.zeros(0, 2, 2, device="cuda"))
    binding.groupNormGradient(x, None, None, 2, torch.zeros(0, 2, 2, device="cuda"), x, x.clone(), ds, db)
    assert not ds.any() and not db.any()


@pytest.mark.parametrize("dims", [(4, 32, 32, 32, 8), (2, 61, 50, 48, 3)])
def test_captured_and_replayed_on_another_stream(dims):
    from paper_1511_05950_amd import binding
    a, b = (Case(*dims, torch.bfloat16, "silu", seed=8) for _ in range(2))
    w1, w2 = a.work(False), a.work(True)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            binding.groupNorm(a.x, a.scale, a.shift, dims[4], a.y, a.stats, activation="silu", workspace=w1)
            binding.groupNormGradient(a.x, a.scale, a.shift, dims[4], a.stats, a.dy, a.dx, a.dscale, a.dshift, activation="silu", workspace=w2)
    for k in range(4):
        for t, s in ((a.x, b.x), (a.dy, b.dy)):
            t.copy_(torch.randn(t.shape, device="cuda") + k)
            s.copy_(t)
        graph.replay()
        b.run()
        torch.cuda.synchronize()
        for name in ("y", "stats", "dx", "dscale", "dshift"):
            assert torch.equal(getattr(a, name), getattr(b, name)), (k, name)


def test_what_the_binding_refuses():
    from paper_1511_05950_amd import binding
    x, y, w = torch.zeros(2, 4, 4, 8, device="cuda"), torch.zeros(2, 4, 4, 8, device="cuda"), torch.ones(8, device="cuda")
    st = torch.zeros(2, 2, 2, device="cuda")
    for args, error in (((x, w, w, 2, y.bfloat16(), st), ValueError), ((x, w, w, 2, y[:1], st), ValueError), ((x, w[:7], w, 2, y, st), ValueError),
                        ((x, w, w.bfloat16(), 2, y, st), TypeError), ((x, w, w, 2, y, st[:1]), ValueError), ((x.double(), w, w, 2, y.double(), st), TypeError),
                        ((x.permute(0, 3, 1, 2), w[:4], w[:4], 2, y.permute(0, 3, 1, 2), None), ValueError), ((x.cpu(), w, w, 2, y, st), ValueError),
                        ((x[:, :, ::2], w, w, 2, y[:, :, ::2].contiguous(), st), None), ((x[:, :, :3], w, w, 2, y[:, :, :3].contiguous(), st), ValueError),
                        ((x, w, w, 3, y, None), binding.SasgdError)):
        if error is None:
            binding.groupNorm(*args)
        else:
            with pytest.raises(error):
                binding.groupNorm(*args)
    with pytest.raises(ValueError):
        binding.groupNormGradient(x, w, w, 2, st, y, x.new_zeros(2, 4, 4, 16)[..., :8], workspace=torch.zeros(4096, device="cuda"))
    with pytest.raises(binding.SasgdError):
        binding.groupNormGradient(x, w, w, 2, st, y, x)             # no workspace
    # expanded tensors: values in one place
    for bad in (x[:1].expand(2, 4, 4, 8), x[:, :1, :1].expand(2, 4, 4, 8)):
        with pytest.raises(ValueError):
            binding.groupNorm(bad, w, w, 2, y, st)
        with pytest.raises(ValueError):
            binding.groupNormGradient(x, w, w, 2, st, bad, y, workspace=torch.zeros(4096, device="cuda"))
    with pytest.raises(ValueError):
        binding.groupNorm(x, w[:1].expand(8), w, 2, y, st)
