"""Operators around a learner's network and the server's step, as cases that can be timed and compared.

  group_norm           binding.groupNorm           group normalisation and the activation behind it, channels last
  group_norm_gradient  binding.groupNormGradient   its backward pass: of the input, the scales and the shifts
  gradient_norm        binding.gradientNorm        the norm over many tensors and the factor that bounds it
  adamw                binding.AdamW.apply         one AdamW step over many tensors (with `bound`, behind gradientNorm), the moments
                                                   in 32 bits or in 8 bits with a scale per 256

A case is a dict of plain values.  With `own` false, run() computes the same in elementary torch operations.  Layer shapes and
parameter vectors are those of workloads' two networks and of networks of a user's own; learners and mini-batches as in the paper's
Section 4 (18 or 30 learners, mini-batches of 4 to 128 images).
"""
import math
import random

import torch

import workloads as wl

own = False

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
NETS = {"cifar3": wl.CIFAR3, "alex8": wl.ALEX8}
BLOCK = 256                      # values of a tensor that share the scale of an 8-bit moment
LARGEST = 448.0                  # largest e4m3 value
RULE = {"alpha0": 1e-4, "beta1": 0.9, "beta2": 0.999, "eps": 1e-8, "weight_decay": 0.01}


# ------------------------------------------------------------------------------------------------ the cases
def listed():
    return [
        # behind the first convolution of the CIFAR-shaped net, one learner with the paper's smallest mini-batch: all latency
        {"name": "norm_cifar_conv1", "op": "group_norm", "images": 4, "height": 32, "width": 32, "channels": 32, "groups": 8, "type": "fp32",
         "activation": "relu", "pixel": 32},
        # behind the first convolution of the AlexNet-shaped net, 18 learners of 16 images
        {"name": "norm_alex_conv1", "op": "group_norm", "images": 288, "height": 54, "width": 54, "channels": 96, "groups": 8, "type": "bf16",
         "activation": "relu", "pixel": 96},
        # a user's wide residual network: groups that are no whole 16 bytes, read out of a wider tensor
        {"name": "norm_wide_silu", "op": "group_norm", "images": 16, "height": 64, "width": 64, "channels": 320, "groups": 32, "type": "bf16",
         "activation": "silu", "pixel": 640},
        # a network of a user's own, no size of it a round number, three learners of 10 images
        {"name": "norm_gradient_odd", "op": "group_norm_gradient", "images": 30, "height": 23, "width": 20, "channels": 43, "groups": 1,
         "type": "fp32", "activation": "none", "pixel": 43},
        # behind the second convolution of the AlexNet-shaped net, 18 learners of 16 images
        {"name": "norm_gradient_alex_conv2", "op": "group_norm_gradient", "images": 288, "height": 27, "width": 27, "channels": 256, "groups": 32,
         "type": "bf16", "activation": "relu", "pixel": 256},
        # behind the first convolution of the CIFAR-shaped net, 18 learners of 128 images
        {"name": "norm_gradient_cifar_18x128", "op": "group_norm_gradient", "images": 2304, "height": 32, "width": 32, "channels": 32, "groups": 8,
         "type": "bf16", "activation": "silu", "pixel": 32},
        # the gradient of the CIFAR-shaped net, tensor by tensor
        {"name": "bound_cifar", "op": "gradient_norm", "net": "cifar3", "type": "fp32", "packed": True, "bound": 0.0},
        # the gradient of the AlexNet-shaped net
        {"name": "bound_alex", "op": "gradient_norm", "net": "alex8", "type": "fp32", "packed": True, "bound": 1.0},
        # 1-softsync server of the CIFAR-shaped net with 30 learners
        {"name": "adamw_cifar_c30", "op": "adamw", "net": "cifar3", "type": "fp32", "packed": True, "states": "fp32", "window": 30,
         "rate": "per_gradient", "copy": False, "bound": 0.0},
        # the AlexNet-shaped net's weights, trained in bf16 behind a bounded gradient
        {"name": "adamw_alex_bounded", "op": "adamw", "net": "alex8", "type": "fp32", "packed": True, "states": "fp32", "window": 1,
         "rate": "constant", "copy": True, "bound": 1.0},
        # the same with the moments in 8 bits, four stale gradients a step
        {"name": "adamw_alex_8bit", "op": "adamw", "net": "alex8", "type": "fp32", "packed": True, "states": "e4m3", "window": 4,
         "rate": "mean_staleness", "copy": True, "bound": 0.0},
        # a model of many tensors of all sizes, bf16 gradients
        {"name": "adamw_many_8bit", "op": "adamw", "net": "many", "tensors": 397, "params": 100_000_000, "mix": 5, "type": "bf16", "packed": False,
         "states": "e4m3", "window": 1, "rate": "constant", "copy": True, "bound": 0.0},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["group_norm", "group_norm_gradient", "gradient_norm", "adamw", "adamw"])
    if op.startswith("group"):
        groups = rng.choice([1, 2, 4, 8, 32, rng.randint(1, 40)])
        channels = groups * _log(rng, 1, max(1, 640 // groups))
        height, width = _log(rng, 1, 96), _log(rng, 1, 96)
        most = 80_000_000 if op == "group_norm" else 60_000_000
        return {"op": op, "images": max(1, min(_log(rng, 1, 2304), most // (height * width * channels))), "height": height, "width": width,
                "channels": channels, "groups": groups, "type": rng.choice(["fp32", "bf16"]), "activation": rng.choice(["none", "relu", "silu"]),
                "pixel": channels + rng.choice([0, 0, 0, rng.randint(1, 64)])}
    tensors = _log(rng, 1, 400)
    case = {"op": op, "net": "many", "tensors": tensors, "params": max(tensors, _log(rng, 1_000, 62_000_000)), "mix": rng.randint(0, 999),
            "type": rng.choice(["fp32", "bf16"]), "packed": rng.random() < 0.4, "bound": rng.choice([0.0, 1.0])}
    if op == "adamw":
        window = rng.choice([1, 1, _log(rng, 1, 30)])
        case = dict(case, states=rng.choice(["fp32", "e4m3"]), window=window, rate=rng.choice(["per_gradient", "mean_staleness", "constant"]),
                    copy=rng.random() < 0.5, params=max(tensors, min(case["params"], 200_000_000 // window)))
    return case


# ------------------------------------------------------------------------------------------------ inputs
def _sizes(case):
    """Numbers of elements of the case's tensors: weights and biases of a network, or sizes of all orders with the given sum."""
    if case["net"] != "many":
        return [n for shape, bias in wl.param_shapes(NETS[case["net"]]) for n in (math.prod(shape), bias)]
    rng = random.Random(case["mix"])
    share = [math.exp(rng.uniform(0, 8)) for _ in range(case["tensors"])]
    spare = case["params"] - case["tensors"]
    sizes = [1 + int(spare * s / sum(share)) for s in share]
    return sizes[:-1] + [sizes[-1] + case["params"] - sum(sizes)]


def _blocks(sizes):
    return [-(-n // BLOCK) for n in sizes]


def _starts(sizes, packed):
    """Where each tensor begins in one flat buffer: right behind the one before, or at the next multiple of BLOCK."""
    at, starts = 0, []
    for n in sizes:
        starts.append(at)
        at += n if packed else -(-n // BLOCK) * BLOCK
    return starts, at


def _places(sizes):
    """For every element of tensors that lie one right behind the other, its place where each begins at a multiple of BLOCK."""
    blocks = _blocks(sizes)
    gaps = torch.tensor([0] + [b * BLOCK - n for b, n in zip(blocks[:-1], sizes[:-1])], device="cuda").cumsum(0)
    return torch.arange(sum(sizes), device="cuda") + torch.repeat_interleave(gaps, torch.tensor(sizes, device="cuda"))


def _views(flat, sizes, starts):
    return [flat[at:at + n] for at, n in zip(starts, sizes)]


def _nearest8(x):
    """A padded vector as e4m3 values and the scale of each BLOCK."""
    x = x.view(-1, BLOCK)
    scale = x.abs().amax(1) / LARGEST
    return (x / scale.clamp_min(1e-30)[:, None]).to(torch.float8_e4m3fn).flatten(), scale


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    randn = lambda *shape: torch.randn(*shape, device="cuda", generator=gen)  # noqa: E731
    s = {"case": case}
    if case["op"].startswith("group"):
        n, h, w, c, g = case["images"], case["height"], case["width"], case["channels"], case["groups"]
        kind = TYPES[case["type"]]
        # layer outputs: every channel with a mean and a spread of its own
        x = randn(n, h, w, case["pixel"])
        x = (x.mul_(randn(case["pixel"]).abs_().add_(0.5)).add_(randn(case["pixel"]))).to(kind)
        s["x"] = x[..., :c]
        s["scale"], s["shift"] = 1 + 0.2 * randn(c), 0.2 * randn(c)
        if case["op"] == "group_norm":
            s["y"] = torch.empty(n, h, w, c, dtype=kind, device="cuda")
            s["stats"] = torch.empty(n, g, 2, device="cuda")
        else:
            s["dy"] = (randn(n, h, w, c) * 1e-2).to(kind)
            s["dx"] = torch.empty_like(s["dy"])
            s["dscale"], s["dshift"] = torch.empty(c, device="cuda"), torch.empty(c, device="cuda")
            v = s["x"].double().reshape(n, h * w, g, c // g)                # what the forward pass has kept
            mean = v.mean((1, 3))
            var = (v - mean[:, None, :, None]).square_().mean((1, 3))
            s["stats"] = torch.stack([mean, (var + 1e-5).rsqrt()], -1).float()
        if own:
            from paper_1511_05950_amd import binding
            s["work"] = torch.empty(binding.groupNormWorkspace(s["x"], g, gradient=case["op"] != "group_norm"), dtype=torch.uint8, device="cuda")
        return s
    sizes = _sizes(case)
    starts, length = _starts(sizes, case["packed"])
    s["place"] = _places(sizes)
    padded = sum(_blocks(sizes)) * BLOCK
    c = case.get("window", 1)

    def storage(std, kind):
        """One flat buffer for all tensors; zeros where none lies."""
        flat = randn(length).mul_(std)
        if case["packed"]:
            return flat.to(kind)
        real = torch.zeros(length, dtype=torch.bool, device="cuda")
        real[s["place"]] = True
        return flat.mul_(real).to(kind)

    s["grads"] = [storage(1e-3, TYPES[case["type"]]) for _ in range(c)]
    s["out"] = torch.zeros(2, device="cuda")
    if own:
        s["work"] = torch.empty(16384, dtype=torch.uint8, device="cuda")
        s["lists"] = [_views(flat, sizes, starts) for flat in s["grads"]]
    if case["op"] == "gradient_norm":
        return s
    rng = random.Random(seed)
    s["stale"] = [rng.randint(0, 2 * c) for _ in range(c)]
    s["step"] = 1000                                                        # a run in progress
    s["theta"] = storage(0.02, torch.float32)
    s["copy"] = s["theta"].to(torch.bfloat16) if case["copy"] else None
    m, v = torch.zeros(padded, device="cuda"), torch.zeros(padded, device="cuda")
    m[s["place"]] = randn(sum(sizes)) * 3e-4
    v[s["place"]] = (randn(sum(sizes)) * 1e-3).square_() + 1e-7
    s["m"], s["v"], s["m_scale"], s["v_scale"] = m, v, None, None
    if case["states"] == "e4m3":
        (s["m"], s["m_scale"]), (s["v"], s["v_scale"]) = _nearest8(m), _nearest8(v.sqrt_())
    if own:
        from paper_1511_05950_amd import binding
        s["opt"] = binding.AdamW(_views(s["theta"], sizes, starts), s["m"], s["v"], s["m_scale"], s["v_scale"],
                                 copies=_views(s["copy"], sizes, starts) if case["copy"] else None, lr_mode=case["rate"], seed=17, **RULE)
    return s


# ------------------------------------------------------------------------------------------------ one pass
def run(s):
    op = s["case"]["op"]
    return {"group_norm": _norm, "group_norm_gradient": _norm_gradient, "gradient_norm": _bound, "adamw": _adamw}[op](s)


def _norm(s):
    case, x, g = s["case"], s["x"], s["case"]["groups"]
    if own:
        from paper_1511_05950_amd import binding
        binding.groupNorm(x, s["scale"], s["shift"], g, s["y"], s["stats"], activation=case["activation"], workspace=s["work"])
        return [s["y"], s["stats"]]
    n, h, w, c = x.shape
    v = x.float().reshape(n, h * w, g, c // g)
    mean = v.mean((1, 3))
    d = v - mean[:, None, :, None]
    r = (d.square().mean((1, 3)) + 1e-5).rsqrt()
    z = (d * r[:, None, :, None]).reshape(x.shape) * s["scale"] + s["shift"]
    if case["activation"] == "relu":
        z = z.clamp_min(0)
    elif case["activation"] == "silu":
        z = z / (1 + torch.exp(-z))
    return [z.to(x.dtype), torch.stack([mean, r], -1)]


def _norm_gradient(s):
    case, x, g = s["case"], s["x"], s["case"]["groups"]
    if own:
        from paper_1511_05950_amd import binding
        binding.groupNormGradient(x, s["scale"], s["shift"], g, s["stats"], s["dy"], s["dx"], s["dscale"], s["dshift"],
                                  activation=case["activation"], workspace=s["work"])
        return [s["dx"], s["dscale"], s["dshift"]]
    n, h, w, c = x.shape
    mean, r = s["stats"][:, None, :, None, 0], s["stats"][:, None, :, None, 1]
    xhat = (x.float().reshape(n, h * w, g, c // g) - mean) * r
    dz = s["dy"].float()
    if case["activation"] != "none":
        z = xhat.reshape(x.shape) * s["scale"] + s["shift"]
        if case["activation"] == "relu":
            dz = dz * (z > 0)
        else:
            sig = 1 / (1 + torch.exp(-z))
            dz = dz * (sig * (1 + z * (1 - sig)))
    dshift = dz.sum((0, 1, 2))
    dscale = (dz * xhat.reshape(x.shape)).sum((0, 1, 2))
    q = (dz * s["scale"]).reshape(xhat.shape)
    dx = r * (q - q.mean((1, 3), keepdim=True) - xhat * (q * xhat).mean((1, 3), keepdim=True))
    return [dx.reshape(x.shape).to(x.dtype), dscale, dshift]


def _bound(s, grads=None):
    """The norm and the factor; in 64 bits, which long sums of squares need."""
    bound = s["case"]["bound"]
    if own:
        from paper_1511_05950_amd import binding
        binding.gradientNorm(s["lists"][0], s["out"], max_norm=bound, workspace=s["work"])
        return s["out"]
    norm = s["grads"][0].double().square().sum().sqrt()
    factor = torch.where(norm > bound, bound / norm, torch.ones_like(norm)) if bound else torch.ones_like(norm)
    return torch.stack([norm, factor]).float()


def _mix(x):
    """32 bits of an integer, scattered."""
    x = x ^ (x >> 16)
    x = (x * 0x6A09E667) & 0xFFFFFFFF
    x = x ^ (x >> 15)
    x = (x * 0xB7E15163) & 0xFFFFFFFF
    return x ^ (x >> 16)


def _chance(n, seed, step):
    """The 32 bits that decide how element 0 .. n - 1 is rounded in this step."""
    key = _mix((seed + step * 0x9E3779B1) & 0xFFFFFFFF)
    e = torch.arange(n, device="cuda")
    return _mix(((e * 0x9E3779B1) & 0xFFFFFFFF) ^ ((e >> 32) * 0x243F6A89 & 0xFFFFFFFF) ^ key)


def _round8(x, chance):
    """Values of 0 .. 448 as e4m3 values: up where the bits cut off and 16 bits of chance carry."""
    small = x < 2.0 ** -6
    x = torch.where(small, x + 2.0 ** -6, x)                    # the even steps below 2^-6 are those of the binade above it
    x = ((x.view(torch.int32) + (chance << 4).int()) & ~0xFFFFF).view(torch.float32)
    return torch.where(small, x - 2.0 ** -6, x).clamp_max(LARGEST)


def _store8(x, chance, floor):
    x = x.view(-1, BLOCK)
    most = x.abs().amax(1)
    most = torch.where(most < 1e-30, 0, most)
    up = torch.where(most > 0, LARGEST / most, 0)
    y = x.abs() * up[:, None]
    y = _round8(y, chance.view(-1, BLOCK)).clamp_min(2.0 ** -9 if floor else 0) * (y > 0)
    return (y * x.sign()).to(torch.float8_e4m3fn).flatten(), most / LARGEST


def _adamw(s):
    case = s["case"]
    s["step"] += 1
    scale = None
    if own:
        if case["bound"]:
            scale = _bound(s)[1:]
        s["opt"].apply(s["lists"], s["step"], staleness=s["stale"], scale=scale)
        return {k: s[k] for k in ("theta", "copy", "m", "v", "m_scale", "v_scale")}
    tau = torch.tensor([float(t) for t in s["stale"]])
    a = {"per_gradient": 1 / tau.clamp_min(1), "mean_staleness": torch.ones_like(tau) / tau.mean().clamp_min(1), "constant": torch.ones_like(tau)}[case["rate"]]
    rate = RULE["alpha0"] * float(a.double().mean())
    share = (a.double() / a.double().sum()).tolist()
    total = s["grads"][0].float() * share[0]
    for g, part in zip(s["grads"][1:], share[1:]):
        total += g.float() * part
    if case["bound"]:
        total = total * _bound(s)[1]
    place, bits8 = s["place"], case["states"] == "e4m3"
    if bits8:
        m = (s["m"].float().view(-1, BLOCK) * s["m_scale"][:, None]).flatten()
        v = (s["v"].float().view(-1, BLOCK) * s["v_scale"][:, None]).flatten().square()
    else:
        m, v = s["m"], s["v"]
    g = torch.zeros_like(m)
    if case["packed"]:
        g[place] = total
    else:
        g += total
    m = m * RULE["beta1"] + g * (1 - RULE["beta1"])
    v = v * RULE["beta2"] + g * g * (1 - RULE["beta2"])
    t = s["step"]
    move = m * (rate / (1 - RULE["beta1"] ** t)) / ((v * (1 / (1 - RULE["beta2"] ** t))).sqrt() + RULE["eps"])
    s["theta"] = s["theta"] * (1 - rate * RULE["weight_decay"]) - (move[place] if case["packed"] else move)
    if case["copy"]:
        s["copy"] = s["theta"].to(torch.bfloat16)
    if bits8:
        chance = _chance(m.numel(), 17, t)
        s["m"], s["m_scale"] = _store8(m, chance >> 16, False)
        s["v"], s["v_scale"] = _store8(v.sqrt(), chance & 0xFFFF, True)
    else:
        s["m"], s["v"] = m, v
    return {k: s[k] for k in ("theta", "copy", "m", "v", "m_scale", "v_scale")}


# ------------------------------------------------------------------------------------------------ work, exact values
def work(case):
    if case["op"].startswith("group"):
        values = case["images"] * case["height"] * case["width"] * case["channels"]
        size = 4 if case["type"] == "fp32" else 2
        if case["op"] == "group_norm":
            return {"bytes": values * size * 2 + case["images"] * case["groups"] * 8 + case["channels"] * 8, "flops": values * 10}
        return {"bytes": values * size * 3 + case["images"] * case["groups"] * 8 + case["channels"] * 16, "flops": values * 20}
    sizes = _sizes(case)
    P, size = sum(sizes), 4 if case["type"] == "fp32" else 2
    if case["op"] == "gradient_norm":
        return {"bytes": P * size, "flops": P * 2}
    state = P * 16 if case["states"] == "fp32" else P * 4 + sum(_blocks(sizes)) * 16
    read = case["window"] * size + (size if case["bound"] else 0)
    return {"bytes": P * (8 + read + (2 if case["copy"] else 0)) + state, "flops": P * (16 + 2 * case["window"])}


def _exact_norm(s):
    """From the definition, image by image in the order (image, group, the group's values)."""
    case, g = s["case"], s["case"]["groups"]
    n, h, w, c = s["x"].shape
    x = s["x"].double().reshape(n, h * w, g, c // g).permute(0, 2, 1, 3).reshape(n, g, -1)
    var, mean = torch.var_mean(x, 2, unbiased=False)
    deviation = torch.sqrt(var + 1e-5)
    if case["op"] == "group_norm_gradient":
        mean, deviation = s["stats"][..., 0].double(), 1 / s["stats"][..., 1].double()
    xhat = ((x - mean[..., None]) / deviation[..., None]).reshape(n, g, h * w, c // g)
    scale, shift = (s[k].double().reshape(1, g, 1, c // g) for k in ("scale", "shift"))
    z = xhat * scale + shift
    back = lambda t: t.permute(0, 2, 1, 3).reshape(n, h, w, c)  # noqa: E731
    if case["op"] == "group_norm":
        y = {"none": z, "relu": torch.where(z > 0, z, 0.0), "silu": z * torch.special.expit(z)}[case["activation"]]
        return [back(y), torch.stack([mean, 1 / deviation], -1)]
    slope = {"none": torch.ones_like(z), "relu": (z > 0).double(), "silu": torch.special.expit(z) + z * torch.special.expit(z) * torch.special.expit(-z)}
    dz = s["dy"].double().reshape(n, h * w, g, c // g).permute(0, 2, 1, 3) * slope[case["activation"]]
    q = dz * scale
    along = (q * xhat).mean((2, 3), keepdim=True)
    dx = (q - q.mean((2, 3), keepdim=True) - xhat * along) / deviation[..., None, None]
    return [back(dx), (dz * xhat).sum((0, 2)).flatten(), dz.sum((0, 2)).flatten()]


def _exact_store8(x, bits, floor):
    """A vector in 8 bits by the grid's own steps: 2^-9 up to 2^-6, an eighth of the power of two below a value beyond."""
    x = x.reshape(-1, BLOCK)
    most = x.abs().max(1, keepdim=True).values
    y = torch.where(most > 1e-30, x.abs() * (LARGEST / most.clamp_min(1e-30)), torch.zeros_like(x))
    step = torch.exp2(torch.floor(torch.log2(y.clamp_min(2.0 ** -6))) - 3)
    grid = (torch.floor(y / step + bits.reshape(-1, BLOCK).double() / 65536) * step).clamp(max=LARGEST)
    if floor:
        grid = torch.where((y > 0) & (grid == 0), torch.full_like(grid, 2.0 ** -9), grid)
    return (torch.sign(x) * grid).flatten(), most.flatten() / LARGEST


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"].startswith("group"):
        return _exact_norm(s)
    first = s["grads"][0].double()
    norm = torch.linalg.vector_norm(first)
    bound = case["bound"]
    factor = (bound / norm if bound and norm > bound else torch.ones_like(norm))
    if case["op"] == "gradient_norm":
        return torch.stack([norm, factor])
    tau = [max(t, 1) for t in s["stale"]]
    c = len(tau)
    if case["rate"] == "per_gradient":
        alpha = [1 / t for t in tau]
    else:
        alpha = [1 / max(sum(s["stale"]) / c, 1) if case["rate"] == "mean_staleness" else 1.0] * c
    rate = RULE["alpha0"] * sum(alpha) / c
    g = sum(x.double() * (a / sum(alpha)) for x, a in zip(s["grads"], alpha)) * factor
    place = s["place"] if case["packed"] else slice(None)
    full = torch.zeros(s["m"].numel(), dtype=torch.float64, device="cuda")
    full[place] = g
    m, v = s["m"].double(), s["v"].double()
    if case["states"] == "e4m3":
        m = m * s["m_scale"].double().repeat_interleave(BLOCK)
        v = (v * s["v_scale"].double().repeat_interleave(BLOCK)) ** 2
    m = m + (1 - RULE["beta1"]) * (full - m)
    v = v + (1 - RULE["beta2"]) * (full * full - v)
    t = s["step"] + 1
    corrected = m / (1 - RULE["beta1"] ** t), v / (1 - RULE["beta2"] ** t)
    old = s["theta"].double()
    theta = old - rate * (RULE["weight_decay"] * old + (corrected[0] / (torch.sqrt(corrected[1]) + RULE["eps"]))[place])
    out = {"theta": theta, "copy": theta if case["copy"] else None, "m": m, "v": v, "m_scale": None, "v_scale": None}
    if case["states"] == "e4m3":
        chance = _chance(m.numel(), 17, t)                                  # an input: whole numbers
        out["m"], out["m_scale"] = _exact_store8(m, chance >> 16, False)
        out["v"], out["v_scale"] = _exact_store8(torch.sqrt(v), chance & 0xFFFF, True)
    return out
