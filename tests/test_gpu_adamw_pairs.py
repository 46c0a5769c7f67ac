"""applyAdamW where a wavefront takes two blocks (8 192 blocks a launch and more): against the formulas, and against the same step in launches small enough for one.

Tolerances are those of test_gpu_adamw.Run."""
import pytest

from test_gpu_adamw import Run

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BLOCK = 256
# 8 515 blocks, an odd number, of tensors with odd numbers of blocks, so that pairs lie across their ends; ends within a block, empty and tiny tensors between
SIZES = [3 * BLOCK, 1, 0, 700_003, 257, 5 * BLOCK - 1, 255, 0, 901_120, 4, 573_440 + 77, BLOCK, 1100]
assert sum(-(-n // BLOCK) for n in SIZES) == 8515


@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("states", ["fp32", "e4m3"])
@pytest.mark.parametrize("c, mode", [(1, "constant"), (3, "per_gradient")])
@pytest.mark.parametrize("shift, outs, factor", [(0, False, None), (0, True, 0.3), (1, False, 0.3)])
def test_steps(kind, states, c, mode, shift, outs, factor):
    r = Run(SIZES, kind, states, c, mode, shift, outs=outs, seed=c + shift)
    r.step(1, factor=factor)
    r.step(2, factor=factor)


@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("states", ["fp32", "e4m3"])
@pytest.mark.parametrize("apart", [0, 1])
def test_flat_vectors(states, apart, kind):
    """Three gradients cut alike out of flat vectors, against the formulas; the same bits as gradients that lie anywhere.  (fp32 vectors start a multiple of 16 bytes apart.)"""
    a, b = (Run(SIZES, kind, states, 3, seed=3) for _ in range(2))
    for l in range(3):
        flat, at, lists = torch.zeros(sum(-(-n // 64) * 64 for n in SIZES) + 64 + apart, device="cuda", dtype=kind), 8 * l * apart, []
        for n, g in zip(b.sizes, b.lists[l]):
            flat[at:at + n] = g
            lists.append(flat[at:at + n])
            at += -(-n // 64) * 64
        b.lists[l] = lists
    for t in (1, 2):
        a.step(t)
        b.step(t)
    assert torch.equal(a.flat, b.flat) and torch.equal(a.m.view(torch.uint8), b.m.view(torch.uint8)) and torch.equal(a.v.view(torch.uint8), b.v.view(torch.uint8))


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
    assert all(torch.equal(x, y) for x, y in zip(before, after))
    assert all(torch.equal(x, y) for x, y in zip(r.theta, r.out))
    assert all(s is None or torch.equal(s, x.bfloat16()) for s, x in zip(r.copies, r.out))


@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("states", ["fp32", "e4m3"])
@pytest.mark.parametrize("c", [1, 3])
def test_the_same_bits_in_small_launches(c, states, kind):
    """Tensor by tensor, fewer than 8 192 blocks each, every one at its place in the moments (by which e4m3 values are rounded): one block a wavefront."""
    from paper_1511_05950_amd import binding
    a, b = (Run(SIZES, kind, states, c, outs=True, seed=8) for _ in range(2))
    alpha0, beta1, beta2, eps, wd = b.hyper
    for t in (1, 2):
        a.opt.apply(a.lists, t, staleness=a.stale)
        for k, n in enumerate(SIZES):
            first = sum(-(-s // BLOCK) for s in SIZES[:k]) * BLOCK
            last = first + -(-n // BLOCK) * BLOCK
            if states == "fp32":
                opt = binding.AdamW([b.theta[k]], b.m[first:last], b.v[first:last], copies=[b.copies[k]], outs=[b.out[k]], alpha0=alpha0, beta1=beta1, beta2=beta2, eps=eps,
                                    weight_decay=wd, lr_mode=b.mode, seed=b.seed)
                if n:
                    opt.apply([[one[k]] for one in b.lists], t, staleness=b.stale)
                continue
            if not n:
                continue
            # tensors of zeros in front of it, so that it lies at its place: a large one and 100 of one element, which fill a launch (of at most 100 tensors)
            blocks = first // BLOCK
            ones = min(blocks, 100)
            sizes = [(blocks - ones) * BLOCK] * (blocks > ones) + [1] * ones
            front = [torch.zeros(s, device="cuda") for s in sizes]
            lists = [[torch.zeros(s, device="cuda", dtype=kind) for s in sizes] + [one[k]] for one in b.lists]
            m, v = b.m.view(torch.uint8)[:last].clone().view(torch.float8_e4m3fn), b.v.view(torch.uint8)[:last].clone().view(torch.float8_e4m3fn)
            ms, vs = b.ms[:last // BLOCK].clone(), b.vs[:last // BLOCK].clone()
            opt = binding.AdamW(front + [b.theta[k]], m, v, ms, vs, copies=[None] * len(front) + [b.copies[k]], outs=front + [b.out[k]], alpha0=alpha0, beta1=beta1, beta2=beta2,
                                eps=eps, weight_decay=wd, lr_mode=b.mode, seed=b.seed)
            opt.apply(lists, t, staleness=b.stale)
            b.m.view(torch.uint8)[first:last] = m.view(torch.uint8)[first:last]
            b.v.view(torch.uint8)[first:last] = v.view(torch.uint8)[first:last]
            b.ms[first // BLOCK:last // BLOCK] = ms[first // BLOCK:]
            b.vs[first // BLOCK:last // BLOCK] = vs[first // BLOCK:]
        for x, y in ((a.out_flat, b.out_flat), (a.copy_flat, b.copy_flat), (a.m.view(torch.uint8), b.m.view(torch.uint8)), (a.v.view(torch.uint8), b.v.view(torch.uint8))):
            assert torch.equal(x, y), t
        if states == "e4m3":
            assert torch.equal(a.ms, b.ms) and torch.equal(a.vs, b.vs)
