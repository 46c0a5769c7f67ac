"""The reference of the AdamW tests: against torch's own optimizer in 64 bits, and the roundings it describes."""
import numpy as np
import pytest

import adamw_reference as ref
from oracle import protocol

torch = pytest.importorskip("torch")


def test_plain_steps_are_torchs_adamw():
    rng = np.random.default_rng(1)
    theta = rng.standard_normal(57)
    p = torch.nn.Parameter(torch.from_numpy(theta.copy()))
    opt = torch.optim.AdamW([p], lr=3e-3, betas=(0.8, 0.95), eps=1e-6, weight_decay=0.1)
    m, v = np.zeros(57), np.zeros(57)
    for t in range(1, 9):
        g = rng.standard_normal(57)
        p.grad = torch.from_numpy(g.copy())
        opt.step()
        theta, m, v = ref.step(theta, [g], m, v, t, [0], "per_gradient", 3e-3, 0.8, 0.95, 1e-6, 0.1)
    assert np.abs(theta - p.detach().numpy()).max() < 1e-14


@pytest.mark.parametrize("mode", ["per_gradient", "mean_staleness", "constant"])
def test_window_is_the_servers(mode):
    """rate times the mean gradient is what the server's momentum step subtracts without momentum and weight decay."""
    rng = np.random.default_rng(2)
    stale, grads, theta = [0, 1, 5, 2], rng.standard_normal((4, 33)), rng.standard_normal(33)
    mean, share = ref.alphas(mode, stale)
    want, _ = protocol.server_update(theta, np.zeros(33), list(grads), stale, 0.1, 0.0, 0.0, mode=mode)
    assert np.abs(theta - 0.1 * mean * (share @ grads) - want).max() < 1e-15


def test_bytes_and_grid():
    vals = ref.e4m3(np.arange(127))
    assert vals[0] == 0 and vals[1] == 2.0 ** -9 and vals[126] == 448 and np.all(np.diff(vals) > 0)
    as_torch = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(vals, as_torch)
    low, gap = ref.grid_below(vals[:-1] * (1 + 1e-12) + 1e-14)
    assert np.array_equal(low, vals[:-1]) and np.allclose(gap, np.diff(vals))


def test_chance_is_even_and_independent_of_the_step():
    n = 1 << 16
    a, b = ref.chance(0, n, 17, 1), ref.chance(0, n, 17, 2)
    for bits in (a >> np.uint64(16), a & np.uint64(0xFFFF), b & np.uint64(0xFFFF)):
        u = bits.astype(np.float64) / 65536
        # mean of n uniform values: sigma = 1 / sqrt(12 n) = 0.0011; five of them.  Shares of 16 ranges: sqrt(p q / n) = 0.00095.
        assert abs(u.mean() - 0.5) < 0.0057
        assert np.abs(np.histogram(u, 16, (0, 1))[0] / n - 1 / 16).max() < 0.0048
    for x, y in ((a >> np.uint64(16), a & np.uint64(0xFFFF)), (a >> np.uint64(16), b >> np.uint64(16)), (a[1:] & np.uint64(0xFFFF), a[:-1] & np.uint64(0xFFFF))):
        c = np.corrcoef(x.astype(np.float64), y.astype(np.float64))[0, 1]
        assert abs(c) < 5 / np.sqrt(n)


def test_storing_keeps_the_expectation():
    """A moment that moves by a thousandth a step follows its target in 8 bits; rounded to the nearest it would stand still."""
    n, target, u = 1 << 14, 4.0, np.ones(1 << 14)
    u[0::256] = 8.0                                    # the largest of each block
    for t in range(1, 401):
        v = u * u * 0.99 + 0.01 * np.where(np.arange(n) % 256 == 0, 64.0, target)
        q, scale, _ = ref.stored(np.sqrt(v), ref.chance(0, n, 3, t) & np.uint64(0xFFFF), True)
        u = (q * scale[:, None]).flatten()
    got = (u[np.arange(n) % 256 != 0] ** 2).mean()
    # v -> 0.99 (v + r) + 0.04, r the variance of a rounded u, at most a quarter of its squared gap (y = 112, gap 8 of 112: 0.143 at u = 2):
    # below 4 + 99 * 0.0051 = 4.51; above 4 less the start's share, 3 * 0.99^400 = 0.054, and five errors of a mean of 16 320 values
    # that spread by about 1.2
    assert 3.9 < got < 4.56
