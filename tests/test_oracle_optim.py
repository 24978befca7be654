"""Pins of the AdamW oracle: none of the expected values comes from the oracle itself."""
import numpy as np
import pytest
import torch

from oracle import optim


def test_matches_the_library_optimizer_in_double():
    rng = np.random.default_rng(1)
    p0 = rng.standard_normal(200)
    w = torch.nn.Parameter(torch.tensor(p0))
    opt = torch.optim.AdamW([w], lr=3e-3, betas=(0.8, 0.95), eps=1e-7, weight_decay=0.2, foreach=False)
    p, m, v = p0.copy(), np.zeros(200), np.zeros(200)
    for t in range(1, 12):
        g = rng.standard_normal(200) * 10.0 ** rng.integers(-4, 2)
        w.grad = torch.tensor(g)
        opt.step()
        p, m, v = optim.adamw(p, g, m, v, t, 3e-3, 0.8, 0.95, 1e-7, 0.2)
        # ten fp64 roundings an element and step
        assert np.max(np.abs(w.detach().numpy() - p)) <= 1e-13


def test_first_step_is_the_sign_of_the_gradient():
    g = np.array([3.0, -1e-4, 7e5, 0.0])
    p, m, v = optim.adamw(np.ones(4), g, np.zeros(4), np.zeros(4), 1, 0.01, 0.9, 0.999, 1e-30, 0.0)
    assert np.allclose(p, 1.0 - 0.01 * np.sign(g), rtol=0, atol=1e-15)
    assert np.allclose(m, 0.1 * g) and np.allclose(v, 0.001 * g * g)


def _all_e4m3():
    v = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).float().numpy()
    return np.unique(v[np.isfinite(v) & (v >= 0)]).astype(np.float64)


def test_e4m3_roundings():
    grid = _all_e4m3()
    assert grid[-1] == optim.TOP and grid[1] == optim.LEAST
    rng = np.random.default_rng(2)
    y = np.concatenate([grid, np.minimum(np.exp(rng.uniform(-8, 6.2, 4000)), 448.0), 0.5 * (grid[1:] + grid[:-1])])
    # to nearest: the library's cast (fp32 holds every y here that is a grid value or a midpoint)
    y32 = y.astype(np.float32).astype(np.float64)
    want = torch.tensor(y32, dtype=torch.float32).to(torch.float8_e4m3fn).float().numpy()
    assert np.array_equal(optim.e4m3_nearest(y32), want)
    # grid values stay, whatever the bits; others land on a neighbour, up with the right frequency over all 65536 bits
    for bits in (0, 1, 32768, 65535):
        assert np.array_equal(optim.e4m3_stochastic(grid, np.full(grid.shape, bits)), grid)
    bits = np.arange(65536)
    for x in (0.0007, 0.0019, 0.013, 0.0161, 0.77, 3.1, 101.0, 447.0, 448.0):
        z = optim.e4m3_stochastic(np.full(65536, x), bits)
        lo, hi = grid[grid <= x][-1], grid[min(np.searchsorted(grid, x), grid.size - 1)]
        assert set(np.unique(z)) <= {lo, hi}
        assert abs(z.mean() - x) <= (hi - lo) / 65536.0


def test_bf16_stochastic_is_right_on_average():
    bits = np.arange(65536)
    for x in (1.0, -1.003, 3.14159e-5, 2.0 ** -130, -77.77, 0.0):
        z = optim.bf16_stochastic(np.full(65536, x), bits)
        assert np.array_equal(torch.tensor(z).to(torch.bfloat16).double().numpy(), z)
        step = max(abs(x), 2.0 ** -126) * 2.0 ** -7
        assert abs(z.mean() - x) <= step / 65536.0


def test_generator_first_values():
    # h(0) of the documented generator, worked with Python's integers
    def h(x):
        mask = (1 << 64) - 1
        x = (x + 0x9E3779B97F4A7C15) & mask
        x = ((x ^ (x >> 30)) * 0xBF58476D1CE4E5B9) & mask
        x = ((x ^ (x >> 27)) * 0x94D049BB133111EB) & mask
        return x ^ (x >> 31)
    assert h(0) == 0xE220A8397B1DCDAF          # the generator's published first output
    key = h(h(h(77) ^ 5) ^ 2)
    low, high = optim.random_bits(77, 5, 2, 5)
    for e in range(5):
        half = h(key ^ (e // 2)) >> (32 * (e % 2)) & 0xFFFFFFFF
        assert (low[e], high[e]) == (half & 0xFFFF, half >> 16)


def test_eight_bit_store():
    rng = np.random.default_rng(3)
    x = rng.standard_normal(600) * np.exp(3 * rng.standard_normal(600))
    x[256:512] *= 1e-35                       # below 2^-100: counts as zero
    x[5] = 0.0
    q, scale = optim.store8(x, None, False)
    back = optim.load8(q, scale)
    assert np.all(back[256:512] == 0) and scale[1] == 0
    big = np.abs(x[:256]).max()
    assert abs(np.abs(back[:256]).max() - big) <= 1e-15 * big          # the largest comes back
    # half a spacing: 1/16 of a value, or of the least one
    assert np.all(np.abs(back[:256] - x[:256]) <= np.maximum(np.abs(x[:256]) / 16, big / 448 * 2.0 ** -10) * (1 + 1e-12))
    r, _ = optim.store8(np.abs(x), None, True)
    assert np.all((r[:256] > 0) == (x[:256] != 0))


@pytest.mark.parametrize("max_norm", [0.0, 1.0, 1e9])
def test_norm(max_norm):
    g = [np.array([3.0, 4.0]), np.array([12.0]), np.zeros(0)]
    norm, f = optim.grad_norm(g, max_norm)
    assert norm == 13.0
    assert f == (1.0 / (13.0 + 1e-6) if max_norm == 1.0 else 1.0)
    assert optim.grad_norm(g + [np.array([np.nan])], max_norm)[1] == 0.0
    assert optim.grad_norm(g + [np.array([np.inf])], max_norm)[1] == 0.0


def test_stochastic_moments_follow_and_nearest_ones_stand():
    """Why the rounding is an option: with gradients whose size falls by half, the held second moment follows on average with
    stochastic rounding and stands with rounding to nearest (one element of each block keeps its size and with it the scale)."""
    rng = np.random.default_rng(4)
    n, beta2 = 256 * 8, 0.99
    size = np.full(n, 1.0)
    keep = np.arange(n) % 256 == 0
    got = {}
    for mode in ("nearest", "stochastic"):
        q, scale = optim.store8(np.where(keep, 4.0, size), None, True)
        for t in range(1, 801):
            v = optim.load8(q, scale) ** 2
            g = np.where(keep, 4.0, 0.5 * size)
            v = beta2 * v + (1 - beta2) * g * g
            bits = rng.integers(0, 65536, n) if mode == "stochastic" else None
            q, scale = optim.store8(np.sqrt(v), bits, True)
        got[mode] = optim.load8(q, scale)[~keep]
    assert np.all(got["nearest"] >= 0.9)
    # the mean of v is right to the second order of the spacing: 12 % in the root is wide
    assert abs(np.sqrt(np.mean(got["stochastic"] ** 2)) - 0.5) <= 0.06
