"""The group norm's statistics where a group's values are equal, or close beside their size, in every form that
the kernels have: what is asked of the mean is its one rounding to fp32, of everything else digits of the
spread.

Values x of a group with mean mu, |x - mu| <= D, D small beside |mu|: x - k is exact for any two of them (Sterbenz),
so the roundings (half a step each, U = 2^-24 relative) are those of sums of differences.
  mean: (a chain of at most C = 128 roundings of terms <= 2 D), and rounded once: 2 C U D + U |mu|
  rstd: relative, half the variance's.  A thread's squares about its first value are (1 + 26) times its share of
        N var at most (no value is further than 5.1 standard deviations from the mean): 27 C U var; its mean about that
        value has an error of 2 C U D, which enters as 2 |o| times that, o the thread's distance from the mean, whose
        mean square is at most var: 4 C U D var^1/2; two roundings for the root and the result.
  y:    from mean and rstd as written: x - mean is exact, two products and a sum, four roundings at most.
"""
import numpy as np
import pytest
import torch

from norm_ref import C, U, within
from test_gpu_group_norm import run_fwd

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def G():
    assert torch.cuda.is_available(), "GPU tests need a HIP device"
    import paper_2512_01678_amd.gcn as G
    return G


FORMS = [
    # n, c, groups, graphs (0: no offsets), pitch over c, offset, rows of the longest graph (0: not told)
    (2708, 16, 4, 0, 0, 0, 0),           # a workgroup a group
    (173, 47, 47, 0, 0, 1, 0),           # the same, 4-byte rows
    (700, 24, 3, 3, 0, 0, 300),          # the same, of three graphs
    (3000, 128, 8, 300, 0, 0, 64),       # a wavefront a graph: groups of several lanes
    (2000, 64, 64, 400, 4, 0, 100),      # four groups a lane
    (2500, 30, 15, 300, 2, 0, 120),      # two groups a lane
    (2500, 48, 4, 300, 0, 0, 300),       # a workgroup a graph
    (1500, 31, 1, 260, 1, 1, 60),        # the same, 4-byte rows
    (9000, 128, 8, 300, 0, 0, 700),      # the same, more rows than its registers hold
    (4000, 64, 4, 0, 0, 0, 0),           # two passes, the second joins the pieces
    (300007, 32, 4, 0, 0, 0, 0),         # two passes, a workgroup joins a group's pieces
    (20000, 64, 8, 30, 0, 0, 0),         # two passes, 16 lanes join them
    (5000, 700, 1, 3, 0, 0, 0),          # groups of several panels
    (2001, 130, 2, 2, 0, 1, 0),          # the same, 4-byte rows
]
ids = dict(ids=lambda f: "x".join(map(str, f)))


def offsets(form, rng):
    n, _, _, k, _, _, longest = form
    if not k:
        return [0, n]
    size = rng.exponential(1.0, k)
    size[rng.random(k) < 0.1] = 0.0
    size[k // 2] = 0.0
    at = np.round(np.cumsum(size) / size.sum() * (n - longest)).astype(np.int64)
    at[k // 2:] += longest
    return [0, *at.tolist()]


def run(G, form, x, gamma, beta, ptr, eps):
    n, c, groups, k, extra, off, longest = form
    hint = max(b - a for a, b in zip(ptr, ptr[1:])) if longest else -1
    Y, _, mean, rstd = run_fwd(G, (n, c, groups, k, 0, 0, extra, off), x, gamma, beta, ptr, 0, eps=eps, max_seg=hint)
    return Y.cpu().numpy(), mean.cpu().numpy(), rstd.cpu().numpy()


@pytest.mark.parametrize("form", FORMS, **ids)
def test_constant_groups(G, form):
    """The mean is the value, the deviations are 0, y is beta: to the last bit, whatever the value and the count."""
    n, c, groups, k = form[:4]
    rng = np.random.default_rng(1)
    ptr = offsets(form, rng)
    beta, gamma = rng.standard_normal(c).astype(np.float32), rng.standard_normal(c).astype(np.float32)
    some = np.diff(ptr) > 0
    for seed, values in enumerate(([0.1, 100.7, -1000.3, 12345.67], [98765.4, -0.3, 1e-3, 3.3e7])):
        v = np.random.default_rng(seed).choice(values, (len(ptr) - 1, groups)).astype(np.float32)
        x = np.repeat(np.repeat(v, np.diff(ptr), axis=0), c // groups, axis=1)
        y, mean, rstd = run(G, form, x, gamma, beta, ptr, 1e-5)
        assert (mean[some] == v[some]).all(), np.abs(mean / v - 1)[some].max()
        assert np.abs(rstd[some] * np.sqrt(1e-5) - 1).max() <= 2 * U
        assert (y == beta).all(), np.abs(y - beta).max()


@pytest.mark.parametrize("size,sigma", [(1000.3, 1e-3), (-12345.67, 0.01), (100.7, 1.0)])
@pytest.mark.parametrize("form", FORMS, **ids)
def test_small_spread_far_from_zero(G, form, size, sigma):
    n, c, groups, k = form[:4]
    rng, eps = np.random.default_rng(2), 1e-12
    ptr = offsets(form, rng)
    x = (size + sigma * np.clip(rng.standard_normal((n, c)), -5.0, 5.0)).astype(np.float32)
    gamma, beta = (1 + 0.3 * rng.standard_normal(c)).astype(np.float32), (0.3 * rng.standard_normal(c)).astype(np.float32)
    y, mean, rstd = run(G, form, x, gamma, beta, ptr, eps)
    d = x.astype(np.float64).reshape(n, groups, -1) - size
    mu, r = np.zeros(mean.shape), np.zeros(mean.shape)
    bmu, br, want, by = np.zeros(mean.shape), np.zeros(mean.shape), np.zeros((n, c)), np.zeros((n, c))
    for s in range(len(ptr) - 1):
        rows = slice(ptr[s], ptr[s + 1])
        v = d[rows]
        if not v.size:
            continue
        m = v.mean((0, 2))
        var = ((v - m[:, None]) ** 2).mean((0, 2))
        far = np.abs(v - m[:, None]).max((0, 2))
        mu[s], r[s] = size + m, 1 / np.sqrt(var + eps)
        bmu[s] = 2 * C * U * far + U * np.abs(mu[s])
        br[s] = (0.5 * (27 * C * U * var + 4 * C * U * far * np.sqrt(var)) * r[s] ** 2 + 2 * U) * r[s]
        xh = (x[rows].astype(np.float64).reshape(v.shape) - mean[s].astype(np.float64)[:, None]) * rstd[s][:, None]
        xh = gamma * xh.reshape(-1, c)
        want[rows], by[rows] = xh + beta, 4 * U * (np.abs(xh) + np.abs(beta))
    within(mean, mu, bmu, "mean")
    within(rstd, r, br, "rstd")
    within(y, want, by, "y")
