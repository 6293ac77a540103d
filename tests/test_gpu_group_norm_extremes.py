"""The gradient behind SiLU where z is far from zero, in the forms with one reading and with two."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def G():
    assert torch.cuda.is_available(), "GPU tests need a HIP device"
    import paper_2512_01678_amd.gcn as G
    return G


@pytest.mark.parametrize("n", [50, 30000])
@pytest.mark.parametrize("z", [-3e38, -1e30, -1e6, -200.0, -88.8, -80.5, 80.5, 1e6, 3e38])
def test_silu_far_from_zero(G, n, z):
    """Far below zero the slope z exp(z) is smaller than 1e-32, far above it is 1 to the last bit: q = 1 / (1 + e), e below
    2^-24, and z e q below 80 exp(-80).  d is dy times that."""
    c = 8
    x = torch.randn(n, c, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    dy = torch.ones(n, c, device="cuda")
    gamma, beta = torch.zeros(c, device="cuda"), torch.full((c,), z, device="cuda")
    mean, rstd = torch.empty(1, 2, device="cuda"), torch.empty(1, 2, device="cuda")
    y = torch.empty_like(x)
    G.group_norm(x, 2, gamma, beta, y, mean, rstd, act=G.ACT_SILU)
    dx, dgamma, dbeta = torch.empty_like(x), torch.empty(c, device="cuda"), torch.empty(c, device="cuda")
    G.group_norm_bwd(x, dy, mean, rstd, 2, gamma, beta, dx, dgamma, dbeta, act=G.ACT_SILU)
    assert not dx.any()  # gamma is 0
    if z < 0:
        assert float(y.abs().max()) <= 1e-32  # z exp(z)
        assert float(dbeta.abs().max()) <= n * 1e-32 and float(dgamma.abs().max()) <= n * 10 * 1e-32
    else:
        # q is the hardware's reciprocal of 1: exact; sums of ones below 2^24 too
        assert float((y / z - 1).abs().max()) <= 2.0 ** -23 and (dbeta == n).all()
