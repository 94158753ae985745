"""The policy loss where probabilities underflow: logits of a type's lowest value beside ordinary ones at any temperature and loss
scale, and the ends of the temperature, in rows of a warp, of clusters and streamed ones."""
import numpy as np
import pytest
import torch

from test_gpu_lm_policy import Case
from test_gpu_lm_vocab import DTYPES, INF, host, rows

pytestmark = pytest.mark.gpu

N = 8


def masked_case(V, dtype, tau, scale, low):
    """Half of each row's logits, or all but a few, are `low` (every third row: -inf), the token's is not."""
    c = Case(V, N, V, dtype, tau=tau, masked=False)
    rng = np.random.default_rng(V)
    z = host(c.z).astype(np.float64)
    for i in range(N):
        out = rng.random(V) < (0.5 if i % 2 else 0.99)
        out[c.tokens[i]] = False
        z[i, out] = -INF if i % 3 == 2 else low
    c.z = rows(z, dtype)
    z = host(c.z).astype(np.float64) / c.how["tau"]
    lp = z - z.max(1, keepdims=True)
    lp = (lp - np.log(np.exp(lp).sum(1, keepdims=True)))[np.arange(N), c.tokens]
    c.old, c.ref = (lp + 0.05).astype(np.float32), (lp - 0.1).astype(np.float32)
    c.scale = np.full(N, scale, np.float32)
    return c


@pytest.mark.parametrize("dtype,scale", [("f32", 1.0), ("f32", 65536.0), ("bf16", 1024.0), ("bf16", 65536.0), ("f16", 1.0), ("f16", 1024.0)])
@pytest.mark.parametrize("tau", [0.7, 1.0, 2.0, 4.0])
@pytest.mark.parametrize("V", [900, 5003, 70001, 1000003])
def test_lowest_values_at_any_temperature(dtype, V, tau, scale):
    """Probability 0 and no gradient, whatever the factors that it would have."""
    low = float(torch.finfo(DTYPES[dtype]).min)
    c = masked_case(V, dtype, tau, scale, low)
    got = c.check()
    assert (got["grad"][host(c.z) <= low] == 0).all()


@pytest.mark.parametrize("V", [900, 5003, 70001, 1000003])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_very_low_logits_at_a_low_temperature(dtype, V):
    """Quotients that just stay in fp32 times factors that take them out of it."""
    c = masked_case(V, dtype, 1e-3, 1024.0, -1e35)
    got = c.check()
    assert (got["grad"][host(c.z) < -1e30] == 0).all()


@pytest.mark.parametrize("tau", [1e-20, 1e-10])
@pytest.mark.parametrize("V", [900, 5003, 70001, 1000003])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_lowest_temperatures(dtype, V, tau):
    """A largest logit of its own has all of the mass: log p is 0, nothing changes it, and its token's loss is exact but for
    the ratio and the KL term."""
    c = Case(V, N, V, dtype, masked=False)
    z = host(c.z).astype(np.float64)
    z[np.arange(N), c.tokens] = z.max(1) + 10
    c.z = rows(z, dtype)
    c.how["tau"] = float(np.float32(tau))
    c.old, c.ref = np.linspace(-0.1, 0.1, N).astype(np.float32), np.linspace(0.3, -0.3, N).astype(np.float32)
    got = c.check()
    assert (got["grad"] == 0).all() and (got["logp"] == 0).all() and (got["entropy"] == 0).all()


@pytest.mark.parametrize("V", [900, 5003, 70001, 1000003])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_two_largest_logits_at_the_lowest_temperature(dtype, V):
    """They share the mass; gradients of 1e20 and zeros side by side."""
    c = Case(V, N, V, dtype, masked=False)
    z = host(c.z).astype(np.float64)
    other = (c.tokens + V // 2) % V
    z[np.arange(N), c.tokens] = z[np.arange(N), other] = z.max(1) + 10
    c.z = rows(z, dtype)
    c.how["tau"] = float(np.float32(1e-20))
    c.old, c.ref = np.full(N, -0.6, np.float32), np.full(N, -0.8, np.float32)
    got = c.check()
    rest = np.ones((N, V), bool)
    rest[np.arange(N), c.tokens] = rest[np.arange(N), other] = False
    assert (got["grad"][rest] == 0).all() and (got["grad"][~rest] != 0).all()


@pytest.mark.parametrize("V", [900, 5003, 70001, 1000003])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_the_highest_temperature(dtype, V):
    Case(V, N, V, dtype, tau=1e20, masked=False).check()
