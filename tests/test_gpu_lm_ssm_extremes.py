"""The selective scan at the ends of its decays: decays past fp32 at a reset, and idle steps in tiles that begin with
an ordinary one."""
import numpy as np
import pytest
import torch

from test_gpu_lm_ssm import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("B,T,N", [(2, 1, 16), (2, 40, 16), (2, 40, 64), (1, 400, 16), (1, 3000, 7)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_reset_under_a_decay_past_fp32(dtype, B, T, N):
    """exp(step A) of e^100 there, where the state before counts as 0; steps of 0 elsewhere: nothing of A is left but in its own
    gradient and the steps'."""
    cut = T // 2 + 3 if T > 1 else 0
    c = Case(16, B, T, 33, N, 1, dtype, softplus=False, bias=False)
    c.reset = torch.zeros((B, T), dtype=torch.bool, device="cuda")
    c.reset[:, cut] = True
    c.dt.zero_()
    c.dt[:, cut] = 1.0
    c.A.zero_()
    want = c.run()
    c.A.fill_(100.0)
    got = c.run()
    for k in ("y", "h_last", "saved", "dx", "dz", "db", "dc", "dskip", "dh0"):
        assert np.isfinite(got[k]).all(), k
        assert np.array_equal(got[k], want[k]), k
    assert np.isfinite(got["dA"]).all() and np.isfinite(got["ddt"]).all() and np.array_equal(got["ddt"][:, cut], want["ddt"][:, cut])


@pytest.mark.parametrize("N", [16, 64])
def test_idle_steps_after_an_ordinary_one(N):
    """Steps of 0 decay by exactly 1 whatever their tile's first step is, from ones that hardly decay to ones that forget."""
    B, D = 3, 64
    c = Case(17, B, 16, D, N, 1, "f32", softplus=False, bias=False)
    c.dt.zero_()
    c.dt[:, 0] = torch.logspace(-5, 1, B * D, device="cuda").view(B, D)
    c.dy.zero_()
    got = c.run()
    one = Case(17, B, 16, D, N, 1, "f32", softplus=False, bias=False)
    one.dims = (B, 1, D, N, 1)
    for k in ("x", "dt", "dy", "z", "b", "c"):
        setattr(one, k, getattr(c, k)[:, :1].contiguous())
    alone = one.run()
    for k in ("h_last", "dh0"):
        assert np.array_equal(got[k], alone[k]), k
    # what later steps read of the state
    c.c = c.c[:, :1].expand(B, 16, 1, N)
    c.z, c.skip = None, None
    y = c.run(backward=False)["y"]
    assert np.array_equal(y, np.broadcast_to(y[:, :1], y.shape))
