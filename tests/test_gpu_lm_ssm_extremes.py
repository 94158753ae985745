"""The selective scan at the ends of its decays."""
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
