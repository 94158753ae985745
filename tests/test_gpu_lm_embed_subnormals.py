"""The embedding gradient below fp32's smallest normal number, 2^-126."""
import numpy as np
import pytest
import torch

from paper_1805_08469_gb300 import lm

pytestmark = pytest.mark.gpu

TINY = 2.0 ** -126


def grad(dout, tokens, table, accumulate):
    N, (V, D) = len(tokens), table.shape
    space = torch.empty(lm.gem_embed_workspace(N, V, D), dtype=torch.uint8, device="cuda")
    lm.gem_embed_grad(dout, torch.tensor(tokens, dtype=torch.int32, device="cuda"), table, space, accumulate=accumulate)
    return table.double().cpu().numpy()


@pytest.mark.parametrize("D", [8, 5])
def test_added_to_an_fp32_table(D):
    """What is added, what the table holds there and their sum may each count as 0; rows without a token keep their bits."""
    held = np.array([1e-40, 1e-40, 1.5e-38, 1.5e-38, 1.0, -3e-39, 0.0])
    add = np.array([0.0, 1e-40, -1.2e-38, 2e-38, 1e-40, 0.0, 5e-39])
    tokens = [0, 1, 2, 3, 4, 6]
    table = torch.tensor(held, dtype=torch.float32, device="cuda")[:, None].repeat(1, D)
    before = table.double().cpu().numpy()
    dout = torch.tensor(add[tokens], dtype=torch.float32, device="cuda")[:, None].repeat(1, D)
    got = grad(dout, tokens, table, True)
    want = before.copy()
    want[tokens] += dout.double().cpu().numpy()
    # both terms count as 0, or one (then the sum is the other, which is not below 2^-126), or their sum does
    assert (np.abs(got - want) <= 2 * TINY + 2.0 ** -24 * np.abs(want)).all()
    assert np.array_equal(got[5], before[5])


@pytest.mark.parametrize("D", [8, 5])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_written_sums_keep_theirs(D, dtype):
    dout = torch.tensor([1e-40, 2e-39, -1e-38, 1e-39], device="cuda").to(dtype)[:, None].repeat(1, D)
    table = torch.full((5, D), float("nan"), dtype=dtype, device="cuda")
    got = grad(dout, [0, 1, 3, 4], table, False)
    want = np.zeros((5, D))
    want[[0, 1, 3, 4]] = dout.double().cpu().numpy()
    assert np.array_equal(got, want)
