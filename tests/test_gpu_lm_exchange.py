"""The exchange of maps in a cluster, also where a block's maps do not come: the wait ends by itself, and nothing
that rests on them is anything but NaN, whatever resets follow."""
import ctypes as C
import subprocess
import time

import numpy as np
import pytest
import torch

from paper_1805_08469_gb300 import _build

pytestmark = pytest.mark.gpu

THREADS = 64


@pytest.fixture(scope="module")
def exchange(tmp_path_factory):
    so = tmp_path_factory.mktemp("exchange") / "exchange.so"
    subprocess.run([_build._nvcc(), "-O3", "-std=c++17", "-Xcompiler", "-fPIC", "-shared", *_build.ARCH, "-I", str(_build.CSRC), "-I",
                    str(_build.ROOT / "include"), "-o", str(so), str(_build.ROOT / "tests" / "lm_exchange.cu")], check=True)
    fn = C.CDLL(str(so)).run_exchange
    fn.argtypes = [C.c_int, C.c_void_p, C.c_int, C.c_int, C.c_int]

    def run(channels, rounds, sent, first_reset):
        out = torch.full((rounds, THREADS, 2, channels), -7.0, device="cuda")
        torch.cuda.synchronize()
        start = time.monotonic()
        assert fn(channels, out.data_ptr(), rounds, sent, first_reset) == 0
        return out.cpu().numpy(), time.monotonic() - start

    return run


def states(rounds, first_reset):
    """(before each warp's chunk, after the round): four chunks a round, two of the first block's warps; a chunk
    halves the state and adds 1, or from round first_reset on sets it to 1."""
    h, before, after = 1.0, [], []
    for r in range(rounds):
        chunk = []
        for _ in range(4):
            chunk.append(h)
            h = 1.0 if r >= first_reset else 0.5 * h + 1.0
        before.append(chunk[:2])
        after.append(h)
    return np.repeat(np.array(before), 32, 1)[..., None], np.array(after)[:, None, None]


@pytest.mark.parametrize("channels", [1, 2])
def test_all_maps_come(channels, exchange):
    got, _ = exchange(channels, 9, 9, 5)
    before, after = states(9, 5)
    assert np.array_equal(got[:, :, 0], np.broadcast_to(before, got[:, :, 0].shape))
    assert np.array_equal(got[:, :, 1], np.broadcast_to(after, got[:, :, 1].shape))


@pytest.mark.parametrize("channels,sent", [(1, 0), (2, 3)])
def test_maps_that_do_not_come(channels, sent, exchange):
    """The wait of two seconds is paid once; resets from the next round on do not bring the states back."""
    got, seconds = exchange(channels, sent + 6, sent, sent + 1)
    before, after = states(sent + 6, sent + 1)
    assert np.array_equal(got[:sent, :, 0], np.broadcast_to(before[:sent], got[:sent, :, 0].shape))
    assert np.array_equal(got[:sent, :, 1], np.broadcast_to(after[:sent], got[:sent, :, 1].shape))
    assert np.isnan(got[sent:]).all()
    assert 1.5 < seconds < 3.5
    exchange(channels, 4, 4, 9)   # (the GPU goes on as before)
