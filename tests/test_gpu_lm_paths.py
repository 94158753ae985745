"""The ways the language-model kernels are cut: rows of a warp, of one block, of clusters and past
them, more rows than are resident at once, with masked, empty and NaN rows between; recurrences of
one block and of clusters of every size, 16-bit rows at odd addresses, broadcast inputs."""
import numpy as np
import pytest
import torch

import lm_reference as ref
from paper_1805_08469_gb300 import lm
from test_gpu_lm_glr import Case, FORMS, host as seq_host, place
from test_gpu_lm_vocab import DTYPES, INF, distill_inputs, distill_run, floats, host, ints, logp_run, rows

pytestmark = pytest.mark.gpu


# ---------------------------------------------------------------------- rows of logits


@pytest.mark.parametrize("dtype,V", [("bf16", 4095), ("bf16", 4096), ("bf16", 4097), ("f16", 4103), ("f16", 4111), ("f32", 2047),
                                     ("f32", 2048), ("f32", 2049), ("f32", 2055), ("bf16", 33280), ("bf16", 33281), ("f32", 16640),
                                     ("f32", 16641)])
def test_rows_on_both_sides_of_the_limits(dtype, V):
    """A warp's longest row and a block's first; one block's longest and a cluster's first."""
    z, idx, top, lse = distill_inputs(V, 330, V, 6, dtype, tail=True, absent=False, pad=3)
    pick = [0, 1, 152, 153, 304, 329]
    want = ref.distill(host(z)[pick], idx[pick], top[pick], 1.0, 0.0, lse[pick], dtype=dtype)
    got = distill_run(z, idx, top, lse=lse)
    for k in want:
        ref.check(got[k][pick], want[k], k)
    assert np.isfinite(got["grad"]).all() and np.isfinite(got["loss"]).all()
    y = np.arange(330) * 7 % V
    got = logp_run(z, ints(y), 1.0, 9, floats(np.ones(330)), floats(np.ones(330)))
    want = ref.token_logp(host(z)[pick], y[pick], 1.0, 9, np.ones(6), np.ones(6), dtype)
    for k in got:
        ref.check(got[k][pick], want[k], k)


@pytest.mark.parametrize("dtype,V,N", [("bf16", 700, 2000), ("f32", 3001, 1400), ("bf16", 40001, 700), ("f16", 140001, 300)])
@pytest.mark.parametrize("tail", [False, True])
def test_more_rows_than_are_resident(dtype, V, N, tail):
    """Each block takes several rows: ordinary, masked, empty and NaN ones side by side, each its own."""
    K = 12
    rng = np.random.default_rng(V)
    idx = (rng.integers(0, V, (N, 1)) + np.arange(K) * rng.integers(1, V // K, (N, 1))) % V
    idx[rng.random(N) < 0.1, 5:] = -1
    idx[rng.random(N) < 0.05] = -1
    idx[rng.random(N) < 0.05, 3] = idx[0, 3]
    top = (2 * rng.standard_normal((N, K))).astype(np.float32)
    lse = (np.log(np.exp(top.astype(np.float64)).sum(1)) + 0.1).astype(np.float32) if tail else None
    z = rows(np.zeros((N, V)), dtype, pad=1)
    z.copy_(2 * torch.randn((N, V), device="cuda", generator=torch.Generator("cuda").manual_seed(V)))
    kind = rng.integers(0, 12, N)
    scale = np.where(kind == 0, 0.0, rng.uniform(0.5, 2.0, N)).astype(np.float32)
    z[ints(np.flatnonzero(kind == 0)).long()] = float("nan")      # masked
    z[ints(np.flatnonzero(kind == 1)).long()] = -INF              # empty
    z[ints(np.flatnonzero(kind == 2)).long(), V // 2] = float("nan")
    got = distill_run(z, idx, top, 1.0, 0.0, lse, scale=scale)
    pick = np.flatnonzero(kind != 2)
    pick = np.unique(np.concatenate([pick[:40], pick[-40:], rng.choice(pick, 40)]))
    want = ref.distill(host(z[ints(pick).long()]), idx[pick], top[pick], 1.0, 0.0, None if lse is None else lse[pick], scale=scale[pick],
                       dtype=dtype)
    for k in want:
        ref.check(got[k][pick], want[k], k)
    bad = np.flatnonzero(kind == 2)
    has = (idx[bad] >= 0).any(1) | tail
    assert np.isnan(got["loss"][bad[has]]).all()
    fine = np.flatnonzero(kind > 2)
    assert np.isfinite(got["grad"][fine]).all() and np.isfinite(got["loss"][fine]).all()

    y = rng.integers(-1, V, N)
    got = logp_run(z, ints(y), 1.0, 21)
    pick = np.flatnonzero((kind != 2) & (kind != 0))
    pick = np.unique(np.concatenate([pick[:60], pick[-60:], rng.choice(pick, 60)]))
    want = ref.token_logp(host(z[ints(pick).long()]), y[pick], 1.0, 21)
    for k in got:
        ref.check(got[k][pick], want[k], k)
    bad = np.flatnonzero(kind == 2)
    assert (got["top_idx"][bad, 0] == V // 2).all() and np.isnan(got["entropy"][bad]).all()


@pytest.mark.parametrize("dtype,V", [("bf16", 900), ("f32", 1500), ("f16", 9000), ("bf16", 70001), ("f32", 200000)])
@pytest.mark.parametrize("K", [1, 7, 64, 256])
def test_ties_in_many_rows(dtype, V, K):
    """Rows of few values, alike ones and ones with fewer finite logits than alternatives, in turn with
    ordinary rows: the exact search of one row does not disturb the next."""
    rng = np.random.default_rng(K)
    N = 24
    v = 2 * rng.standard_normal((N, V))
    v[0::4] = 1.0
    v[1::4] = rng.integers(-2, 3, (6, V))
    v[2::4] = np.where(rng.random((6, V)) < 5.0 / V, v[2::4], -INF)
    z = rows(v, dtype)
    y = rng.integers(0, V, N)
    got = logp_run(z, ints(y), 1.3, K)
    want = ref.token_logp(host(z), y, float(np.float32(1.3)), K)
    for k in got:
        ref.check(got[k], want[k], k)


# ---------------------------------------------------------------------- recurrences


@pytest.mark.parametrize("B,T,D", [(1, 129, 32), (1, 2100, 64), (2, 1300, 96), (3, 700, 352), (5, 513, 480), (2, 400, 1600), (1, 200, 4096),
                                   (7, 150, 1100), (20, 100, 1000), (33, 40, 2000)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_every_cut(B, T, D, dtype):
    """From clusters of sixteen blocks to blocks of a few warps, with and without resets."""
    Case(B * T, B, T, D, dtype).check()
    lengths = [(b * 37) % (T + 1) for b in range(B)]
    Case(B * T + 1, B, T, D, dtype, "add", lengths=lengths, resets=0.02).check()


@pytest.mark.parametrize("B,T,D", [(1, 1, 1), (1, 3, 1), (1, 17, 1), (2, 40, 63), (1, 700, 65), (3, 300, 127), (2, 90, 129), (30, 50, 191)])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("layout", ["dense", "half", "odd", "time_major"])
def test_odd_rows(B, T, D, dtype, layout):
    """16-bit rows that start in the middle of a word, from a tensor's first element to its last; what lies
    between the rows of the outputs is not touched."""
    Case(B + T + D, B, T, D, dtype, resets=0.03, lengths=[T - b % 3 for b in range(B)], layout=layout).check()
    if layout == "half":
        x = place(np.random.default_rng(D).standard_normal((B, T, D)), dtype, "dense")
        both = torch.full((B, T, 2 * D), 5.0, dtype=DTYPES[dtype], device="cuda")
        lm.gem_glr_forward(x, x, both[..., D:])
        assert bool((both[..., :D] == 5).all())
        kept = both[..., D:].clone()
        both.fill_(5.0)
        lm.gem_glr_forward(x, x, both[..., :D])
        assert bool((both[..., D:] == 5).all()) and torch.equal(both[..., :D], kept)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("D", [33, 34, 64])
def test_broadcast_inputs_of_every_kind(D, dtype):
    """Strides of 0: a gate for all steps, an input for all sequences, a gradient for all of both."""
    rng = np.random.default_rng(D)
    t = DTYPES[dtype]
    f = torch.from_numpy(rng.standard_normal((2, 1, D))).to(t).cuda().expand(2, 90, D)
    x = torch.from_numpy(rng.standard_normal((1, 90, D))).to(t).cuda().expand(2, 90, D)
    dh = torch.from_numpy(rng.standard_normal((1, 1, D))).to(t).cuda().expand(2, 90, D)
    new = lambda: torch.empty((2, 90, D), dtype=t, device="cuda")  # noqa: E731
    h, dx, df, saved = new(), new(), new(), torch.empty((2, 6, D), device="cuda")
    lm.gem_glr_forward(x, f, h, form=FORMS["add"], saved=saved)
    lm.gem_glr_backward(x, f, saved, dh, dx, df, form=FORMS["add"])
    want = ref.glr(seq_host(x), seq_host(f), False, dh=seq_host(dh), dtype=dtype)
    for k, v in (("h", h), ("dx", dx), ("df", df)):
        ref.check(seq_host(v), want[k], k)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_long_state_through_a_cluster(dtype):
    """Gates so near 1 that the first step is still there after thousands, over many rounds of a cluster."""
    c = Case(1, 1, 12000, 24, dtype, "add")
    c.f.copy_(torch.full_like(c.f, 12.0 if dtype == "f32" else 9.0))
    c.check()
