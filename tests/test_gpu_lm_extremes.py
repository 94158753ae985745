"""The language-model operators at the ends of their ranges: logits with a common offset, temperatures down to
the lowest one, a student far surer than its rest, losses of one term only, states that are infinite."""
import numpy as np
import pytest
import torch

import lm_reference as ref
from lm_reference import U
from paper_1805_08469_gb300 import lm
from test_gpu_lm_glr import Case
from test_gpu_lm_vocab import INF, distill_inputs, distill_run, floats, host, ints, logp_run, rows

pytestmark = pytest.mark.gpu


# ---------------------------------------------------------------------- the scores' gradient


def grad_reference(z, y, tau, dl, dH, dtype):
    """(value, bound) of the scores' gradient.  The bound has the errors of (z - max) / tau and of the entropy,
    neither of which grows with max / tau; subnormal factors of a product add their step."""
    N, V = z.shape
    _, lp, p, err_lp, rel_p, _, _ = ref._softmax(z, tau)
    H, eH = (v[:, None] for v in ref.token_logp(z, y, tau, 0)["entropy"])
    dl, dH = dl.astype(np.float64)[:, None], dH.astype(np.float64)[:, None]
    lp = np.where(p > 0, lp, 0)
    hit = (np.arange(V)[None] == np.asarray(y)[:, None]).astype(np.float64)
    dl = np.where(np.asarray(y)[:, None] < 0, 0, dl)
    g = (hit * dl - p * (dl + dH * (lp + H))) / tau
    size = np.abs(dl) + np.abs(dH) * (np.abs(lp) + np.abs(H))
    e = p * ((rel_p + 8 * U) * size + np.abs(dH) * (err_lp + 4 * U * np.abs(lp) + eH)) + 2.0 ** -147 * (1 + size)
    e = (e + 4 * U * hit * np.abs(dl)) / tau + 4 * U * np.abs(g)
    return g, 1.01 * e + ref.rounded(g, dtype)


def check_grad(v, dtype, tau, pad=1):
    rng = np.random.default_rng(v.shape[1])
    N, V = v.shape
    z = rows(v, dtype, pad=pad)
    y = rng.integers(-1, V, N)
    dl, dH = floats(tau * rng.standard_normal(N)), floats(0.1 * tau * rng.standard_normal(N))
    got = logp_run(z, ints(y), tau, 0, dl, dH)["grad"]
    ref.check(got, grad_reference(host(z), y, float(np.float32(tau)), host(dl), host(dH), dtype), "grad")
    assert np.array_equal(logp_run(z, ints(y), tau, 0, dl, dH, grad=z)["grad"], got)   # in place


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("V", [9, 3000, 40001])
@pytest.mark.parametrize("offset", [1e4, -1e4])
def test_gradient_of_logits_with_a_common_offset(V, dtype, offset):
    """Beside ordinary rows, whose values and places they leave alone."""
    v = 2 * np.random.default_rng(V).standard_normal((6, V))
    v[1::2] += offset
    check_grad(v, dtype, 1.0)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("V", [9, 3000, 40001])
@pytest.mark.parametrize("tau", [1e-3, 1e-6, 1e-8, 1e-20])
def test_gradient_at_low_temperatures(V, dtype, tau):
    """Equal top logits share the mass; neighbouring fp32 numbers lie near tau apart for one of the temperatures."""
    rng = np.random.default_rng(V)
    v = rng.standard_normal((5, V))
    v[0, [1, V - 1]] = 10.3
    v[1] = -10.3
    v[2] = np.float32(10.3) + 2.0 ** -20 * rng.integers(-6, 1, V)
    v[3, V // 2] = 50.0
    check_grad(v, dtype, tau)


def test_gradient_where_the_log_sum_exp_is_past_fp32():
    v = np.full((4, 700), -1e19)
    v[0, [3, 600]] = 1e19
    v[2] = -INF
    v[3] = 1.0
    check_grad(v, "f32", 1e-20)


def test_gradient_of_rows_that_are_not_finite_beside_an_offset():
    v = np.random.default_rng(1).standard_normal((4, 9001)) + 1e5
    v[1, 7] = np.nan
    v[2, 9000] = INF
    z = rows(v, "f32")
    y, one = np.array([3, 3, 3, 3]), np.ones(4)
    got = logp_run(z, ints(y), 1.0, 0, floats(one), floats(one))["grad"]
    assert np.isnan(got[1:3]).all()
    value, bound = grad_reference(host(z)[[0, 3]], y[:2], 1.0, one[:2], one[:2], "f32")
    ref.check(got[[0, 3]], (value, bound), "grad")


# ---------------------------------------------------------------------- the rest as a class


def check_distill(z, dtype, idx, top, shown, tau, alpha=0.0, lse=None, labels=None):
    """shown: the teacher's logits as the 64-bit form gets them."""
    want = ref.distill(host(z), idx, shown, float(np.float32(tau)), alpha, lse, labels, dtype=dtype)
    got = distill_run(z, idx, top, tau, alpha, lse, labels)
    for k in want:
        ref.check(got[k], want[k], k)


@pytest.mark.parametrize("dtype,V", [("f32", 5000), ("f32", 50000), ("f32", 500009), ("bf16", 800001)])
def test_a_student_far_surer_than_its_rest(dtype, V):
    """The rest's mass is below fp32's range relative to the row's largest; its class counts all the same."""
    rng = np.random.default_rng(V)
    N, K = 5, 4
    v = rng.standard_normal((N, V))
    idx = np.stack([rng.choice(V, K, replace=False) for _ in range(N)]).astype(np.int32)
    for n, gap in enumerate([20, 40, 48, 52, 60]):
        v[n, idx[n]] = gap + rng.standard_normal(K)
    top = rng.standard_normal((N, K)).astype(np.float32)
    lse = (np.log(np.exp(2 * top.astype(np.float64)).sum(1)) - np.log1p(-np.array([0.3, 0.1, 0.02, 0.5, 0.2]))).astype(np.float32)
    check_distill(rows(v, dtype), dtype, idx, top, top, 0.5, lse=lse)


# ---------------------------------------------------------------------- the teacher's entries


SIZES = [("f32", 500), ("bf16", 500), ("f16", 20001), ("f32", 50000), ("f32", 500009)]


@pytest.mark.parametrize("dtype,V", SIZES)
@pytest.mark.parametrize("tau,offset", [(1.0, 1e4), (1.0, -3e4), (1e-3, 10.3), (1e-5, 10.3)])
def test_teacher_logits_with_a_common_offset(dtype, V, tau, offset):
    """The softmax of the entries does not know the offset: neither does the bound, which gets the differences
    from the largest (exact in 64 bits)."""
    z, idx, top, _ = distill_inputs(V, 3, V, 12, dtype, absent=False)
    top = (offset + tau * top).astype(np.float32)
    exact = top.astype(np.float64)
    check_distill(z, dtype, idx, top, exact - exact.max(1, keepdims=True), tau)


@pytest.mark.parametrize("dtype,V", SIZES)
def test_an_entry_of_the_lowest_value_stays_an_entry(dtype, V):
    """A logit that is finite, but not after its division by tau, has no mass and is none of the rest."""
    z, idx, top, lse = distill_inputs(V, 3, V, 6, dtype, tau=0.5, tail=True, absent=False)
    top[:, 4] = np.finfo(np.float32).min
    for n in range(3):
        z[n, int(idx[n, 4])] = 6.0
    check_distill(z, dtype, idx, top, top, 0.5, lse=lse)


# ---------------------------------------------------------------------- losses of one term


@pytest.mark.parametrize("dtype,V", SIZES)
@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("tau", [1.0, 2.0, 3.0])
def test_labels_only(dtype, V, tail, tau):
    """alpha = 1: the teacher's term is not there, whatever it would be."""
    z, idx, top, lse = distill_inputs(V, 4, V, 6, dtype, tail=tail, absent=False)
    for n in range(2):
        z[n, int(idx[n, 2])] = -INF
    top[2, 1] = np.nan
    labels = [int(idx[0, 0]), 7, 3, -1]
    want = ref.distill(host(z), np.full((4, 0), -1), np.zeros((4, 0)), tau, 1.0, None, labels, dtype=dtype)
    got = distill_run(z, idx, top, tau, 1.0, lse, labels)
    for k in want:
        ref.check(got[k], want[k], k)


@pytest.mark.parametrize("dtype,V", SIZES)
@pytest.mark.parametrize("tau", [1e-20, 1e19, 5e19, 1e20])
@pytest.mark.parametrize("alpha", [0.0, 0.5])
def test_no_teacher_at_the_ends_of_the_temperatures(dtype, V, tau, alpha):
    z, _, _, _ = distill_inputs(V, 3, V, 6, dtype, absent=False)
    none, labels = np.full((3, 2), -1), [5, -1, V - 1]
    want = ref.distill(host(z), none, np.zeros((3, 2)), float(np.float32(tau)), alpha, None, labels, dtype=dtype)
    got = distill_run(z, none, np.zeros((3, 2)), tau, alpha, None, labels)
    for k in want:
        ref.check(got[k], want[k], k)


@pytest.mark.parametrize("dtype,V", SIZES)
@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("alpha", [0.0, 0.5])
def test_a_row_of_nan_without_a_teacher(dtype, V, tail, alpha):
    """What is not a number in a row shows in its loss as in its gradient, with entries or without."""
    z, idx, top, lse = distill_inputs(V, 4, V, 6, dtype, tail=tail, absent=False)
    idx[1:] = -1
    z[1, V // 2] = float("nan")
    z[2, 3] = INF
    got = distill_run(z, idx, top, 1.0, alpha, lse, [-1] * 4)
    for k in got:
        assert np.isnan(got[k][1:3]).all() and np.isfinite(got[k][[0, 3]]).all(), k
    assert got["loss"][3] == 0


# ---------------------------------------------------------------------- infinite states


@pytest.mark.parametrize("form", ["lerp", "add"])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("B,T,D,resets", [(2, 700, 66, 0.0), (2, 700, 66, 0.004), (200, 70, 64, 0.0), (200, 70, 64, 0.03)])
def test_an_infinite_state_stays_one(B, T, D, resets, dtype, form):
    """However little the gates of a chunk let through, some of an infinity is one: as in calls of a step each."""
    c = Case(B + T, B, T, D, dtype, form, resets=resets)
    c.f.fill_(-12.0)
    c.h0[0, ::2], c.h0[1, ::3] = INF, -INF
    got, want = c.run(), c.reference()
    for k in ("h", "h_last", "saved", "dx", "dh0"):
        ref.check(got[k], want[k], k)
    state = c.h0.clone()
    one = torch.empty((B, 1, D), dtype=c.x.dtype, device="cuda")
    for t in range(40):
        lm.gem_glr_forward(c.x[:, t:t + 1], c.f[:, t:t + 1], one, form=lm.GEM_GLR_LERP if form == "lerp" else lm.GEM_GLR_ADD, h0=state,
                           reset=None if c.reset is None else c.reset[:, t:t + 1].contiguous(), h_last=state)
        h, step = got["h"][:, t], host(one)[:, 0]
        assert np.array_equal(np.isinf(h), np.isinf(step)) and not np.isnan(h).any()


@pytest.mark.parametrize("form", ["lerp", "add"])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("B,T,D,resets", [(2, 700, 66, 0.0), (2, 700, 66, 0.004), (200, 70, 64, 0.0), (200, 70, 64, 0.03)])
def test_an_infinite_gradient_stays_one(B, T, D, resets, dtype, form):
    """From the last state's and from single steps', at the end, the middle and the start of a chunk."""
    c = Case(B + T, B, T, D, dtype, form, resets=resets)
    c.f.fill_(-12.0)
    c.dh_last[0, ::2] = INF
    for t, d in ((47, 1), (40, 5), (32, 9)):
        c.dh[1, t, d] = -INF
    c.dh[1, T - 1, 13] = INF
    got, want = c.run(), c.reference()
    for k in ("h", "dx", "dh0"):
        ref.check(got[k], want[k], k)
    assert np.array_equal(np.isfinite(got["df"]), np.isfinite(want["df"][0]))
