"""The policy loss and its gradient against their definitions in 64 bits: rows of a warp, of blocks, of
clusters and past them, every type, pitches and alignments, masked rows, all terms and their absence, borders,
infinities and NaN, and the gradient against differences."""
import numpy as np
import pytest
import torch

import lm_layers_reference as ref
from lm_reference import check
from paper_1805_08469_gb300 import lm
from test_gpu_lm_vocab import DTYPES, INF, floats, host, ints, rows

pytestmark = pytest.mark.gpu


class Case:
    def __init__(self, seed, N, V, dtype="f32", tau=1.0, low=0.2, high=0.2, kl=0.05, bonus=0.01, pad=0, masked=True, spread=2.0):
        rng = np.random.default_rng(seed)
        self.dtype = dtype
        self.how = dict(tau=float(np.float32(tau)), low=float(np.float32(low)), high=float(np.float32(high)), kl=float(np.float32(kl)),
                        bonus=float(np.float32(bonus)))
        z = spread * rng.standard_normal((N, V))
        y = rng.integers(0, V, N)
        z[np.arange(N), y] += 8 * rng.random(N)
        self.z = rows(z, dtype, pad=pad)
        if masked:
            y[rng.random(N) < 0.1] = -1
        self.tokens = y
        v = host(self.z).astype(np.float64) / self.how["tau"]
        with np.errstate(divide="ignore"):
            lse = np.log(np.exp(v - v.max(1, keepdims=True)).sum(1)) + v.max(1)
        logp = v[np.arange(N), np.clip(y, 0, V - 1)] - lse
        moved = 0.2 * rng.standard_normal(N)
        r = np.exp(moved)
        moved = np.where((np.abs(r - 1 + self.how["low"]) < 1e-2) | (np.abs(r - 1 - self.how["high"]) < 1e-2), 0.001, moved)
        self.old = (logp - moved).astype(np.float32)
        self.ref = (logp + 0.3 * rng.standard_normal(N)).astype(np.float32) if kl else None
        self.A = rng.standard_normal(N).astype(np.float32)
        self.scale = np.where(rng.random(N) < 0.1, 0, rng.uniform(0.5, 2, N)).astype(np.float32) if masked else None

    def run(self, z=None, grad=True, in_place=False, pad=0):
        z = self.z if z is None else z
        N, V = z.shape
        nan = lambda: torch.full((N,), float("nan"), device="cuda")  # noqa: E731
        out = {"loss": nan(), "logp": nan(), "entropy": nan()}
        g = z if in_place else rows(np.full((N, V), np.nan), self.dtype, pad=pad) if grad else None
        h = self.how
        lm.gem_policy(z, ints(self.tokens), floats(self.old), floats(self.A), out["loss"], g, ref_logp=None if self.ref is None else floats(self.ref),
                      row_scale=None if self.scale is None else floats(self.scale), temperature=h["tau"], clip_low=h["low"], clip_high=h["high"],
                      kl=h["kl"], bonus=h["bonus"], logp=out["logp"], entropy=out["entropy"])
        if g is not None:
            out["grad"] = g
        torch.cuda.synchronize()
        return {k: host(v) for k, v in out.items()}

    def reference(self, pick=slice(None), z=None):
        sub = lambda v: None if v is None else v[pick]  # noqa: E731
        return ref.policy((host(self.z) if z is None else z)[pick], self.tokens[pick], self.old[pick], self.A[pick], sub(self.ref), sub(self.scale),
                          dtype=self.dtype, **self.how)

    def check(self, pick=slice(None), **kw):
        want = self.reference(pick)
        got = self.run(**kw)
        for k in got:
            check(got[k][pick], want[k], k)
        return got


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("V", [1, 2, 7, 8, 9, 31, 33, 100, 1000, 1001, 2048, 2049, 4096, 4097, 5000, 16641, 33281, 50001])
def test_row_lengths(V, dtype):
    Case(V, 21, V, dtype).check()


@pytest.mark.parametrize("dtype,V", [("f32", 131072), ("bf16", 200003), ("bf16", 700001), ("f32", 400001), ("bf16", 1000003)])
def test_long_rows(V, dtype):
    """Clusters of every size, and rows past them, which a block streams."""
    Case(V, 5, V, dtype).check()


@pytest.mark.parametrize("V", [200, 3001, 40001])
@pytest.mark.parametrize("how", [dict(kl=0.0), dict(bonus=0.0), dict(kl=0.0, bonus=0.0), dict(tau=0.7), dict(tau=3.0, high=0.5), dict(low=0.0, high=0.0),
                                 dict(low=1.0), dict(bonus=-0.02), dict(masked=False), dict(kl=3.0, bonus=2.0)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_terms(how, V, dtype):
    Case(V, 40, V, dtype, **how).check()


@pytest.mark.parametrize("pad", [1, 3, 8])
@pytest.mark.parametrize("V", [1000, 5000, 40000])
@pytest.mark.parametrize("dtype", ["f32", "f16"])
def test_pitches(V, pad, dtype):
    c = Case(V + pad, 9, V, dtype, pad=pad)
    a = c.check(pad=pad)
    b = c.run(pad=0)          # gradient rows at other offsets from 16 bytes than the logits'
    for k in a:
        assert np.array_equal(a[k], b[k]), k


@pytest.mark.parametrize("V", [1000, 5000, 60001, 1000003])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_in_place_and_without_a_gradient(V, dtype):
    c = Case(V, 6, V, dtype)
    want = c.run()
    none = c.run(grad=False)
    for k in none:
        assert np.array_equal(none[k], want[k]), k
    got = c.run(z=c.z.clone(), in_place=True)
    for k in got:
        assert np.array_equal(got[k], want[k]), k


@pytest.mark.parametrize("dtype,V,N", [("bf16", 700, 2000), ("f32", 3001, 1400), ("bf16", 40001, 700), ("f16", 140001, 300)])
def test_more_rows_than_are_resident(dtype, V, N):
    """Each block takes several rows: ordinary, masked, empty and NaN ones side by side, each its own."""
    c = Case(V, N, V, dtype, pad=1)
    rng = np.random.default_rng(N)
    kind = rng.integers(0, 12, N)
    c.tokens = np.where(c.tokens < 0, 0, c.tokens)
    c.scale = np.where(kind == 0, 0.0, 1.0).astype(np.float32)
    v = c.reference(np.flatnonzero(kind > 3)[:60])
    c.z[ints(np.flatnonzero(kind == 0)).long()] = float("nan")      # masked
    c.tokens = np.where(kind == 1, -1, c.tokens)                     # without a token
    c.z[ints(np.flatnonzero(kind == 1)).long()] = float("nan")
    c.z[ints(np.flatnonzero(kind == 2)).long(), V // 2] = float("nan")
    c.z[ints(np.flatnonzero(kind == 3)).long()] = -INF               # empty
    got = c.run()
    for k in got:
        check(got[k][np.flatnonzero(kind > 3)[:60]], v[k], k)
        assert (got[k][kind <= 1] == 0).all() and np.isfinite(got[k][kind > 3]).all()
    for k in ("loss", "grad"):
        assert np.isnan(got[k][kind == 2]).all() and np.isnan(got[k][kind == 3]).all(), k


@pytest.mark.parametrize("V", [900, 5003, 70001, 1000003])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_masked_logits(V, dtype):
    """Logits of -inf and of the type's lowest value: probability 0, and no gradient."""
    c = Case(V, 12, V, dtype)
    rng = np.random.default_rng(V)
    y = np.maximum(c.tokens, 0)
    z = host(c.z).astype(np.float64)
    for i in range(12):
        out = rng.random(V) < (0.5 if i % 3 else 0.99)
        out[y[i]] = False
        z[i, out] = -INF if i % 2 else float(torch.finfo(DTYPES[dtype]).min)
    c.z = rows(z, dtype)
    z = host(c.z).astype(np.float64)
    lp = z - z.max(1, keepdims=True)
    lp = (lp - np.log(np.exp(lp).sum(1, keepdims=True)))[np.arange(12), y]
    c.old, c.ref = (lp + 0.05).astype(np.float32), (lp - 0.1).astype(np.float32)
    got = c.check()
    assert (got["grad"][z < -1e30] == 0).all()


@pytest.mark.parametrize("V", [64, 5000, 50000, 1000003])
def test_borders(V):
    """Ratios on a bound of the clipping, and logits for which everything is exact: a row of equal logits, V a power of two
    times a token's chance of 1 / V."""
    z = np.zeros((4, V))
    logp = -np.log(V)
    c = Case(1, 4, V, kl=0.0, bonus=0.0, masked=False)
    c.z, c.tokens = rows(z, "f32"), np.array([0, V - 1, V // 2, 1])
    c.A = np.array([1.0, -1.0, 1.0, -1.0], np.float32)
    c.old = np.array([logp + 1.0, logp + 1.0, logp - 1.0, logp - 1.0], np.float32)   # ratios of 1/e and e
    got = c.run()
    # (advantage 1 and a small ratio: not clipped; -1 and a small one: clipped; 1 and a large one: clipped; -1 and a large one: not)
    assert np.abs(got["grad"][0]).max() > 0 and np.abs(got["grad"][3]).max() > 0
    assert (got["grad"][1] == 0).all() and (got["grad"][2] == 0).all()
    check(got["loss"], (np.array([-np.exp(-1), 0.8, -1.2, np.e]), 1e-5), "loss")


def test_tokens_out_of_range():
    c = Case(2, 5, 300, masked=False)
    c.tokens = np.array([0, -7, 300, 2**31 - 1, 299])
    want = c.reference()
    got = c.run()
    for k in ("loss", "logp", "grad"):
        assert np.isnan(got[k][2:4]).all() and (got[k][1] == 0).all(), k
        check(got[k][[0, 4]], (want[k][0][[0, 4]], want[k][1][[0, 4]]), k)


@pytest.mark.parametrize("V", [500, 9000, 60000, 900001])
@pytest.mark.parametrize("bad", ["nan", "inf"])
def test_nan_and_infinite_logits(V, bad):
    c = Case(3, 6, V, "f32", masked=False)
    for i, j in enumerate([0, 1, V // 2, V - 2, V - 1]):
        c.z[i, j] = float(bad)
    got = c.run()
    for k in ("loss", "grad"):
        assert np.isnan(got[k][:5]).all() and np.isfinite(got[k][5]).all(), k


@pytest.mark.parametrize("offset", [-3e4, 500.0, 4e4])
@pytest.mark.parametrize("V", [1000, 9001])
def test_a_common_offset_changes_nothing(offset, V):
    """Logits in steps of 2^-7 that an offset keeps exact: the same differences, the same bits."""
    c = Case(4, 8, V, "f32", masked=False)
    v = np.round(host(c.z).astype(np.float64) * 128) / 128
    c.z = rows(v, "f32")
    want = c.run()
    c.z = rows(v + offset, "f32")
    got = c.run()
    for k in got:
        assert np.array_equal(got[k], want[k]), k


@pytest.mark.parametrize("V", [900, 20000, 1000003])
def test_offsets_past_32_bits(V):
    """Rows that begin more than 2^31 elements apart."""
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 40 GB")
    c = Case(7, 4, V, "bf16", masked=False)
    want = c.run()
    far = torch.empty(3 * (1 << 30) + V, dtype=torch.bfloat16, device="cuda").as_strided((4, V), (1 << 30, 1))
    far.copy_(c.z)
    got = c.run(z=far, in_place=True)
    for k in got:
        assert np.array_equal(got[k], want[k]), k


def test_one_row_of_logits_for_all():
    c = Case(5, 7, 4000, "f32", masked=False)
    z = c.z[:1].expand(7, 4000)
    full = c.z[:1].repeat(7, 1)
    a = c.run(z=z)
    c.z = full
    b = c.run()
    for k in a:
        assert np.array_equal(a[k], b[k]), k


def test_gradients_against_differences():
    """Central differences of the call's own losses: a step of 2^-6 leaves an error of h^2 / 6 times third derivatives below 4, and
    rounding of 2^-22 over 2 h."""
    c = Case(6, 4, 9, "f32", tau=0.9, kl=0.3, bonus=0.2, masked=False, spread=1.0)
    got = c.run()
    h = 2.0 ** -6
    for j in range(9):
        up, down = c.z.clone(), c.z.clone()
        up[:, j] += h
        down[:, j] -= h
        wide = (host(up)[:, j] - host(down)[:, j]).astype(np.float64)
        d = (c.run(z=up)["loss"].astype(np.float64) - c.run(z=down)["loss"].astype(np.float64)) / wide
        r = np.exp(c.run()["logp"] - c.old)
        clear = (np.abs(r - 0.8) > 0.03) & (np.abs(r - 1.2) > 0.03)     # no bound of the clipping within the step
        assert (np.abs(d - got["grad"][:, j])[clear] < 4e-4).all() and clear.any(), j
