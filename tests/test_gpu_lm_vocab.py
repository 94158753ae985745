"""Distillation loss and token log probabilities against their definitions in 64 bits: vocabularies
from one entry to ones larger than a cluster's shared memory, every type, odd pitches and
addresses, absent and repeated entries, masked rows full of NaN, masks of -inf and of the type's
lowest value, ties, and gradients against differences."""
import numpy as np
import pytest
import torch

import lm_reference as ref
from paper_1805_08469_gb300 import lm

pytestmark = pytest.mark.gpu

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
INF = float("inf")


def rows(v, dtype, pad=0, shift=0):
    """[N, V] CUDA tensor of these values with a pitch of V + pad, `shift` elements into its buffer."""
    N, V = v.shape
    buf = torch.full((N * (V + pad) + shift + 8,), float("nan"), dtype=DTYPES[dtype], device="cuda")
    t = buf[shift:shift + N * (V + pad)].view(N, V + pad)[:, :V]
    t.copy_(torch.from_numpy(v))
    return t


def host(t):
    return None if t is None else t.detach().double().cpu().numpy()


def ints(a):
    return torch.as_tensor(np.asarray(a), dtype=torch.int32).cuda()


def floats(a):
    return torch.as_tensor(np.asarray(a, dtype=np.float32)).cuda()


# ---------------------------------------------------------------------- token log probabilities


def logp_run(z, tokens, tau=1.0, K=0, dlogp=None, dentropy=None, grad=None):
    N, V = z.shape
    out = {k: torch.full((N,), float("nan"), device="cuda") for k in ("logp", "entropy", "lse")}
    if K:
        out["top_idx"] = torch.full((N, K), -7, dtype=torch.int32, device="cuda")
        out["top_logp"] = torch.full((N, K), float("nan"), device="cuda")
    lm.gem_token_logp(z, tokens, out["logp"], out["entropy"], temperature=tau, lse=out["lse"], top_idx=out.get("top_idx"),
                      top_logp=out.get("top_logp"))
    if dlogp is not None or dentropy is not None:
        out["grad"] = torch.full_like(z, float("nan")) if grad is None else grad
        lm.gem_token_logp_grad(z, tokens, out["lse"], out["entropy"], dlogp, dentropy, out["grad"], temperature=tau)
    torch.cuda.synchronize()
    return {k: v.cpu().numpy() if v.dtype == torch.int32 else host(v) for k, v in out.items()}


def logp_check(v, dtype, tau=1.0, K=0, pad=0, shift=0, seed=0, grad=True, tokens=None):
    rng = np.random.default_rng(seed)
    N, V = v.shape
    z = rows(v, dtype, pad, shift)
    y = rng.integers(0, V, N) if tokens is None else np.asarray(tokens)
    dl, dH = (floats(rng.standard_normal(N)), floats(0.1 * rng.standard_normal(N))) if grad else (None, None)
    got = logp_run(z, ints(y), tau, K, dl, dH)
    tau = float(np.float32(tau))
    want = ref.token_logp(host(z), y, tau, K, host(dl), host(dH), dtype)
    for k in got:
        ref.check(got[k], want[k], k)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("V", [1, 2, 7, 8, 9, 31, 33, 255, 256, 257, 1000, 1023, 4097, 10007, 32000, 50001])
def test_vocabularies(V, dtype):
    rng = np.random.default_rng(V)
    logp_check(3 * rng.standard_normal((3, V)), dtype, K=min(V, 20), seed=V)


@pytest.mark.parametrize("dtype,V", [("bf16", 131072), ("f16", 131073), ("f32", 100003), ("f32", 262144), ("bf16", 262147),
                                     ("f32", 500009), ("f16", 1100001)])
def test_large_vocabularies(dtype, V):
    """Rows up to and past what the blocks of a cluster hold on chip together."""
    rng = np.random.default_rng(V)
    logp_check(2 * rng.standard_normal((2, V)), dtype, K=64, seed=V, tau=0.8)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("K", [1, 2, 5, 31, 32, 33, 64, 127, 128, 129, 255, 256])
@pytest.mark.parametrize("V", [256, 1111, 20000])
def test_numbers_of_alternatives(K, V, dtype):
    rng = np.random.default_rng(K)
    logp_check(2 * rng.standard_normal((2, V)), dtype, K=K, grad=False)


@pytest.mark.parametrize("N", [1, 2, 31, 700, 3000])
def test_numbers_of_rows(N):
    rng = np.random.default_rng(N)
    logp_check(2 * rng.standard_normal((N, 517)), "bf16", K=4, seed=N)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("pad,shift", [(0, 1), (1, 0), (3, 3), (8, 0), (8, 5), (7, 2)])
@pytest.mark.parametrize("V", [5, 1001, 40000])
def test_pitches_and_addresses(V, pad, shift, dtype):
    """Rows that start anywhere between 16-byte boundaries; what lies between the rows is NaN."""
    rng = np.random.default_rng(V + pad)
    logp_check(2 * rng.standard_normal((4, V)), dtype, K=5, pad=pad, shift=shift, tau=1.3)


@pytest.mark.parametrize("tau", [1e-3, 0.05, 0.7, 1.0, 3.0, 1e4])
def test_temperatures(tau):
    rng = np.random.default_rng(4)
    logp_check(3 * rng.standard_normal((3, 1500)), "f32", tau=tau, K=10)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("V", [300, 9000, 50001])
def test_tokens_and_masks(V, dtype):
    """Positions without a token, tokens outside the vocabulary, logits masked with -inf and with the
    type's lowest value, rows that masks leave nothing or one entry of, logits far apart."""
    rng = np.random.default_rng(V)
    low = float(torch.finfo(DTYPES[dtype]).min)
    v = 2 * rng.standard_normal((9, V))
    v[1, rng.random(V) < 0.7] = -INF
    v[2, rng.random(V) < 0.7] = low
    v[3] = -INF
    v[4] = low
    v[5] = -INF
    v[5, V // 3] = 1.5
    v[6] = np.where(np.arange(V) < 4, [[50000.0, 49984.0, -50000.0, 0.0]][0] + [0] * (V - 4), -60000.0)
    v[7] = low
    v[7, V - 1] = 3.0
    y = np.array([-1, 5, V, 3, 0, V // 3, 1, V - 1, -2147483648])
    z = rows(v, dtype)
    dl, dH = floats(np.arange(1, 10)), floats(np.full(9, 0.1))
    got = logp_run(z, ints(y), 1.0, 10, dl, dH)
    want = ref.token_logp(host(z), y, 1.0, 10, host(dl), host(dH), dtype)
    for k in got:
        ref.check(got[k], want[k], k)
    assert got["entropy"][3] == 0 and np.all(got["top_logp"][3] == -INF)
    assert np.array_equal(got["top_idx"][3], np.arange(10)) and np.array_equal(got["top_idx"][4], np.arange(10))


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("V", [300, 33000])
def test_rows_that_are_not_finite(V, dtype):
    """A NaN or +inf makes its own row's values NaN and no other's; the order puts NaN first."""
    rng = np.random.default_rng(V)
    v = rng.standard_normal((6, V))
    v[1, [V - 2, 0, 77]] = np.nan
    v[2, 200] = INF
    v[3] = np.nan
    v[4, :] = -INF
    v[4, 99] = np.nan
    z = rows(v, dtype)
    y = np.full(6, 3)
    got = logp_run(z, ints(y), 1.0, 5, floats(np.ones(6)), floats(np.ones(6)))
    good = [0, 5]
    want = ref.token_logp(host(z)[good], y[good], 1.0, 5, np.ones(2), np.ones(2), dtype)
    for k in got:
        ref.check(got[k][good], want[k], k)
        if k != "top_idx":
            assert np.isnan(got[k][1:5]).all(), k
    zh = host(z)
    for n in range(6):
        nan_first = sorted(range(V), key=lambda j: (0 if np.isnan(zh[n, j]) else 1, 0 if np.isnan(zh[n, j]) else -zh[n, j], j))
        assert list(got["top_idx"][n]) == nan_first[:5], n


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("V", [64, 1000, 33333, 131072])
def test_ties_and_adverse_orders(V, dtype):
    """Equal logits by index; all alike; both zeros; few values; ascending, descending; the large
    ones gathered at one place or at one distance (one thread's, one warp's) from one another."""
    rng = np.random.default_rng(V)
    j = np.arange(V)
    v = [np.zeros(V), np.where(j % 2 == 0, -0.0, 0.0), rng.integers(0, 3, V), rng.integers(-4, 4, V) / 4, j / V, -j / V,
         np.where(j == V // 2, 1.0, 0.0), np.where(j < 40, 5.0, 0.0), np.where(j >= V - 40, 5.0, 0.0)]
    for step in (8, 32, 256, 1024, 2048, 4096, 8192):
        v.append(np.where(j % step == min(3, V - 1), 10 + (j // step % 13) / 8, rng.standard_normal(V)))
        v.append(np.where(j % step < 8, 10 + rng.standard_normal(V), rng.standard_normal(V)))
    for K in (1, 20, 64):
        logp_check(np.stack(v), dtype, K=K, grad=False)


def test_log_probabilities_of_optional_outputs_and_in_place_gradient():
    rng = np.random.default_rng(5)
    z = rows(rng.standard_normal((4, 900)), "bf16", pad=4)
    y = ints([1, 2, 3, 4])
    full = logp_run(z, y, 1.0, 7, floats(np.ones(4)), floats(np.ones(4)))
    e = torch.empty(4, device="cuda")
    lm.gem_token_logp(z, None, None, e)
    assert np.array_equal(host(e), full["entropy"])
    lm.gem_token_logp(z, y, e)
    assert np.array_equal(host(e), full["logp"])
    i, t = torch.empty((4, 7), dtype=torch.int32, device="cuda"), torch.empty((4, 7), device="cuda")
    lm.gem_token_logp(z, top_idx=i, top_logp=t)
    assert np.array_equal(i.cpu().numpy(), full["top_idx"]) and np.array_equal(host(t), full["top_logp"])
    lse, H = floats(full["lse"]), floats(full["entropy"])
    a, b = torch.empty_like(z), torch.empty_like(z)
    lm.gem_token_logp_grad(z, y, lse, None, floats(np.ones(4)), None, a)
    want = ref.token_logp(host(z), [1, 2, 3, 4], 1.0, 0, np.ones(4), None, "bf16")
    ref.check(host(a), want["grad"], "grad")
    lm.gem_token_logp_grad(z, None, lse, H, None, floats(np.ones(4)), b)
    want = ref.token_logp(host(z), [-1] * 4, 1.0, 0, None, np.ones(4), "bf16")
    ref.check(host(b), want["grad"], "grad")
    lm.gem_token_logp_grad(z, y, lse, H, floats(np.ones(4)), floats(np.ones(4)), z)
    assert np.array_equal(host(z), full["grad"])


def test_one_row_of_logits_for_all():
    rng = np.random.default_rng(6)
    z = rows(rng.standard_normal((1, 700)), "f32").expand(5, 700)
    got = logp_run(z, ints([0, 1, 2, 3, 699]), 1.0, 3)
    want = ref.token_logp(host(z), [0, 1, 2, 3, 699], 1.0, 3)
    for k in got:
        ref.check(got[k], want[k], k)


def test_offsets_past_32_bits():
    """Rows more than 2^32 elements apart."""
    far = (1 << 32) + 12345
    if torch.cuda.mem_get_info()[0] < 6 * far:
        pytest.skip("needs 26 GB of device memory")
    buf = torch.zeros(far + 1000, dtype=torch.bfloat16, device="cuda")
    z = buf.as_strided((2, 1000), (far, 1))
    z.copy_(torch.randn((2, 1000), device="cuda"))
    dl = np.ones(2)
    got = logp_run(z, ints([7, 999]), 1.0, 5, floats(dl), None, grad=z.clone().contiguous())
    want = ref.token_logp(host(z), [7, 999], 1.0, 5, dl, None, "bf16")
    for k in got:
        ref.check(got[k], want[k], k)


# ---------------------------------------------------------------------- distillation


def distill_inputs(seed, N, V, K, dtype, tau=1.0, tail=False, absent=True, pad=0, shift=0):
    rng = np.random.default_rng(seed)
    K_ = min(K, V)
    idx = np.stack([rng.choice(V, K_, replace=False) for _ in range(N)]) if K_ else np.zeros((N, 0))
    if K > K_:
        idx = np.concatenate([idx, np.full((N, K - K_), -1)], 1)
    top = 2 + 2 * rng.standard_normal((N, K))
    v = 2 * rng.standard_normal((N, V))
    for n in range(N):
        for k in range(K_):
            v[n, idx[n, k]] += 0.5 * top[n, k]
    if absent and N > 1 and K:
        idx[1, rng.random(K) < 0.5] = -1
        if N > 2:
            idx[2, :] = -1
        if N > 3:
            idx[3, ::2] = np.where(np.arange(len(idx[3, ::2])) % 2, V, 2147483647)
            top[3, 1::3] = -INF
    top = top.astype(np.float32)
    lse = None
    if tail:
        full = np.log(np.exp(top.astype(np.float64) / tau).sum(1) + 1e-30) - np.log1p(-rng.uniform(0.001, 0.4, N))
        lse = full.astype(np.float32)
    return rows(v, dtype, pad, shift), idx.astype(np.int32), top, lse


def distill_run(z, idx, top, tau=1.0, alpha=0.0, lse=None, labels=None, scale=None, grad="new"):
    loss = torch.full((z.shape[0],), float("nan"), device="cuda")
    g = torch.full_like(z, float("nan")) if isinstance(grad, str) else grad
    lm.gem_distill(z, ints(idx), floats(top), loss, g, teacher_lse=None if lse is None else floats(lse),
                   labels=None if labels is None else ints(labels), row_scale=None if scale is None else floats(scale),
                   temperature=tau, alpha=alpha)
    torch.cuda.synchronize()
    return {"loss": host(loss)} | ({} if g is None else {"grad": host(g)})


def distill_check(z, dtype, idx, top, tau=1.0, alpha=0.0, lse=None, labels=None, scale=None):
    want = ref.distill(host(z), idx, top, float(np.float32(tau)), float(np.float32(alpha)), lse, labels,
                       None if scale is None else np.asarray(scale, np.float32), dtype)
    got = distill_run(z, idx, top, tau, alpha, lse, labels, scale)
    for k in want:
        ref.check(got[k], want[k], k)
    return got


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("V", [1, 2, 9, 33, 257, 1000, 4097, 32000, 50001])
def test_distill_vocabularies(V, dtype, tail):
    K = min(V, 20)
    z, idx, top, lse = distill_inputs(V, 5, V, K, dtype, tail=tail)
    distill_check(z, dtype, idx, top, lse=lse)


@pytest.mark.parametrize("dtype,V", [("bf16", 131072), ("f16", 131073), ("f32", 100003), ("f32", 262144), ("f32", 500009), ("f16", 1100001)])
def test_distill_large_vocabularies(dtype, V):
    z, idx, top, lse = distill_inputs(V, 2, V, 128, dtype, tau=2.0, tail=True)
    distill_check(z, dtype, idx, top, 2.0, 0.25, lse, [3, V - 1])
    distill_check(z, dtype, idx, top, 1.0, 0.0)


@pytest.mark.parametrize("K", [0, 1, 2, 31, 32, 33, 100, 255, 256])
@pytest.mark.parametrize("tail", [False, True])
def test_distill_numbers_of_entries(K, tail):
    z, idx, top, lse = distill_inputs(K, 4, 777, K, "f32", tail=tail)
    distill_check(z, "f32", idx, top, lse=lse)


def test_more_entries_than_the_vocabulary():
    z, idx, top, _ = distill_inputs(1, 4, 5, 9, "f32")
    distill_check(z, "f32", idx, top)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("tau,alpha", [(1.0, 0.5), (2.0, 0.3), (0.5, 0.9), (4.0, 0.0), (3.0, 1.0)])
@pytest.mark.parametrize("tail", [False, True])
def test_temperatures_and_labels(dtype, tau, alpha, tail):
    z, idx, top, lse = distill_inputs(3, 6, 1300, 16, dtype, tau=tau, tail=tail)
    labels = [5, idx[1, 0] if idx[1, 0] >= 0 else 0, -1, 1299, 1300, -100]
    distill_check(z, dtype, idx, top, tau, alpha, lse, labels, [1.0, 0.5, 2.0, 1e-3, 1.0, -1.0])


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("pad,shift", [(0, 1), (1, 0), (3, 3), (8, 0), (7, 2)])
@pytest.mark.parametrize("V", [5, 1001, 40000])
def test_distill_pitches_and_addresses(V, pad, shift, dtype):
    z, idx, top, lse = distill_inputs(V, 4, V, min(V, 6), dtype, tail=True, pad=pad, shift=shift)
    want = ref.distill(host(z), idx, top, 1.0, 0.0, lse, dtype=dtype)
    got = distill_run(z, idx, top, lse=lse)
    for k in want:
        ref.check(got[k], want[k], k)
    # the gradient in rows of another pitch and address, and what lies between them untouched
    N = 4
    buf = torch.full((N * (V + 5) + 3,), 7.0, dtype=DTYPES[dtype], device="cuda")
    g = buf[3:].view(N, V + 5)[:, :V]
    got2 = distill_run(z, idx, top, lse=lse, grad=g)
    assert np.array_equal(got2["grad"], got["grad"])
    assert bool((buf[:3] == 7).all()) and bool((buf[3:].view(N, V + 5)[:, V:] == 7).all())
    # in place
    got3 = distill_run(z, idx, top, lse=lse, grad=z)
    assert np.array_equal(got3["grad"], got["grad"]) and np.array_equal(got3["loss"], got["loss"])


def test_loss_without_a_gradient():
    z, idx, top, lse = distill_inputs(2, 5, 3001, 10, "bf16", tail=True)
    a, b = distill_run(z, idx, top, lse=lse), distill_run(z, idx, top, lse=lse, grad=None)
    assert np.array_equal(a["loss"], b["loss"])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tail", [False, True])
def test_entries_with_the_same_index_add_up(dtype, tail):
    z, idx, top, lse = distill_inputs(4, 5, 500, 12, dtype, tail=tail, absent=False)
    idx[0, :] = 7
    idx[1, ::2] = 499
    idx[2, 3:6] = [0, 0, 1]
    distill_check(z, dtype, idx, top, lse=lse)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("V", [300, 20001])
def test_masked_rows_and_logits(V, dtype):
    """Rows whose scale is 0 hold NaN and give zeros; logits of -inf and of the type's lowest value, on
    and off the teacher's entries; rows with nothing left."""
    low = float(torch.finfo(DTYPES[dtype]).min)
    for tail in (False, True):
        z, idx, top, lse = distill_inputs(V, 9, V, 8, dtype, tail=tail, absent=False)
        off = torch.ones((9, V), dtype=torch.bool, device="cuda").scatter_(1, ints(idx).long(), False)
        z[0] = float("nan")
        z[1][off[1] & (torch.rand(V, device="cuda") < 0.6)] = -INF
        z[2][off[2] & (torch.rand(V, device="cuda") < 0.6)] = low
        z[3][off[3]] = -INF            # only the teacher's entries are left
        z[4, int(idx[4, 2])] = -INF    # the teacher gives mass to what the student masks
        z[5] = -INF
        z[6] = low
        z[7][~off[7]] = -INF           # only what is not the teacher's
        scale = np.array([0, 1, 1, 1, 1, 1, 1, 1, 0], np.float32)
        got = distill_check(z, dtype, idx, top, lse=lse, scale=scale)
        assert np.all(got["grad"][[0, 8]] == 0) and np.all(got["loss"][[0, 8]] == 0)
        assert np.isposinf(got["loss"][[4, 5, 7]]).all()


def test_confident_student_and_teacher():
    """Almost all mass on the entries on both sides: the rest is a sum of its own, not 1 - sum p."""
    rng = np.random.default_rng(8)
    N, V, K = 4, 5000, 4
    v = rng.standard_normal((N, V))
    idx = np.stack([rng.choice(V, K, replace=False) for _ in range(N)]).astype(np.int32)
    for n in range(N):
        v[n, idx[n]] = 25 + rng.standard_normal(K)
    top = rng.standard_normal((N, K)).astype(np.float32)
    lse = (np.log(np.exp(top.astype(np.float64)).sum(1)) - np.log1p(-np.array([0.3, 0.1, 0.02, 0.5]))).astype(np.float32)
    distill_check(rows(v, "f32"), "f32", idx, top, lse=lse)


def test_a_row_of_nan_stays_its_own():
    z, idx, top, lse = distill_inputs(9, 4, 2000, 8, "f32", absent=False)
    want = distill_run(z, idx, top)
    z[1, 1500] = float("nan")
    z[2, 3] = INF
    got = distill_run(z, idx, top)
    for k in got:
        assert np.isnan(got[k][1:3]).all() and np.array_equal(got[k][[0, 3]], want[k][[0, 3]])


@pytest.mark.parametrize("tail", [False, True])
def test_distill_gradient_against_differences(tail):
    z, idx, top, lse = distill_inputs(10, 4, 400, 10, "f32", tau=1.5, tail=tail)
    labels, scale = [5, -1, 7, int(idx[3, 1])], np.array([1.0, 0.5, 2.0, 1.0], np.float32)
    got = distill_run(z, idx, top, 1.5, 0.25, lse, labels, scale)["grad"]
    rng = np.random.default_rng(11)
    zh = host(z)

    def value(v):
        return (ref.distill(v, idx, top, 1.5, 0.25, lse, labels, scale)["loss"][0] * scale).sum()

    for _ in range(5):
        v = rng.standard_normal(zh.shape)
        slope = (value(zh + 1e-4 * v) - value(zh - 1e-4 * v)) / 2e-4
        # truncation below step^2 times third derivatives of order 1; fp32 gradients
        assert abs((got * v).sum() - slope) <= 1e-5 * np.abs(got * v).sum() + 1e-6


def test_log_probability_gradient_against_differences():
    rng = np.random.default_rng(12)
    z = rows(rng.standard_normal((3, 300)), "f32")
    y, dl, dH = [4, -1, 299], rng.standard_normal(3), rng.standard_normal(3)
    got = logp_run(z, ints(y), 0.8, 0, floats(dl), floats(dH))["grad"]
    zh = host(z)
    dl, dH = np.float32(dl), np.float32(dH)

    def value(v):
        r = ref.token_logp(v, y, float(np.float32(0.8)), 0)
        return (r["logp"][0] * dl + r["entropy"][0] * dH).sum()

    for _ in range(5):
        v = rng.standard_normal(zh.shape)
        slope = (value(zh + 1e-4 * v) - value(zh - 1e-4 * v)) / 2e-4
        assert abs((got * v).sum() - slope) <= 1e-5 * np.abs(got * v).sum() + 1e-6


def test_runs_repeat_bit_for_bit_on_any_stream():
    z, idx, top, lse = distill_inputs(13, 40, 30001, 50, "bf16", tail=True)
    first, one = distill_run(z, idx, top, 2.0, 0.0, lse), logp_run(z, ints(np.arange(40)), 1.0, 50)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(3):
            again, two = distill_run(z, idx, top, 2.0, 0.0, lse), logp_run(z, ints(np.arange(40)), 1.0, 50)
            assert all(np.array_equal(first[k], again[k]) for k in first)
            assert all(np.array_equal(one[k], two[k]) for k in one)


def test_inside_a_graph():
    z, idx, top, lse = distill_inputs(14, 6, 9001, 20, "f16", tail=True)
    want = distill_run(z, idx, top, lse=lse)
    i, t, l = ints(idx), floats(top), floats(lse)  # noqa: E741
    loss, grad = torch.empty(6, device="cuda"), torch.empty_like(z)
    H = torch.empty(6, device="cuda")

    def calls():
        lm.gem_distill(z, i, t, loss, grad, teacher_lse=l)
        lm.gem_token_logp(grad, None, None, H)

    calls()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        calls()
    want_H = H.clone()
    for x in (loss, grad, H):
        x.fill_(float("nan"))
    g.replay()
    torch.cuda.synchronize()
    assert np.array_equal(host(loss), want["loss"]) and np.array_equal(host(grad), want["grad"]) and torch.equal(H, want_H)


def test_scores_of_a_teacher_feed_the_distillation():
    """The alternatives and log-sum-exp of gem_token_logp are the teacher's entries of gem_distill: a
    student equal to the teacher has a loss and a gradient of zero up to rounding."""
    rng = np.random.default_rng(15)
    z = rows(2 * rng.standard_normal((5, 3000)), "f32")
    K, tau = 32, 2.0
    i, t = torch.empty((5, K), dtype=torch.int32, device="cuda"), torch.empty((5, K), device="cuda")
    lm.gem_token_logp(z, top_idx=i, top_logp=t, temperature=tau)
    loss, grad = torch.empty(5, device="cuda"), torch.empty_like(z)
    lm.gem_distill(z, i, t * tau, loss, grad, teacher_lse=torch.zeros(5, device="cuda"), temperature=tau)
    # log p and q within the bounds of their forms (about 300 U each at this size), times tau^2
    assert float(loss.abs().max()) < 1e-3 * tau * tau and float(grad.abs().max()) < 1e-4
