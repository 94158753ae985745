"""The embedding and its table's gradient against their definitions in 64 bits: every pair of types,
odd widths, strides and alignments, tokens out of range, heavy and absent tokens, orders of tokens."""
import numpy as np
import pytest
import torch

import lm_layers_reference as ref
from lm_reference import check
from paper_1805_08469_gb300 import lm

pytestmark = pytest.mark.gpu

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def matrix(v, dtype, pad=0, shift=0):
    """A CUDA matrix of these values, `pad` elements between rows, `shift` before the first, in a poisoned buffer."""
    N, D = v.shape
    buf = torch.full((N * (D + pad) + shift + 1,), float("nan"), dtype=DTYPES[dtype], device="cuda")
    out = buf[shift:shift + N * (D + pad)].view(N, D + pad)[:, :D]
    out.copy_(torch.from_numpy(np.asarray(v, np.float64)))
    return out


def host(t):
    return t.detach().double().cpu().numpy()


def ints(v):
    return torch.from_numpy(np.asarray(v, np.int32)).cuda()


def grad(dout, tokens, dtable, scale=1.0, accumulate=False):
    (V, D), N = dtable.shape, len(tokens)
    size = lm.gem_embed_workspace(N, V, D)
    space = torch.full((size + 64,), 0xA5, dtype=torch.uint8, device="cuda")
    lm.gem_embed_grad(dout, ints(tokens), dtable, space[:size], scale=scale, accumulate=accumulate)
    torch.cuda.synchronize()
    assert bool((space[size:] == 0xA5).all()), "written past the workspace"


def both(seed, N, V, D, dtype="f32", table="f32", grad_type="f32", pads=(0, 0, 0, 0), shift=0, scale=1.3, tokens=None, accumulate=False):
    rng = np.random.default_rng(seed)
    if tokens is None:
        tokens = rng.integers(0, V, N)
        tokens[rng.random(N) < 0.1] = -1
    tokens = np.asarray(tokens)
    scale = float(np.float32(scale))
    t = matrix(rng.standard_normal((V, D)), table, pads[0], shift)
    out = matrix(np.full((N, D), np.nan), dtype, pads[1], shift)
    lm.gem_embed(t, ints(tokens), out, scale=scale)
    torch.cuda.synchronize()
    check(host(out), ref.embed(host(t), tokens, scale, dtype)["out"], "out")
    dout = matrix(rng.standard_normal((N, D)), dtype, pads[2], shift)
    old = rng.standard_normal((V, D)) if accumulate else np.full((V, D), np.nan)
    dt = matrix(old, grad_type, pads[3], shift)
    before = host(dt) if accumulate else None
    grad(dout, tokens, dt, scale, accumulate)
    check(host(dt), ref.embed_grad(host(dout), tokens, V, scale, grad_type, before)["dtable"], "dtable")


@pytest.mark.parametrize("table", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_types(table, dtype):
    both(1, 70, 40, 96, dtype, table, table)
    both(2, 70, 40, 33, dtype, table, table, accumulate=True)


@pytest.mark.parametrize("D", [1, 2, 3, 4, 7, 8, 31, 32, 64, 100, 127, 128, 129, 255, 256, 257, 512, 1000, 1001, 2056])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_widths(D, dtype):
    both(D, 90, 23, D, dtype, accumulate=D % 2 == 0)


@pytest.mark.parametrize("N", [1, 2, 31, 32, 33, 63, 64, 65, 255, 256, 257, 1000, 1023, 1025, 5000])
@pytest.mark.parametrize("V", [1, 2, 511, 513])
def test_counts(N, V):
    both(N, N, V, 40, "bf16")


@pytest.mark.parametrize("pads", [(1, 0, 0, 0), (0, 1, 0, 0), (0, 0, 1, 0), (0, 0, 0, 1), (8, 8, 8, 8), (3, 5, 7, 9)])
@pytest.mark.parametrize("shift", [0, 1, 4])
@pytest.mark.parametrize("dtype", ["f32", "f16"])
def test_layouts(pads, shift, dtype):
    """Row pitches and first elements off the boundaries that wide loads want; nothing between the rows is touched."""
    both(7, 130, 61, 264, dtype, dtype, "f32", pads, shift)
    both(8, 130, 61, 67, dtype, "f32", dtype, pads, shift, accumulate=True)
    buf = torch.full((61, 80), 5.0, device="cuda")
    grad(matrix(np.ones((9, 64)), dtype), np.arange(9) * 5, buf[:, 8:72])
    assert bool((buf[:, :8] == 5).all() and (buf[:, 72:] == 5).all())


@pytest.mark.parametrize("kind", ["all one", "two", "sorted", "reversed", "none", "heavy", "first and last", "distinct"])
@pytest.mark.parametrize("N,V", [(1000, 700), (20000, 50000), (40001, 300)])
def test_orders_of_tokens(kind, N, V):
    rng = np.random.default_rng(N)
    t = rng.integers(0, V, N)
    t = {"all one": np.full(N, V // 2), "two": np.where(rng.random(N) < 0.5, 0, V - 1), "sorted": np.sort(t), "reversed": np.sort(t)[::-1],
         "none": np.full(N, -1), "heavy": np.where(rng.random(N) < 0.6, 7, t), "first and last": np.where(np.arange(N) % 3 == 0, 0, V - 1),
         "distinct": np.arange(N) * 7 % V}[kind]
    both(N, N, V, 24, "f16", tokens=t)
    both(N + 1, N, V, 9, "f32", tokens=t, accumulate=True)


@pytest.mark.parametrize("V", [255, 256, 257, 65535, 65536, 262145, 3000001])
def test_large_tables(V):
    rng = np.random.default_rng(V)
    t = np.concatenate([rng.integers(0, V, 700), [0, V - 1, V - 1, 0, -1, -5]])
    both(V, len(t), V, 16 if V > 1000000 else 40, "bf16", tokens=t)


@pytest.mark.parametrize("D", [3, 8])
def test_many_tokens(D):
    """More chunks than the blocks look at once, with runs of one chunk, of two and of thousands."""
    rng = np.random.default_rng(D)
    N, V = 480001, 150000
    t = np.minimum(rng.integers(0, V, N), (V * rng.random(N) ** 4).astype(np.int64))
    t[rng.random(N) < 0.2] = 77777
    both(D, N, V, D, "bf16", tokens=t, accumulate=D == 8)


def test_tokens_out_of_range():
    """Negative ones have no row; those past the table give NaN, and no gradient; what dout holds there is not used."""
    tokens = np.array([0, -1, 5, 6, -2**31, 2**31 - 1, 3, 3])
    table = matrix(np.random.default_rng(0).standard_normal((6, 20)), "f32")
    out = torch.empty((8, 20), device="cuda")
    lm.gem_embed(table, ints(tokens), out)
    check(host(out), ref.embed(host(table), tokens, 1.0, "f32")["out"], "out")
    dout = matrix(np.random.default_rng(1).standard_normal((8, 20)), "f32")
    want = ref.embed_grad(host(dout), tokens, 6, 1.0, "f32")["dtable"]
    for i in (1, 3, 4, 5):
        dout[i] = float("nan")
    dt = torch.full((6, 20), float("nan"), device="cuda")
    grad(dout, tokens, dt)
    check(host(dt), want, "dtable")


def test_infinities_and_nan_stay_in_their_rows():
    dout = torch.ones((40, 48), device="cuda")
    dout[3] = float("nan")
    dout[7] = float("inf")
    dt = torch.empty((40, 48), device="cuda")
    grad(dout, np.arange(40) // 2, dt)
    assert bool(dt[1].isnan().all() and dt[3].isinf().all())
    dt[[1, 3]] = 2.0
    assert bool((dt[:20] == 2).all() and (dt[20:] == 0).all())


def test_empty_sizes():
    dt = torch.full((5, 12), float("nan"), device="cuda")
    grad(torch.empty((0, 12), device="cuda"), np.zeros(0), dt)
    assert bool((dt == 0).all())
    dt.fill_(3.0)
    grad(torch.empty((0, 12), device="cuda"), np.zeros(0), dt, accumulate=True)
    assert bool((dt == 3).all())
    grad(torch.empty((4, 0), device="cuda"), np.arange(4), torch.empty((5, 0), device="cuda"))
    lm.gem_embed(torch.empty((5, 0), device="cuda"), ints(np.arange(4)), torch.empty((4, 0), device="cuda"))


def test_the_same_bits_every_time():
    """Whatever else runs, and whatever the workspace held."""
    rng = np.random.default_rng(5)
    t = np.minimum(rng.zipf(1.3, 30000) - 1, 8999)
    dout = torch.randn((30000, 136), device="cuda").bfloat16()
    first = torch.empty((9000, 136), device="cuda")
    grad(dout, t, first)
    size = lm.gem_embed_workspace(30000, 9000, 136)
    for k in range(3):
        space = torch.randint(0, 256, (size,), dtype=torch.uint8, device="cuda")
        again = torch.full_like(first, float("nan"))
        lm.gem_embed_grad(dout, ints(t), again, space)
        assert torch.equal(first, again)


def test_offsets_past_32_bits():
    """Rows that begin more than 2^31 elements into the table and the gradients."""
    V, D = 70001, 32768
    free = torch.cuda.mem_get_info()[0]
    if free < 24 << 30:
        pytest.skip("needs 24 GB")
    table = torch.zeros((V, D), dtype=torch.bfloat16, device="cuda")
    table[V - 1] = 1.5
    table[65537] = 2.5
    out = torch.empty((3, D), dtype=torch.bfloat16, device="cuda")
    tokens = ints([V - 1, 65537, 0])
    lm.gem_embed(table, tokens, out, scale=2.0)
    assert bool((out[0] == 3).all() and (out[1] == 5).all() and (out[2] == 0).all())
    table.fill_(7.0)
    grad(out, [V - 1, 65537, V - 1], table)
    assert bool((table[V - 1] == 3).all() and (table[65537] == 5).all() and (table[:65537] == 0).all() and (table[65538:V - 1] == 0).all())
