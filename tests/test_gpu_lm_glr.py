"""The gated linear recurrence against its definition in 64 bits: lengths from none to long ones,
odd channel counts, every type, strided tensors, resets and ragged lengths with poison in the
places they hide, the state carried from call to call, and the gradients against differences."""
import numpy as np
import pytest
import torch

import lm_reference as ref
from paper_1805_08469_gb300 import lm

pytestmark = pytest.mark.gpu

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
FORMS = {"lerp": lm.GEM_GLR_LERP, "add": lm.GEM_GLR_ADD}


def place(v, dtype, layout):
    """A CUDA tensor of these values in one of several memory layouts, in a poisoned buffer."""
    B, T, D = v.shape
    t = DTYPES[dtype]
    if layout == "time_major":
        out = torch.full((T, B, D), float("nan"), dtype=t, device="cuda").transpose(0, 1)
    elif layout == "half":
        out = torch.full((B, T, 2 * D), float("nan"), dtype=t, device="cuda")[..., D:]
    elif layout == "odd":
        out = torch.full((B, T + 1, D + 3), float("nan"), dtype=t, device="cuda")[:, 1:, 1:D + 1]
    else:
        out = torch.full((B, T, D), float("nan"), dtype=t, device="cuda")
    out.copy_(torch.from_numpy(v))
    return out


def host(t):
    return None if t is None else t.detach().double().cpu().numpy()


class Case:
    def __init__(self, seed, B, T, D, dtype, form="lerp", h0=True, lengths=None, resets=0.0, layout="dense"):
        rng = np.random.default_rng(seed)
        self.dims, self.dtype, self.form, self.layout = (B, T, D), dtype, form, layout
        self.x = place(rng.standard_normal((B, T, D)), dtype, layout)
        self.f = place(1.5 * rng.standard_normal((B, T, D)) + rng.uniform(-2, 6, D), dtype, layout)
        self.dh = place(rng.standard_normal((B, T, D)), dtype, layout)
        self.h0 = torch.from_numpy(rng.standard_normal((B, D)).astype(np.float32)).cuda() if h0 else None
        self.dh_last = torch.from_numpy(rng.standard_normal((B, D)).astype(np.float32)).cuda() if h0 else None
        self.lengths = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda")
        self.reset = None
        if resets:
            self.reset = torch.from_numpy((rng.random((B, T)) < resets).astype(np.uint8)).cuda()

    def run(self, backward=True):
        B, T, D = self.dims
        new = lambda: place(np.zeros((B, T, D)), self.dtype, self.layout).fill_(float("nan"))  # noqa: E731
        out = {"h": new(), "h_last": torch.full((B, D), float("nan"), device="cuda"),
               "saved": torch.full((B, -(-T // 16), D), float("nan"), device="cuda")}
        lm.gem_glr_forward(self.x, self.f, out["h"], form=FORMS[self.form], h0=self.h0, lengths=self.lengths, reset=self.reset,
                           h_last=out["h_last"], saved=out["saved"])
        if backward:
            out |= {"dx": new(), "df": new(), "dh0": torch.full((B, D), float("nan"), device="cuda")}
            lm.gem_glr_backward(self.x, self.f, out["saved"], self.dh, out["dx"], out["df"], form=FORMS[self.form], lengths=self.lengths,
                                reset=self.reset, dh_last=self.dh_last, dh0=out["dh0"])
        torch.cuda.synchronize()
        return {k: host(v) for k, v in out.items()}

    def reference(self):
        return ref.glr(host(self.x), host(self.f), self.form == "lerp", host(self.h0),
                       None if self.lengths is None else self.lengths.cpu().numpy(),
                       None if self.reset is None else self.reset.cpu().numpy(), host(self.dh), host(self.dh_last), self.dtype)

    def check(self):
        got, want = self.run(), self.reference()
        for k in want:
            ref.check(got[k], want[k], k)


@pytest.mark.parametrize("form", ["lerp", "add"])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("T", [1, 2, 15, 16, 17, 127, 128, 129, 300])
def test_lengths_of_time(T, dtype, form):
    Case(T, 2, T, 66, dtype, form).check()


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("D", [1, 2, 3, 31, 32, 33, 63, 64, 65, 127, 200, 513, 1000])
def test_channel_counts(D, dtype):
    Case(D, 3, 45, D, dtype, resets=0.05).check()


@pytest.mark.parametrize("dtype,T,D", [("f32", 5000, 7), ("f32", 2049, 256), ("bf16", 4097, 96), ("f16", 1777, 130), ("bf16", 9001, 2)])
def test_long_sequences(dtype, T, D):
    Case(T, 1, T, D, dtype, resets=0.002).check()


@pytest.mark.parametrize("B,T,D", [(1, 700, 2048), (40, 257, 64), (9, 513, 640), (300, 33, 70), (700, 1, 65)])
def test_many_and_few_channels(B, T, D):
    """Shapes for which the work is split over time, over channels, and not at all."""
    for dtype in ("f32", "bf16"):
        Case(B, B, T, D, dtype, "add" if B > 9 else "lerp", resets=0.01).check()


@pytest.mark.parametrize("layout", ["time_major", "half", "odd"])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("D", [64, 37])
def test_layouts(layout, dtype, D):
    Case(5, 3, 150, D, dtype, layout=layout, resets=0.03).check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_no_initial_state_and_no_last_gradient(dtype):
    Case(6, 2, 100, 40, dtype, h0=False).check()


@pytest.mark.parametrize("form", ["lerp", "add"])
@pytest.mark.parametrize("dtype", ["f32", "f16"])
def test_ragged_lengths_hide_what_lies_past_them(dtype, form):
    """Empty, single, chunk-edge and full sequences; a length outside the range is clipped; NaN and
    infinities past the length reach no output."""
    lengths = [0, 1, 15, 16, 17, 128, 129, 333, -3, 1000]
    c = Case(7, len(lengths), 333, 48, dtype, form, lengths=lengths, resets=0.02)
    clean = c.run()
    for b, n in enumerate(lengths):
        n = min(max(n, 0), 333)
        for t, v in ((c.x, float("nan")), (c.f, float("inf")), (c.dh, float("nan"))):
            t[b, n:] = v
    got, want = c.run(), None
    for k in got:
        assert np.array_equal(got[k], clean[k]), k
    x, f, dh = host(c.x), host(c.f), host(c.dh)
    want = ref.glr(np.nan_to_num(x), np.clip(f, -50, 50), form == "lerp", host(c.h0), np.array(lengths), c.reset.cpu().numpy(),
                   np.nan_to_num(dh), host(c.dh_last), dtype)
    for k in want:
        ref.check(got[k], want[k], k)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("T", [40, 400])
def test_a_reset_drops_any_state(bad, T):
    """A state that holds NaN or infinity ends at a reset, in the forward and the backward pass."""
    c = Case(8, 2, T, 33, "f32", "add")
    cut = T // 2 + 3
    c.reset = torch.zeros((2, T), dtype=torch.uint8, device="cuda")
    c.reset[:, cut] = 255
    c.h0[0] = bad
    c.x[1, 3] = bad
    got = c.run()
    assert not np.isfinite(got["h"][0, :cut]).any() and not np.isfinite(got["h"][1, 3:cut]).any()
    clean = Case(8, 2, T, 33, "f32", "add")
    clean.reset = c.reset
    want = clean.reference()
    for k, part in (("h", np.s_[:, cut:]), ("dx", np.s_[:, :]), ("df", np.s_[:, cut:]), ("h_last", np.s_[:])):
        ref.check(got[k][part], (want[k][0][part], np.broadcast_to(want[k][1], want[k][0].shape)[part]), k)
    # backward: a gradient that is not finite after the reset does not reach what lies before it
    c = Case(8, 2, T, 33, "f32", "add")
    c.reset = clean.reset
    c.dh[:, cut + 2] = bad
    got = c.run()
    ref.check(got["dx"][:, :cut], (want["dx"][0][:, :cut], np.broadcast_to(want["dx"][1], want["dx"][0].shape)[:, :cut]), "dx")
    assert np.isfinite(got["dh0"]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_gates_at_their_ends(dtype):
    """Gates of 0 and 1, to infinity: nothing but the formula's values, and no NaN."""
    big = 3e38 if dtype == "f32" else 6e4 if dtype == "f16" else 3e38
    vals = np.array([-np.inf, -big, -200.0, -88.0, -30.0, -1e-30, 0.0, 1e-30, 30.0, 88.0, 200.0, big, np.inf])
    c = Case(9, 2, 40, len(vals), dtype)
    c.f.copy_(torch.from_numpy(np.broadcast_to(vals, (2, 40, len(vals))).copy()))
    got, want = c.run(), c.reference()
    for k in want:
        ref.check(got[k], (want[k][0], want[k][1] + 1e-30), k)


def test_no_steps():
    """T = 0: the state and its gradient pass through."""
    x = torch.empty((3, 0, 5), device="cuda")
    h0 = torch.randn((3, 5), device="cuda")
    out = torch.full((3, 5), float("nan"), device="cuda")
    lm.gem_glr_forward(x, x, x, h0=h0, h_last=out, saved=torch.empty((3, 0, 5), device="cuda"))
    assert torch.equal(out, h0)
    lm.gem_glr_forward(x, x, x, h_last=out)
    assert torch.equal(out, torch.zeros_like(out))
    out.fill_(float("nan"))
    lm.gem_glr_backward(x, x, torch.empty((3, 0, 5), device="cuda"), x, x, x, dh_last=h0, dh0=out)
    assert torch.equal(out, h0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("cuts", [[0, 1, 2, 3, 30], [0, 16, 30], [0, 7, 30]])
def test_the_state_goes_on_in_place(dtype, cuts):
    """A sequence in several calls whose h_last is their h0: the same bound as in one call."""
    c = Case(10, 2, 30, 70, dtype)
    want = c.reference()
    state = c.h0.clone()
    parts = []
    for a, b in zip(cuts, cuts[1:]):
        h = torch.empty((2, b - a, 70), dtype=DTYPES[dtype], device="cuda")
        lm.gem_glr_forward(c.x[:, a:b], c.f[:, a:b], h, h0=state, h_last=state)
        parts.append(host(h))
    ref.check(np.concatenate(parts, 1), want["h"], "h")
    ref.check(host(state), want["h_last"], "h_last")


def test_last_gradient_in_place_and_optional_outputs():
    c = Case(11, 2, 50, 40, "f32")
    full = c.run()
    g = c.dh_last.clone()
    saved = torch.from_numpy(full["saved"]).float().cuda()
    dx, df = torch.empty_like(c.x), torch.empty_like(c.x)
    lm.gem_glr_backward(c.x, c.f, saved, c.dh, dx, df, dh_last=g, dh0=g)
    assert np.array_equal(host(g), full["dh0"]) and np.array_equal(host(dx), full["dx"])
    lm.gem_glr_backward(c.x, c.f, saved, c.dh, dx, df, dh_last=c.dh_last)
    assert np.array_equal(host(df), full["df"])
    h = torch.empty_like(c.x)
    lm.gem_glr_forward(c.x, c.f, h, h0=c.h0)
    assert np.array_equal(host(h), full["h"])


def test_broadcast_inputs():
    """Inputs with strides of 0: one gate for all steps, one input for all sequences."""
    rng = np.random.default_rng(12)
    f = torch.from_numpy(rng.standard_normal((2, 1, 48)).astype(np.float32)).cuda().expand(2, 90, 48)
    x = torch.from_numpy(rng.standard_normal((1, 90, 48)).astype(np.float32)).cuda().expand(2, 90, 48)
    h = torch.empty((2, 90, 48), device="cuda")
    lm.gem_glr_forward(x, f, h)
    ref.check(host(h), ref.glr(host(x), host(f), True)["h"], "h")


@pytest.mark.parametrize("form", ["lerp", "add"])
def test_gradients_against_differences(form):
    """<gradient, direction> against the central difference of the 64-bit definition."""
    c = Case(13, 2, 70, 20, "f32", form, resets=0.03, lengths=[70, 51])
    got = c.run()
    rng = np.random.default_rng(14)
    x, f, h0, dh, dl = host(c.x), host(c.f), host(c.h0), host(c.dh), host(c.dh_last)
    lengths, reset = c.lengths.cpu().numpy(), c.reset.cpu().numpy()

    def value(x, f, h0):
        r = ref.glr(x, f, form == "lerp", h0, lengths, reset)
        return (r["h"][0] * dh).sum() + (r["h_last"][0] * dl).sum()

    for k, name in enumerate(("dx", "df", "dh0")):
        v = rng.standard_normal(got[name].shape)
        args = [x, f, h0]
        lo, hi = list(args), list(args)
        lo[k], hi[k] = args[k] - 1e-4 * v, args[k] + 1e-4 * v
        slope = (value(*hi) - value(*lo)) / 2e-4
        # truncation: step^2 / 6 times third derivatives of order 1 on each of the 2,800 terms;
        # rounding: fp32 gradients within 1e-4 of their own scale
        assert abs((got[name] * v).sum() - slope) <= 1e-4 * np.abs(got[name] * v).sum() + 1e-5, name


def test_runs_repeat_bit_for_bit_on_any_stream():
    c = Case(15, 3, 1000, 200, "bf16", resets=0.01)
    first = c.run()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = c.run()
    for k in first:
        assert np.array_equal(first[k], again[k]), k


def test_inside_a_graph():
    c = Case(16, 2, 300, 96, "bf16")
    want = c.run()
    h, last = torch.empty_like(c.x), torch.empty((2, 96), device="cuda")
    saved = torch.empty((2, 19, 96), device="cuda")
    dx, df, dh0 = torch.empty_like(c.x), torch.empty_like(c.x), torch.empty((2, 96), device="cuda")

    def both():
        lm.gem_glr_forward(c.x, c.f, h, h0=c.h0, h_last=last, saved=saved)
        lm.gem_glr_backward(c.x, c.f, saved, c.dh, dx, df, dh_last=c.dh_last, dh0=dh0)

    both()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        both()
    for t in (h, last, saved, dx, df, dh0):
        t.fill_(float("nan"))
    g.replay()
    torch.cuda.synchronize()
    for k, t in (("h", h), ("h_last", last), ("dx", dx), ("df", df), ("dh0", dh0)):
        assert np.array_equal(host(t), want[k]), k


def test_offsets_past_32_bits():
    """A view whose last steps lie more than 2^32 elements from its first."""
    far = (1 << 32) + 4096
    if torch.cuda.mem_get_info()[0] < 3 * far * 2:
        pytest.skip("needs 26 GB of device memory")
    buf = torch.zeros(far, dtype=torch.bfloat16, device="cuda")
    x = buf.as_strided((1, 2, 64), (far, far - 64, 1))
    x.copy_(torch.randn((1, 2, 64), device="cuda"))
    f, h = torch.randn((1, 2, 64), device="cuda").bfloat16(), torch.empty((1, 2, 64), dtype=torch.bfloat16, device="cuda")
    lm.gem_glr_forward(x, f, h)
    ref.check(host(h), ref.glr(host(x), host(f), True, dtype="bf16")["h"], "h")
