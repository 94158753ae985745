"""The short convolution against its definition in 64 bits: every width and type, lengths around the
segments that time is cut into, strided tensors, resets and ragged lengths with poison in the places they
hide, the state carried from call to call, and the gradients against differences."""
import numpy as np
import pytest
import torch

import lm_layers_reference as ref
from lm_reference import check
from paper_1805_08469_gb300 import lm
from test_gpu_lm_glr import DTYPES, host, place

pytestmark = pytest.mark.gpu

FORMS = {"linear": lm.GEM_CONV_LINEAR, "silu": lm.GEM_CONV_SILU}


def floats(v):
    return torch.from_numpy(np.asarray(v, np.float32)).cuda()


class Case:
    def __init__(self, seed, B, T, D, W=4, dtype="f32", form="silu", state=True, bias=True, lengths=None, resets=0.0, layout="dense"):
        rng = np.random.default_rng(seed)
        self.dims, self.dtype, self.form, self.layout = (B, T, D, W), dtype, form, layout
        self.x = place(rng.standard_normal((B, T, D)), dtype, layout)
        self.dy = place(rng.standard_normal((B, T, D)), dtype, layout)
        self.w = floats(rng.standard_normal((D, W)))
        self.bias = floats(rng.standard_normal(D)) if bias else None
        self.state = floats(rng.standard_normal((B, W - 1, D))) if state else None
        self.dlast = floats(rng.standard_normal((B, W - 1, D))) if state else None
        self.lengths = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda")
        self.reset = torch.from_numpy((rng.random((B, T)) < resets).astype(np.uint8)).cuda() if resets else None

    def run(self, backward=True):
        B, T, D, W = self.dims
        nan = lambda *s: torch.full(s, float("nan"), device="cuda")  # noqa: E731
        new = lambda: place(np.zeros((B, T, D)), self.dtype, self.layout).fill_(float("nan"))  # noqa: E731
        out = {"y": new(), "state_last": nan(B, W - 1, D)}
        lm.gem_conv_forward(self.x, self.w, out["y"], form=FORMS[self.form], bias=self.bias, state=self.state, lengths=self.lengths, reset=self.reset,
                            state_last=out["state_last"])
        if backward:
            out |= {"dx": new(), "dweight": nan(D, W), "dbias": nan(D), "dstate": nan(B, W - 1, D)}
            size = lm.gem_conv_workspace(B, T, D, W)
            space = nan(size + 16)
            lm.gem_conv_backward(self.x, self.w, self.dy, out["dx"], out["dweight"], space[:size], form=FORMS[self.form], bias=self.bias,
                                 dbias=out["dbias"], state=self.state, lengths=self.lengths, reset=self.reset, dstate_last=self.dlast,
                                 dstate=out["dstate"])
            torch.cuda.synchronize()
            assert bool(space[size:].isnan().all())
        torch.cuda.synchronize()
        return {k: host(v) for k, v in out.items()}

    def reference(self):
        cpu = lambda t: None if t is None else t.cpu().numpy()  # noqa: E731
        return ref.conv(host(self.x), host(self.w), self.form == "silu", host(self.bias), host(self.state), cpu(self.lengths), cpu(self.reset),
                        host(self.dy), host(self.dlast), self.dtype)

    def check(self):
        got, want = self.run(), self.reference()
        for k in want:
            check(got[k], want[k], k)


@pytest.mark.parametrize("W", [2, 3, 4])
@pytest.mark.parametrize("form", ["linear", "silu"])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("T", [1, 2, 3, 4, 5, 63, 64, 65, 67, 130, 300])
def test_lengths_of_time(T, dtype, form, W):
    Case(T, 2, T, 36, W, dtype, form).check()


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("D", [1, 2, 3, 4, 5, 31, 32, 33, 127, 128, 129, 260, 513])
def test_channel_counts(D, dtype):
    Case(D, 2, 70, D, 4, dtype, resets=0.05).check()


@pytest.mark.parametrize("layout", ["time_major", "half", "odd"])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("D", [64, 37])
def test_layouts(layout, dtype, D):
    Case(5, 3, 150, D, 3, dtype, layout=layout, resets=0.03).check()


@pytest.mark.parametrize("B,T,D", [(1, 5000, 8), (70, 9, 40), (3, 1025, 200), (300, 1, 65)])
def test_shapes(B, T, D):
    Case(T, B, T, D, 4, "bf16", resets=0.01).check()


@pytest.mark.parametrize("B,T,D", [(701, 9, 40), (650, 1, 65), (90, 500, 70), (3, 5000, 260), (1, 70001, 8), (333, 65, 128), (1201, 64, 5)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_blocks_of_several_segments(B, T, D, dtype):
    """Blocks whose warps have segments of one sequence, of several, and none."""
    lengths = np.random.default_rng(B).integers(-1, T + 2, B).tolist()
    Case(B, B, T, D, 4 if T > 1 else 3, dtype, resets=0.05, lengths=lengths).check()


def test_without_state_bias_and_last_gradient():
    Case(6, 2, 100, 40, 4, "f32", state=False, bias=False).check()


@pytest.mark.parametrize("W", [2, 4])
@pytest.mark.parametrize("dtype", ["f32", "f16"])
def test_ragged_lengths_hide_what_lies_past_them(dtype, W):
    lengths = [0, 1, 2, 3, 4, 63, 64, 65, 66, 67, 128, 200, -3, 1000]
    c = Case(7, len(lengths), 200, 48, W, dtype, lengths=lengths, resets=0.02)
    clean, want = c.run(), c.reference()
    for k in want:
        check(clean[k], want[k], k)
    for b, n in enumerate(lengths):
        n = min(max(n, 0), 200)
        c.x[b, n:] = float("nan")
        c.dy[b, n:] = float("inf")
    got = c.run()
    for k in got:
        assert np.array_equal(got[k], clean[k]), k


@pytest.mark.parametrize("at", [0, 1, 2, 3, 62, 63, 64, 65, 66, 99])
@pytest.mark.parametrize("W", [2, 3, 4])
def test_a_reset_drops_every_earlier_input(at, W):
    """NaN and infinity before a reset do not reach what follows, nor gradients what went before."""
    c = Case(8, 2, 100, 20, W, "f32")
    c.reset = torch.zeros((2, 100), dtype=torch.bool, device="cuda")
    c.reset[:, at] = True
    want = c.reference()
    if at:
        c.x[0, :at] = float("nan")
        c.x[1, :at] = float("inf")
    c.state[:] = float("nan")
    got = c.run()
    part = np.s_[:, at:]
    for k in ("y", "dx"):
        check(got[k][part], (want[k][0][part], np.broadcast_to(want[k][1], want[k][0].shape)[part]), k)
    if at <= 97:
        check(got["state_last"], want["state_last"], "state_last")
    c = Case(8, 2, 100, 20, W, "f32")
    c.reset = torch.zeros((2, 100), dtype=torch.uint8, device="cuda")
    c.reset[:, at] = 255
    c.dy[:, at:] = float("nan")
    got = c.run()
    check(got["dx"][:, :at], (want["dx"][0][:, :at], np.broadcast_to(want["dx"][1], want["dx"][0].shape)[:, :at]), "dx")
    if at == 0:
        assert (got["dstate"] == 0).all()


@pytest.mark.parametrize("cuts", [[0, 1, 2, 3, 100], [0, 64, 100], [0, 7, 99, 100], [0, 100]])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_the_state_goes_on_in_place(dtype, cuts):
    """A sequence in several calls whose state_last is their state: the same as in one call."""
    c = Case(10, 2, 100, 70, 4, dtype, resets=0.05)
    want = c.run(backward=False)
    state = c.state.clone()
    parts = []
    for a, b in zip(cuts, cuts[1:]):
        y = torch.empty((2, b - a, 70), dtype=DTYPES[dtype], device="cuda")
        lm.gem_conv_forward(c.x[:, a:b], c.w, y, bias=c.bias, state=state, reset=c.reset[:, a:b].contiguous(), state_last=state)
        parts.append(host(y))
    assert np.array_equal(np.concatenate(parts, 1), want["y"])
    assert np.array_equal(host(state), want["state_last"])


def test_no_steps():
    x = torch.empty((3, 0, 8), device="cuda")
    w, s = torch.randn((8, 4), device="cuda"), torch.randn((3, 3, 8), device="cuda")
    out = torch.full_like(s, float("nan"))
    lm.gem_conv_forward(x, w, x, state=s, state_last=out)
    assert torch.equal(out, s)
    dw, db = torch.full((8, 4), float("nan"), device="cuda"), torch.full((8,), float("nan"), device="cuda")
    out.fill_(float("nan"))
    lm.gem_conv_backward(x, w, x, x, dw, torch.empty(lm.gem_conv_workspace(3, 0, 8, 4), device="cuda"), dbias=db, dstate_last=s, dstate=out)
    assert torch.equal(out, s) and bool((dw == 0).all() and (db == 0).all())
    none = torch.empty((0, 5, 8), device="cuda")
    dw.fill_(float("nan"))
    lm.gem_conv_backward(none, w, none, none, dw, None)
    assert bool((dw == 0).all())


def test_offsets_past_32_bits():
    """Steps and outputs that lie more than 2^31 elements apart."""
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 40 GB")
    T, D, far = 4, 66, 1 << 30
    c = Case(15, 1, T, D, 4, "bf16")
    want = c.run()
    stretch = lambda t: torch.empty(far * (T - 1) + D, dtype=t.dtype, device="cuda").as_strided(t.shape, (far * T, far, 1))  # noqa: E731
    x, y = stretch(c.x), stretch(c.x)
    x.copy_(c.x)
    lm.gem_conv_forward(x, c.w, y, bias=c.bias, state=c.state)
    assert np.array_equal(host(y), want["y"])
    dw = torch.empty_like(c.w)
    lm.gem_conv_backward(x, c.w, c.dy, y, dw, torch.empty(lm.gem_conv_workspace(1, T, D, 4), device="cuda"), bias=c.bias, state=c.state,
                         dstate_last=c.dlast)
    assert np.array_equal(host(y), want["dx"]) and np.array_equal(host(dw), want["dweight"])


def test_parts_of_the_gradient():
    c = Case(12, 2, 90, 30, 3, "f32")
    full = c.run()
    dx = torch.empty_like(c.x)
    lm.gem_conv_backward(c.x, c.w, c.dy, dx, None, None, bias=c.bias, state=c.state, dstate_last=c.dlast)
    assert np.array_equal(host(dx), full["dx"])


@pytest.mark.parametrize("form", ["linear", "silu"])
def test_gradients_against_differences(form):
    """Central differences of the fp32 forward call, of a step h that balances its truncation against rounding: an error
    of h^2 (third derivatives of up to some 10) and 2^-24 / h of the loss' terms."""
    B, T, D, W = 1, 9, 3, 4
    c = Case(13, B, T, D, W, "f32", form, resets=0.2)
    got = c.run()

    def loss():
        y, last = torch.empty_like(c.x), torch.empty_like(c.state)
        lm.gem_conv_forward(c.x, c.w, y, form=FORMS[form], bias=c.bias, state=c.state, reset=c.reset, state_last=last)
        return float((y.double() * c.dy.double()).sum() + (last.double() * c.dlast.double()).sum())

    h = 2.0 ** -7
    for t, g in ((c.x, got["dx"]), (c.w, got["dweight"]), (c.bias, got["dbias"]), (c.state, got["dstate"])):
        flat = t.view(-1)
        for i in range(flat.numel()):
            keep = flat[i].item()
            flat[i] = keep + h
            up, above = loss(), flat[i].item()
            flat[i] = keep - h
            down, below = loss(), flat[i].item()
            flat[i] = keep
            assert abs((up - down) / (above - below) - g.reshape(-1)[i]) < 3e-3, i
