"""The selective state space scan against its definition in 64 bits: state counts, groups, types and
layouts, lengths from none to long ones on both sides of the cuts of time, resets and ragged lengths with poison in
the places they hide, the state carried from call to call, and the gradients against differences."""
import numpy as np
import pytest
import torch

import lm_layers_reference as ref
from lm_reference import check
from paper_1805_08469_gb300 import lm
from test_gpu_lm_glr import DTYPES, host, place

pytestmark = pytest.mark.gpu


def floats(v):
    return torch.from_numpy(np.asarray(v, np.float32)).cuda()


def states(v, dtype, layout):
    """b or c [B, T, G, N] in one of the layouts of test_gpu_lm_glr.place."""
    B, T, G, N = v.shape
    t = place(v.reshape(B, T, G * N), dtype, layout)
    return t.unflatten(2, (G, N))


class Case:
    def __init__(self, seed, B, T, D, N=16, G=1, dtype="f32", gate=True, skip=True, bias=True, softplus=True, h0=True, lengths=None, resets=0.0,
                 layout="dense", slow=False):
        rng = np.random.default_rng(seed)
        self.dims, self.dtype, self.layout, self.softplus = (B, T, D, N, G), dtype, layout, softplus
        seq = lambda s=1.0, m=0.0: place(m + s * rng.standard_normal((B, T, D)), dtype, layout)  # noqa: E731
        self.x, self.dy = seq(), seq()
        # steps from 0.001 (memories of a thousand steps) to 1
        self.dt = seq(0.7, (-6.0 if slow else -2.0) if softplus and not bias else 0.0)
        if not softplus:
            self.dt.copy_(torch.from_numpy(np.exp(rng.uniform(np.log(1e-3), 0.0, (B, T, D)))))
        self.bias = floats(rng.uniform(-7, -5 if slow else 0, D) if softplus else 0.01 * rng.random(D)) if bias else None
        self.z = seq() if gate else None
        self.b, self.c = (states(rng.standard_normal((B, T, G, N)), dtype, layout) for _ in range(2))
        self.A = floats(-np.arange(1, N + 1) * np.exp(0.1 * rng.standard_normal((D, N))))
        self.skip = floats(rng.standard_normal(D)) if skip else None
        self.h0 = floats(rng.standard_normal((B, D, N))) if h0 else None
        self.dlast = floats(rng.standard_normal((B, D, N))) if h0 else None
        self.lengths = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda")
        self.reset = torch.from_numpy((rng.random((B, T)) < resets).astype(np.uint8)).cuda() if resets else None

    def run(self, backward=True, fill=float("nan")):
        B, T, D, N, G = self.dims
        full = lambda *s: torch.full(s, fill, device="cuda")  # noqa: E731
        new = lambda: place(np.zeros((B, T, D)), self.dtype, self.layout).fill_(fill)  # noqa: E731
        new_states = lambda: states(np.zeros((B, T, G, N)), self.dtype, self.layout).fill_(fill)  # noqa: E731
        out = {"y": new(), "h_last": full(B, D, N), "saved": full(B, -(-T // 16), D, N)}
        size = lm.gem_ssm_workspace(B, T, D, N, G, backward=backward)
        space = torch.full((size + 16,), fill, device="cuda")
        more = dict(z=self.z, skip=self.skip, dt_bias=self.bias, softplus=self.softplus, lengths=self.lengths, reset=self.reset, workspace=space[:size])
        lm.gem_ssm_forward(self.x, self.dt, self.A, self.b, self.c, out["y"], h0=self.h0, h_last=out["h_last"], saved=out["saved"], **more)
        if backward:
            out |= {"dx": new(), "ddt": new(), "db": new_states(), "dc": new_states(), "dA": full(D, N), "dskip": full(D), "ddt_bias": full(D),
                    "dh0": full(B, D, N)}
            if self.z is not None:
                out["dz"] = new()
            space[:size].fill_(fill)
            lm.gem_ssm_backward(self.x, self.dt, self.A, self.b, self.c, out["saved"], self.dy, out["dx"], out["ddt"], out["dA"], out["db"], out["dc"],
                                dz=out.get("dz"), dskip=out["dskip"], ddt_bias=out["ddt_bias"], dh_last=self.dlast, dh0=out["dh0"], **more)
        torch.cuda.synchronize()
        assert bool((space[size:] == fill).all() if fill == fill else space[size:].isnan().all()), "written past the workspace"
        return {k: host(v) for k, v in out.items()}

    def reference(self):
        cpu = lambda t: None if t is None else t.cpu().numpy()  # noqa: E731
        return ref.ssm(host(self.x), host(self.dt), host(self.A), host(self.b), host(self.c), host(self.z), host(self.skip), host(self.bias),
                       self.softplus, host(self.h0), cpu(self.lengths), cpu(self.reset), host(self.dy), host(self.dlast), self.dtype)

    def check(self):
        got, want = self.run(), self.reference()
        self.compare(got, want)
        return got

    def compare(self, got, want):
        for k, (value, bound) in want.items():
            if k == "saved" and self.lengths is not None:   # what lies past a sequence's end is not written
                on = np.arange(value.shape[1])[None] * 16 < np.clip(self.lengths.cpu().numpy(), 0, self.dims[1])[:, None]
                check(got[k][on], (value[on], bound[on]), k)
            else:
                check(got[k], (value, bound), k)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("T", [1, 2, 15, 16, 17, 31, 32, 33, 64, 65, 150])
def test_lengths_of_time(T, dtype):
    Case(T, 2, T, 40, 16, 1, dtype).check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N", [1, 2, 3, 4, 5, 8, 13, 15, 16, 17, 20, 31, 32, 33, 48, 63, 64])
def test_state_counts(N, dtype):
    Case(N, 2, 50, 37, N, 1, dtype).check()


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("D", [1, 2, 7, 8, 16, 31, 32, 33, 63, 64, 65, 100, 130])
def test_channel_counts(D, dtype):
    Case(D, 2, 40, D, 16, 1, dtype, resets=0.04).check()


@pytest.mark.parametrize("D,G", [(8, 2), (30, 3), (64, 4), (130, 2), (96, 96), (200, 5)])
@pytest.mark.parametrize("N", [16, 7, 32, 64])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_groups(D, G, N, dtype):
    Case(D, 2, 37, D, N, G, dtype).check()


@pytest.mark.parametrize("layout", ["time_major", "half", "odd"])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("D,N,G", [(64, 16, 1), (37, 5, 1), (72, 32, 3)])
def test_layouts(layout, dtype, D, N, G):
    Case(5, 2, 50, D, N, G, dtype, layout=layout, resets=0.03).check()


@pytest.mark.parametrize("form", [dict(gate=False), dict(skip=False), dict(bias=False), dict(softplus=False), dict(softplus=False, bias=False),
                                  dict(h0=False), dict(gate=False, skip=False, bias=False, h0=False)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_what_may_be_left_out(form, dtype):
    Case(6, 2, 90, 40, 16, 1, dtype, **form).check()


@pytest.mark.parametrize("B,T,D,N,G", [(1, 2500, 24, 16, 1), (1, 700, 200, 16, 2), (40, 33, 64, 16, 1), (3, 513, 64, 32, 1), (1, 1100, 16, 64, 2),
                                       (200, 3, 40, 8, 1)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_cuts_of_time(B, T, D, N, G, dtype):
    """One split, few and many; with and without resets, and with sequences that end in every split."""
    Case(T, B, T, D, N, G, dtype).check()
    Case(T + 1, B, T, D, N, G, dtype, lengths=[(b * 53 + 700) % (T + 1) for b in range(B)], resets=0.004).check()


@pytest.mark.parametrize("B,T,D,N,G", [(600, 5, 20, 7, 1), (300, 18, 66, 64, 2), (17, 40, 33, 16, 1)])
def test_many_sequences(B, T, D, N, G):
    """The parameters' gradients are sums over more sequences than a thread reads at a time."""
    Case(B, B, T, D, N, G, "bf16", resets=0.05).check()


def test_slow_decays_over_a_long_sequence():
    """States that remember thousands of steps, through every split."""
    Case(3, 1, 6000, 16, 16, 1, "f32", slow=True).check()


@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("T", [70, 333])
def test_ragged_lengths_hide_what_lies_past_them(dtype, T):
    lengths = [0, 1, 15, 16, 17, 64, 65, T - 1, T, -3, 1000]
    c = Case(7, len(lengths), T, 24, 16, 1, dtype, lengths=lengths, resets=0.02)
    clean = c.run(fill=3.0)
    c.compare(clean, c.reference())
    for b, n in enumerate(lengths):
        n = min(max(n, 0), T)
        for t, v in ((c.x, float("nan")), (c.dt, float("inf")), (c.z, float("nan")), (c.b, float("inf")), (c.c, float("nan")), (c.dy, float("nan"))):
            t[b, n:] = v
    got = c.run(fill=3.0)
    for k in got:
        assert np.array_equal(got[k], clean[k]), k


def test_an_idle_step_keeps_the_state_to_the_bit():
    """Steps past the end, and steps of 0, decay by exactly 1."""
    c = Case(9, 2, 400, 64, 16, 1, "f32", softplus=False, bias=False, lengths=[3, 0])
    got = c.run()
    assert np.array_equal(got["h_last"][1], host(c.h0)[1]) and np.array_equal(got["dh0"][1], host(c.dlast)[1])
    c.lengths = None
    c.dt.zero_()
    got = c.run()
    assert np.array_equal(got["h_last"], host(c.h0))


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("B,T", [(2, 40), (2, 400)])
def test_a_reset_drops_any_state(bad, B, T):
    """A state that holds NaN or infinity ends at a reset, in the forward and the backward pass."""
    cut = T // 2 + 3
    c = Case(8, B, T, 33, 16, 1, "f32")
    c.reset = torch.zeros((B, T), dtype=torch.bool, device="cuda")
    c.reset[:, cut] = True
    want = c.reference()
    part = lambda k, s: (want[k][0][s], np.broadcast_to(want[k][1], want[k][0].shape)[s])  # noqa: E731
    c.h0[0] = bad
    c.x[1, 3] = bad
    got = c.run()
    assert not np.isfinite(got["y"][0, 0]).any() and not np.isfinite(got["y"][1, 3]).any()
    late = np.s_[:, cut:]
    for k in ("y", "ddt", "dx", "dz", "dc", "db"):
        check(got[k][late], part(k, late), k)
    check(got["h_last"], want["h_last"], "h_last")
    c = Case(8, B, T, 33, 16, 1, "f32")
    c.reset = torch.zeros((B, T), dtype=torch.uint8, device="cuda")
    c.reset[:, cut] = 255
    c.dy[:, cut + 2] = bad
    got = c.run()
    early = np.s_[:, :cut]
    for k in ("dx", "ddt", "dz", "db", "dc"):
        check(got[k][early], part(k, early), k)
    check(got["dh0"], want["dh0"], "dh0")


def test_an_infinite_state_stays_not_finite():
    """Over many splits, whatever the decays between."""
    for T in (50, 3000):
        c = Case(2, 1, T, 24, 16, 1, "f32")
        c.h0[:] = float("inf")
        got = c.run(backward=False)
        assert not np.isfinite(got["h_last"]).any()


def test_growing_states():
    """Negative steps let states grow, over many splits by more than fp32 holds as one factor; a state of 0 stays 0."""
    B, T, D, N = 1, 3000, 24, 2
    c = Case(14, B, T, D, N, 1, "f32", softplus=False, bias=False)
    c.dt.copy_(-0.02 * torch.rand((B, T, D), device="cuda") - 0.001)      # growth by e^30 and e^60
    c.h0.mul_(1e-20)
    got, want = c.run(backward=False), c.reference()
    for k in got:
        check(got[k], want[k], k)
    c.dt.fill_(-1.0)
    c.x.zero_()
    c.h0.zero_()
    got = c.run(backward=False)
    assert (got["h_last"] == 0).all() and (got["y"] == 0).all()


def test_offsets_past_32_bits():
    """Steps, states and outputs that lie more than 2^31 elements apart."""
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 40 GB")
    T, D, N, far = 3, 40, 16, 1 << 30
    c = Case(15, 1, T, D, N, 1, "bf16")
    want = c.run()
    stretch = lambda t: torch.empty(far * (T - 1) + t.shape[2:].numel(), dtype=t.dtype, device="cuda").as_strided(  # noqa: E731
        t.shape, (far * T, far) + t.stride()[2:])
    for name in ("x", "b"):
        t = stretch(getattr(c, name))
        t.copy_(getattr(c, name))
        setattr(c, name, t)
    y = stretch(c.dy)
    lm.gem_ssm_forward(c.x, c.dt, c.A, c.b, c.c, y, z=c.z, skip=c.skip, dt_bias=c.bias, h0=c.h0)
    assert np.array_equal(host(y), want["y"])


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_extreme_steps(dtype):
    """Steps from 0 to ones that forget everything; nothing but the formula's values."""
    big = 3e4
    vals = np.array([-np.inf, -big, -200.0, -100.0, -80.0, -20.0, -1e-30, 0.0, 1e-3, 1.0, 20.0, 80.0, 200.0, big])
    c = Case(9, 2, 40, len(vals), 16, 1, dtype, bias=False)
    c.dt.copy_(torch.from_numpy(np.broadcast_to(vals, (2, 40, len(vals))).copy()))
    got = c.run()
    c.dt[c.dt == -float("inf")] = -300.0
    want = c.reference()
    for k, (value, bound) in want.items():
        if dtype == "f16" and k in ("y", "dx", "ddt", "dz", "db", "dc"):
            # the largest fp16 is 65504, and what lies half a step (16) above it or further rounds to infinity
            value = np.where(np.abs(value) >= 65520, np.copysign(np.inf, value), value)
        check(got[k], (value, bound + 1e-30), k)


@pytest.mark.parametrize("cuts", [[0, 1, 2, 3, 100], [0, 16, 100], [0, 37, 99, 100]])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_the_state_goes_on_in_place(dtype, cuts):
    """A sequence in several calls whose h_last is their h0: the same bound as in one call."""
    c = Case(10, 2, 100, 70, 16, 2, dtype, resets=0.03)
    want = c.reference()
    state = c.h0.clone()
    parts = []
    for a, e in zip(cuts, cuts[1:]):
        y = torch.empty((2, e - a, 70), dtype=DTYPES[dtype], device="cuda")
        space = torch.empty(lm.gem_ssm_workspace(2, e - a, 70, 16, 2), device="cuda")
        lm.gem_ssm_forward(c.x[:, a:e], c.dt[:, a:e], c.A, c.b[:, a:e], c.c[:, a:e], y, z=c.z[:, a:e], skip=c.skip, dt_bias=c.bias, h0=state,
                           h_last=state, reset=c.reset[:, a:e].contiguous(), workspace=space)
        parts.append(host(y))
    check(np.concatenate(parts, 1), want["y"], "y")
    check(host(state), want["h_last"], "h_last")


@pytest.mark.parametrize("T", [40, 3000])
def test_states_in_place_of_their_own_gradients(T):
    """h_last may be h0 and dh0 may be dh_last, with one split of time and with many."""
    c = Case(11, 1, T, 24, 16, 1, "f32")
    want = c.run()
    B, T, D, N, G = c.dims
    state, grad = c.h0.clone(), c.dlast.clone()
    space = torch.empty(lm.gem_ssm_workspace(B, T, D, N, G, backward=True), device="cuda")
    y, saved = torch.empty_like(c.x), torch.empty((B, -(-T // 16), D, N), device="cuda")
    more = dict(z=c.z, skip=c.skip, dt_bias=c.bias, workspace=space)
    lm.gem_ssm_forward(c.x, c.dt, c.A, c.b, c.c, y, h0=state, h_last=state, saved=saved, **more)
    new = [torch.empty_like(c.x) for _ in range(3)]
    db, dc = torch.empty_like(c.b), torch.empty_like(c.c)
    lm.gem_ssm_backward(c.x, c.dt, c.A, c.b, c.c, saved, c.dy, new[0], new[1], None, db, dc, dz=new[2], dh_last=grad, dh0=grad, **more)
    for a, k in ((y, "y"), (state, "h_last"), (grad, "dh0"), (new[0], "dx"), (new[1], "ddt"), (new[2], "dz"), (db, "db"), (dc, "dc")):
        assert np.array_equal(host(a), want[k]), k


def test_no_steps():
    x, b = torch.empty((3, 0, 8), device="cuda"), torch.empty((3, 0, 1, 16), device="cuda")
    A, h0 = -torch.ones((8, 16), device="cuda"), torch.randn((3, 8, 16), device="cuda")
    out = torch.full_like(h0, float("nan"))
    lm.gem_ssm_forward(x, x, A, b, b, x, h0=h0, h_last=out)
    assert torch.equal(out, h0)
    out.fill_(float("nan"))
    dA = torch.full_like(A, float("nan"))
    space = torch.empty(lm.gem_ssm_workspace(3, 0, 8, 16, 1, backward=True), device="cuda")
    lm.gem_ssm_backward(x, x, A, b, b, torch.empty((3, 0, 8, 16), device="cuda"), x, x, x, dA, b, b, dh_last=h0, dh0=out, workspace=space)
    assert torch.equal(out, h0) and bool((dA == 0).all())
    x, b = torch.empty((0, 5, 8), device="cuda"), torch.empty((0, 5, 1, 16), device="cuda")
    dA.fill_(float("nan"))
    lm.gem_ssm_backward(x, x, A, b, b, torch.empty((0, 1, 8, 16), device="cuda"), x, x, x, dA, b, b)
    assert bool((dA == 0).all())


def test_broadcast_inputs():
    """Strides of 0: a step size for all steps, an input for all sequences, b for all of both."""
    rng = np.random.default_rng(4)
    B, T, D, N = 3, 70, 40, 16
    c = Case(4, B, T, D, N, 1, "f32")
    c.dt = floats(rng.standard_normal((B, 1, D)) - 2).expand(B, T, D)
    c.x = floats(rng.standard_normal((1, T, D))).expand(B, T, D)
    c.b = floats(rng.standard_normal((1, 1, 1, N))).expand(B, T, 1, N)
    c.check()


def test_gradients_against_differences():
    """Central differences of the fp32 forward call: a step of 2^-7 leaves an error of h^2 times third derivatives of up to
    some 20, and rounding of the loss' terms, 2^-24 of some 200, over 2 h."""
    B, T, D, N = 1, 6, 3, 2
    c = Case(13, B, T, D, N, 1, "f32", resets=0.2)
    got = c.run()

    def loss():
        y, last = torch.empty_like(c.x), torch.empty_like(c.h0)
        lm.gem_ssm_forward(c.x, c.dt, c.A, c.b, c.c, y, z=c.z, skip=c.skip, dt_bias=c.bias, h0=c.h0, reset=c.reset, h_last=last)
        return float((y.double() * c.dy.double()).sum() + (last.double() * c.dlast.double()).sum())

    h = 2.0 ** -7
    for t, k in ((c.x, "dx"), (c.dt, "ddt"), (c.z, "dz"), (c.b, "db"), (c.c, "dc"), (c.A, "dA"), (c.skip, "dskip"), (c.bias, "ddt_bias"),
                 (c.h0, "dh0")):
        flat = t.view(-1)
        for i in range(flat.numel()):
            keep = flat[i].item()
            flat[i] = keep + h
            up, above = loss(), flat[i].item()
            flat[i] = keep - h
            down, below = loss(), flat[i].item()
            flat[i] = keep
            assert abs((up - down) / (above - below) - got[k].reshape(-1)[i]) < 3e-3, (k, i)
