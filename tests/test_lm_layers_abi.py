"""Embedding, convolution, scan and policy loss without a GPU: sizes, refusals on the host, and the binding's
checks of its tensors.  No call here passes every check with work to do, so nothing is launched."""
import ctypes as C

import numpy as np
import pytest
import torch

import lm_layers_reference as ref
from paper_1805_08469_gb300 import _lib, lm
from paper_1805_08469_gb300._build import build_library

OK, EINVAL = 0, -1
PTR = 1 << 20          # an aligned address; a refused call never reads it
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def L():
    build_library()
    return _lib.lib()


def seq(data=PTR, sb=1000, st=10):
    return _lib.GemSeq(data, sb, st)


def policy(L, dtype=0, N=2, V=100, logits=PTR, ld=100, tokens=PTR, old=PTR, adv=PTR, ref=PTR, scale=0, tau=1.0, low=0.2, high=0.2, kl=0.1,
           bonus=0.0, loss=PTR, logp=0, entropy=0, grad=PTR, grad_ld=100):
    return L.gem_policy(dtype, N, V, logits, ld, tokens, old, adv, ref, scale, tau, low, high, kl, bonus, loss, logp, entropy, grad, grad_ld, 0)


@pytest.mark.parametrize("bad", [
    dict(dtype=3), dict(dtype=-1), dict(N=-1), dict(N=1 << 28), dict(V=0), dict(V=1 << 31), dict(logits=0), dict(logits=PTR + 2), dict(ld=99),
    dict(ld=-100), dict(ld=0), dict(ld=1 << 50), dict(tokens=0), dict(tokens=PTR + 1), dict(old=0), dict(old=PTR + 2), dict(adv=0), dict(adv=PTR + 3),
    dict(ref=0), dict(ref=PTR + 2), dict(scale=PTR + 2), dict(tau=0.0), dict(tau=NAN), dict(tau=1e-30), dict(tau=INF), dict(low=-0.1), dict(low=1.5),
    dict(low=NAN), dict(high=-0.1), dict(high=INF), dict(high=NAN), dict(kl=-1.0), dict(kl=NAN), dict(kl=INF), dict(bonus=INF), dict(bonus=NAN),
    dict(loss=0), dict(loss=PTR + 2), dict(logp=PTR + 2), dict(entropy=PTR + 1), dict(grad=PTR + 2), dict(grad_ld=99), dict(grad_ld=104)])
def test_policy_refuses(L, bad):
    assert policy(L, **bad) == EINVAL       # (grad is logits here: another pitch is refused too)


def embed(L, table_dtype=0, dtype=1, N=4, V=9, D=8, table=PTR, table_ld=8, tokens=PTR, out=PTR, out_ld=8):
    return L.gem_embed(table_dtype, dtype, N, V, D, table, table_ld, tokens, 1.0, out, out_ld, 0)


@pytest.mark.parametrize("bad", [
    dict(table_dtype=3), dict(dtype=-1), dict(N=-1), dict(N=1 << 28), dict(V=0), dict(V=1 << 31), dict(D=-1), dict(D=1 << 25), dict(table=0),
    dict(table=PTR + 2), dict(table_ld=7), dict(table_ld=-8), dict(tokens=0), dict(tokens=PTR + 2), dict(out=0), dict(out=PTR + 1), dict(out_ld=7),
    dict(out_ld=1 << 50)])
def test_embed_refuses(L, bad):
    assert embed(L, **bad) == EINVAL


def embed_grad(L, dtype=1, grad_dtype=0, N=4, V=9, D=8, dout=PTR, dout_ld=8, tokens=PTR, accumulate=0, dtable=PTR, dtable_ld=8, space=PTR):
    return L.gem_embed_grad(dtype, grad_dtype, N, V, D, dout, dout_ld, tokens, 1.0, accumulate, dtable, dtable_ld, space, 0)


@pytest.mark.parametrize("bad", [
    dict(dtype=3), dict(grad_dtype=5), dict(N=-1), dict(N=1 << 28), dict(V=0), dict(D=-1), dict(dout=0), dict(dout=PTR + 1), dict(dout_ld=7),
    dict(tokens=0), dict(tokens=PTR + 2), dict(accumulate=2), dict(accumulate=-1), dict(dtable=0), dict(dtable=PTR + 2), dict(dtable_ld=3), dict(space=0),
    dict(space=PTR + 4)])
def test_embed_grad_refuses(L, bad):
    assert embed_grad(L, **bad) == EINVAL


def conv(L, dtype=0, form=1, B=2, T=4, D=10, W=4, x=None, weight=PTR, bias=0, state=0, lengths=0, y=None, last=0):
    return L.gem_conv_forward(dtype, form, B, T, D, W, C.byref(x or seq()), weight, bias, state, lengths, 0, C.byref(y or seq()), last, 0)


def conv_back(L, dtype=0, form=1, B=2, T=4, D=10, W=4, x=None, weight=PTR, bias=0, state=0, lengths=0, dy=None, dlast=0, dx=None, dw=PTR, db=0, ds=0,
              space=PTR):
    x, dy, dx = (C.byref(t or seq()) for t in (x, dy, dx))
    return L.gem_conv_backward(dtype, form, B, T, D, W, x, weight, bias, state, lengths, 0, dy, dlast, dx, dw, db, ds, space, 0)


SIZES = [dict(dtype=3), dict(dtype=-1), dict(B=-1), dict(T=-1), dict(D=-1), dict(B=1 << 31), dict(T=1 << 31), dict(x=seq(0)), dict(x=seq(PTR + 2)),
         dict(x=seq(sb=-1)), dict(x=seq(st=-10)), dict(x=seq(sb=1 << 60)), dict(lengths=PTR + 1)]


@pytest.mark.parametrize("bad", SIZES + [
    dict(form=2), dict(form=-1), dict(W=1), dict(W=5), dict(W=0), dict(B=1 << 20, T=1 << 20), dict(B=1, T=1, D=(1 << 30) + 1), dict(weight=0), dict(weight=PTR + 2), dict(bias=PTR + 1),
    dict(state=PTR + 2), dict(last=PTR + 2), dict(y=seq(0)), dict(y=seq(st=9)), dict(y=seq(sb=39)), dict(y=seq(st=0))])
def test_conv_refuses(L, bad):
    assert conv(L, **bad) == EINVAL


@pytest.mark.parametrize("bad", SIZES + [
    dict(form=2), dict(W=1), dict(W=5), dict(weight=0), dict(dy=seq(0)), dict(dx=seq(0)), dict(dx=seq(st=3)), dict(dlast=PTR + 2), dict(dw=PTR + 2),
    dict(db=PTR + 1), dict(ds=PTR + 3), dict(space=0), dict(space=PTR + 2), dict(ds=PTR, dlast=PTR)])
def test_conv_backward_refuses(L, bad):
    assert conv_back(L, **bad) == EINVAL


def ssm_in(B=2, T=4, D=10, N=4, G=1, x=None, dt=None, b=None, c=None, z=None, A=PTR, skip=0, bias=0, lengths=0, reset=0):
    none = _lib.GemSeq()
    return _lib.GemSsm(B, T, D, N, G, 1, x or seq(), dt or seq(), b or seq(), c or seq(), z or none, A, skip, bias, lengths, reset)


def ssm(L, dtype=0, h0=0, y=None, last=0, saved=0, space=0, **kw):
    return L.gem_ssm_forward(dtype, C.byref(ssm_in(**kw)), h0, C.byref(y or seq()), last, saved, space, 0)


def ssm_back(L, dtype=0, saved=PTR, dy=None, dlast=0, dx=None, ddt=None, db=None, dc=None, dz=None, dA=0, dskip=0, dbias=0, dh0=0, space=PTR, **kw):
    out = _lib.GemSsmGrad(dx or seq(), ddt or seq(), db or seq(), dc or seq(), dz or seq(), dA, dskip, dbias, dh0)
    return L.gem_ssm_backward(dtype, C.byref(ssm_in(**kw)), saved, C.byref(dy or seq()), dlast, C.byref(out), space, 0)


SSM = SIZES + [dict(N=0), dict(N=65), dict(B=1, T=1, D=(1 << 30) + 4), dict(B=1, T=1, D=1 << 26, G=1 << 25, N=64), dict(G=0), dict(G=3), dict(G=-1), dict(dt=seq(0)), dict(b=seq(0)), dict(c=seq(PTR + 2)), dict(b=seq(st=-1)),
               dict(z=seq(PTR + 1)), dict(A=0), dict(A=PTR + 2), dict(skip=PTR + 1), dict(bias=PTR + 2)]


@pytest.mark.parametrize("bad", SSM + [dict(h0=PTR + 2), dict(last=PTR + 1), dict(saved=PTR + 2), dict(space=PTR + 2), dict(y=seq(0)), dict(y=seq(st=9)),
                                       dict(T=4000, x=seq(sb=40000), y=seq(sb=40000), space=0)])
def test_ssm_refuses(L, bad):
    assert ssm(L, **bad) == EINVAL


@pytest.mark.parametrize("bad", SSM + [
    dict(saved=0), dict(saved=PTR + 2), dict(dy=seq(0)), dict(dx=seq(0)), dict(ddt=seq(st=9)), dict(db=seq(0)), dict(dc=seq(st=3)), dict(dlast=PTR + 2),
    dict(dA=PTR + 1), dict(dskip=PTR + 2), dict(dbias=PTR + 2), dict(dh0=PTR + 1), dict(space=0, dA=PTR), dict(z=seq(), dz=seq(0))])
def test_ssm_backward_refuses(L, bad):
    assert ssm_back(L, **bad) == EINVAL


def test_null_structures_are_refused(L):
    one = seq()
    ref_one, ref_in, ref_out = C.byref(one), C.byref(ssm_in()), C.byref(_lib.GemSsmGrad(one, one, one, one, one))
    assert L.gem_ssm_forward(0, None, 0, ref_one, 0, 0, 0, 0) == EINVAL
    assert L.gem_ssm_forward(0, ref_in, 0, None, 0, 0, 0, 0) == EINVAL
    assert L.gem_ssm_backward(0, None, PTR, ref_one, 0, ref_out, PTR, 0) == EINVAL
    assert L.gem_ssm_backward(0, ref_in, PTR, ref_one, 0, None, PTR, 0) == EINVAL
    assert L.gem_ssm_backward(0, ref_in, PTR, None, 0, ref_out, PTR, 0) == EINVAL
    assert L.gem_conv_forward(0, 0, 1, 1, 1, 4, None, PTR, 0, 0, 0, 0, ref_one, 0, 0) == EINVAL
    assert L.gem_conv_forward(0, 0, 1, 1, 1, 4, ref_one, PTR, 0, 0, 0, 0, None, 0, 0) == EINVAL


def test_empty_sizes_leave_nothing_to_do(L):
    none = seq(0)
    assert policy(L, N=0, logits=0, tokens=0, loss=0, grad=0) == OK
    assert embed(L, N=0, table=0, tokens=0, out=0) == OK and embed(L, D=0, table=0, out=0) == OK
    assert embed_grad(L, N=0, accumulate=1, dout=0, tokens=0, dtable=0, space=0) == OK and embed_grad(L, D=0, dout=0, dtable=0) == OK
    assert conv(L, B=0, x=none, y=none, weight=0) == OK and conv(L, D=0, x=none, y=none, weight=0) == OK and conv(L, T=0, x=none, y=none) == OK
    assert conv_back(L, D=0, x=none, dy=none, dx=none, weight=0) == OK
    assert ssm(L, B=0, x=none, dt=none, b=none, c=none, y=none, A=0) == OK and ssm(L, D=0, x=none, dt=none, y=none, b=none, c=none, A=0) == OK
    assert ssm(L, T=0, x=none, dt=none, b=none, c=none, y=none) == OK
    assert ssm_back(L, B=0, saved=0, space=0) == OK


def test_counts(L):
    for B, T, D, N, want in [(2, 1, 5, 3, 30), (2, 16, 5, 3, 30), (2, 17, 5, 3, 60), (3, 0, 4, 2, 0), (0, 9, 9, 9, 0), (-1, 1, 1, 1, -1), (1, -1, 1, 1, -1),
                             (1, 1, 1, 0, -1), (1, 1, 1, 65, -1)]:
        assert L.gem_ssm_saved_count(B, T, D, N) == want
    assert L.gem_ssm_workspace(4, 1, 64, 16, 1, 0) == 0
    assert L.gem_ssm_workspace(1, 100000, 64, 16, 1, 0) > 0
    assert L.gem_ssm_workspace(1, 100, 64, 16, 3, 0) == -1 and L.gem_ssm_workspace(-1, 1, 1, 1, 1, 1) == -1
    assert L.gem_ssm_workspace(1 << 20, 1 << 20, 1 << 20, 64, 1, 1) == -1
    assert L.gem_conv_workspace(2, 100, 10, 4) > 0 and L.gem_conv_workspace(2, 100, 10, 5) == -1 and L.gem_conv_workspace(0, 1, 1, 2) == 0
    assert L.gem_embed_workspace(-1, 1, 1) == -1 and L.gem_embed_workspace(1, 0, 1) == -1 and L.gem_embed_workspace(1000, 50, 8) > 0


def test_the_binding_checks_its_tensors():
    """Tensors of the host, of another type, shape or layout are refused before the library is called."""
    z, i, f = torch.zeros(2, 8), torch.zeros(2, dtype=torch.int32), torch.zeros(2)
    for call in (lambda: lm.gem_policy(z, i, f, f, f), lambda: lm.gem_embed(z, i, z), lambda: lm.gem_embed_grad(z, i, z, None),
                 lambda: lm.gem_conv_forward(torch.zeros(1, 2, 8), torch.zeros(8, 4), torch.zeros(1, 2, 8))):
        with pytest.raises((TypeError, ValueError)):
            call()
    x, b = torch.zeros(1, 2, 4), torch.zeros(1, 2, 1, 3)
    with pytest.raises(TypeError):
        lm.gem_ssm_forward(x, x, torch.zeros(4, 3), b, b, x)
    with pytest.raises(ValueError):
        lm.gem_ssm_forward(x[0], x[0], torch.zeros(4, 3), b, b, x[0])
    with pytest.raises(ValueError):
        lm.gem_conv_forward(x[0], torch.zeros(4, 4), x[0])


def test_structure_layouts():
    """The structures' sizes, and that they packed into bytes are the same."""
    assert C.sizeof(_lib.GemSsm) == 24 + 16 + 5 * 24 + 5 * 8 and C.sizeof(_lib.GemSsmGrad) == 5 * 24 + 4 * 8
    s = [_lib.GemSeq(10 * k, 10 * k + 1, 10 * k + 2) for k in range(1, 6)]
    flat = [v for q in s for v in (q.data, q.stride_b, q.stride_t)]
    assert bytes(s[0]) == _lib.pack_seq(*flat[:3])
    assert bytes(_lib.GemSsm(1, 2, 3, 4, 5, 1, *s, 6, 7, 8, 9, 10)) == _lib.pack_ssm(1, 2, 3, 4, 5, True, *flat, 6, 7, 8, 9, 10)
    assert bytes(_lib.GemSsmGrad(*s, 6, 7, 8, 9)) == _lib.pack_ssm_grad(*flat, 6, 7, 8, 9)


# ---------------------------------------------------------------------- the definitions themselves


def differences(f, arrays, got, names, h=1e-5):
    for name, a in zip(names, arrays):
        flat, g = a.reshape(-1), got[name][0].reshape(-1)
        for k in range(flat.size):
            keep = flat[k]
            flat[k] = keep + h
            up = f()
            flat[k] = keep - h
            down = f()
            flat[k] = keep
            assert abs((up - down) / (2 * h) - g[k]) < 1e-6 * max(1, abs(g[k])), (name, k)


def test_the_conv_reference_s_gradients():
    rng = np.random.default_rng(1)
    B, T, D, W = 3, 7, 2, 4
    x, w, bias, s = rng.standard_normal((B, T, D)), rng.standard_normal((D, W)), rng.standard_normal(D), rng.standard_normal((B, W - 1, D))
    dy, dl = rng.standard_normal((B, T, D)), rng.standard_normal((B, W - 1, D))
    how = dict(lengths=np.array([7, 2, 0]), reset=(rng.random((B, T)) < 0.3))

    def loss():
        r = ref.conv(x, w, True, bias, s, **how)
        return (r["y"][0] * dy).sum() + (r["state_last"][0] * dl).sum()

    got = ref.conv(x, w, True, bias, s, dy=dy, dstate_last=dl, **how)
    differences(loss, (x, w, bias, s), got, ("dx", "dweight", "dbias", "dstate"))


def test_the_scan_reference_s_gradients():
    rng = np.random.default_rng(2)
    B, T, D, N, G = 2, 5, 4, 3, 2
    x, dt, z = (rng.standard_normal((B, T, D)) for _ in range(3))
    b, c = (rng.standard_normal((B, T, G, N)) for _ in range(2))
    A, skip, bias, h0 = -rng.random((D, N)) - 0.5, rng.standard_normal(D), rng.standard_normal(D), rng.standard_normal((B, D, N))
    dy, dl = rng.standard_normal((B, T, D)), rng.standard_normal((B, D, N))
    how = dict(lengths=np.array([5, 3]), reset=np.array([[0, 0, 1, 0, 0], [1, 0, 0, 0, 1]]))

    def loss():
        r = ref.ssm(x, dt, A, b, c, z, skip, bias, True, h0, **how)
        return (r["y"][0] * dy).sum() + (r["h_last"][0] * dl).sum()

    got = ref.ssm(x, dt, A, b, c, z, skip, bias, True, h0, dy=dy, dh_last=dl, **how)
    differences(loss, (x, dt, A, b, c, z, skip, bias, h0), got, ("dx", "ddt", "dA", "db", "dc", "dz", "dskip", "ddt_bias", "dh0"))


def test_the_policy_reference_s_gradients():
    rng = np.random.default_rng(3)
    N, V = 3, 6
    z, y, old, A = rng.standard_normal((N, V)), rng.integers(0, V, N), -1.8 + 0.2 * rng.standard_normal(N), rng.standard_normal(N)
    r = rng.standard_normal(N) - 2
    how = dict(tau=0.8, kl=0.3, bonus=0.1)
    got = ref.policy(z, y, old, A, r, **how)
    differences(lambda: ref.policy(z, y, old, A, r, **how)["loss"][0].sum(), (z,), got, ("grad",))
