"""Language-model operators without a GPU: sizes, refusals on the host, and the binding's checks
of its tensors.  No call here passes every check with work to do, so nothing is launched."""
import ctypes as C

import pytest
import torch

from paper_1805_08469_gb300 import _lib, lm
from paper_1805_08469_gb300._build import build_library

OK, EINVAL = 0, -1
PTR = 1 << 20          # an aligned address; a refused call never reads it


@pytest.fixture(scope="module")
def L():
    build_library()
    return _lib.lib()


def seq(data=PTR, sb=1000, st=10):
    return _lib.GemSeq(data, sb, st)


def fwd(L, dtype=0, form=0, B=2, T=4, D=10, x=None, f=None, h0=0, lengths=0, reset=0, h=None, h_last=0, saved=0):
    return L.gem_glr_forward(dtype, form, B, T, D, x or seq(), f or seq(), h0, lengths, reset, h or seq(), h_last, saved, 0)


def bwd(L, dtype=0, form=0, B=2, T=4, D=10, saved=PTR, dh=None, dx=None, df=None, dh_last=0, dh0=0):
    return L.gem_glr_backward(dtype, form, B, T, D, seq(), seq(), 0, 0, saved, dh or seq(), dh_last, dx or seq(), df or seq(), dh0, 0)


@pytest.mark.parametrize("bad", [
    dict(dtype=-1), dict(dtype=3), dict(form=2), dict(form=-1), dict(B=-1), dict(T=-1), dict(D=-1),
    dict(B=1 << 31), dict(T=1 << 31), dict(B=1 << 20, D=1 << 20),
    dict(x=seq(0)), dict(f=seq(0)), dict(h=seq(0)), dict(x=seq(PTR + 2)), dict(dtype=1, f=seq(PTR + 1)),
    dict(x=seq(sb=-1)), dict(f=seq(st=-10)), dict(x=seq(sb=1 << 60)),
    dict(h=seq(st=9)), dict(h=seq(sb=39)), dict(h=seq(sb=9, st=100)), dict(h=seq(sb=0)), dict(h=seq(st=0)),
    dict(h=seq(sb=10, st=19)),
    dict(h0=PTR + 2), dict(lengths=PTR + 1), dict(h_last=PTR + 2), dict(saved=PTR + 3)])
def test_glr_forward_refuses(L, bad):
    assert fwd(L, **bad) == EINVAL


@pytest.mark.parametrize("bad", [
    dict(dtype=7), dict(form=3), dict(T=-2), dict(saved=0), dict(saved=PTR + 1), dict(dh=seq(0)), dict(dx=seq(0)),
    dict(df=seq(st=3)), dict(dx=seq(sb=0)), dict(dh_last=PTR + 2), dict(dh0=PTR + 1), dict(dh=seq(sb=-5))])
def test_glr_backward_refuses(L, bad):
    assert bwd(L, **bad) == EINVAL


def test_null_tensors_are_refused(L):
    args = [0, 0, 1, 1, 1]
    one = seq()
    for k in range(3):
        t = [one, one, one]
        t[k] = None
        assert L.gem_glr_forward(*args, t[0], t[1], 0, 0, 0, t[2], 0, 0, 0) == EINVAL
    for k in range(5):
        t = [one] * 5
        t[k] = None
        assert L.gem_glr_backward(*args, t[0], t[1], 0, 0, PTR, t[2], 0, t[3], t[4], 0, 0) == EINVAL


def test_empty_sizes_leave_nothing_to_do(L):
    none = seq(0)
    assert fwd(L, B=0, x=none, f=none, h=none) == OK
    assert fwd(L, D=0, x=none, f=none, h=none) == OK
    assert fwd(L, T=0, x=none, f=none, h=none) == OK
    assert bwd(L, T=0, saved=0) == OK
    assert distill(L, N=0, logits=0, loss=0, grad=0) == OK
    assert logp(L, N=0, logits=0, logp=0) == OK
    assert logp_grad(L, N=0, logits=0, grad=0) == OK


def test_saved_count(L):
    for B, T, D, want in [(2, 1, 5, 10), (2, 16, 5, 10), (2, 17, 5, 20), (3, 0, 4, 0), (0, 9, 9, 0),
                          (1, 100003, 1024, 6251 * 1024), (-1, 1, 1, -1), (1, -1, 1, -1), (1, 1, -1, -1)]:
        assert L.gem_glr_saved_count(B, T, D) == want


def distill(L, dtype=0, N=2, V=100, logits=PTR, ld=100, K=3, idx=PTR, top=PTR, lse=0, labels=0, scale=0, tau=1.0,
            alpha=0.0, loss=PTR, grad=PTR, grad_ld=100):
    return L.gem_distill(dtype, N, V, logits, ld, K, idx, top, lse, labels, scale, tau, alpha, loss, grad, grad_ld, 0)


NAN, INF = float("nan"), float("inf")


@pytest.mark.parametrize("bad", [
    dict(dtype=3), dict(N=-1), dict(N=1 << 31), dict(V=0), dict(V=1 << 31), dict(logits=0), dict(logits=PTR + 2),
    dict(ld=99), dict(ld=-100), dict(ld=1 << 50), dict(K=-1), dict(K=257), dict(idx=0), dict(top=0), dict(idx=PTR + 1),
    dict(lse=PTR + 2), dict(scale=PTR + 2), dict(loss=0), dict(loss=PTR + 2), dict(alpha=0.5), dict(alpha=0.5, labels=PTR + 2),
    dict(alpha=-0.1), dict(alpha=1.1), dict(alpha=NAN), dict(tau=0.0), dict(tau=-1.0), dict(tau=NAN), dict(tau=INF),
    dict(tau=1e-30), dict(grad_ld=99), dict(grad=PTR + 2), dict(grad_ld=101), dict(ld=0)])
def test_distill_refuses(L, bad):
    assert distill(L, **bad) == EINVAL      # (grad is logits here: another pitch is refused too)


def logp(L, dtype=1, N=2, V=100, logits=PTR, ld=100, tokens=PTR, tau=1.0, K=0, logp=PTR, entropy=0, lse=0, idx=0, top=0):
    return L.gem_token_logp(dtype, N, V, logits, ld, tokens, tau, K, logp, entropy, lse, idx, top, 0)


@pytest.mark.parametrize("bad", [
    dict(dtype=-1), dict(N=-1), dict(V=0), dict(logits=0), dict(logits=PTR + 1), dict(ld=50), dict(tokens=0),
    dict(tokens=PTR + 2), dict(tau=0.0), dict(tau=NAN), dict(K=-1), dict(K=257, V=1000, ld=1000, idx=PTR, top=PTR),
    dict(K=101, idx=PTR, top=PTR), dict(K=5), dict(K=5, idx=PTR), dict(K=5, top=PTR), dict(entropy=PTR + 2), dict(lse=PTR + 1)])
def test_token_logp_refuses(L, bad):
    assert logp(L, **bad) == EINVAL


def logp_grad(L, dtype=2, N=2, V=100, logits=PTR, ld=100, tokens=PTR, tau=1.0, lse=PTR, entropy=PTR, dlogp=PTR, dentropy=PTR,
              grad=PTR, grad_ld=100):
    return L.gem_token_logp_grad(dtype, N, V, logits, ld, tokens, tau, lse, entropy, dlogp, dentropy, grad, grad_ld, 0)


@pytest.mark.parametrize("bad", [
    dict(dtype=9), dict(N=-1), dict(V=-1), dict(logits=0), dict(ld=10), dict(tokens=0), dict(tau=-2.0), dict(lse=0),
    dict(entropy=0), dict(dlogp=PTR + 2), dict(dentropy=PTR + 2), dict(grad=0), dict(grad=PTR + 1), dict(grad_ld=99),
    dict(grad_ld=108)])
def test_token_logp_grad_refuses(L, bad):
    assert logp_grad(L, **bad) == EINVAL


def test_the_binding_checks_its_tensors():
    """Tensors of the host, of another type, shape or layout are refused before the library is called."""
    z = torch.zeros(2, 8)
    with pytest.raises(TypeError):
        lm.gem_token_logp(z, torch.zeros(2, dtype=torch.int32), torch.zeros(2))
    with pytest.raises(TypeError):
        lm.gem_distill(z, torch.zeros(2, 1, dtype=torch.int32), torch.zeros(2, 1), torch.zeros(2))
    with pytest.raises(TypeError):
        lm.gem_token_logp(z.t(), torch.zeros(8, dtype=torch.int32), torch.zeros(8))
    with pytest.raises(ValueError):
        lm.gem_token_logp(z[0], None, None)
    with pytest.raises(ValueError):
        lm.gem_token_logp(z, None, None, top_idx=torch.zeros(2, 1, dtype=torch.int32))
    x = torch.zeros(1, 2, 4)
    with pytest.raises(TypeError):
        lm.gem_glr_forward(x, x, x)
    with pytest.raises(ValueError):
        lm.gem_glr_forward(x[0], x[0], x[0])


def test_gem_seq_layout():
    assert C.sizeof(_lib.GemSeq) == 24
