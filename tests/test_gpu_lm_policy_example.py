"""The example that uses embedding, convolution, scan and policy loss together: its gradient against that of
plain operations in 64 bits, its answers token by token against whole sequences, and the operators in a captured graph."""
import sys

import pytest
import torch

from conftest import ROOT
from paper_1805_08469_gb300 import lm

pytestmark = pytest.mark.gpu

sys.path.insert(0, str(ROOT / "examples"))


def plain_loss(m, flat, read, sampled, old, advantage, bonus, ref, kl):
    """The mean loss in elementary operations, from a leaf in 64 bits."""
    v = m.views(flat)
    (B, T), D, N = read.shape, m.D, m.N
    e = v["embed"][read.long()] * m.d ** 0.5
    both = e @ v["inward"].t()
    x, z = both[..., :D], both[..., D:]
    padded = torch.cat([torch.zeros(B, 3, D, dtype=x.dtype, device=x.device), x], 1)
    p = v["taps_bias"] + sum(padded[:, k:k + T] * v["taps"][:, k] for k in range(4))
    u = p * torch.sigmoid(p)
    mixed = u @ v["mix"].t()
    step = torch.nn.functional.softplus(mixed[..., :D] + v["dt_bias"])
    b, c = mixed[..., D:D + N], mixed[..., D + N:]
    A = -v["A_log"].exp()
    h, ys = torch.zeros(B, D, N, dtype=x.dtype, device=x.device), []
    for t in range(T):
        h = torch.exp(step[:, t, :, None] * A) * h + (step[:, t] * u[:, t])[..., None] * b[:, t, None]
        ys.append((h * c[:, t, None]).sum(-1) + v["skip"] * u[:, t])
    y = torch.stack(ys, 1) * z * torch.sigmoid(z)
    lp = torch.log_softmax(y @ v["outward"].t(), -1).view(B * T, -1)
    logp = lp.gather(1, sampled.reshape(-1, 1).long())[:, 0]
    r = torch.exp(logp - old)
    far = ref - logp
    H = -(lp.exp() * lp).sum(1)
    loss = torch.maximum(-r * advantage, -r.clamp(0.8, 1.2) * advantage) + kl * (far.exp() - far - 1) - bonus * H
    return loss.mean()


def test_the_whole_model_s_gradient():
    """Every fp32 operation is the exact one on values moved by up to 2^-24 of themselves.  What such moves of the parameters alone
    do to the exact gradient is measured here (logits of several hundred make it some 1e-4); the operations on the way, eight
    products and sums between a parameter and the loss and as many back, may do sixteen times that if all agree."""
    import async_policy

    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    m = async_policy.Model(50, 12, 20, 5)
    flat = m.init(g)
    read = torch.randint(0, 50, (3, 37), device="cuda", generator=g, dtype=torch.int32)
    sampled = torch.randint(0, 50, (3, 37), device="cuda", generator=g, dtype=torch.int32)
    logits, _ = m.forward(flat, read)
    logp = torch.log_softmax(logits.double(), 1).gather(1, sampled.reshape(-1, 1).long())[:, 0]
    # ratios of 0.9, 1.1 and beyond the bounds, none on one
    moved = torch.tensor([-0.5, -0.1, 0.1, 0.5], device="cuda")[torch.randint(0, 4, (111,), device="cuda", generator=g)]
    old, ref = (logp - moved).float(), (logp + 0.3).float()
    advantage = torch.randn(111, device="cuda", generator=g)
    loss, grad = async_policy.loss_and_gradient(m, flat, read, sampled, old, advantage, 0.05, ref, 0.1)

    def exact_of(theta):
        leaf = theta.detach().clone().requires_grad_()
        value = plain_loss(m, leaf, read, sampled, old.double(), advantage.double(), 0.05, ref.double(), 0.1)
        value.backward()
        return value.item(), m.views(leaf.grad)

    value, exact = exact_of(flat.double())
    moves = [exact_of(flat.double() * (1 + 2.0 ** -24 * torch.randn(m.P, device="cuda", dtype=torch.float64, generator=g)))[1] for _ in range(4)]
    assert abs(loss.item() - value) < 1e-4 * abs(value)
    for name, got in m.views(grad).items():
        bound = 16 * max((v[name] - exact[name]).norm() for v in moves)
        assert bound < 0.01 * exact[name].norm(), name      # (the test says something)
        assert (got - exact[name]).norm() <= bound, name


def test_answers_token_by_token_are_the_sequence_s():
    """Log probabilities given one by one, with the states carried on, are those of the whole sequence."""
    import async_policy

    g = torch.Generator(device="cuda")
    g.manual_seed(2)
    m = async_policy.Model(60, 16, 24, 16)
    flat = m.init(g)
    first = torch.arange(8, device="cuda", dtype=torch.int32)
    sampled, scores = m.answer(flat, first, 40, g)
    logits, _ = m.forward(flat, torch.cat([first[:, None], sampled[:, :-1]], 1))
    logp = torch.log_softmax(logits.double(), 1).gather(1, sampled.reshape(-1, 1).long()).view(8, 40)
    assert (logp - scores).abs().max() < 1e-4


def test_it_runs():
    import async_policy

    rewards, losses = async_policy.main(commits=12, B=8, T=10, verbose=False)
    assert bool(torch.isfinite(rewards).all() and torch.isfinite(losses).all())


def test_a_captured_step_gives_the_same():
    """Forward, loss and backward captured into a graph and replayed on other inputs, on a stream of its own."""
    import async_policy

    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    m = async_policy.Model(70, 16, 32, 16)
    flat = m.init(g)
    make = lambda: (torch.randint(0, 70, (2, 300), device="cuda", generator=g, dtype=torch.int32),  # noqa: E731
                    torch.randint(0, 70, (2, 300), device="cuda", generator=g, dtype=torch.int32), -4 * torch.rand(600, device="cuda", generator=g),
                    torch.randn(600, device="cuda", generator=g))
    inputs = [t.clone() for t in make()]
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        async_policy.loss_and_gradient(m, flat, *inputs)      # (a first call outside the graph)
    stream.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        loss, grad = async_policy.loss_and_gradient(m, flat, *inputs)
    for _ in range(3):
        other = make()
        for a, b in zip(inputs, other):
            a.copy_(b)
        graph.replay()
        torch.cuda.synchronize()
        got = loss.clone(), grad.clone()
        want = async_policy.loss_and_gradient(m, flat, *other)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_two_calls_at_once():
    """Two streams with buffers of their own give what each gives alone."""
    import async_policy

    g = torch.Generator(device="cuda")
    g.manual_seed(4)
    m = async_policy.Model(90, 16, 64, 16)
    flat = m.init(g)
    data = [(torch.randint(0, 90, (4, 500), device="cuda", generator=g, dtype=torch.int32),
             torch.randint(0, 90, (4, 500), device="cuda", generator=g, dtype=torch.int32), -4 * torch.rand(2000, device="cuda", generator=g),
             torch.randn(2000, device="cuda", generator=g)) for _ in range(2)]
    want = [async_policy.loss_and_gradient(m, flat, *d) for d in data]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [None, None]
    for _ in range(4):
        for i, s in enumerate(streams):
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                got[i] = async_policy.loss_and_gradient(m, flat, *data[i])
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_the_explicit_stream_is_used():
    """A call on a stream that waits for its inputs' producer, while the current stream does not."""
    side = torch.cuda.Stream()
    table, tokens = torch.randn(50, 64, device="cuda"), torch.arange(50, device="cuda", dtype=torch.int32)
    out = torch.zeros(50, 64, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        big = torch.randn(4096, 4096, device="cuda")
        for _ in range(20):
            big = big @ big * 1e-3
        table.mul_(2.0)
    lm.gem_embed(table, tokens, out, stream=side)
    side.synchronize()
    assert torch.equal(out, table)
