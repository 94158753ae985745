"""Asynchronous policy gradients of a small selective state space language model.

Workers answer prompts with their own stale snapshots of the model, score the answers and commit the
gradients of the clipped policy loss with Gradient Energy Matching.  A worker's step runs the library's operators:

  answer    gem_embed, gem_conv_forward and gem_ssm_forward with one step and their states carried on
  train     gem_embed, gem_conv_forward, gem_ssm_forward, gem_policy (loss and gradient of the logits),
            gem_ssm_backward, gem_conv_backward, gem_embed_grad
  commit    gem_commit at the central variable

The matrix products are torch's.  The task: after each token t comes one of the tokens that 3 t + 1 gives modulo
a tenth of the vocabulary.

    python examples/async_policy.py [commits]
"""
from __future__ import annotations

import sys
from pathlib import Path

import torch

sys.path.insert(0, str(Path(__file__).resolve().parents[1]))

from paper_1805_08469_gb300 import gem, lm, sim  # noqa: E402

W = 4   # taps of the convolution


class Model:
    """embedding [V, d] -> input and gate [2 D, d] -> convolution -> step sizes, b and c [D + 2 N, D] -> scan, gated -> logits
    [V, D], its parameters views into one flat vector."""

    def __init__(self, V: int, d: int, D: int, N: int):
        self.V, self.d, self.D, self.N = V, d, D, N
        self.shapes = {"embed": (V, d), "inward": (2 * D, d), "taps": (D, W), "taps_bias": (D,), "mix": (D + 2 * N, D), "A_log": (D, N),
                       "skip": (D,), "dt_bias": (D,), "outward": (V, D)}
        self.P = sum(torch.Size(s).numel() for s in self.shapes.values())

    def views(self, flat):
        out, at = {}, 0
        for name, shape in self.shapes.items():
            n = torch.Size(shape).numel()
            out[name] = flat[at:at + n].view(shape)
            at += n
        return out

    def init(self, generator):
        flat = torch.empty(self.P, device="cuda")
        v = self.views(flat)
        for name, scale in dict(embed=1.0, inward=self.d ** -0.5, taps=W ** -0.5, taps_bias=0.0, mix=self.D ** -0.5, outward=self.D ** -0.5).items():
            v[name].copy_(scale * torch.randn(v[name].shape, device="cuda", generator=generator))
        v["A_log"].copy_(torch.arange(1, self.N + 1, device="cuda").float().log().expand(self.D, self.N))
        v["skip"].fill_(1.0)
        step = 10 ** (-2 + 1.5 * torch.rand(self.D, device="cuda", generator=generator))
        v["dt_bias"].copy_(step + torch.log(-torch.expm1(-step)))
        return flat

    def state(self, B: int):
        """What a sequence carries from token to token: the convolution's last inputs and the scan's states."""
        return torch.zeros(B, W - 1, self.D, device="cuda"), torch.zeros(B, self.D, self.N, device="cuda")

    def forward(self, flat, tokens, state=None, keep=False):
        """Logits [B T, V] of tokens [B, T], from `state` on (which is replaced in place), and what the backward pass needs."""
        (B, T), D, N = tokens.shape, self.D, self.N
        v = self.views(flat)
        new = lambda *shape: torch.empty(shape, device="cuda")  # noqa: E731
        e = new(B * T, self.d)
        lm.gem_embed(v["embed"], tokens.reshape(-1), e, scale=self.d ** 0.5)
        both = (e @ v["inward"].t()).view(B, T, 2 * D)
        x, z = both[..., :D], both[..., D:]
        conv, h = state if state is not None else (None, None)
        u, y = new(B, T, D), new(B, T, D)
        lm.gem_conv_forward(x, v["taps"].contiguous(), u, bias=v["taps_bias"], state=conv, state_last=conv)
        mixed = (u.view(-1, D) @ v["mix"].t()).view(B, T, D + 2 * N)
        dt, b, c = mixed[..., :D], mixed[..., D:D + N].unflatten(2, (1, N)), mixed[..., D + N:].unflatten(2, (1, N))
        A = -v["A_log"].exp()
        saved = new(B, -(-T // lm.GEM_SSM_CHUNK), D, N) if keep else None
        space = new(lm.gem_ssm_workspace(B, T, D, N, backward=keep))
        lm.gem_ssm_forward(u, dt, A, b, c, y, z=z, skip=v["skip"], dt_bias=v["dt_bias"], h0=h, h_last=h, saved=saved, workspace=space)
        return y.view(-1, D) @ v["outward"].t(), (e, x, z, u, dt, b, c, A, y, saved, space)

    def backward(self, flat, tokens, kept, dlogits):
        """The gradient as a flat vector (sequences that began without a state)."""
        (B, T), D, N = tokens.shape, self.D, self.N
        e, x, z, u, dt, b, c, A, y, saved, space = kept
        v, grad = self.views(flat), torch.empty(self.P, device="cuda")
        g = self.views(grad)
        new = lambda *shape: torch.empty(shape, device="cuda")  # noqa: E731
        g["outward"].copy_(dlogits.t() @ y.view(-1, D))
        dy = (dlogits @ v["outward"]).view(B, T, D)
        dboth, dmixed, du, dA = new(B, T, 2 * D), new(B, T, D + 2 * N), new(B, T, D), new(D, N)
        part = lambda lo: dmixed[..., lo:lo + N].unflatten(2, (1, N))  # noqa: E731
        lm.gem_ssm_backward(u, dt, A, b, c, saved, dy, du, dmixed[..., :D], dA, part(D), part(D + N), z=z, dz=dboth[..., D:], skip=v["skip"],
                            dskip=g["skip"], dt_bias=v["dt_bias"], ddt_bias=g["dt_bias"], workspace=space)
        g["A_log"].copy_(dA * A)
        flat_mixed = dmixed.view(-1, D + 2 * N)
        g["mix"].copy_(flat_mixed.t() @ u.view(-1, D))
        du += (flat_mixed @ v["mix"]).view(B, T, D)
        lm.gem_conv_backward(x, v["taps"], du, dboth[..., :D], g["taps"], new(lm.gem_conv_workspace(B, T, D, W)), bias=v["taps_bias"],
                             dbias=g["taps_bias"])
        flat_both = dboth.view(-1, 2 * D)
        g["inward"].copy_(flat_both.t() @ e)
        room = torch.empty(lm.gem_embed_workspace(B * T, self.V, self.d), dtype=torch.uint8, device="cuda")
        lm.gem_embed_grad(flat_both @ v["inward"], tokens.reshape(-1), g["embed"], room, scale=self.d ** 0.5)
        return grad

    def answer(self, flat, first, steps: int, generator):
        """Tokens [B, steps] sampled one by one after `first` [B], with their log probabilities."""
        B = first.shape[0]
        state, token, tokens, scores = self.state(B), first, [], []
        for _ in range(steps):
            logits, _ = self.forward(flat, token[:, None], state)
            token = torch.multinomial(logits.softmax(1), 1, generator=generator)[:, 0].to(torch.int32)
            logp = torch.empty(B, device="cuda")
            lm.gem_token_logp(logits, token, logp)
            tokens.append(token)
            scores.append(logp)
        return torch.stack(tokens, 1), torch.stack(scores, 1)


def loss_and_gradient(model, flat, read, sampled, old_logp, advantage, bonus: float = 0.01, ref_logp=None, kl: float = 0.0):
    """The mean policy loss of tokens `sampled` [B, T] after the tokens `read` [B, T], and its gradient."""
    n = sampled.numel()
    logits, kept = model.forward(flat, read, keep=True)
    loss = torch.empty(n, device="cuda")
    lm.gem_policy(logits, sampled.reshape(-1), old_logp.reshape(-1), advantage.reshape(-1), loss, logits, ref_logp=ref_logp,
                  row_scale=torch.full((n,), 1.0 / n, device="cuda"), kl=kl, bonus=bonus)   # in place
    return loss.mean(), model.backward(flat, read, kept, logits)


def main(commits: int = 300, n: int = 4, V: int = 200, B: int = 32, T: int = 24, eta: float = 0.002, seed: int = 5, verbose: bool = True):
    """Returns the mean rewards and losses of the commits."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    model = Model(V, 32, 64, 16)
    order, _ = sim.gem_schedule_uniform(seed, n, commits)
    rewards, losses = torch.empty(commits, device="cuda"), torch.empty(commits, device="cuda")
    with gem.Gem(model.P, n, eta=eta, mu=0.9, eps=1e-8, stream=torch.cuda.current_stream()) as G:
        theta = model.init(g)
        model.views(theta)["outward"].mul_(0.02)              # (nearly even chances to begin with)
        G.set_theta(theta)
        for t, w in enumerate(order.tolist()):
            flat = G.snapshot(w)                              # the worker's stale parameters
            first = torch.randint(0, V, (B,), device="cuda", generator=g, dtype=torch.int32)
            sampled, old = model.answer(flat, first, T, g)
            read = torch.cat([first[:, None], sampled[:, :-1]], 1)
            reward = (sampled % (V // 10) == (3 * read + 1) % (V // 10)).float()
            losses[t], grad = loss_and_gradient(model, flat, read, sampled, old, reward - reward.mean())
            G.commit(w, grad)
            rewards[t] = reward.mean()
            if verbose and (t + 1) % max(1, commits // 8) == 0:
                print(f"commit {t + 1}: reward {rewards[max(0, t - 9):t + 1].mean().item():.4f}")
        G.sync()
    return rewards, losses


if __name__ == "__main__":
    main(int(sys.argv[1]) if len(sys.argv) > 1 else 300)
