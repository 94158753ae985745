"""Asynchronous distillation of a small gated recurrent language model.

Workers train a student against a fixed teacher and commit their gradients with Gradient Energy
Matching, in the order of a seeded schedule.  Each worker's step runs the library's operators at
the worker's stale snapshot:

  teacher   gem_glr_forward, then gem_token_logp: its top entries and log-sum-exp
  student   gem_glr_forward, gem_distill (loss and gradient of the logits), gem_glr_backward
  commit    gem_commit at the central variable

and in the end the student answers token by token (gem_glr_forward with one step and the state
carried on, gem_token_logp for the most likely token).  The matrix products are torch's.

    python examples/async_distill.py [commits]
"""
from __future__ import annotations

import sys
from pathlib import Path

import torch

sys.path.insert(0, str(Path(__file__).resolve().parents[1]))

from paper_1805_08469_gb300 import gem, lm, sim  # noqa: E402


class Model:
    """embedding [V, d] -> candidate and gate [2 D, d] -> gated linear recurrence -> logits [V, D], its
    parameters views into one flat vector."""

    def __init__(self, V: int, d: int, D: int):
        self.V, self.d, self.D = V, d, D
        self.shapes = [(V, d), (2 * D, d), (V, D)]
        self.P = sum(a * b for a, b in self.shapes)

    def views(self, flat):
        out, at = [], 0
        for a, b in self.shapes:
            out.append(flat[at:at + a * b].view(a, b))
            at += a * b
        return out

    def init(self, generator):
        flat = torch.empty(self.P, device="cuda")
        for v, scale in zip(self.views(flat), (1.0, 1.5 / self.d ** 0.5, 3.0 / self.D ** 0.5)):
            v.copy_(scale * torch.randn(v.shape, device="cuda", generator=generator))
        return flat

    def forward(self, flat, tokens, saved=None):
        """Logits [B T, V], and what the backward pass needs."""
        embed, inward, outward = self.views(flat)
        e = embed[tokens]                                   # [B, T, d]
        both = e @ inward.t()                               # [B, T, 2 D]: candidate and gate side by side
        x, f = both[..., :self.D], both[..., self.D:]
        h = torch.empty(x.shape, device="cuda")
        lm.gem_glr_forward(x, f, h, saved=saved)
        return h.view(-1, self.D) @ outward.t(), (e, x, f, h)

    def backward(self, flat, tokens, kept, saved, dlogits):
        """The gradient as a flat vector."""
        _, inward, outward = self.views(flat)
        e, x, f, h = kept
        grad = torch.zeros(self.P, device="cuda")
        d_embed, d_inward, d_outward = self.views(grad)
        d_outward.copy_(dlogits.t() @ h.view(-1, self.D))
        dh = (dlogits @ outward).view(h.shape)
        both = torch.empty(*h.shape[:2], 2 * self.D, device="cuda")
        lm.gem_glr_backward(x, f, saved, dh, both[..., :self.D], both[..., self.D:])
        flat_both = both.view(-1, 2 * self.D)
        d_inward.copy_(flat_both.t() @ e.view(-1, self.d))
        d_embed.index_add_(0, tokens.reshape(-1), flat_both @ inward)
        return grad

    def generate(self, flat, first, steps: int):
        """The most likely continuation of one token for each sequence, a call per token."""
        embed, inward, outward = self.views(flat)
        B = first.shape[0]
        state = torch.zeros(B, self.D, device="cuda")
        h = torch.empty(B, 1, self.D, device="cuda")
        best, logp = torch.empty(B, 1, dtype=torch.int32, device="cuda"), torch.empty(B, 1, device="cuda")
        out, token = [], first
        for _ in range(steps):
            both = (embed[token] @ inward.t())[:, None]
            lm.gem_glr_forward(both[..., :self.D], both[..., self.D:], h, h0=state, h_last=state)
            lm.gem_token_logp(h[:, 0] @ outward.t(), top_idx=best, top_logp=logp)
            token = best[:, 0].long()
            out.append(token)
        return torch.stack(out, 1)


def teach(teacher, flat, tokens, K: int, tau: float):
    """The teacher's top K entries of every position, and its log-sum-exp (both at temperature tau)."""
    logits, _ = teacher.forward(flat, tokens)
    N = logits.shape[0]
    idx = torch.empty(N, K, dtype=torch.int32, device="cuda")
    top, lse = torch.empty(N, K, device="cuda"), torch.empty(N, device="cuda")
    lm.gem_token_logp(logits, temperature=tau, lse=lse, top_idx=idx, top_logp=top)
    return idx, (top + lse[:, None]) * tau, lse


def main(commits: int = 400, n: int = 4, V: int = 500, B: int = 8, T: int = 64, K: int = 16, tau: float = 1.0, eta: float = 5.0, seed: int = 7,
         verbose: bool = True):
    """Returns the mean losses of the first and the last tenth of the commits, and the share of tokens on
    which the student continues a sequence as the teacher does."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    teacher, student = Model(V, 32, 64), Model(V, 32, 64)
    teacher_flat = teacher.init(g)
    order, _ = sim.gem_schedule_uniform(seed, n, commits)
    saved = torch.empty(B, -(-T // lm.GEM_GLR_CHUNK), student.D, device="cuda")
    losses = torch.empty(commits, device="cuda")
    scale = torch.full((B * T,), 1.0 / (B * T), device="cuda")
    with gem.Gem(student.P, n, eta=eta, mu=0.9, eps=1e-8, stream=torch.cuda.current_stream()) as G:
        G.set_theta(0.3 * student.init(g))
        for t, w in enumerate(order.tolist()):
            tokens = torch.randint(0, V, (B, T), device="cuda", generator=g)
            idx, top, lse = teach(teacher, teacher_flat, tokens, K, tau)
            flat = G.snapshot(w)                            # the worker's stale parameters
            logits, kept = student.forward(flat, tokens, saved)
            loss = torch.empty(B * T, device="cuda")
            lm.gem_distill(logits, idx, top, loss, logits, teacher_lse=lse, row_scale=scale, temperature=tau)   # in place
            G.commit(w, student.backward(flat, tokens, kept, saved, logits))
            losses[t] = loss.mean()
            if verbose and (t + 1) % max(1, commits // 8) == 0:
                print(f"commit {t + 1}: loss {losses[max(0, t - 9):t + 1].mean().item():.4f}")
        first = torch.arange(64, device="cuda") % V
        a, b = teacher.generate(teacher_flat, first, 16), student.generate(G.theta(), first, 16)
        G.sync()
    tenth = max(1, commits // 10)
    result = losses[:tenth].mean().item(), losses[-tenth:].mean().item(), (a == b).float().mean().item()
    if verbose:
        print("mean loss of the first tenth {:.4f}, of the last {:.4f}; tokens as the teacher's: {:.1%}".format(*result))
    return result


if __name__ == "__main__":
    main(int(sys.argv[1]) if len(sys.argv) > 1 else 400)
