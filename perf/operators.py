"""Performance cases of the sequence-model operators: what a program whose workers train, or
answer with, a gated recurrent language model has the library do.

  glr      the gated linear recurrence: one token at a time with the state carried on
           (serving), a whole prompt (forward), or forward and backward (training)
  distill  the loss of a student's logits against a teacher's top entries, with its gradient
  logp     log probabilities of given tokens with entropy and the top alternatives, or (in
           training) log probability and entropy with the gradient of both

A pass is one call that a user makes (two in training, where the backward pass needs what the
forward pass computed), on buffers that the program owns.  The plain forms are elementary torch
operations in 32 bits, rounded once at the end.
"""
from __future__ import annotations

import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}


def listed():
    return [
        # serving: one token for each of 4 sequences, the state updated in place
        dict(name="glr_step_b4", op="glr", pass_="step", form="lerp", dtype="bf16", B=4, T=1, D=1024, ragged=0, resets=0, fused=0),
        # a batch of prompts of different lengths, an even channel count that is no power of two
        dict(name="glr_prompts_f16", op="glr", pass_="forward", form="add", dtype="f16", B=12, T=1777, D=1000, ragged=1, resets=0, fused=0),
        # training on full sequences; candidate and gate are the halves of one projection's output
        dict(name="glr_train_bf16", op="glr", pass_="train", form="lerp", dtype="bf16", B=8, T=4096, D=2048, ragged=0, resets=0, fused=1),
        # training on one long stream of packed documents, the state dropped where one begins
        dict(name="glr_train_long_f32", op="glr", pass_="train", form="lerp", dtype="f32", B=1, T=100003, D=1024, ragged=0, resets=1, fused=0),
        # distilling a small classifier: a few short rows, where latency counts
        dict(name="distill_small_f32", op="distill", dtype="f32", N=64, V=1000, K=8, tau=1.0, alpha=0.0, tail=0),
        # the usual recipe: softened teacher, hard labels mixed in, padded positions masked
        dict(name="distill_v32k_bf16", op="distill", dtype="bf16", N=4096, V=32000, K=64, tau=2.0, alpha=0.3, tail=0),
        # an odd vocabulary (rows between alignments), the teacher's remaining mass as one class
        dict(name="distill_tail_odd_f16", op="distill", dtype="f16", N=1023, V=50001, K=20, tau=1.0, alpha=0.0, tail=1),
        # a large vocabulary and many teacher entries: the largest batch
        dict(name="distill_v131k_bf16", op="distill", dtype="bf16", N=4096, V=131072, K=128, tau=1.0, alpha=0.0, tail=0),
        # serving: the next token's log probability and its alternatives for one sequence
        dict(name="logp_next_token", op="logp", dtype="bf16", N=1, V=131072, K=20, tau=1.0, grad=0),
        # serving a batch at a sampling temperature, odd vocabulary
        dict(name="logp_batch_odd_f16", op="logp", dtype="f16", N=64, V=50001, K=5, tau=0.7, grad=0),
        # scoring a corpus, or writing out a teacher's top entries for distillation
        dict(name="logp_score_bf16", op="logp", dtype="bf16", N=4096, V=131072, K=64, tau=1.0, grad=0),
        # training on log probabilities with an entropy bonus: forward and gradient
        dict(name="logp_train_f32", op="logp", dtype="f32", N=2048, V=32000, K=0, tau=1.0, grad=1),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["glr", "glr", "distill", "logp"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    if op == "glr":
        pass_ = rng.choice(["step", "forward", "train", "train"])
        while True:
            B, D = _log_int(rng, 1, 64), _log_int(rng, 64, 4096)
            T = 1 if pass_ == "step" else _log_int(rng, 2, 60000)
            if B * T * D <= 67108864:
                break
        if rng.random() < 0.6:
            D = max(8, D // 8 * 8)
        several = pass_ != "step"
        return dict(op="glr", pass_=pass_, form=rng.choice(["lerp", "add"]), dtype=dtype, B=B, T=T, D=D,
                    ragged=rng.randint(0, 1) if several else 0, resets=rng.randint(0, 1) if several else 0,
                    fused=rng.randint(0, 1))
    while True:
        N, V = _log_int(rng, 1, 8192), _log_int(rng, 500, 160000)
        if N * V <= (2.6e8 if dtype == "f32" else 5.3e8):
            break
    if rng.random() < 0.5:
        V = V // 8 * 8
    if op == "distill":
        return dict(op="distill", dtype=dtype, N=N, V=V, K=_log_int(rng, 1, 128), tau=rng.choice([1.0, 2.0, rng.uniform(0.5, 4.0)]),
                    alpha=rng.choice([0.0, 0.0, 0.5, rng.uniform(0.05, 0.95)]), tail=rng.randint(0, 1))
    grad = rng.choice([0, 0, 1])
    return dict(op="logp", dtype=dtype, N=N, V=V, K=0 if grad else _log_int(rng, 1, 128), tau=rng.choice([1.0, 1.0, rng.uniform(0.5, 2.0)]), grad=grad)


def work(case):
    e = BYTES[case["dtype"]]
    if case["op"] == "glr":
        B, T, D = case["B"], case["T"], case["D"]
        n = B * T * D
        if case["pass_"] == "train":   # x, f, dh in; h, dx, df out; the last state, its gradient, dh0
            return {"bytes": 6 * n * e + 12 * B * D, "flops": 25 * n}
        return {"bytes": 3 * n * e + 8 * B * D, "flops": 10 * n}
    N, V, K = case["N"], case["V"], case["K"]
    if case["op"] == "distill":
        return {"bytes": 2 * N * V * e + N * (8 * K + 16), "flops": N * V * 8}
    return {"bytes": (2 if case["grad"] else 1) * N * V * e + N * (8 * K + 12), "flops": N * V * (12 if case["grad"] else 6)}


# ---------------------------------------------------------------------------- inputs


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _glr_inputs(case, seed):
    g = _generator(seed)
    B, T, D, t = case["B"], case["T"], case["D"], TYPES[case["dtype"]]
    s = {}

    def pair():
        if case["fused"]:
            both = torch.empty((B, T, 2 * D), dtype=t, device="cuda")
            return both[..., :D], both[..., D:]
        return torch.empty((B, T, D), dtype=t, device="cuda"), torch.empty((B, T, D), dtype=t, device="cuda")

    s["x"], s["f"] = pair()
    s["x"].copy_(torch.randn((B, T, D), device="cuda", generator=g))
    # trained gates: most channels remember for a few to a few hundred steps
    s["f"].copy_(1.5 * torch.randn((B, T, D), device="cuda", generator=g) + (7.0 * torch.rand(D, device="cuda", generator=g) - 1.0))
    s["h0"] = torch.randn((B, D), device="cuda", generator=g)
    s["lengths"] = torch.randint(0, T + 1, (B,), device="cuda", generator=g, dtype=torch.int32) if case["ragged"] else None
    s["reset"] = (torch.rand((B, T), device="cuda", generator=g) < 1.0 / 700).to(torch.uint8) if case["resets"] else None
    s["h"] = torch.empty((B, T, D), dtype=t, device="cuda")
    s["h_last"] = torch.empty((B, D), device="cuda")
    if case["pass_"] == "train":
        s["dh"] = torch.randn((B, T, D), device="cuda", generator=g).to(t)
        s["dh_last"] = torch.randn((B, D), device="cuda", generator=g)
        s["dx"], s["df"] = pair()
        s["dh0"] = torch.empty((B, D), device="cuda")
        # what the forward pass keeps for the backward pass: the state before every 16th step
        s["saved"] = torch.empty((B, -(-T // 16), D), device="cuda")
    return s


def _logits(g, N, V, t):
    z = torch.empty((N, V), dtype=t, device="cuda")
    step = max(1, 33554432 // V)
    for a in range(0, N, step):
        z[a:a + step] = 2.0 * torch.randn((min(step, N - a), V), device="cuda", generator=g)
    return z


def _distill_inputs(case, seed):
    g = _generator(seed)
    N, V, K, t = case["N"], case["V"], min(case["K"], case["V"]), TYPES[case["dtype"]]
    s = {"logits": _logits(g, N, V, t)}
    # distinct entries of each row, at odd distances; the last rows of a padded batch have fewer
    first = torch.randint(0, V, (N, 1), device="cuda", generator=g)
    gap = torch.randint(1, max(1, V // K) + 1, (N, 1), device="cuda", generator=g)
    idx = (first + gap * torch.arange(K, device="cuda")) % V
    top = (3.0 + 2.5 * torch.randn((N, K), device="cuda", generator=g)).sort(dim=1, descending=True).values
    # a student on its way to the teacher: its logits rise at the teacher's entries
    near = s["logits"].gather(1, idx).float() + top * torch.rand((N, 1), device="cuda", generator=g)
    s["logits"].scatter_(1, idx, near.to(t))
    filled = torch.where(torch.rand((N, 1), device="cuda", generator=g) < 0.1, torch.randint(0, K + 1, (N, 1), device="cuda", generator=g), K)
    s["idx"] = torch.where(torch.arange(K, device="cuda") < filled, idx, -1).to(torch.int32).contiguous()
    s["top"] = top
    s["teacher_lse"] = None
    if case["tail"]:
        tail = 0.01 + 0.3 * torch.rand(N, device="cuda", generator=g)
        s["teacher_lse"] = (top / case["tau"]).exp().sum(1).log() - torch.log1p(-tail)
    s["labels"] = None
    if case["alpha"]:
        some = torch.where(torch.rand(N, device="cuda", generator=g) < 0.8, idx[:, 0], torch.randint(0, V, (N,), device="cuda", generator=g))
        s["labels"] = torch.where(torch.rand(N, device="cuda", generator=g) < 0.05, -1, some).to(torch.int32)
    keep = (torch.rand(N, device="cuda", generator=g) < 0.95).float()
    keep[0] = 1.0
    # the mean over the kept rows; 16-bit floats of few exponents under a loss scale
    s["row_scale"] = keep / keep.sum() * (4096.0 if case["dtype"] == "f16" else 1.0)
    s["loss"] = torch.empty(N, device="cuda")
    s["grad"] = torch.empty_like(s["logits"])
    return s


def _logp_inputs(case, seed):
    g = _generator(seed)
    N, V, t = case["N"], case["V"], TYPES[case["dtype"]]
    K = min(case["K"], V)
    s = {"logits": _logits(g, N, V, t)}
    s["tokens"] = torch.randint(0, V, (N,), device="cuda", generator=g, dtype=torch.int32)
    # most given tokens are likely ones; a few positions have none
    at = s["tokens"].long()[:, None]
    s["logits"].scatter_(1, at, (s["logits"].gather(1, at).float() + 12.0 * torch.rand((N, 1), device="cuda", generator=g)).to(t))
    if N > 1:
        s["tokens"][torch.rand(N, device="cuda", generator=g) < 0.03] = -1
    s["logp"], s["entropy"], s["lse"] = (torch.empty(N, device="cuda") for _ in range(3))
    s["top_idx"] = torch.empty((N, K), dtype=torch.int32, device="cuda") if K else None
    s["top_logp"] = torch.empty((N, K), device="cuda") if K else None
    if case["grad"]:
        s["dlogp"] = torch.randn(N, device="cuda", generator=g)
        s["dentropy"] = 0.01 * torch.rand(N, device="cuda", generator=g) + 0.01
        s["grad"] = torch.empty_like(s["logits"])
    return s


def prepare(case, seed):
    s = {"glr": _glr_inputs, "distill": _distill_inputs, "logp": _logp_inputs}[case["op"]](case, seed)
    s["case"] = case
    return s


# ---------------------------------------------------------------------------- the framework's calls


def _own(s):
    from paper_1805_08469_gb300 import lm

    c = s["case"]
    if c["op"] == "glr":
        form = lm.GEM_GLR_LERP if c["form"] == "lerp" else lm.GEM_GLR_ADD
        if c["pass_"] == "step":   # the state is read and replaced in place in serving; here both stay
            lm.gem_glr_forward(s["x"], s["f"], s["h"], form=form, h0=s["h0"], h_last=s["h_last"])
            return {"h": s["h"], "h_last": s["h_last"]}
        if c["pass_"] == "forward":
            lm.gem_glr_forward(s["x"], s["f"], s["h"], form=form, h0=s["h0"], lengths=s["lengths"], reset=s["reset"], h_last=s["h_last"])
            return {"h": s["h"], "h_last": s["h_last"]}
        lm.gem_glr_forward(s["x"], s["f"], s["h"], form=form, h0=s["h0"], lengths=s["lengths"], reset=s["reset"],
                           h_last=s["h_last"], saved=s["saved"])
        lm.gem_glr_backward(s["x"], s["f"], s["saved"], s["dh"], s["dx"], s["df"], form=form, lengths=s["lengths"],
                            reset=s["reset"], dh_last=s["dh_last"], dh0=s["dh0"])
        return {k: s[k] for k in ("h", "h_last", "dx", "df", "dh0")}
    if c["op"] == "distill":
        lm.gem_distill(s["logits"], s["idx"], s["top"], s["loss"], s["grad"], teacher_lse=s["teacher_lse"], labels=s["labels"],
                       row_scale=s["row_scale"], temperature=c["tau"], alpha=c["alpha"])
        return {"loss": s["loss"], "grad": s["grad"]}
    lm.gem_token_logp(s["logits"], s["tokens"], s["logp"], s["entropy"], temperature=c["tau"], lse=s["lse"],
                      top_idx=s["top_idx"], top_logp=s["top_logp"])
    out = {"logp": s["logp"], "entropy": s["entropy"]}
    if s["top_idx"] is not None:
        out |= {"top_idx": s["top_idx"], "top_logp": s["top_logp"]}
    if c["grad"]:
        lm.gem_token_logp_grad(s["logits"], s["tokens"], s["lse"], s["entropy"], s["dlogp"], s["dentropy"], s["grad"],
                               temperature=c["tau"])
        out["grad"] = s["grad"]
    return out


# ---------------------------------------------------------------------------- the plain forms


def _scan(a, u):
    """h_t = a_t h_{t-1} + u_t from h_{-1} = 0 along dim 1, by doubling."""
    a, u, s = a.clone(), u.clone(), 1
    while s < a.shape[1]:
        u[:, s:] += a[:, s:] * u[:, :-s]
        a[:, s:] = a[:, s:] * a[:, :-s]
        s *= 2
    return u


def _plain_glr(s):
    c = s["case"]
    x, f, lerp = s["x"].float(), s["f"].float(), c["form"] == "lerp"
    a, b = torch.sigmoid(f), torch.sigmoid(-f)
    u, carry = (b * x if lerp else x.clone()), a.clone()
    T = c["T"]
    if s["reset"] is not None:
        carry.masked_fill_((s["reset"] != 0)[..., None], 0.0)
    if s["lengths"] is not None:
        past = (torch.arange(T, device=x.device) >= s["lengths"][:, None])[..., None]
        carry.masked_fill_(past, 1.0)
        u.masked_fill_(past, 0.0)
    u[:, 0] += carry[:, 0] * s["h0"]
    h = _scan(carry, u)
    shown = h if s["lengths"] is None else h.masked_fill(past, 0.0)
    out = {"h": shown.to(s["x"].dtype), "h_last": h[:, -1].clone()}
    if c["pass_"] != "train":
        return out
    g = s["dh"].float()
    if s["lengths"] is not None:
        g = g.masked_fill(past, 0.0)
    else:
        g = g.clone()
    g[:, -1] += s["dh_last"]
    back = torch.cat([torch.zeros_like(carry[:, :1]), carry.flip(1)[:, :-1]], 1)
    g = _scan(back, g.flip(1)).flip(1)
    before = torch.cat([s["h0"][:, None], h[:, :-1]], 1)
    if s["reset"] is not None:
        before.masked_fill_((s["reset"] != 0)[..., None], 0.0)
    dx = b * g if lerp else g.clone()
    df = g * ((before - x) if lerp else before) * a * b
    if s["lengths"] is not None:
        dx.masked_fill_(past, 0.0)
        df.masked_fill_(past, 0.0)
    return out | {"dx": dx.to(s["x"].dtype), "df": df.to(s["x"].dtype), "dh0": carry[:, 0] * g[:, 0]}


def _plain_distill(s):
    c = s["case"]
    tau, alpha, N, V = c["tau"], c["alpha"], c["N"], c["V"]
    z = s["logits"].float()
    y = z / tau
    m = y.amax(1, keepdim=True)
    p = (y - m).exp()
    total = p.sum(1, keepdim=True)
    there = s["idx"] >= 0
    at = s["idx"].clamp(min=0).long()
    t = (s["top"] / tau).masked_fill(~there, -math.inf)
    if s["teacher_lse"] is None:
        mt = t.amax(1, keepdim=True)
        mt = mt.masked_fill(mt == -math.inf, 0.0)
        t = t - mt
        mass = t.exp().sum(1, keepdim=True)
        logq = t - mass.log()
    else:
        logq = t - s["teacher_lse"][:, None]
    logq = logq.masked_fill(~there, -math.inf)
    q = logq.exp()
    logp = (y.gather(1, at) - m) - total.log()
    kl = torch.where(there, q * (logq - logp), 0.0).sum(1)
    full = torch.zeros_like(p).scatter_add_(1, at, q)
    mean = q.sum(1, keepdim=True)
    if s["teacher_lse"] is not None:
        inside = torch.zeros_like(p).scatter_add_(1, at, there.float()) > 0
        rest = p.masked_fill(inside, 0.0).sum(1, keepdim=True)
        qr = torch.where(rest > 0, (1.0 - mean).clamp(min=0.0), 0.0)
        kl = kl + torch.where(qr > 0, qr * (qr.log() - (rest.log() - total.log())), 0.0)[:, 0]
        p /= total
        g = p * torch.where(inside, mean + qr, mean + qr - torch.where(qr > 0, qr * total / rest, 0.0)) - full
    else:
        p /= total
        g = p * mean - full
    loss, g = (1.0 - alpha) * tau * tau * kl, g * ((1.0 - alpha) * tau)
    if s["labels"] is not None:
        given = (s["labels"] >= 0)[:, None]
        label = s["labels"].clamp(min=0).long()[:, None]
        m = z.amax(1, keepdim=True)
        p = (z - m).exp()
        total = p.sum(1, keepdim=True)
        loss = loss + torch.where(given, -alpha * ((z.gather(1, label) - m) - total.log()), 0.0)[:, 0]
        p = p / total
        p.scatter_add_(1, label, torch.full_like(total, -1.0))
        g += torch.where(given, alpha * p, 0.0)
    kept = s["row_scale"] != 0
    g *= s["row_scale"][:, None]
    return {"loss": torch.where(kept, loss, 0.0), "grad": g.to(s["logits"].dtype)}


def _plain_logp(s):
    c = s["case"]
    raw = s["logits"].float()
    z = raw / c["tau"]
    m = z.amax(1, keepdim=True)
    d = z - m
    p = d.exp()
    total = p.sum(1, keepdim=True)
    entropy = total.log() - (p * d).sum(1, keepdim=True) / total
    given = (s["tokens"] >= 0)[:, None]
    at = s["tokens"].clamp(min=0).long()[:, None]
    logp = torch.where(given, d.gather(1, at) - total.log(), 0.0)
    out = {"logp": logp[:, 0], "entropy": entropy[:, 0]}
    if s["top_idx"] is not None:
        K = s["top_idx"].shape[1]
        order = raw.sort(dim=1, descending=True, stable=True).indices[:, :K]
        out |= {"top_idx": order.to(torch.int32), "top_logp": d.gather(1, order) - total.log()}
    if c["grad"]:
        p /= total
        dl = torch.where(given, s["dlogp"][:, None], 0.0)
        g = -p * (dl + s["dentropy"][:, None] * (d - total.log() + entropy))
        g.scatter_add_(1, at, dl)
        out["grad"] = (g / c["tau"]).to(s["logits"].dtype)
    return out


def run(state):
    if own:
        return _own(state)
    return {"glr": _plain_glr, "distill": _plain_distill, "logp": _plain_logp}[state["case"]["op"]](state)


# ---------------------------------------------------------------------------- the definitions in 64 bits


def _exact_glr(s):
    c = s["case"]
    B, T, D = c["B"], c["T"], c["D"]
    x, f, lerp = s["x"].double(), s["f"].double(), c["form"] == "lerp"
    a, b = 1 / (1 + torch.exp(-f)), 1 / (1 + torch.exp(f))
    u = b * x if lerp else x.clone()
    k = a.clone()
    ends = torch.full((B,), T) if s["lengths"] is None else s["lengths"].cpu()
    for i in range(B):
        k[i, int(ends[i]):] = 1.0
        u[i, int(ends[i]):] = 0.0
        if s["reset"] is not None:
            k[i, :int(ends[i])][s["reset"][i, :int(ends[i])] != 0] = 0.0
    k, u = k.transpose(0, 1).contiguous(), u.transpose(0, 1).contiguous()      # [T][B][D], one step at a time
    h = torch.empty_like(u)
    state = s["h0"].double()
    for kt, ut, ht in zip(k.unbind(0), u.unbind(0), h.unbind(0)):
        state = torch.addcmul(ut, kt, state, out=ht)
    live = torch.ones((T, B, 1), dtype=torch.bool, device="cuda")
    for i in range(B):
        live[int(ends[i]):, i] = False
    out = {"h": (h * live).transpose(0, 1), "h_last": h[-1].clone()}
    if c["pass_"] != "train":
        return out
    g = s["dh"].double().transpose(0, 1) * live
    g[-1] += s["dh_last"].double()
    steps, carries = g.unbind(0), k.unbind(0)
    for t in range(T - 2, -1, -1):
        steps[t].addcmul_(carries[t + 1], steps[t + 1])
    before = torch.cat([s["h0"].double()[None], h[:-1]])
    before = torch.where(k == 0, 0.0, before) if s["reset"] is not None else before
    x, a, b = x.transpose(0, 1), a.transpose(0, 1), b.transpose(0, 1)
    dx = (g * b if lerp else g) * live
    df = g * (before - x if lerp else before) * a * b * live
    return out | {"dx": dx.transpose(0, 1), "df": df.transpose(0, 1), "dh0": k[0] * g[0]}


def _exact_distill(s):
    c = s["case"]
    tau, alpha = c["tau"], c["alpha"]
    loss, grad = [], []
    step = max(1, 16777216 // c["V"])
    for a in range(0, c["N"], step):
        r = slice(a, a + step)
        z = s["logits"][r].double()
        n = z.shape[0]
        idx, t = s["idx"][r].long(), s["top"][r].double() / tau
        there = idx >= 0
        t = torch.where(there, t, -torch.inf)
        lse = torch.logsumexp(t, 1) if s["teacher_lse"] is None else s["teacher_lse"][r].double()
        lse = torch.where(there.any(1), lse, 0.0)
        logq = t - lse[:, None]
        # the student's log probabilities over a row with one more column, for entries that are absent
        logp = torch.cat([torch.log_softmax(z / tau, 1), torch.zeros((n, 1), dtype=z.dtype, device=z.device)], 1)
        at = torch.where(there, idx, c["V"])
        q = torch.where(there, logq.exp(), 0.0)
        kl = torch.where(there, q * (logq - logp.gather(1, at)), 0.0).sum(1)
        target = torch.zeros_like(logp).scatter_add_(1, at, q)[:, :-1]
        logp = logp[:, :-1]
        if s["teacher_lse"] is not None:
            out = torch.ones((n, c["V"] + 1), dtype=torch.bool, device=z.device).scatter_(1, at, False)[:, :-1]
            qr = (1 - q.sum(1)).clamp(min=0.0)
            logr = torch.logsumexp(torch.where(out, logp, -torch.inf), 1)
            qr = torch.where(logr > -torch.inf, qr, 0.0)
            kl = kl + torch.where(qr > 0, qr * (qr.log() - logr), 0.0)
            # the rest's mass is spread over its entries as the student spreads it
            target = torch.where(out, qr[:, None] * (logp - torch.where(qr > 0, logr, 0.0)[:, None]).exp(), target)
        g = (1 - alpha) * tau * (logp.exp() * target.sum(1, keepdim=True) - target)
        total = (1 - alpha) * tau ** 2 * kl
        if s["labels"] is not None:
            y = s["labels"][r].long()
            lp = torch.log_softmax(z, 1)
            rows = torch.nonzero(y >= 0)[:, 0]
            total[rows] -= alpha * lp[rows, y[rows]]
            hard = lp.exp()
            hard[rows, y[rows]] -= 1
            g[rows] += alpha * hard[rows]
        w = s["row_scale"][r].double()
        loss.append(torch.where(w != 0, total, 0.0))
        grad.append(g * w[:, None])
    return {"loss": torch.cat(loss), "grad": torch.cat(grad)}


def _exact_logp(s):
    c = s["case"]
    parts = []
    step = max(1, 16777216 // c["V"])
    for a in range(0, c["N"], step):
        r = slice(a, a + step)
        lp = torch.log_softmax(s["logits"][r].double() / c["tau"], 1)
        H = -(lp.exp() * lp).sum(1)
        y = s["tokens"][r].long()
        rows = torch.nonzero(y >= 0)[:, 0]
        logp = torch.zeros_like(H)
        logp[rows] = lp[rows, y[rows]]
        part = {"logp": logp, "entropy": H}
        if s["top_idx"] is not None:
            part["top_logp"] = lp.topk(s["top_idx"].shape[1], 1).values
        if c["grad"]:
            dl = torch.where(y >= 0, s["dlogp"][r].double(), 0.0)
            g = -lp.exp() * (dl[:, None] + s["dentropy"][r].double()[:, None] * (lp + H[:, None]))
            g[rows, y[rows]] += dl[rows]
            part["grad"] = g / c["tau"]
        parts.append(part)
    out = {k: torch.cat([p[k] for p in parts]) for k in parts[0]}
    if s["top_idx"] is not None:
        out["top_idx"] = None
    return out


def exact(case, seed):
    s = prepare(case, seed)
    for k in ("grad", "dx", "df", "h", "saved"):   # the program's output buffers are not needed here
        s.pop(k, None)
    return {"glr": _exact_glr, "distill": _exact_distill, "logp": _exact_logp}[case["op"]](s)
