"""Performance cases of the operators around the sequence model's layers: what a program whose
workers train a selective state space language model by policy gradients, or answer with it, has
the library do from the tokens to the loss.

  embed    tokens to rows of the embedding table, scaled; in training also the table's gradient
  conv     the short causal convolution in front of the scan: one token, or forward and backward
  ssm      the selective state space scan: one token with the state carried on (serving), a whole
           prompt (forward), or forward and backward (training)
  policy   the clipped policy loss with a KL term and an entropy bonus, and its gradient

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
        # serving: the embeddings of one new token for each of 32 sequences
        dict(name="embed_next_tokens", op="embed", pass_="forward", table="bf16", dtype="bf16", N=32, V=32000, D=1024, tied=0),
        # a table that is also the output layer: its gradient is added to that layer's; odd widths
        dict(name="embed_tied_odd_f16", op="embed", pass_="train", table="f32", dtype="f16", N=16383, V=50001, D=1001, tied=1),
        # training with a large vocabulary, fp32 parameters and bf16 activations
        dict(name="embed_train_v131k", op="embed", pass_="train", table="f32", dtype="bf16", N=65536, V=131072, D=1024, tied=0),
        # serving: one token of 16 sequences through the convolution, its last inputs carried on
        dict(name="conv_step_b16", op="conv", pass_="step", dtype="bf16", B=16, T=1, D=2048, W=4, silu=1, ragged=0, resets=0),
        # training on full sequences
        dict(name="conv_train_bf16", op="conv", pass_="train", dtype="bf16", B=8, T=4096, D=2048, W=4, silu=1, ragged=0, resets=0),
        # serving: one token of 16 sequences through the scan
        dict(name="ssm_step_b16", op="ssm", pass_="step", dtype="bf16", B=16, T=1, D=2048, N=16, G=1, gate=1, ragged=0, resets=0),
        # prompts of different lengths, a large state shared by two groups, channels that are no power of two
        dict(name="ssm_prompts_f16", op="ssm", pass_="forward", dtype="f16", B=3, T=1777, D=1000, N=64, G=2, gate=1, ragged=1, resets=0),
        # training on full sequences; input and gate are the halves of one projection's output
        dict(name="ssm_train_bf16", op="ssm", pass_="train", dtype="bf16", B=8, T=2048, D=2048, N=16, G=1, gate=1, ragged=0, resets=0),
        # training on one long stream of packed documents, the state dropped where one begins
        dict(name="ssm_train_long_f32", op="ssm", pass_="train", dtype="f32", B=1, T=50021, D=512, N=16, G=1, gate=0, ragged=0, resets=1),
        # tuning a small classifier of actions: a few short rows, where latency counts
        dict(name="policy_small_f32", op="policy", dtype="f32", N=64, V=1000, tau=1.0, low=0.2, high=0.2, kl=0.05, bonus=0.01),
        # an odd vocabulary (rows between alignments), sampled at a temperature, asymmetric clipping
        dict(name="policy_odd_f16", op="policy", dtype="f16", N=1023, V=50001, tau=0.7, low=0.2, high=0.28, kl=0.0, bonus=0.0),
        # a large vocabulary with all terms: the largest batch
        dict(name="policy_v131k_bf16", op="policy", dtype="bf16", N=4096, V=131072, tau=1.0, low=0.2, high=0.2, kl=0.04, bonus=0.003),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["embed", "conv", "ssm", "ssm", "policy"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    if op == "embed":
        while True:
            N, V, D = _log_int(rng, 1, 65536), _log_int(rng, 500, 131072), _log_int(rng, 64, 4096)
            if V * D <= 134217728 and N * D <= 67108864:
                break
        if rng.random() < 0.6:
            D = D // 8 * 8
        return dict(op="embed", pass_=rng.choice(["forward", "train", "train"]), table=rng.choice(["f32", dtype]), dtype=dtype, N=N, V=V, D=D,
                    tied=rng.choice([0, 0, 1]))
    if op == "policy":
        while True:
            N, V = _log_int(rng, 1, 8192), _log_int(rng, 500, 160000)
            if N * V <= (2.6e8 if dtype == "f32" else 5.3e8):
                break
        if rng.random() < 0.5:
            V = V // 8 * 8
        return dict(op="policy", dtype=dtype, N=N, V=V, tau=rng.choice([1.0, 1.0, rng.uniform(0.5, 2.0)]), low=rng.choice([0.2, rng.uniform(0.1, 0.3)]),
                    high=rng.choice([0.2, rng.uniform(0.1, 0.4)]), kl=rng.choice([0.0, 0.04, rng.uniform(0.001, 0.2)]),
                    bonus=rng.choice([0.0, 0.01, rng.uniform(0.001, 0.05)]))
    pass_ = rng.choice(["step", "forward", "train", "train"])
    several = pass_ != "step"
    if op == "conv":
        while True:
            B, D = _log_int(rng, 1, 64), _log_int(rng, 64, 4096)
            T = _log_int(rng, 2, 60000) if several else 1
            if B * T * D <= 67108864:
                break
        if rng.random() < 0.6:
            D = max(8, D // 8 * 8)
        return dict(op="conv", pass_=pass_, dtype=dtype, B=B, T=T, D=D, W=rng.choice([4, 4, 3, 2]), silu=rng.choice([1, 1, 0]),
                    ragged=rng.randint(0, 1) if several else 0, resets=rng.randint(0, 1) if several else 0)
    N = rng.choice([16, 16, 16, 8, 32, 64, rng.randint(1, 64)])
    G = rng.choice([1, 1, 1, 2, 4])
    while True:
        B, D = _log_int(rng, 1, 64), G * _log_int(rng, 64 / G, 4096 / G)
        T = _log_int(rng, 2, 50000) if several else 1
        if B * T * D * N <= 536870912:
            break
    if rng.random() < 0.6:
        D = max(8 * G, D // (8 * G) * 8 * G)
    return dict(op="ssm", pass_=pass_, dtype=dtype, B=B, T=T, D=D, N=N, G=G, gate=rng.choice([1, 1, 0]),
                ragged=rng.randint(0, 1) if several else 0, resets=rng.randint(0, 1) if several else 0)


def work(case):
    e = BYTES[case["dtype"]]
    if case["op"] == "embed":
        N, V, D = case["N"], case["V"], case["D"]
        b = N * D * (BYTES[case["table"]] + e) + 4 * N
        if case["pass_"] == "train":   # the gradient rows in, the table's gradient out (all of it, or the rows of N tokens in and out)
            b += N * D * e + 4 * N + (2 * min(N, V) * D * 4 if case["tied"] else V * D * 4)
        return {"bytes": b, "flops": 2 * N * D}
    if case["op"] == "policy":
        N, V = case["N"], case["V"]
        return {"bytes": 2 * N * V * e + 28 * N, "flops": N * V * (12 if case["bonus"] else 8)}
    B, T, D = case["B"], case["T"], case["D"]
    n = B * T * D
    if case["op"] == "conv":
        W = case["W"]
        state = 8 * B * (W - 1) * D + 4 * D * (W + 1)
        if case["pass_"] == "train":   # x, dy in; y, dx out; the parameters' gradients
            return {"bytes": 4 * n * e + 2 * state, "flops": n * (6 * W + 20)}
        return {"bytes": 2 * n * e + state, "flops": n * (2 * W + 6)}
    N, bc, rows = case["N"], 2 * B * T * case["G"] * case["N"], 3 + case["gate"]
    state = 8 * B * D * N + 4 * D * (N + 2)
    if case["pass_"] == "train":       # x, dt, z, dy in; y, dx, ddt, dz out; b, c in, their gradients out
        return {"bytes": (2 * rows * n + 2 * bc) * e + 2 * state, "flops": 28 * n * N}
    return {"bytes": (rows * n + bc) * e + state, "flops": 7 * n * N}


# ---------------------------------------------------------------------------- inputs


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _embed_inputs(case, seed):
    g = _generator(seed)
    N, V, D, t = case["N"], case["V"], case["D"], TYPES[case["dtype"]]
    s = {"table": torch.randn((V, D), device="cuda", generator=g).mul_(0.02).to(TYPES[case["table"]])}
    # words by their rank's frequency; the ends of padded sequences hold no token
    rank = torch.exp(torch.rand(N, device="cuda", generator=g, dtype=torch.float64) * math.log(V)).long() - 1
    shuffle = torch.randperm(V, device="cuda", generator=g)
    s["tokens"] = shuffle[rank.clamp(0, V - 1)].to(torch.int32)
    if N > 64:
        s["tokens"][torch.rand(N, device="cuda", generator=g) < 0.03] = -1
    s["scale"] = math.sqrt(D)
    s["out"] = torch.empty((N, D), dtype=t, device="cuda")
    if case["pass_"] == "train":
        s["dout"] = torch.randn((N, D), device="cuda", generator=g).to(t)
        # where the table is tied, what the output layer's gradient left there
        s["dtable"] = torch.randn((V, D), device="cuda", generator=g) if case["tied"] else torch.empty((V, D), device="cuda")
    return s


def _ragged(case, g, s):
    B, T = case["B"], case["T"]
    s["lengths"] = torch.randint(0, T + 1, (B,), device="cuda", generator=g, dtype=torch.int32) if case["ragged"] else None
    s["reset"] = (torch.rand((B, T), device="cuda", generator=g) < 1.0 / 700).to(torch.uint8) if case["resets"] else None


def _conv_inputs(case, seed):
    g = _generator(seed)
    B, T, D, W, t = case["B"], case["T"], case["D"], case["W"], TYPES[case["dtype"]]
    # the layer's input is half of a projection's output
    s = {"x": torch.randn((B, T, 2 * D), device="cuda", generator=g).to(t)[..., :D]}
    s["weight"] = torch.randn((D, W), device="cuda", generator=g) / math.sqrt(W)
    s["bias"] = 0.1 * torch.randn(D, device="cuda", generator=g)
    s["state"] = torch.randn((B, W - 1, D), device="cuda", generator=g)
    _ragged(case, g, s)
    s["y"] = torch.empty((B, T, D), dtype=t, device="cuda")
    s["state_last"] = torch.empty_like(s["state"])
    if case["pass_"] == "train":
        s["dy"] = torch.randn((B, T, D), device="cuda", generator=g).to(t)
        s["dstate_last"] = torch.randn((B, W - 1, D), device="cuda", generator=g)
        s["dx"] = torch.empty((B, T, D), dtype=t, device="cuda")
        s["dweight"], s["dbias"], s["dstate"] = torch.empty_like(s["weight"]), torch.empty_like(s["bias"]), torch.empty_like(s["state"])
    return s


def _ssm_inputs(case, seed):
    g = _generator(seed)
    B, T, D, N, G, t = case["B"], case["T"], case["D"], case["N"], case["G"], TYPES[case["dtype"]]
    randn = lambda *shape: torch.randn(shape, device="cuda", generator=g)  # noqa: E731
    s = {"x": torch.nn.functional.silu(randn(B, T, D)).to(t), "z": None}
    if case["gate"]:
        s["z"] = randn(B, T, 2 * D).to(t)[..., D:]
    s["dt"] = (0.5 * randn(B, T, D)).to(t)
    # steps of 0.001 to 0.1 from their bias, decays of 1 to N as such layers begin with
    step = torch.exp(math.log(1e-3) + torch.rand(D, device="cuda", generator=g) * math.log(100.0))
    s["dt_bias"] = step + torch.log(-torch.expm1(-step))
    s["A"] = -torch.arange(1, N + 1, device="cuda").float() * torch.exp(0.1 * randn(D, N))
    both = randn(B, T, 2, G, N).to(t)     # b and c beside each other in a projection's output
    s["b"], s["c"] = both[:, :, 0], both[:, :, 1]
    s["skip"] = 1.0 + 0.1 * randn(D)
    s["h0"] = randn(B, D, N)
    _ragged(case, g, s)
    s["y"] = torch.empty((B, T, D), dtype=t, device="cuda")
    s["h_last"] = torch.empty_like(s["h0"])
    if case["pass_"] == "train":
        s["dy"] = randn(B, T, D).to(t)
        s["dh_last"] = randn(B, D, N)
        for k in ("dx", "ddt") + (("dz",) if case["gate"] else ()):
            s[k] = torch.empty((B, T, D), dtype=t, device="cuda")
        for k in ("db", "dc"):
            s[k] = torch.empty((B, T, G, N), dtype=t, device="cuda")
        for k, like in (("dA", "A"), ("dskip", "skip"), ("ddt_bias", "dt_bias"), ("dh0", "h0")):
            s[k] = torch.empty_like(s[like])
        # what the forward pass keeps for the backward pass: the state before every 16th step
        s["saved"] = torch.empty((B, -(-T // 16), D, N), device="cuda")
    return s


def _policy_inputs(case, seed):
    g = _generator(seed)
    N, V, t = case["N"], case["V"], TYPES[case["dtype"]]
    z = torch.empty((N, V), dtype=t, device="cuda")
    step = max(1, 33554432 // V)
    for a in range(0, N, step):
        z[a:a + step] = 2.0 * torch.randn((min(step, N - a), V), device="cuda", generator=g)
    s = {"logits": z, "tokens": torch.randint(0, V, (N,), device="cuda", generator=g, dtype=torch.int32)}
    # sampled tokens are likely ones
    at = s["tokens"].long()[:, None]
    z.scatter_(1, at, (z.gather(1, at).float() + 14.0 * torch.rand((N, 1), device="cuda", generator=g)).to(t))
    logp = torch.empty(N, device="cuda", dtype=torch.float64)
    for a in range(0, N, step):
        y = z[a:a + step].double() / case["tau"]
        logp[a:a + step] = (y.gather(1, at[a:a + step]) - y.logsumexp(1, keepdim=True))[:, 0]
    # the policy has moved since the tokens were sampled; no ratio lies so near a bound that rounding decides
    moved = 0.15 * torch.randn(N, device="cuda", generator=g, dtype=torch.float64)
    ratio = moved.exp()
    near = ((ratio - (1 - case["low"])).abs() < 1e-3) | ((ratio - (1 + case["high"])).abs() < 1e-3)
    s["old_logp"] = (logp - torch.where(near, 0.01, moved)).float()
    s["ref_logp"] = (logp + 0.2 * torch.randn(N, device="cuda", generator=g, dtype=torch.float64)).float() if case["kl"] else None
    s["advantage"] = torch.randn(N, device="cuda", generator=g)
    # prompts and padding are masked; the mean over the others, 16-bit floats of few exponents under a loss scale
    keep = (torch.rand(N, device="cuda", generator=g) < 0.9).float()
    keep[0] = 1.0
    s["row_scale"] = keep / keep.sum() * (4096.0 if case["dtype"] == "f16" else 1.0)
    s["loss"], s["logp"], s["entropy"] = (torch.empty(N, device="cuda") for _ in range(3))
    s["grad"] = torch.empty_like(z)
    return s


def prepare(case, seed):
    s = {"embed": _embed_inputs, "conv": _conv_inputs, "ssm": _ssm_inputs, "policy": _policy_inputs}[case["op"]](case, seed)
    s["case"] = case
    return s


# ---------------------------------------------------------------------------- the framework's calls


def _workspace(s, size, dtype):
    """A workspace that the program makes once and keeps."""
    if "workspace" not in s:
        s["workspace"] = torch.empty(size, dtype=dtype, device="cuda") if size else None
    return s["workspace"]


def _own(s):
    from paper_1805_08469_gb300 import lm

    c = s["case"]
    if c["op"] == "embed":
        lm.gem_embed(s["table"], s["tokens"], s["out"], scale=s["scale"])
        if c["pass_"] == "forward":
            return {"out": s["out"]}
        space = _workspace(s, lm.gem_embed_workspace(c["N"], c["V"], c["D"]), torch.uint8)
        lm.gem_embed_grad(s["dout"], s["tokens"], s["dtable"], space, scale=s["scale"], accumulate=bool(c["tied"]))
        return {"out": s["out"], "dtable": s["dtable"]}
    if c["op"] == "conv":
        form = lm.GEM_CONV_SILU if c["silu"] else lm.GEM_CONV_LINEAR
        lm.gem_conv_forward(s["x"], s["weight"], s["y"], form=form, bias=s["bias"], state=s["state"], lengths=s["lengths"], reset=s["reset"],
                            state_last=s["state_last"])
        if c["pass_"] != "train":
            return {"y": s["y"], "state_last": s["state_last"]}
        space = _workspace(s, lm.gem_conv_workspace(c["B"], c["T"], c["D"], c["W"]), torch.float32)
        lm.gem_conv_backward(s["x"], s["weight"], s["dy"], s["dx"], s["dweight"], space, form=form, bias=s["bias"], dbias=s["dbias"],
                             state=s["state"], lengths=s["lengths"], reset=s["reset"], dstate_last=s["dstate_last"], dstate=s["dstate"])
        return {k: s[k] for k in ("y", "state_last", "dx", "dweight", "dbias", "dstate")}
    if c["op"] == "ssm":
        space = _workspace(s, lm.gem_ssm_workspace(c["B"], c["T"], c["D"], c["N"], c["G"], backward=c["pass_"] == "train"), torch.float32)
        more = dict(z=s["z"], skip=s["skip"], dt_bias=s["dt_bias"], lengths=s["lengths"], reset=s["reset"], workspace=space)
        lm.gem_ssm_forward(s["x"], s["dt"], s["A"], s["b"], s["c"], s["y"], h0=s["h0"], h_last=s["h_last"], saved=s.get("saved"), **more)
        if c["pass_"] != "train":
            return {"y": s["y"], "h_last": s["h_last"]}
        lm.gem_ssm_backward(s["x"], s["dt"], s["A"], s["b"], s["c"], s["saved"], s["dy"], s["dx"], s["ddt"], s["dA"], s["db"], s["dc"],
                            dz=s.get("dz"), dskip=s["dskip"], ddt_bias=s["ddt_bias"], dh_last=s["dh_last"], dh0=s["dh0"], **more)
        return {k: s[k] for k in ("y", "h_last", "dx", "ddt", "dA", "db", "dc", "dz", "dskip", "ddt_bias", "dh0") if k in s}
    lm.gem_policy(s["logits"], s["tokens"], s["old_logp"], s["advantage"], s["loss"], s["grad"], ref_logp=s["ref_logp"], row_scale=s["row_scale"],
                  temperature=c["tau"], clip_low=c["low"], clip_high=c["high"], kl=c["kl"], bonus=c["bonus"], logp=s["logp"], entropy=s["entropy"])
    return {k: s[k] for k in ("loss", "logp", "entropy", "grad")}


# ---------------------------------------------------------------------------- the plain forms


def _plain_embed(s):
    c = s["case"]
    none = (s["tokens"] < 0)[:, None]
    at = s["tokens"].clamp(min=0).long()
    rows = (s["table"][at].float() * s["scale"]).masked_fill(none, 0.0)
    out = {"out": rows.to(s["out"].dtype)}
    if c["pass_"] == "forward":
        return out
    g = (s["dout"].float() * s["scale"]).masked_fill(none, 0.0)
    if c["tied"]:
        s["dtable"].index_add_(0, at, g)
        return out | {"dtable": s["dtable"]}
    return out | {"dtable": torch.zeros((c["V"], c["D"]), device=g.device).index_add_(0, at, g)}


def _past(s):
    """Where a step lies past its sequence's end, [B, T, 1]."""
    c = s["case"]
    if s["lengths"] is None:
        return torch.zeros((c["B"], c["T"], 1), dtype=torch.bool, device="cuda")
    return (torch.arange(c["T"], device="cuda") >= s["lengths"][:, None])[..., None]


def _plain_conv(s):
    c = s["case"]
    B, T, D, W = c["B"], c["T"], c["D"], c["W"]
    past = _past(s)
    x = torch.cat([s["state"], s["x"].float().masked_fill(past, 0.0)], 1)              # [B, W - 1 + T, D]
    part = torch.zeros((B, W - 1 + T), dtype=torch.int64, device="cuda")               # the document of each input
    if s["reset"] is not None:
        part[:, W - 1:] = (s["reset"] != 0).long().cumsum(1)
    same = [(part[:, k:k + T] == part[:, W - 1:])[..., None] for k in range(W)]        # tap k reaches step t's own document
    w = s["weight"]
    pre = s["bias"] + sum((torch.where(same[k], x[:, k:k + T], 0.0) * w[:, k] for k in range(W)), torch.zeros((), device="cuda"))
    sig = torch.sigmoid(pre)
    y = (pre * sig if c["silu"] else pre).masked_fill(past, 0.0)
    n = torch.full((B,), T, device="cuda") if s["lengths"] is None else s["lengths"].long()
    at = n[:, None] + torch.arange(W - 1, device="cuda")                               # the last W - 1 inputs
    end = torch.where(n > 0, part.gather(1, (n + W - 2).clamp(min=0)[:, None])[:, 0], 0)[:, None]
    kept = (part.gather(1, at) == end)[..., None]
    row = at[..., None].expand(B, W - 1, D)
    out = {"y": y.to(s["y"].dtype), "state_last": torch.where(kept, x.gather(1, row), 0.0)}
    if c["pass_"] != "train":
        return out
    dpre = s["dy"].float().masked_fill(past, 0.0)
    if c["silu"]:
        dpre = dpre * sig * (1.0 + pre * (1.0 - sig))
    dx = torch.zeros_like(x).scatter_add_(1, row, torch.where(kept, s["dstate_last"], 0.0))
    dw = torch.empty_like(w)
    for k in range(W):
        g = torch.where(same[k], dpre, 0.0)
        dx[:, k:k + T] += g * w[:, k]
        dw[:, k] = (g * x[:, k:k + T]).sum((0, 1))
    return out | {"dx": dx[:, W - 1:].masked_fill(past, 0.0).to(s["y"].dtype), "dweight": dw, "dbias": dpre.sum((0, 1)), "dstate": dx[:, :W - 1].clone()}


def _scan(a, u):
    """h_t = a_t h_{t-1} + u_t from h_{-1} = 0 along dim 1, by doubling, in place."""
    s = 1
    while s < a.shape[1]:
        u[:, s:] += a[:, s:] * u[:, :-s]
        a[:, s:] = a[:, s:] * a[:, :-s]
        s *= 2
    return u


def _softplus(v):
    return v.clamp(min=0.0) + torch.log1p(torch.exp(-v.abs()))


def _plain_ssm(s):
    c = s["case"]
    B, T, D, N, G = (c[k] for k in "BTDNG")
    past = _past(s)
    t = s["x"].dtype
    wide = lambda v: v.float().masked_fill(past[..., None], 0.0).repeat_interleave(D // G, 2)  # noqa: E731  [B, T, G, N] to channels
    x, raw = s["x"].float().masked_fill(past, 0.0), s["dt"].float() + s["dt_bias"]
    step = _softplus(raw).masked_fill(past, 0.0)
    a = torch.exp(step[..., None] * s["A"])                                            # [B, T, D, N]
    if s["reset"] is not None:
        a.masked_fill_((s["reset"] != 0)[..., None, None], 0.0)
    if c["ragged"]:
        a.masked_fill_(past[..., None], 1.0)
    b = wide(s["b"])
    u = (step * x)[..., None] * b
    u[:, 0] += a[:, 0] * s["h0"]
    h = _scan(a.clone(), u)
    cc = wide(s["c"])
    mixed = (cc * h).sum(-1) + s["skip"] * x
    out = {"h_last": h[:, -1].clone()}
    gate, sig = 1.0, None
    if s["z"] is not None:
        z = s["z"].float()
        sig = torch.sigmoid(z)
        gate = z * sig
    out["y"] = (mixed * gate).masked_fill(past, 0.0).to(t)
    if c["pass_"] != "train":
        return out
    dy = s["dy"].float().masked_fill(past, 0.0)
    if sig is not None:
        out["dz"] = (dy * mixed * sig * (1.0 + z * (1.0 - sig))).masked_fill(past, 0.0).to(t)
        dy = (dy * gate).masked_fill(past, 0.0)
    over = lambda v: v.view(B, T, G, D // G, N).sum(3).to(t)  # noqa: E731  a group's channels
    out["dc"] = over(dy[..., None] * h)
    before = torch.cat([s["h0"][:, None], h[:, :-1]], 1).mul_(a)                        # a_t h_{t-1}
    del h
    g = cc.mul_(dy[..., None])
    g[:, -1] += s["dh_last"]
    back = torch.cat([torch.zeros_like(a[:, :1]), a.flip(1)[:, :-1]], 1)
    g = _scan(back, g.flip(1)).flip(1)
    del back
    out["dh0"] = a[:, 0] * g[:, 0]
    out["db"] = over(g * (step * x)[..., None])
    through = (g * b).sum(-1)
    g *= before
    out["dA"] = (g * step[..., None]).sum((0, 1))
    draw_ = ((g * s["A"]).sum(-1) + through * x) * torch.sigmoid(raw)
    out["ddt"] = draw_.masked_fill(past, 0.0).to(t)
    out["ddt_bias"] = draw_.masked_fill(past, 0.0).sum((0, 1))
    out["dx"] = (through * step + s["skip"] * dy).masked_fill(past, 0.0).to(t)
    out["dskip"] = (dy * x).sum((0, 1))
    return out


def _plain_policy(s):
    c = s["case"]
    z = s["logits"].float() / c["tau"]
    d = z - z.amax(1, keepdim=True)
    p = d.exp()
    total = p.sum(1, keepdim=True)
    logs = total.log()
    at = s["tokens"].long()[:, None]
    logp = (d.gather(1, at) - logs)[:, 0]
    entropy = (logs - (p * d).sum(1, keepdim=True) / total)[:, 0]
    ratio = (logp - s["old_logp"]).exp()
    A = s["advantage"]
    plain, clipped = ratio * A, ratio.clamp(1.0 - c["low"], 1.0 + c["high"]) * A
    loss = -torch.minimum(plain, clipped) - c["bonus"] * entropy
    dlogp = torch.where(plain <= clipped, -plain, 0.0)
    if s["ref_logp"] is not None:
        far = s["ref_logp"] - logp
        loss = loss + c["kl"] * (torch.expm1(far) - far)
        dlogp = dlogp - c["kl"] * torch.expm1(far)
    p /= total
    g = p * ((c["bonus"] * (d - logs + entropy[:, None])) - dlogp[:, None])
    g.scatter_add_(1, at, dlogp[:, None])
    g *= (s["row_scale"] / c["tau"])[:, None]
    kept = s["row_scale"] != 0
    hide = lambda v: torch.where(kept, v, 0.0)  # noqa: E731
    return {"loss": hide(loss), "logp": hide(logp), "entropy": hide(entropy), "grad": g.to(s["logits"].dtype)}


def run(state):
    if own:
        return _own(state)
    return {"embed": _plain_embed, "conv": _plain_conv, "ssm": _plain_ssm, "policy": _plain_policy}[state["case"]["op"]](state)


# ---------------------------------------------------------------------------- the definitions in 64 bits


def _exact_embed(s):
    c = s["case"]
    y = s["tokens"].long()
    there = torch.nonzero(y >= 0)[:, 0]
    rows = torch.zeros((c["N"], c["D"]), dtype=torch.float64, device="cuda")
    rows[there] = s["table"].double()[y[there]] * s["scale"]
    out = {"out": rows}
    if c["pass_"] == "train":
        order = there[torch.argsort(y[there], stable=True)]
        tokens, count = torch.unique_consecutive(y[order], return_counts=True)
        total = torch.cumsum(s["dout"][order].double(), 0)
        ends = torch.cumsum(count, 0) - 1
        upto = torch.cat([torch.zeros_like(total[:1]), total[ends]])
        out["dtable"] = s["dtable"].double() if c["tied"] else torch.zeros((c["V"], c["D"]), dtype=torch.float64, device="cuda")
        out["dtable"][tokens] += s["scale"] * (upto[1:] - upto[:-1])
    return out


def _ends(s):
    c = s["case"]
    return [c["T"]] * c["B"] if s["lengths"] is None else s["lengths"].tolist()


def _exact_conv(s):
    """Sequence by sequence and document by document, each padded by its own past."""
    c = s["case"]
    B, T, D, W = c["B"], c["T"], c["D"], c["W"]
    w, bias = s["weight"].double(), s["bias"].double()
    new = lambda *shape: torch.zeros(shape, dtype=torch.float64, device="cuda")  # noqa: E731
    out = {"y": new(B, T, D), "state_last": new(B, W - 1, D)}
    train = c["pass_"] == "train"
    if train:
        out |= {"dx": new(B, T, D), "dweight": new(D, W), "dbias": new(D), "dstate": new(B, W - 1, D)}
    resets = None if s["reset"] is None else s["reset"].cpu().numpy()
    for i, n in enumerate(_ends(s)):
        starts = [] if resets is None else [int(k) for k in resets[i, :n].nonzero()[0]]
        cuts = [0] + starts + [n]           # (the first part may be empty: a reset at step 0 drops the state)
        for j, (lo, hi) in enumerate(zip(cuts, cuts[1:])):
            before = s["state"][i].double() if j == 0 else new(W - 1, D)
            full = torch.cat([before, s["x"][i, lo:hi].double()])
            taps = full.unfold(0, W, 1) if hi > lo else new(0, D, W)                    # [steps, D, W]
            pre = (taps * w).sum(-1) + bias
            out["y"][i, lo:hi] = pre / (1 + torch.exp(-pre)) if c["silu"] else pre
            last = j == len(cuts) - 2
            if last:
                out["state_last"][i] = full[full.shape[0] - (W - 1):]
            if not train:
                continue
            g = s["dy"][i, lo:hi].double()
            if c["silu"]:
                sig = 1 / (1 + torch.exp(-pre))
                g = g * (sig + pre * sig * (1 - sig))
            dfull = torch.zeros_like(full)
            for k in range(W):
                dfull[k:k + hi - lo] += g * w[:, k]
            if last:
                dfull[full.shape[0] - (W - 1):] += s["dstate_last"][i].double()
            out["dweight"] += (taps * g[..., None]).sum(0)
            out["dbias"] += g.sum(0)
            out["dx"][i, lo:hi] = dfull[W - 1:]
            if j == 0:
                out["dstate"][i] = dfull[:W - 1]
    return out


def _exact_ssm(s):
    """The recurrences one step at a time, [T][B][D][N]; all else in products over whole tensors."""
    c = s["case"]
    B, T, D, N, G = (c[k] for k in "BTDNG")
    lead = lambda v: v.double().transpose(0, 1)  # noqa: E731
    live = torch.ones((T, B, 1), dtype=torch.bool, device="cuda")
    for i, n in enumerate(_ends(s)):
        live[n:, i] = False
    pick = lambda v: torch.where(live, lead(v), 0.0)  # noqa: E731
    x, raw = pick(s["x"]), pick(s["dt"]) + s["dt_bias"].double()
    step = torch.where(live, torch.logaddexp(raw, torch.zeros_like(raw)), 0.0)
    b, cc = (torch.where(live[..., None], lead(s[k]), 0.0)[:, :, :, None].expand(T, B, G, D // G, N).reshape(T, B, D, N).contiguous() for k in "bc")
    a = (step[..., None] * s["A"].double()).exp_()
    if s["reset"] is not None:
        a[(s["reset"].t() != 0) & live[..., 0]] = 0.0
    h = b * (step * x)[..., None]
    state = s["h0"].double()
    for at, ht in zip(a.unbind(0), h.unbind(0)):
        state = torch.addcmul(ht, at, state, out=ht)
    mixed = torch.einsum("tbdn,tbdn->tbd", cc, h) + s["skip"].double() * x
    gate = 1.0
    if s["z"] is not None:
        z = pick(s["z"])
        sig = 1 / (1 + torch.exp(-z))
        gate = z * sig
    back = lambda v: v.transpose(0, 1)  # noqa: E731
    out = {"y": back(mixed * gate), "h_last": h[-1].clone()}
    if c["pass_"] != "train":
        return out
    dy = pick(s["dy"])
    if s["z"] is not None:
        out["dz"] = back(dy * mixed * (sig + gate * (1 - sig)))
        dy = dy * gate
    out["dc"] = back(torch.einsum("tbgd,tbgdn->tbgn", dy.view(T, B, G, -1), h.view(T, B, G, -1, N)))
    g = cc.mul_(dy[..., None])
    g[-1] += s["dh_last"].double()
    steps, decays = g.unbind(0), a.unbind(0)
    for t in range(T - 2, -1, -1):
        steps[t].addcmul_(decays[t + 1], steps[t + 1])
    out["dh0"] = a[0] * g[0]
    out["db"] = back(torch.einsum("tbgd,tbgdn->tbgn", (step * x).view(T, B, G, -1), g.view(T, B, G, -1, N)))
    through = torch.einsum("tbdn,tbdn->tbd", g, b)
    del b
    g.mul_(a)                                       # the gradient of log a_t: g_t a_t h_{t-1}
    g[1:] *= h[:-1]
    g[0] *= s["h0"].double()
    out["dA"] = torch.einsum("tbdn,tbd->dn", g, step)
    dstep = torch.einsum("tbdn,dn->tbd", g, s["A"].double()) + through * x
    draw_ = torch.where(live, dstep / (1 + torch.exp(-raw)), 0.0)
    out["ddt"], out["ddt_bias"] = back(draw_), draw_.sum((0, 1))
    out["dx"], out["dskip"] = back(through * step + s["skip"].double() * dy), (dy * x).sum((0, 1))
    return out


def _exact_policy(s):
    c = s["case"]
    parts = []
    step = max(1, 16777216 // c["V"])
    for k in range(0, c["N"], step):
        r = slice(k, k + step)
        lp = torch.log_softmax(s["logits"][r].double() / c["tau"], 1)
        p = lp.exp()
        H = -(p * lp).sum(1)
        rows = torch.arange(lp.shape[0], device="cuda")
        y = s["tokens"][r].long()
        logp = lp[rows, y]
        A, w = s["advantage"][r].double(), s["row_scale"][r].double()
        ratio = torch.exp(logp - s["old_logp"][r].double())
        outside = ((A > 0) & (ratio > 1 + c["high"])) | ((A < 0) & (ratio < 1 - c["low"]))
        loss = -torch.where(outside, ratio.clamp(1 - c["low"], 1 + c["high"]), ratio) * A - c["bonus"] * H
        dl = torch.where(outside, 0.0, -A * ratio)
        if s["ref_logp"] is not None:
            far = s["ref_logp"][r].double() - logp
            loss += c["kl"] * (torch.exp(far) - far - 1)
            dl += c["kl"] * (1 - torch.exp(far))
        hit = torch.zeros_like(p)
        hit[rows, y] = 1
        g = (dl[:, None] * (hit - p) + c["bonus"] * p * (lp + H[:, None])) * (w / c["tau"])[:, None]
        on = w != 0
        parts.append({"loss": loss * on, "logp": logp * on, "entropy": H * on, "grad": g})
    return {k: torch.cat([q[k] for q in parts]) for k in parts[0]}


def exact(case, seed):
    s = prepare(case, seed)
    return {"embed": _exact_embed, "conv": _exact_conv, "ssm": _exact_ssm, "policy": _exact_policy}[case["op"]](s)
