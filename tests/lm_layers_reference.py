"""Embedding, short convolution, selective scan and policy loss in 64 bits, each with a bound on what
fp32 arithmetic and one rounding of the output may differ by.

U = 2^-24 is the largest relative error of one fp32 operation.  The fast exponential is within 4 U and 2 U
times the size of its argument, a fast reciprocal within 2 U; a sum of n terms in any order within n U of the sum of
their sizes.
"""
import numpy as np

from lm_reference import U, _softmax, rounded

TINY = 1e-36    # what fast functions flush to zero, times factors up to 100


def sigmoid(v):
    with np.errstate(over="ignore"):
        return 1 / (1 + np.exp(-v))


def e_sigmoid(v):
    """Bound of the sigmoid's error: an exponential, a sum, a reciprocal."""
    return sigmoid(v) * U * (8 + 2 * np.minimum(np.abs(v), 200)) + TINY


def silu(v):
    return v * sigmoid(v)


def dsilu(v):
    s = sigmoid(v)
    return s * (1 + v * (1 - s))


def e_dsilu(v, ev):
    """Bound of the error of silu's derivative at v, which is itself known to ev (its slope is below 0.6)."""
    return e_sigmoid(v) * (1 + 2 * np.abs(v)) + 0.6 * ev + 8 * U * sigmoid(v) * (1 + np.abs(v)) + TINY


# ---------------------------------------------------------------------- embedding


def embed(table, tokens, scale, dtype):
    V = table.shape[0]
    ok = (tokens >= 0) & (tokens < V)
    rows = np.where(ok[:, None], table.astype(np.float64)[np.where(ok, tokens, 0)] * scale, 0.0)
    rows = np.where((tokens >= V)[:, None], np.nan, rows)
    return {"out": (rows, 2 * U * np.abs(np.nan_to_num(rows)) + rounded(np.nan_to_num(rows), dtype))}


def embed_grad(dout, tokens, V, scale, dtype, old=None):
    D = dout.shape[1]
    ok = (tokens >= 0) & (tokens < V)
    sums, sizes, count = np.zeros((V, D)), np.zeros((V, D)), np.zeros((V, 1))
    np.add.at(sums, tokens[ok], dout.astype(np.float64)[ok])
    np.add.at(sizes, tokens[ok], np.abs(dout.astype(np.float64))[ok])
    np.add.at(count, tokens[ok], 1.0)
    g = sums * scale
    e = (count + 2) * U * sizes * abs(scale)
    if old is not None:
        g = g + old
        e = e + 2 * U * np.abs(g)
    e = np.where(count > 0, e + rounded(g, dtype), 0.0)   # rows without a token are exact
    return {"dtable": (g, e)}


# ---------------------------------------------------------------------- convolution


def conv(x, w, silu_form, bias=None, state=None, lengths=None, reset=None, dy=None, dstate_last=None, dtype="f32"):
    """{name: (value, bound)} of y, state_last, and with dy of dx, dweight, dbias, dstate; step by step."""
    B, T, D = x.shape
    W = w.shape[1]
    w = w.astype(np.float64)
    b0 = np.zeros(D) if bias is None else bias.astype(np.float64)
    n = np.full(B, T) if lengths is None else np.clip(lengths, 0, T)
    y, ey = np.zeros((B, T, D)), np.zeros((B, T, D))
    last = np.zeros((B, W - 1, D))
    out = {"dx": np.zeros((B, T, D)), "dweight": np.zeros((D, W)), "dbias": np.zeros(D), "dstate": np.zeros((B, W - 1, D))}
    err = {k: np.zeros_like(v) for k, v in out.items()}
    size = {k: np.zeros_like(v) for k, v in out.items()}
    for i in range(B):
        ext = np.concatenate([np.zeros((W - 1, D)) if state is None else state[i].astype(np.float64), x[i].astype(np.float64)])
        dext, eext, sext = np.zeros_like(ext), np.zeros_like(ext), np.zeros_like(ext)
        oldest = 0          # of the inputs that still count
        for t in range(n[i]):
            if reset is not None and reset[i, t]:
                oldest = t + W - 1
            taps = np.stack([ext[t + k] if t + k >= oldest else np.zeros(D) for k in range(W)])
            p = b0 + (w.T * taps).sum(0)
            ep = (W + 2) * U * (np.abs(b0) + np.abs(w.T * taps).sum(0))
            if silu_form:
                y[i, t] = silu(p)
                ey[i, t] = 1.1 * ep + np.abs(p) * e_sigmoid(p) + 2 * U * np.abs(y[i, t]) + TINY
            else:
                y[i, t], ey[i, t] = p, ep
            if dy is None:
                continue
            g = dy[i, t].astype(np.float64)
            eg = np.zeros(D)
            if silu_form:
                f = dsilu(p)
                eg = np.abs(g) * e_dsilu(p, ep) + 2 * U * np.abs(g * f)
                g = g * f
            for k in range(W):
                if t + k >= oldest:
                    dext[t + k] += g * w[:, k]
                    eext[t + k] += eg * np.abs(w[:, k])
                    sext[t + k] += np.abs(g * w[:, k])
                out["dweight"][:, k] += g * taps[k]
                err["dweight"][:, k] += eg * np.abs(taps[k])
                size["dweight"][:, k] += np.abs(g * taps[k])
            out["dbias"] += g
            err["dbias"] += eg
            size["dbias"] += np.abs(g)
        ends = np.stack([ext[n[i] + j] if n[i] + j >= oldest else np.zeros(D) for j in range(W - 1)])
        last[i] = ends
        if dy is not None:
            if dstate_last is not None:
                for j in range(W - 1):
                    if n[i] + j >= oldest:
                        dext[n[i] + j] += dstate_last[i, j]
                        sext[n[i] + j] += np.abs(dstate_last[i, j])
            out["dx"][i, :n[i]] = dext[W - 1:W - 1 + n[i]]
            err["dx"][i, :n[i]] = (eext + (W + 2) * U * sext)[W - 1:W - 1 + n[i]]
            out["dstate"][i] = dext[:W - 1]
            err["dstate"][i] = (eext + (W + 2) * U * sext)[:W - 1]
    res = {"y": (y, ey + rounded(y, dtype)), "state_last": (last, 0.0 * last)}
    if dy is not None:
        terms = 80 + n.sum() / 64
        res["dx"] = (out["dx"], err["dx"] + rounded(out["dx"], dtype))
        res["dstate"] = (out["dstate"], err["dstate"] + 2 * U * np.abs(out["dstate"]))
        for k in ("dweight", "dbias"):
            res[k] = (out[k], err[k] + terms * U * size[k])
    return res


# ---------------------------------------------------------------------- selective scan


def ssm(x, dt, A, b, c, z=None, skip=None, dt_bias=None, softplus=True, h0=None, lengths=None, reset=None, dy=None, dh_last=None, dtype="f32"):
    """{name: (value, bound)} of y, h_last, saved, and with dy of every gradient; step by step."""
    x, dt, b, c = (v.astype(np.float64) for v in (x, dt, b, c))
    B, T, D = x.shape
    G, N = b.shape[2:]
    per = D // G
    A = A.astype(np.float64)
    n = np.full(B, T) if lengths is None else np.clip(lengths, 0, T)
    live = (np.arange(T)[None] < n[:, None])[..., None]
    fresh = np.zeros((B, T), bool) if reset is None else (reset != 0)
    clean = lambda v: np.where(live, np.nan_to_num(v), 0.0)  # noqa: E731
    x, dt = clean(x), clean(dt)
    b, c = (np.repeat(np.where(live[..., None], np.nan_to_num(v), 0.0), per, axis=2) for v in (b, c))
    D0 = np.zeros(D) if skip is None else skip.astype(np.float64)
    raw = dt + (0.0 if dt_bias is None else dt_bias.astype(np.float64))
    if softplus:
        small = np.log1p(np.exp(-np.abs(raw)))
        step = np.maximum(raw, 0) + small
        e_step = U * small * (16 + 2 * np.abs(raw)) + 2 * U * step + sigmoid(raw) * 2 * U * np.abs(raw) + TINY
    else:
        step, e_step = raw, U * np.abs(raw)
    step, e_step = np.where(live, step, 0.0), np.where(live, e_step, 0.0)
    sx, e_sx = step * x, np.abs(x) * e_step + 2 * U * np.abs(step * x)

    def decay(t):
        arg = step[:, t, :, None] * A
        a = np.exp(arg)
        rel = np.where(live[:, t, :, None], 4.4 * U + 3 * U * np.abs(arg) + np.abs(A) * e_step[:, t, :, None], 0.0)
        # (below 2^-126 a decay is 0 in fp32)
        return a, a * rel + 1.2e-38 * (a < 1e-30)

    h = np.zeros((B, D, N)) if h0 is None else h0.astype(np.float64).copy()
    e = np.zeros_like(h)
    mixed, e_mixed = np.zeros((B, T, D)), np.zeros((B, T, D))
    H, E, saved = np.zeros((T + 1, B, D, N)), np.zeros((T + 1, B, D, N)), []
    H[0], E[0] = h, e
    drop = lambda t: (fresh[:, t] & live[:, t, 0])[:, None, None]  # noqa: E731
    for t in range(T):
        if t % 16 == 0:
            saved.append((h.copy(), e.copy()))
        a, ea = decay(t)
        h, e = np.where(drop(t), 0.0, h), np.where(drop(t), 0.0, e)
        u = sx[:, t, :, None] * b[:, t]
        eu = e_sx[:, t, :, None] * np.abs(b[:, t]) + 2 * U * np.abs(u)
        e = 1.0001 * (a * e + ea * np.abs(h) + eu + np.where(live[:, t, :, None], 2 * U * (np.abs(a * h) + np.abs(u)), 0.0))
        h = a * h + u
        H[t + 1], E[t + 1] = h, e
        mixed[:, t] = (c[:, t] * h).sum(-1) + D0 * x[:, t]
        e_mixed[:, t] = (np.abs(c[:, t]) * e).sum(-1) + (N + 6) * U * (np.abs(c[:, t] * h).sum(-1) + np.abs(D0 * x[:, t]))
    out = {"h_last": (h, 1.05 * e + 2 * U * np.abs(h))}
    if saved:
        out["saved"] = tuple(np.stack(v, 1) for v in zip(*saved))
        out["saved"] = (out["saved"][0], 1.05 * out["saved"][1] + 2 * U * np.abs(out["saved"][0]))
    gate, e_gate = np.ones((B, T, D)), np.zeros((B, T, D))
    if z is not None:
        z = clean(z.astype(np.float64))
        gate = silu(z)
        e_gate = np.abs(z) * e_sigmoid(z) + 2 * U * np.abs(gate)
    y = np.where(live, mixed * gate, 0.0)
    out["y"] = (y, 1.05 * np.where(live, np.abs(gate) * e_mixed + np.abs(mixed) * e_gate + 2 * U * np.abs(y), 0.0) + rounded(y, dtype))
    if dy is None:
        return out
    dy = clean(dy.astype(np.float64))
    gy, e_gy = dy * gate, np.abs(dy) * e_gate + 2 * U * np.abs(dy * gate)
    if z is not None:
        f, ef = dsilu(z), e_dsilu(z, 0.0)
        dz = dy * mixed * f
        e_dz = np.abs(dy) * (e_mixed * np.abs(f) + np.abs(mixed) * ef) + 4 * U * np.abs(dz)
        out["dz"] = (dz, 1.05 * e_dz + rounded(dz, dtype))
    g = np.zeros((B, D, N)) if dh_last is None else dh_last.astype(np.float64).copy()
    e = np.zeros_like(g)
    names = {"dx": (B, T, D), "ddt": (B, T, D), "db": (B, T, G, N), "dc": (B, T, G, N)}
    val, err = {k: np.zeros(s) for k, s in names.items()}, {k: np.zeros(s) for k, s in names.items()}
    dA, e_dA, s_dA = (np.zeros((D, N)) for _ in range(3))
    over = lambda v: v.reshape(B, G, per, N).sum(2)  # noqa: E731
    for t in range(T - 1, -1, -1):
        a, ea = decay(t)
        ht, eh, hp, ehp = H[t + 1], E[t + 1], np.where(drop(t), 0.0, H[t]), np.where(drop(t), 0.0, E[t])
        on = live[:, t, :, None]
        cg = c[:, t] * gy[:, t, :, None]
        e = e + np.abs(c[:, t]) * e_gy[:, t, :, None] + np.where(on, 3 * U * (np.abs(g) + np.abs(cg)), 0.0)
        g = g + cg
        v = gy[:, t, :, None] * ht
        val["dc"][:, t] = over(v)
        err["dc"][:, t] = over(np.abs(ht) * e_gy[:, t, :, None] + np.abs(gy[:, t, :, None]) * eh) + (per + 10) * U * over(np.abs(v))
        v = g * sx[:, t, :, None]
        val["db"][:, t] = over(v)
        err["db"][:, t] = over(np.abs(sx[:, t, :, None]) * e + np.abs(g) * e_sx[:, t, :, None]) + (per + 10) * U * over(np.abs(v))
        q = g * a * hp
        eq = np.abs(a * hp) * e + np.abs(g) * (a * ehp + ea * np.abs(hp)) + 4 * U * np.abs(q)
        sb = (g * b[:, t]).sum(-1)
        e_sb = (np.abs(b[:, t]) * e).sum(-1) + (N + 6) * U * np.abs(g * b[:, t]).sum(-1)
        sq = (A * q).sum(-1)
        e_sq = (np.abs(A) * eq).sum(-1) + (N + 8) * U * np.abs(A * q).sum(-1)
        d = sq + x[:, t] * sb
        ed = e_sq + np.abs(x[:, t]) * e_sb + 3 * U * (np.abs(sq) + np.abs(x[:, t] * sb))
        if softplus:
            s = sigmoid(raw[:, t])
            ed = s * ed + np.abs(d) * (e_sigmoid(raw[:, t]) + U * np.abs(raw[:, t]) * s) + 2 * U * np.abs(d * s)
            d = d * s
        val["ddt"][:, t], err["ddt"][:, t] = np.where(live[:, t], d, 0.0), np.where(live[:, t], ed, 0.0)
        val["dx"][:, t] = sb * step[:, t] + D0 * gy[:, t]
        err["dx"][:, t] = (e_sb * step[:, t] + np.abs(sb) * e_step[:, t] + np.abs(D0) * e_gy[:, t]
                           + 3 * U * (np.abs(sb * step[:, t]) + np.abs(D0 * gy[:, t])))
        v = q * step[:, t, :, None]
        dA += v.sum(0)
        s_dA += np.abs(v).sum(0)
        e_dA += (eq * step[:, t, :, None] + np.abs(q) * e_step[:, t, :, None]).sum(0)
        gn = a * g
        e = 1.0001 * (a * e + ea * np.abs(g) + np.where(on, 2 * U * np.abs(gn), 0.0))
        g, e = np.where(drop(t), 0.0, gn), np.where(drop(t), 0.0, e)
    for k in names:
        out[k] = (val[k], 1.05 * err[k] + rounded(val[k], dtype))
    terms = U * (T + B * 130 + 40)
    out["dA"] = (dA, 1.05 * e_dA + terms * s_dA)
    out["dskip"] = ((gy * x).sum((0, 1)), (e_gy * np.abs(x)).sum((0, 1)) + terms * np.abs(gy * x).sum((0, 1)))
    out["ddt_bias"] = (val["ddt"].sum((0, 1)), 1.05 * err["ddt"].sum((0, 1)) + terms * np.abs(val["ddt"]).sum((0, 1)))
    out["dh0"] = (g, 1.05 * e + 2 * U * np.abs(g))
    return out


# ---------------------------------------------------------------------- policy loss


def policy(z, tokens, old, A, ref=None, scale=None, tau=1.0, low=0.2, high=0.2, kl=0.0, bonus=0.0, dtype="f32"):
    """{name: (value, bound)} of loss, logp, entropy and grad; rows without NaN and +inf, ratios apart from the bounds."""
    N, V = z.shape
    d, lp, p, err_lp, rel_p, _, _ = _softmax(z, tau)
    with np.errstate(invalid="ignore"):
        logs = np.where(np.isfinite(d), d - lp, 0).max(1)
        terms = np.where(p > 0, p * lp, 0)
    H = -terms.sum(1)
    eH = ((np.abs(terms) * rel_p).sum(1) + (p * err_lp).sum(1) + err_lp.min(1) + U * (64 + V / 32) * np.abs(terms).sum(1) + 6 * U * (np.abs(H) + np.abs(logs)))
    rows = np.arange(N)
    y = np.asarray(tokens, np.int64)
    yc = np.clip(y, 0, V - 1)
    w = np.ones(N) if scale is None else scale.astype(np.float64)
    on = (y >= 0) & (w != 0)
    old, A = old.astype(np.float64), A.astype(np.float64)
    l, el = lp[rows, yc], err_lp[rows, yc] + 2 * U * np.abs(lp[rows, yc]) + 2 * U
    diff = l - old
    r = np.exp(diff)
    er = r * (el + U * np.abs(diff) + 4 * U + U * np.abs(diff) * 2)
    first, second = -r * A, -np.clip(r, 1 - low, 1 + high) * A
    keep = first >= second
    loss = np.where(keep, first, second)
    e = np.where(keep, np.abs(A) * er, 0.0) + 3 * U * np.abs(loss)
    D = np.where(keep, first, 0.0)
    eD = np.where(keep, np.abs(A) * er + 2 * U * np.abs(first), 0.0)
    if kl:
        far = ref.astype(np.float64) - l
        more = np.expm1(far)
        e_far = el + U * np.abs(far)
        loss = loss + kl * (more - far)
        e = e + kl * (np.abs(more) * e_far + 5 * U * np.abs(more) + 3 * U * np.abs(far)) + 2 * U * np.abs(loss)
        D = D - kl * more
        eD = eD + kl * ((1 + np.abs(more)) * e_far + 6 * U * np.abs(more)) + 2 * U * np.abs(D)
    if bonus:
        loss = loss - bonus * H
        e = e + abs(bonus) * (eH + 2 * U * np.abs(H)) + 2 * U * np.abs(loss)
    hit = np.zeros_like(p)
    hit[rows, yc] = 1
    lp0 = np.where(p > 0, lp, 0)
    d0 = np.where(np.isfinite(d), np.abs(d), 0)
    g = (D[:, None] * (hit - p) + bonus * p * (lp0 + H[:, None])) * w[:, None] / tau
    inner = np.abs(D)[:, None] + abs(bonus) * (np.abs(H)[:, None] + np.abs(logs)[:, None] + d0)
    eg = p * ((rel_p + 12 * U) * inner + eD[:, None] + abs(bonus) * eH[:, None]) + hit * (eD + 3 * U * np.abs(D))[:, None] + 2.0 ** -126 * inner
    eg = eg * np.abs(w)[:, None] / tau + 3 * U * np.abs(g)
    bad = on & (y >= V)
    blank = lambda v, nan=True: np.where(bad if v.ndim == 1 else bad[:, None], np.nan if nan else 0.0, np.where(on if v.ndim == 1 else on[:, None], v, 0.0))  # noqa: E731
    fix = lambda v: np.where(on if v.ndim == 1 else on[:, None], v, 0.0)  # noqa: E731
    return {"loss": (blank(loss), fix(e) + 2.0 ** -140), "logp": (blank(l), fix(el) + 2.0 ** -140),
            "entropy": (fix(H), fix(eH) + 2.0 ** -140), "grad": (blank(g), 1.01 * fix(eg) + rounded(fix(g), dtype))}
