"""The language-model operators in 64 bits, each with a bound on what fp32 arithmetic and one
rounding of the output may differ by.

U = 2^-24 is the largest relative error of one fp32 operation.  Bounds count operations: a gate
(exp, sum, quotient, product) is within GATE = 12 U, plus 8 U |f| where the argument of the exponential
carries its error (the documented bound of the fast exponential, 2 + 1.16 |f| units in the last
place of 2 U each, and what scaling the argument adds); a recurrence step adds 4 U of its terms.
"""
import numpy as np

U = 2.0 ** -24
# relative rounding of the output type, and its smallest step near zero
ROUND = {"f32": (2.0 ** -24, 2.0 ** -149), "bf16": (2.0 ** -8, 2.0 ** -133), "f16": (2.0 ** -11, 2.0 ** -24)}


def rounded(value, dtype):
    rel, step = ROUND[dtype]
    return rel * np.abs(value) + step


def glr(x, f, lerp, h0=None, lengths=None, reset=None, dh=None, dh_last=None, dtype="f32"):
    """{name: (value, bound)} of h, h_last, saved, and with dh of dx, df, dh0."""
    x, f = x.astype(np.float64), f.astype(np.float64)
    B, T, D = x.shape
    with np.errstate(over="ignore"):
        a, b = 1 / (1 + np.exp(-f)), 1 / (1 + np.exp(f))
    gate = 12 * U + 8 * U * np.abs(np.clip(np.nan_to_num(f), -100, 100))
    u = b * x if lerp else x
    n = np.full(B, T) if lengths is None else np.clip(lengths, 0, T)
    live = (np.arange(T)[None] < n[:, None])[..., None]
    fresh = np.zeros((B, T, 1), bool) if reset is None else (reset != 0)[..., None]
    h = np.zeros((B, D)) if h0 is None else h0.astype(np.float64).copy()
    e = np.zeros_like(h)
    H, E = np.zeros((B, T, D)), np.zeros((B, T, D))
    before, ebefore = np.zeros((B, T, D)), np.zeros((B, T, D))
    saved, esaved = [], []
    for t in range(T):
        if t % 16 == 0:
            saved.append(h.copy())
            esaved.append(e.copy())
        with np.errstate(invalid="ignore"):
            before[:, t], ebefore[:, t] = np.where(fresh[:, t], 0, h), np.where(fresh[:, t], 0, e)
            hn = a[:, t] * before[:, t] + u[:, t]
            en = a[:, t] * ebefore[:, t] + (gate[:, t] + 4 * U) * (np.abs(a[:, t] * before[:, t]) + np.abs(u[:, t]))
        h, e = np.where(live[:, t], hn, h), np.where(live[:, t], en, e)
        H[:, t], E[:, t] = np.where(live[:, t], h, 0), np.where(live[:, t], e, 0)
    out = {"h": (H, 1.01 * E + rounded(H, dtype)), "h_last": (h, e + 2 * U * np.abs(h))}
    out["saved"] = (np.stack(saved, 1), np.stack(esaved, 1)) if saved else (np.zeros((B, 0, D)),) * 2
    if dh is None:
        return out
    g = np.zeros((B, D)) if dh_last is None else dh_last.astype(np.float64).copy()
    e = np.zeros_like(g)
    dx, edx, df, edf = (np.zeros((B, T, D)) for _ in range(4))
    for t in range(T - 1, -1, -1):
        on = live[:, t]
        with np.errstate(invalid="ignore"):
            gt = dh[:, t].astype(np.float64) + g
            et = e + 4 * U * (np.abs(dh[:, t]) + np.abs(g))
            w = b[:, t] if lerp else np.ones_like(gt)
            dx[:, t], edx[:, t] = np.where(on, w * gt, 0), np.where(on, w * (et + (gate[:, t] + 2 * U) * np.abs(gt)), 0)
            c = before[:, t] - x[:, t] if lerp else before[:, t]
            ec = ebefore[:, t] + 2 * U * (np.abs(before[:, t]) + (np.abs(x[:, t]) if lerp else 0))
            ab = a[:, t] * b[:, t]
            df[:, t] = np.where(on, gt * c * ab, 0)
            edf[:, t] = np.where(on, ab * (et * np.abs(c) + np.abs(gt) * ec + (2 * gate[:, t] + 4 * U) * np.abs(gt * c)), 0)
            gn, gerr = a[:, t] * gt, a[:, t] * (et + (gate[:, t] + 2 * U) * np.abs(gt))
            gn, gerr = np.where(fresh[:, t], 0, gn), np.where(fresh[:, t], 0, gerr)
        g, e = np.where(on, gn, g), np.where(on, gerr, e)
    out["dx"] = (dx, 1.01 * edx + rounded(dx, dtype))
    out["df"] = (df, 1.01 * edf + rounded(df, dtype))
    out["dh0"] = (g, e + 2 * U * np.abs(g))
    return out


def _softmax(z, tau):
    """Reference log p of each row, with the bound of log p, of p relative to it, and of log-sum-exp."""
    z = z.astype(np.float64)
    V = z.shape[1]
    m = z.max(1, keepdims=True)
    ref = np.where(m == -np.inf, 0, m)
    d = (z - ref) / tau
    with np.errstate(divide="ignore", invalid="ignore"):
        s = np.exp(d).sum(1, keepdims=True)
        logs = np.where(s > 0, np.log(s), 0)
        lp = np.where(s > 0, d - logs, -np.inf)
    near = np.where(np.isfinite(d), np.minimum(np.abs(d), 200), 200)
    # exponent: 4 roundings of |d|; the exponential itself 12 U; the sum: its terms in sequence in
    # a thread, then a tree, with the terms' errors weighted by their mass
    rel = U * (12 + 8 * near)
    p = np.exp(np.where(np.isfinite(lp), lp, -np.inf))
    rel_s = (p * rel).sum(1, keepdims=True) + U * (64 + V / 32)
    err_lp = U * (4 * near + 2 * np.abs(logs)) + rel_s
    err_lse = U * (6 * np.abs(ref / tau) + 4 * np.abs(logs)) + rel_s
    lse = np.where(s > 0, ref / tau + logs, -np.inf)
    return d, lp, p, err_lp, rel + rel_s + 8 * U, lse, err_lse


def token_logp(z, tokens, tau, K, dlogp=None, dentropy=None, dtype="f32"):
    """{name: (value, bound)}; rows without NaN and +inf."""
    N, V = z.shape
    d, lp, p, err_lp, rel_p, lse, err_lse = _softmax(z, tau)
    with np.errstate(invalid="ignore"):
        terms = np.where(p > 0, p * lp, 0)
    H = -terms.sum(1)
    eH = ((np.abs(terms) * rel_p).sum(1) + (p * err_lp).sum(1) + err_lp.min(1) + U * (64 + V / 32) * np.abs(terms).sum(1) + 4 * U * np.abs(H))
    own = lambda v: rounded(np.where(np.isfinite(v), v, 0), "f32")  # noqa: E731  (the output's rounding)
    out = {"entropy": (H, eH + own(H)), "lse": (lse[:, 0], err_lse[:, 0] + 2 * own(lse[:, 0]))}
    rows = np.arange(N)
    y = np.asarray(tokens, np.int64)
    ok = (y >= 0) & (y < V)
    yc = np.where(ok, y, 0)
    out["logp"] = (np.where(y < 0, 0.0, np.where(y >= V, np.nan, lp[rows, yc])), err_lp[rows, yc] + 2 * U + own(lp[rows, yc]))
    if K:
        order = np.argsort(-z.astype(np.float64), axis=1, kind="stable")[:, :K]
        out["top_idx"] = (order, None)
        out["top_logp"] = (np.take_along_axis(lp, order, 1), np.take_along_axis(err_lp + own(lp), order, 1) + 2 * U)
    if dlogp is not None or dentropy is not None:
        dl = np.zeros(N) if dlogp is None else dlogp.astype(np.float64)
        dl = np.where(y < 0, 0.0, np.where(y >= V, np.nan, dl)) if dlogp is not None else dl
        dH = np.zeros(N) if dentropy is None else dentropy.astype(np.float64)
        with np.errstate(invalid="ignore"):
            lp0 = np.where(p > 0, lp, 0)
            g = -p * (dl[:, None] + dH[:, None] * (lp0 + H[:, None]))
        hit = np.zeros_like(p)
        hit[rows[ok], y[ok]] = 1
        g = (g + hit * dl[:, None]) / tau
        # log p is formed from the stored lse here
        e_lp = err_lse + U * (4 * np.minimum(np.abs(np.where(np.isfinite(z), z, 0) / tau), 1e6) + 4 * np.abs(lp0))
        rel = e_lp + U * (16 + 8 * np.abs(lp0))
        e = p * (rel * (np.abs(dl)[:, None] + np.abs(dH)[:, None] * np.abs(lp0 + H[:, None])) + np.abs(dH)[:, None] * (e_lp + eH[:, None])
                 + 8 * U * (np.abs(dl)[:, None] + np.abs(dH)[:, None] * (np.abs(lp0) + np.abs(H)[:, None])))
        e += 2.0 ** -150 * (np.abs(dl)[:, None] + np.abs(dH)[:, None] * np.abs(lp0 + H[:, None]))   # a subnormal p
        e = (e + 4 * U * hit * np.abs(dl)[:, None]) / tau + 4 * U * np.abs(g)
        out["grad"] = (g, 1.01 * e + rounded(g, dtype))
    return out


def distill(z, idx, top, tau, alpha, teacher_lse=None, labels=None, scale=None, dtype="f32"):
    """{name: (value, bound)} of loss and grad; rows with finite or -inf logits."""
    N, V = z.shape
    w = np.ones(N) if scale is None else scale.astype(np.float64)
    loss, eloss = np.zeros(N), np.zeros(N)
    grad, egrad = np.zeros((N, V)), np.zeros((N, V))
    for n in range(N):
        if w[n] == 0:
            continue
        zn = z[n:n + 1].astype(np.float64)
        d, lp, p, err_lp, rel_p, _, _ = (v[0] for v in _softmax(zn, tau))
        entries = [(int(j), float(t) / tau) for j, t in zip(idx[n], top[n]) if 0 <= j < V and t > -np.inf]
        kl = e_kl = mass = e_mass = 0.0
        q_at, e_at = np.zeros(V), np.zeros(V)
        factor, e_factor = np.zeros(V), np.zeros(V)
        if entries:
            t = np.array([v for _, v in entries])
            j = np.array([v for v, _ in entries])
            lse = np.log(np.exp(t - t.max()).sum()) + t.max() if teacher_lse is None else float(teacher_lse[n])
            logq = t - lse
            e_lq = U * (8 * np.abs(t) + 4 * abs(lse) + 8 * np.abs(t - t.max()) + 80 + len(t))
            q = np.exp(logq)
            rel_q = e_lq + U * (16 + 8 * np.minimum(np.abs(logq), 200))
            mass, e_mass = q.sum(), (q * (rel_q + U * 40)).sum()
            with np.errstate(invalid="ignore"):
                gap = np.where(q > 0, logq - lp[j], 0)
                kl = (q * gap).sum()
                e_kl = (q * (rel_q * np.abs(gap) + e_lq + err_lp[j] + 4 * U * (np.abs(logq) + np.abs(lp[j])) + U * 40 * np.abs(gap)))
                e_kl = np.where(q > 0, e_kl, 0).sum()
            np.add.at(q_at, j, q)
            np.add.at(e_at, j, q * (rel_q + 40 * U))
        factor += mass
        e_factor += e_mass
        if teacher_lse is not None:
            inside = np.zeros(V, bool)
            inside[[j for j, _ in entries]] = True
            rest = p[~inside].sum()
            if rest > 0 and 1 - mass > -1e-3:
                qr, e_qr = max(0.0, 1 - mass), e_mass + 4 * U
                rel_r = (p[~inside] * rel_p[~inside]).sum() / rest + U * (64 + V / 32)
                if qr > 0:
                    log_r = np.log(rest)
                    kl += qr * (np.log(qr) - log_r)
                    e_kl += e_qr * (abs(np.log(qr)) + abs(log_r) + 1) + qr * (rel_r + U * 8 * (abs(log_r) + abs(np.log(qr)) + 4))
                    factor += qr
                    factor[~inside] -= qr / rest
                    e_factor += e_qr
                    e_factor[~inside] += e_qr / rest + qr / rest * (rel_r + 16 * U)
        soft = (1 - alpha) * tau
        loss[n], eloss[n] = soft * tau * kl, soft * tau * (e_kl + 8 * U * abs(kl))
        g = soft * (p * factor - q_at)
        e = soft * (p * np.abs(factor) * (rel_p + 16 * U) + p * e_factor + e_at + 8 * U * (p * np.abs(factor) + q_at))
        if alpha > 0 and labels[n] >= 0:
            if labels[n] >= V:
                loss[n] = np.nan
                grad[n] = np.nan
                continue
            y = int(labels[n])
            _, lp1, p1, err1, rel1, _, _ = (v[0] for v in _softmax(zn, 1.0))
            loss[n] -= alpha * lp1[y]
            eloss[n] += alpha * (err1[y] + 4 * U * (abs(lp1[y]) if np.isfinite(lp1[y]) else 0))
            hit = np.zeros(V)
            hit[y] = 1
            g = g + alpha * (p1 - hit)
            e = e + alpha * (p1 * (rel1 + 8 * U) + 4 * U * hit) + 4 * U * np.abs(g)
        if np.isfinite(loss[n]):
            eloss[n] += 8 * U * abs(loss[n])
        grad[n], egrad[n] = w[n] * g, abs(w[n]) * e + 4 * U * np.abs(w[n] * g)
    return {"loss": (loss, eloss + 2.0 ** -140), "grad": (grad, 1.01 * egrad + rounded(grad, dtype))}


def check(got, want, name):
    """Every element of got within its bound of want; infinities and NaN in the same places."""
    value, bound = want
    got = np.asarray(got, np.float64 if bound is not None else None)
    assert got.shape == value.shape, (name, got.shape, value.shape)
    if bound is None:
        assert np.array_equal(got, value), f"{name}: {np.sum(got != value)} of {got.size} differ"
        return
    bound = np.broadcast_to(bound, value.shape)
    fine = np.isfinite(value)
    assert np.array_equal(np.isnan(got), np.isnan(value)), f"{name}: NaN in other places"
    assert np.array_equal(got[~fine & ~np.isnan(value)], value[~fine & ~np.isnan(value)]), f"{name}: other infinities"
    assert np.isfinite(got[fine]).all(), f"{name}: not finite"
    off = np.abs(got[fine] - value[fine]) - bound[fine]
    assert off.size == 0 or off.max() <= 0, \
        f"{name}: {np.sum(off > 0)} of {off.size} outside, worst by {off.max():.3g} (bound {bound[fine][off.argmax()]:.3g})"
