"""The forecasting operators in 64 bits, step by step, each value with a bound on what 32-bit arithmetic may differ by.

The bounds follow the formulas: every operation contributes its own rounding, carried through the recurrence by the
magnitudes it meets.  EPS is the unit roundoff of 32 bits; the exponential unit and the functions built on it are
taken at 4 EPS relative plus the rounding of their argument (|argument| EPS).
"""
import numpy as np

EPS = 2.0 ** -24
ROUND = {"float32": 0.0, "float16": 2.0 ** -11, "bfloat16": 2.0 ** -8}     # bf16: 8 bits; half an ulp is 2^-9, doubled below
TINY = {"float32": 0.0, "float16": 2.0 ** -24, "bfloat16": 0.0}            # spacing of the smallest values
FLUSH = 2.0 ** -120                                                        # what a flushed subnormal may lose


def silu(v, ev):
    """silu(v) and its error for an argument off by ev (its slope stays below 1.1)."""
    with np.errstate(over="ignore"):
        s = v / (1.0 + np.exp(-v))
    return s, 1.1 * ev + np.abs(s) * (8 + 2 * np.abs(v)) * EPS + FLUSH


def softplus(v, ev):
    s = np.maximum(v, 0.0) + np.log1p(np.exp(-np.abs(v)))
    # log1p(e^-|v|): the inner exponential's relative error, and the rounding of the sum
    return s, ev + (np.log1p(np.exp(-np.abs(v))) * (8 + 2 * np.abs(v)) + s * 4) * EPS + FLUSH


def ssm(xbc, dt, z, off, A, skip, dt_bias, conv_w, conv_b, G, state, history):
    """state (S, D, N) and history (S, W - 1, rows) per job, float64; returns y, its bound, state, its bound, history."""
    D, N = A.shape
    W = 0 if conv_w is None else conv_w.shape[1]
    T = xbc.shape[0]
    y, ey = np.full((T, D), np.nan), np.zeros((T, D))
    state, history = state.copy(), history.copy()
    estate = np.zeros_like(state)
    for s in range(len(off) - 1):
        h, eh = state[s], np.zeros((D, N))
        window = list(history[s]) if W > 1 else []
        for t in range(off[s], off[s + 1]):
            row = xbc[t]
            if W == 0:
                u, eu = row, np.zeros_like(row)
            else:
                taps = np.stack(window + [row], axis=1)
                prod = taps * conv_w
                v = prod.sum(axis=1) + conv_b
                u, eu = silu(v, (np.abs(prod).sum(axis=1) + np.abs(conv_b)) * (W + 1) * EPS)
                window = (window + [row])[1:]
            x, ex = u[:D], eu[:D]
            B, eB = (np.repeat(q[D:D + G * N].reshape(G, N), D // G, axis=0) for q in (u, eu))
            C, eC = (np.repeat(q[D + G * N:].reshape(G, N), D // G, axis=0) for q in (u, eu))
            raw = dt[t] + dt_bias
            d, ed = softplus(raw, np.abs(raw) * EPS)
            arg = d[:, None] * A
            decay = np.exp(arg)
            # the argument in base 2: A log2(e), then the product, are rounded; d itself is off by ed
            edecay = decay * (ed[:, None] * np.abs(A) + 4 * np.abs(arg) * EPS + 4 * EPS) + FLUSH
            dx = (d * x)[:, None]
            edx = (ed * np.abs(x) + d * ex)[:, None] + 2 * np.abs(dx) * EPS
            inp, einp = dx * B, edx * np.abs(B) + np.abs(dx) * eB + 2 * np.abs(dx * B) * EPS
            eh = decay * eh + edecay * (np.abs(h) + eh) + einp
            h = decay * h + inp
            eh = eh + np.abs(h) * EPS + FLUSH
            prod = C * h
            o = prod.sum(axis=1) + skip * x
            eo = (np.abs(C) * eh + eC * (np.abs(h) + eh)).sum(axis=1) + np.abs(skip) * ex
            eo = eo + (np.abs(prod).sum(axis=1) + np.abs(skip * x)) * (N + 3) * EPS
            if z is not None:
                gate, eg = silu(z[t], 0.0)
                eo = eo * (np.abs(gate) + eg) + np.abs(o) * eg + np.abs(o * gate) * EPS
                o = o * gate
            y[t], ey[t] = o, eo
        state[s], estate[s] = h, eh
        if W > 1:
            history[s] = np.stack(window)
    return y, ey, state, estate, history


def token_stats(logits, tokens, top, scale):
    """logits float64 (R, V); returns logp, entropy, top_logp, top_ids and a bound on the first three (one per row)."""
    R, V = logits.shape
    logp, entropy = np.zeros(R), np.zeros(R)
    top_logp, top_ids, bound = np.full((R, top), -np.inf), np.full((R, top), -1, np.int32), np.zeros(R)
    for r in range(R):
        x = logits[r]
        l = x * scale
        with np.errstate(invalid="ignore", over="ignore"):
            if np.isnan(x).any() or (x == np.inf).any():
                lp, entropy[r] = np.where(x == -np.inf, -np.inf, np.nan), np.nan
            elif (x == -np.inf).all():
                lp = np.full(V, -np.inf)
            else:
                lse = l.max() + np.log(np.exp(l - l.max()).sum())
                lp = l - lse
                p = np.exp(lp)
                entropy[r] = -(p[p > 0] * lp[p > 0]).sum()
        t = tokens[r]
        logp[r] = 0.0 if t < 0 else np.nan if t >= V else lp[t]
        order = np.lexsort((np.arange(V), np.where(np.isnan(x), np.inf, -x)))        # NaN: below -inf
        nan_last = np.concatenate([order[~np.isnan(x[order])], np.sort(order[np.isnan(x[order])])])
        k = min(top, V)
        top_ids[r, :k], top_logp[r, :k] = nan_last[:k], lp[nan_last[:k]]
        finite = np.abs(l[np.isfinite(l)])
        # scaled logits and reference rounded at their size; sums of V positive terms, at most V / 32 of them in a row,
        # each off by the exponential's error and its argument's; the weighted sum meets differences of up to 2 max
        most = finite.max() if finite.size else 0.0
        bound[r] = EPS * (8 * most + (V / 32 + 32 + 4 * most) * (1 + np.log(V) + min(2 * most, 100.0) * 0.25))
    return logp, entropy, top_logp, top_ids, bound
