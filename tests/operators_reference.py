"""The operators on logits and sequences as they are defined, in 64 bits on the CPU, with a bound for what an
evaluation in binary32 may be off.  Test infrastructure only.

Rounding: `EPS` = 2^-24 is half a unit in the last place of binary32.  `UNIT` is the same for the element type that a
result is rounded to in the end, `TINY` half its smallest subnormal.  The bounds count roundings: every operation adds one,
an exponential of an argument x adds |x| of them for the rounded argument (twice, for its scaling) and two of its own,
and a sum of n terms at most n, of which a workgroup's threads do n / 64 one after the other at most here."""

import numpy as np

EPS = 2.0 ** -24
UNIT = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
TINY = {"f32": 2.0 ** -150, "f16": 2.0 ** -25, "bf16": 2.0 ** -134}


def rounded(bound, value, dtype):
    """A bound for a result that is off by `bound` before it is rounded to `dtype`."""
    return bound + (np.abs(value) + bound) * UNIT[dtype] + TINY[dtype]


# --- rows of logits -----------------------------------------------------------
def top(z, k):
    """(idx, val): the k largest of every row, ties by ascending index; NaN and -inf never."""
    z = np.asarray(z, np.float64)
    idx = np.full((z.shape[0], k), -1, np.int32)
    val = np.full((z.shape[0], k), -np.inf)
    for r in range(z.shape[0]):
        row = np.where(np.isnan(z[r]), -np.inf, z[r])
        order = np.argsort(-row, kind="stable")[:k]
        order = order[row[order] > -np.inf]
        idx[r, :len(order)] = order
        val[r, :len(order)] = row[order]
    return idx, val


def lse(z, temperature):
    z = np.asarray(z, np.float64) / temperature
    with np.errstate(invalid="ignore", divide="ignore", over="ignore"):
        m = z.max(axis=1, keepdims=True)
        shift = np.where(m == -np.inf, 0.0, m)
        return (shift + np.log(np.exp(z - shift).sum(1, keepdims=True)))[:, 0]


def sum_roundings(n):
    return 8 + n / 64.0


def lse_bound(z, temperature):
    """|log-sum-exp|: its own magnitude's roundings, and the relative ones of the sum: of its terms those within 2^-24 of
    the largest count (arguments up to 17), the others add less than n 2^-24 altogether."""
    value = np.abs(lse(z, temperature))
    return EPS * (4.0 * (np.where(np.isfinite(value), value, 0.0) + 1.0) + 4 * 17 + sum_roundings(z.shape[1]))


def distill(z, top_idx, top_val, temperature, hard, labels=None, top_lse=None, weight=None):
    """(loss, grad, loss_bound, grad_bound) of every row."""
    z = np.asarray(z, np.float64)
    rows, vocab = z.shape
    loss, grad = np.zeros(rows), np.zeros_like(z)
    loss_bound, grad_bound = np.zeros(rows), np.zeros_like(z)
    for r in range(rows):
        w = 1.0 if weight is None else float(weight[r])
        if w == 0.0 or np.all(z[r] == -np.inf):
            continue
        with np.errstate(over="ignore", invalid="ignore", divide="ignore"):
            log_q = z[r] / temperature - lse(z[r:r + 1], temperature)[0]
            log_q1 = z[r] - lse(z[r:r + 1], 1.0)[0]
        q, q1 = np.exp(log_q), np.exp(log_q1)
        # an element's probability: the argument's roundings and the sum's
        far = np.where(np.isfinite(log_q1), np.minimum(np.abs(log_q1), 200.0), 0.0) + np.log(vocab)
        relative = EPS * (4 * far + 4 * 17 + 8 + sum_roundings(vocab))
        pairs = [(int(i), float(t) / temperature) for i, t in zip(top_idx[r], top_val[r]) if 0 <= i < vocab]
        t = np.array([p[1] for p in pairs])
        kl = kl_bound = 0.0
        p = np.zeros(len(pairs))
        p_bound = np.zeros(len(pairs))
        if len(pairs) and (top_lse is not None or np.any(t > -np.inf)):
            c = float(top_lse[r]) if top_lse is not None else t.max() + np.log(np.exp(t - t.max()).sum())
            log_p = t - c
            p = np.exp(log_p)
            size = np.where(np.isfinite(log_p), np.abs(log_p) + np.abs(t) + abs(c), 0.0)
            p_bound = p * EPS * (4 * size + 4 * 17 + 16 + len(pairs))
            for i, (j, _) in enumerate(pairs):
                if p[i] > 0.0:
                    kl += p[i] * (log_p[i] - log_q[j])
                    both = abs(log_p[i]) + abs(log_q[j])
                    kl_bound += p_bound[i] * both + p[i] * EPS * (4 * (size[i] + abs(log_q[j]) + np.log(vocab)) + 4 * 17 +
                                                                  sum_roundings(vocab) + len(pairs))
        y = -1 if labels is None or hard == 0.0 else int(labels[r])
        y = y if y < vocab else -1
        ce = -log_q1[y] if y >= 0 else 0.0
        ce_bound = EPS * (8 * (abs(ce) + np.log(vocab)) + 4 * 17 + sum_roundings(vocab)) if y >= 0 else 0.0
        soft = (1.0 - hard) * temperature
        loss[r] = w * (soft * temperature * kl + hard * ce)
        loss_bound[r] = abs(w) * (soft * temperature * kl_bound + hard * ce_bound) + 8 * EPS * abs(w) * (
            soft * temperature * abs(kl) + hard * abs(ce))
        mass = p.sum()
        g = soft * mass * q
        b = soft * (mass * q * (relative + 8 * EPS) + q * p_bound.sum())
        if y >= 0:
            g = g + hard * q1
            b = b + hard * q1 * (relative + 8 * EPS)
        for i, (j, _) in enumerate(pairs):
            g[j] -= soft * p[i]
            b[j] += soft * (p_bound[i] + 8 * EPS * p[i])
        if y >= 0:
            g[y] -= hard
            b[y] += 8 * EPS * hard
        grad[r], grad_bound[r] = w * g, abs(w) * b
    return loss, grad, loss_bound, grad_bound


# --- the recurrence -----------------------------------------------------------
def _sigmoid(f):
    with np.errstate(over="ignore"):
        t = np.exp(-np.abs(f))
    return np.where(f >= 0, 1.0 / (1.0 + t), t / (1.0 + t)), np.where(f >= 0, t / (1.0 + t), 1.0 / (1.0 + t))


def _gate_roundings(f):
    """Of a sigmoid: exponential (argument |f|), sum, reciprocal (two), product; and two of the step that uses it."""
    return 12.0 + 4.0 * np.where(np.isfinite(f), np.minimum(np.abs(f), 200.0), 0.0)


def scan_forward(gate, x, lengths, h0, free):
    """h, h_last and bounds of both.  All coefficients are positive, so that a bound obeys the recurrence itself,
    fed with the roundings of the terms' magnitudes; it holds for every order in which terms are joined."""
    gate, x = np.asarray(gate, np.float64), np.asarray(x, np.float64)
    a, b = _sigmoid(gate)
    drive = x if free else b * x
    per = _gate_roundings(gate) * EPS
    h, bound = np.zeros_like(x), np.zeros_like(x)
    last = np.zeros((len(lengths), x.shape[1])) if h0 is None else np.asarray(h0, np.float64).copy()
    last_bound = np.zeros_like(last)
    before, before_bound = np.zeros_like(x), np.zeros_like(x)
    row = 0
    for s, length in enumerate(lengths):
        state, big, err = last[s], np.abs(last[s]), np.zeros(x.shape[1])
        for t in range(row, row + length):
            before[t], before_bound[t] = state, err
            err = a[t] * err + per[t] * (a[t] * big + np.abs(drive[t]))
            big = a[t] * big + np.abs(drive[t])
            state = a[t] * state + drive[t]
            h[t], bound[t] = state, err
        last[s], last_bound[s] = state, err
        row += length
    return dict(h=h, h_bound=bound, last=last, last_bound=last_bound, before=before, before_bound=before_bound)


def scan_backward(gate, x, lengths, h0, dh, dh_last, free):
    gate, x, dh = (np.asarray(v, np.float64) for v in (gate, x, dh))
    f = scan_forward(gate, x, lengths, h0, free)
    a, b = _sigmoid(gate)
    per = _gate_roundings(gate) * EPS
    g, g_bound = np.zeros_like(x), np.zeros_like(x)
    flow0 = np.zeros((len(lengths), x.shape[1])) if dh_last is None else np.asarray(dh_last, np.float64).copy()
    flow_bound = np.zeros_like(flow0)
    row = sum(lengths)
    for s in reversed(range(len(lengths))):
        row -= lengths[s]
        flow, big, err = flow0[s], np.abs(flow0[s]), np.zeros(x.shape[1])
        for t in reversed(range(row, row + lengths[s])):
            gt, big_t = dh[t] + flow, np.abs(dh[t]) + big
            err = err + 2 * EPS * big_t
            g[t], g_bound[t] = gt, err
            flow, big, err = a[t] * gt, a[t] * big_t, a[t] * err + per[t] * a[t] * big_t
        flow0[s], flow_bound[s] = flow, err
    ab = a * b
    dx = g if free else b * g
    dx_bound = g_bound if free else b * g_bound + per * np.abs(dx)
    inner = f["before"] if free else f["before"] - x
    inner_size = np.abs(f["before"]) + (0.0 if free else np.abs(x))
    dgate = g * inner * ab
    dgate_bound = ab * (g_bound * np.abs(inner) + (np.abs(g) + g_bound) * f["before_bound"]
                        + np.abs(g) * inner_size * 2 * per)
    return dict(dx=dx, dx_bound=dx_bound, dgate=dgate, dgate_bound=dgate_bound, dh0=flow0, dh0_bound=flow_bound)
