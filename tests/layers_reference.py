"""The layers of recurrent language models with matrix states as they are defined, in 64 bits on the CPU, with a bound for
what an evaluation in binary32 may be off.  Test infrastructure only.

The bounds count roundings as tests/operators_reference.py does: EPS = 2^-24 for each of binary32, twice that for an addition
inside a matrix unit, which need not round to the nearest; UNIT for the one to the element type."""

import numpy as np

from tests.operators_reference import EPS, UNIT


# --- rotary -----------------------------------------------------------------
def frequencies(n, base=10000.0, factor=1.0, context=0.0, low=1.0, high=32.0):
    f = base ** (-2.0 * np.arange(n // 2) / max(n, 1))
    kept = np.clip((f * context / (2.0 * np.pi) - low) / (high - low), 0.0, 1.0)
    return f * (kept + (1.0 - kept) / factor)


def rotary(x, positions, f, half, magnitude, inverse):
    """(value, bound).  cos and sin are off by the rounding of the angle (two, of an eighth of a turn at most), four of the
    series and what it leaves out (2e-9): 8 EPS; a product with the magnitude, one with the element, and a sum."""
    n = 2 * len(f)
    value, bound = x.copy(), np.zeros_like(x)
    angle = (np.asarray(positions, np.float64)[:, None] * f * (-1.0 if inverse else 1.0))[:, None]
    c, s = magnitude * np.cos(angle), magnitude * np.sin(angle)
    i = np.arange(n // 2)
    p, q = (i, i + n // 2) if half else (2 * i, 2 * i + 1)
    value[..., p] = x[..., p] * c - x[..., q] * s
    value[..., q] = x[..., p] * s + x[..., q] * c
    bound[..., p] = bound[..., q] = 11 * EPS * abs(magnitude) * (np.abs(x[..., p]) + np.abs(x[..., q]))
    return value, bound


# --- linear attention ---------------------------------------------------------
def _walk(a, b, c, log_decay, first, scale, out_scale, late, dtype):
    """out, last and their bounds for one sequence: a, b [steps, heads, da], c [steps, heads, dc].

    `size` is the same recurrence of absolute values, `off` bounds what a state is off: a step rounds it a few times (8:
    the product, the parts that are left out, sums of up to 64 products inside a matrix unit are counted where they are
    read), and a power of the decay is off by the rounding of its exponent.  Shares and a state that is read are taken as two
    bfloat16 parts for results in 16 bits, the first cut off (2^-7 of it is left at most), the second rounded (2^-8 of that):
    2^-15 of each term."""
    parts = 0.0 if dtype == "f32" else 2.0 ** -15
    steps, heads, da = a.shape
    d = np.exp(log_decay.astype(np.float64))[:, None, None]
    rate = np.abs(np.where(np.isinf(log_decay), 0.0, log_decay))[:, None, None]
    state = np.zeros((heads, da, c.shape[2])) if first is None else first.astype(np.float64)
    size, off = np.abs(state), np.zeros_like(state)
    out, bound = np.empty((steps, heads, c.shape[2])), np.empty((steps, heads, c.shape[2]))

    def decay():
        nonlocal state, size, off
        off = d * (off + 4 * EPS * rate * size)
        state, size = d * state, d * size

    for t in range(steps):
        if not late:
            decay()
        kv = scale * b[t][:, :, None] * c[t][:, None, :]
        state, size = state + kv, size + np.abs(kv)
        off = off + (8 + 2 * 64) * EPS * size
        out[t] = out_scale * np.einsum("hi,hij->hj", a[t], state)
        absolute = np.abs(a[t])
        bound[t] = abs(out_scale) * (np.einsum("hi,hij->hj", absolute, off) +
                                     (2 * (da + 8) * EPS + parts) * np.einsum("hi,hij->hj", absolute, size))
        if late:
            decay()
    return out, bound, state, off


def attention(q, k, v, log_decay, state0, scale, lengths, do=None, dstate_last=None, dtype="f32"):
    """{name: (value, bound)}: o, state_last, and with `do` dq, dk, dv, dstate0."""
    n, heads, dk, dv = q.shape[0], q.shape[1], q.shape[2], v.shape[2]
    result = {name: (np.zeros((n, heads, d)), np.zeros((n, heads, d))) for name, d in
              (("o", dv), ("dq", dk), ("dk", dk), ("dv", dv))}
    for name in ("state_last", "dstate0"):
        result[name] = (np.zeros((len(lengths), heads, dk, dv)), np.zeros((len(lengths), heads, dk, dv)))
    turned = lambda x: None if x is None else np.swapaxes(x, -1, -2)
    start = 0
    for s, length in enumerate(lengths):
        there = slice(start, start + length)
        first = None if state0 is None else state0[s]
        out = _walk(q[there], k[there], v[there], log_decay, first, 1.0, scale, False, dtype)
        result["o"][0][there], result["o"][1][there] = out[:2]
        result["state_last"][0][s], result["state_last"][1][s] = out[2:]
        if do is not None:
            back = lambda x: x[there][::-1]
            out = _walk(do[there], v[there], k[there], log_decay, turned(first), 1.0, scale, False, dtype)
            result["dq"][0][there], result["dq"][1][there] = out[:2]
            flow = None if dstate_last is None else dstate_last[s]
            out = _walk(back(v), back(do), back(q), log_decay, turned(flow), scale, 1.0, True, dtype)
            result["dk"][0][there], result["dk"][1][there] = out[0][::-1], out[1][::-1]
            out = _walk(back(k), back(q), back(do), log_decay, flow, scale, 1.0, True, dtype)
            result["dv"][0][there], result["dv"][1][there] = out[0][::-1], out[1][::-1]
            result["dstate0"][0][s], result["dstate0"][1][s] = out[2:]
        start += length
    return result


# --- vocabulary loss ----------------------------------------------------------
def vocab_loss(hidden, weight, labels, row_weight, dtype, alone=False):
    """{name: (value, bound)}: loss, lse, dhidden, dweight.

    A logit is off by 2 EPS for each of its products; a share by that, the log-sum-exp's error, the rounding of its exponent
    and of the exponential; it is rounded to the element type after its product with the row's weight; then the sums.

    With `alone`: what a row may be off by itself, whatever the others hold.  In binary32 every element is held as three parts
    of bfloat16, cut off, of which nothing is lost; of the products those of the parts 1 and 2, 2 and 1, 2 and 2 are left out,
    2 * 2^-8 * 2^-16 and less: 2 EPS.  In binary16 a share is scaled by 2^14 for dhidden, whatever its row weighs, and for dweight
    by 2^14 over the largest weight: 2^-39 is lost at most, of one or of the largest weight.

    Without: as much as two parts of binary16 are off that share a scale, which is more.  2^-22 of an element is lost at most,
    and the product of the small parts, 2^-22 of a product, is left out: 3 * 2^-22 = 12 EPS.  Shares in binary16, one part or
    two, and the parts of binary32 are scaled so that the array's largest is 2^14 or more, where the smallest step is 2^-24:
    2^-25 / 2^14 = 2^-39 of the largest may be lost whatever the element is."""
    rows, vocab, width = hidden.shape[0], weight.shape[0], hidden.shape[1]
    w = np.where((labels < 0) | (labels >= vocab), 0.0, np.ones(rows) if row_weight is None else row_weight)
    y = np.where((labels < 0) | (labels >= vocab), 0, labels)
    dead = w == 0.0
    seen = np.where(dead[:, None] & ~np.isfinite(hidden), 0.0, hidden)   # counts nothing in a row without weight
    z = seen @ weight.T
    off = (2 * width + ((6 if alone else 16) if dtype == "f32" else 4)) * EPS * (np.abs(seen) @ np.abs(weight).T)
    step = 2.0 ** -39
    most = lambda x: step * np.abs(x).max(initial=0.0) if dtype == "f32" and not alone else 0.0
    sizes = (np.abs(seen).sum(1, keepdims=True), np.abs(weight).sum(1))
    off = off + sizes[0] * most(weight) + sizes[1] * most(seen)
    top = z.max(1, keepdims=True)
    e = np.exp(z - top)
    lse = top[:, 0] + np.log(e.sum(1))
    p = e / e.sum(1, keepdims=True)
    far = np.abs(z - lse[:, None])
    lse_off = (p * (off + (4 + 2 * np.abs(z - top)) * EPS)).sum(1) + 2 * (vocab / 16 + 16) * EPS + 4 * EPS * np.abs(lse)
    at = np.arange(rows)
    loss = w * (lse - z[at, y])
    loss_off = np.abs(w) * (lse_off + off[at, y] + 2 * EPS * np.abs(lse - z[at, y]))
    share = p.copy()
    share[at, y] -= 1.0
    share_off = p * (off + lse_off[:, None] + (4 + 2 * far) * EPS) + 2 * EPS * np.abs(share)
    unit = 4 * EPS if dtype == "f32" else UNIT[dtype] + 2.0 ** -24
    share_off = share_off + unit * np.abs(share)
    over = step * (np.abs(w).max(initial=0.0) / np.where(dead, 1.0, np.abs(w)))[:, None]
    own = share_off + step if dtype == "f16" else share_off
    if dtype == "f16" or dtype == "f32" and not alone:
        share_off = share_off + over
    a = np.abs
    dhidden = w[:, None] * (share @ weight)
    dhidden_off = a(w)[:, None] * ((own if alone else share_off) @ a(weight) + 2 * (vocab + 8) * EPS * (a(share) @ a(weight)) +
                                 a(share).sum(1, keepdims=True) * most(weight))
    h = np.where(dead[:, None], 0.0, seen)
    dweight = (share * w[:, None]).T @ h
    dweight_off = ((share_off * a(w)[:, None]).T @ a(h)) + 2 * (rows + 8) * EPS * ((a(share) * a(w)[:, None]).T @ a(h))
    dweight_off = dweight_off + (a(share) * a(w)[:, None]).sum(0)[:, None] * most(h)
    return dict(loss=(loss, loss_off), lse=(lse, lse_off), dhidden=(dhidden, dhidden_off), dweight=(dweight, dweight_off))
