"""The operators of a distilled recurrent language model, as cases to measure.

A case is one pass through one operator:

  top      a teacher's k largest logits of every row as (index, value) pairs, largest first, ties to the lowest
           index, and the row's log-sum-exp at a temperature (`Distillation.dgc_top_logits`)
  distill  loss and gradient of a student's logits against such pairs, mixed with hard labels
           (`Distillation.dgc_distill_loss`), or the loss alone
  scan     the gated linear recurrence h_t = a_t h_{t-1} + b_t x_t with a = sigmoid(gate) and b = 1 - a (or 1), over
           sequences of equal or of different lengths laid behind each other: forward alone, or forward and backward
           (`GatedScan.dgc_gated_scan_forward`, `GatedScan.dgc_gated_scan_backward`)

Where `own` is false, `run` computes the same from elementary torch operations in 32 bits; `exact` in 64 bits.
"""

from __future__ import annotations

import math
import random
from typing import List

import torch

own = False

DEVICE = "cuda"
DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}


# ---------------------------------------------------------------------------
# Cases
# ---------------------------------------------------------------------------
def _top(**kw) -> dict:
    return dict(dict(op="top", rows=1, vocab=1, k=1, dtype="f32", temperature=1.0, padding=0, masks=False), **kw)


def _distill(**kw) -> dict:
    return dict(dict(op="distill", rows=1, vocab=1, k=1, dtype="f32", temperature=1.0, hard=0.0, tail=False, grad=True,
                     padding=0, masks=False), **kw)


def _scan(**kw) -> dict:
    return dict(dict(op="scan", sequences=1, length=1, channels=1, dtype="f32", free=False, train=False, packed=False,
                     joint=False, initial=True, resets=False, layout_seed=0), **kw)


def listed() -> List[dict]:
    return [
        # a teacher asked for the next token of a few streams: latency
        _top(name="top_serve", rows=8, vocab=32768, k=16, dtype="bf16"),
        # a batch of 20 x 35 tokens of the LSTM language model's vocabulary
        _top(name="top_lm", rows=700, vocab=10000, k=64, dtype="f32", temperature=2.0),
        # an odd vocabulary, part of it masked by -inf or by the type's lowest value, some rows wholly
        _top(name="top_odd", rows=333, vocab=50001, k=100, dtype="f16", masks=True),
        # labelling a corpus with a large vocabulary
        _top(name="top_large", rows=4096, vocab=131072, k=64, dtype="bf16"),
        # one time step of the language model's batch, loss and gradient: latency
        _distill(name="distill_small", rows=20, vocab=10000, k=8, dtype="f32", hard=0.5, temperature=2.0),
        # validation: the loss alone, in a buffer whose rows are padded
        _distill(name="distill_eval", rows=1024, vocab=50000, k=32, dtype="bf16", grad=False, padding=48),
        # odd vocabulary, masked logits, padded pair lists, rows of weight zero, the teacher's whole log-sum-exp
        _distill(name="distill_odd", rows=1111, vocab=32771, k=50, dtype="f16", temperature=2.0, hard=0.1, tail=True,
                 masks=True),
        # the training step of a large vocabulary, soft and hard targets
        _distill(name="distill_large", rows=4096, vocab=131072, k=64, dtype="bf16", temperature=2.0, hard=0.1),
        # one token for each of 64 streams, the state carried in 32 bits: latency
        _scan(name="scan_step", sequences=64, length=1, channels=1500, dtype="f32"),
        # a training step of the LSTM language model's shape: 20 sequences of 35 steps, 1500 channels
        _scan(name="scan_lm", sequences=20, length=35, channels=1500, dtype="f32", train=True),
        # utterances of very different lengths behind each other, 1200 channels, gate and candidate from one projection
        _scan(name="scan_packed", sequences=48, length=1500, channels=1200, dtype="f16", packed=True, joint=True,
              initial=False),
        # one long document, training, with places where the state starts again
        _scan(name="scan_long", sequences=1, length=65536, channels=2048, dtype="bf16", train=True, joint=True,
              resets=True),
    ]


def draw(rng) -> dict:
    """One more case of the ranges above: vocabularies of 29 (the speech model's letters) to 131072, up to 4096 rows,
    sequences of 1 to 65536 steps, 32 to 4096 channels, odd sizes among them."""
    def spread(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    dtype = rng.choice(("f32", "f16", "bf16", "bf16"))
    op = rng.choice(("top", "distill", "scan", "scan"))
    if op == "scan":
        train = rng.random() < 0.6
        channels = spread(32, 4096)
        if rng.random() < 0.5:
            channels = (channels + 7) // 8 * 8
        length = spread(1, 65536)
        sequences = max(1, min(spread(1, 256), (1 << 26) // (length * channels)))
        return _scan(sequences=sequences, length=length, channels=channels, dtype=dtype, train=train,
                     free=rng.random() < 0.3, packed=rng.random() < 0.5, joint=rng.random() < 0.5,
                     initial=rng.random() < 0.7, resets=rng.random() < 0.3, layout_seed=rng.randrange(1 << 20))
    vocab = spread(29, 131072)
    if rng.random() < 0.5:
        vocab = (vocab + 7) // 8 * 8
    rows = max(1, min(spread(1, 4096), (1 << 27) // vocab))
    common = dict(rows=rows, vocab=vocab, k=min(spread(1, 256), vocab), dtype=dtype,
                  temperature=rng.choice((1.0, 1.0, 2.0, 4.0)), padding=rng.choice((0, 0, 16, 3)),
                  masks=rng.random() < 0.4)
    if op == "top":
        return _top(**common)
    return _distill(hard=rng.choice((0.0, 0.1, 0.5)), tail=rng.random() < 0.5, grad=rng.random() < 0.8, **common)


def work(case: dict) -> dict:
    b = BYTES[case["dtype"]]
    if case["op"] == "scan":
        lengths = _lengths(case)
        n, s, d = sum(lengths), len(lengths), case["channels"]
        carried = s * d * 4 * (2 if case["initial"] else 1)           # first state read, last state written
        if not case["train"]:
            return {"bytes": 3 * n * d * b + carried, "flops": 8 * n * d}
        # forward: gate, x -> h; backward: gate, x, dh -> dgate, dx, and the gradients of the states
        return {"bytes": 8 * n * d * b + 2 * carried, "flops": 24 * n * d}
    r, v, k = case["rows"], case["vocab"], case["k"]
    if case["op"] == "top":
        return {"bytes": r * v * b + r * (k * 8 + 4), "flops": 4 * r * v}
    two = 2 if case["hard"] > 0.0 and case["temperature"] != 1.0 else 1
    bytes_ = r * v * b * (2 if case["grad"] else 1) + r * (k * 8 + 8)
    bytes_ += r * 4 * (int(case["hard"] > 0.0) + int(case["tail"]))
    return {"bytes": bytes_, "flops": (8 if case["grad"] else 4) * two * r * v}


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------
def _generator(seed: int, salt: int) -> torch.Generator:
    g = torch.Generator(device=DEVICE)
    g.manual_seed((int(seed) * 1000003 + salt) % (1 << 62))
    return g


def _lengths(case: dict) -> List[int]:
    """The sequences' lengths: all alike, or from one eighth of `length` to all of it, now and then none at all."""
    s, t = case["sequences"], case["length"]
    if not case["packed"]:
        return [t] * s
    rng = random.Random(case["layout_seed"])
    out = [0 if rng.random() < 0.03 else rng.randint(max(1, t // 8), t) for _ in range(s)]
    out[0] = t
    return out


def _logits(case: dict, gen: torch.Generator) -> torch.Tensor:
    """Rows of a model's logits: a bulk of standard deviation 2.5 with a heavier upper tail, in a buffer whose rows are
    `padding` elements further apart than they are long.  With `masks`, some columns of every third row are -inf or
    the type's lowest value, and every 16th row is nothing but -inf."""
    r, v, dt = case["rows"], case["vocab"], DTYPES[case["dtype"]]
    buffer = torch.empty(r, v + case["padding"], dtype=dt, device=DEVICE)
    z = buffer[:, :v]
    step = max(1, (1 << 26) // v)
    for i in range(0, r, step):
        part = torch.randn(min(step, r - i), v, generator=gen, device=DEVICE)
        z[i:i + step] = (2.5 * part + 0.35 * part.clamp_min(0.0) ** 2).to(dt)
    if case["padding"]:
        buffer[:, v:] = float("nan")                                  # nothing there may be read into a result
    if case["masks"]:
        columns = torch.rand(v, generator=gen, device=DEVICE)
        z[0::3, columns < 0.2] = float("-inf")
        z[1::3, columns > 0.6] = torch.finfo(dt).min
        if r >= 16:
            z[15::16] = float("-inf")
    return z


def _inputs(case: dict, seed: int) -> dict:
    gen = _generator(seed, 17)
    if case["op"] == "scan":
        lengths = _lengths(case)
        n, s, d, dt = sum(lengths), len(lengths), case["channels"], DTYPES[case["dtype"]]
        starts = [0]
        for length in lengths:
            starts.append(starts[-1] + length)
        if case["joint"]:
            both = torch.empty(n, 2 * d, dtype=dt, device=DEVICE)
            gate, x = both[:, :d], both[:, d:]
        else:
            gate, x = (torch.empty(n, d, dtype=dt, device=DEVICE) for _ in range(2))
        gate.copy_(torch.randn(n, d, generator=gen, device=DEVICE).mul_(1.5).add_(2.0))
        if case["resets"]:
            gate[torch.rand(n, generator=gen, device=DEVICE) < 1e-3] = float("-inf")
        x.copy_(torch.randn(n, d, generator=gen, device=DEVICE))
        state = dict(gate=gate, x=x, starts=starts, h0=None, dh=None, dh_last=None)
        if case["initial"]:
            state["h0"] = torch.randn(s, d, generator=gen, device=DEVICE) * 0.5
        if case["train"]:
            state["dh"] = torch.randn(n, d, generator=gen, device=DEVICE).mul_(0.1).to(dt)
            if case["initial"]:
                state["dh_last"] = torch.randn(s, d, generator=gen, device=DEVICE) * 0.1
        return state
    state = dict(logits=_logits(case, gen))
    if case["op"] == "distill":
        # the teacher's pairs: distinct indices, values of a model that is close to the student
        r, v, k = case["rows"], case["vocab"], case["k"]
        offset = torch.randint(0, v, (r, 1), generator=gen, device=DEVICE)
        stride = 1
        for p in (7919, 104729, 31, 1):                               # a step that meets no column twice
            if math.gcd(p, v) == 1:
                stride = p
                break
        idx = ((offset + torch.arange(k, device=DEVICE) * stride) % v).to(torch.int32)
        val = torch.randn(r, k, generator=gen, device=DEVICE).mul_(1.5).add_(9.0).sort(dim=1, descending=True).values
        if case["masks"]:
            cut = torch.randint(0, k + 1, (r, 1), generator=gen, device=DEVICE)
            none = (torch.arange(k, device=DEVICE) >= cut) & (torch.arange(r, device=DEVICE)[:, None] % 4 == 1)
            seen = state["logits"].gather(1, idx.long()) > torch.finfo(state["logits"].dtype).min
            none |= ~seen                                             # a teacher masks what its student masks
            idx = torch.where(none, torch.full_like(idx, -1), idx)
            val = torch.where(none, torch.full_like(val, float("-inf")), val)
        state.update(top_idx=idx.contiguous(), top_val=val.contiguous(), top_lse=None, labels=None, row_weight=None)
        if case["tail"]:
            state["top_lse"] = torch.logsumexp(val / case["temperature"], 1) + torch.rand(
                r, generator=gen, device=DEVICE) * 0.5
        if case["hard"] > 0.0:
            labels = torch.randint(0, v, (r,), generator=gen, device=DEVICE, dtype=torch.int32)
            if case["masks"]:
                seen = state["logits"].gather(1, labels.long()[:, None])[:, 0] > torch.finfo(state["logits"].dtype).min
                labels = torch.where(seen, labels, torch.full_like(labels, -1))
            state["labels"] = labels
        # the mean over the rows, times the loss scaling that gradients in 16 bits with 5 bits of exponent are kept with
        state["row_weight"] = torch.full((r,), (4096.0 if case["dtype"] == "f16" else 1.0) / r, device=DEVICE)
        if case["masks"]:
            state["row_weight"][torch.rand(r, generator=gen, device=DEVICE) < 0.1] = 0.0
    return state


def prepare(case: dict, seed: int) -> dict:
    state = _inputs(case, seed)
    state["case"] = case
    if not own:
        return state
    from paper_1712_01887_amd import binding as B
    if case["op"] == "scan":
        s, d, dt = len(state["starts"]) - 1, case["channels"], DTYPES[case["dtype"]]
        n = state["starts"][-1]
        offsets = torch.tensor(state["starts"], dtype=torch.int64, device=DEVICE) if case["packed"] else None
        plan = B.GatedScan(s, case["length"], d, dt, free_input=case["free"], row_offsets=offsets, rows=n)
        state["plan"] = plan
        state["h"] = torch.empty(n, d, dtype=dt, device=DEVICE)
        state["h_last"] = torch.empty(s, d, device=DEVICE)
        state["states"] = plan.alloc_states() if case["train"] else None
        if case["train"]:
            if case["joint"]:
                both = torch.empty(n, 2 * d, dtype=dt, device=DEVICE)
                state["dgate"], state["dx"] = both[:, :d], both[:, d:]
            else:
                state["dgate"], state["dx"] = (torch.empty(n, d, dtype=dt, device=DEVICE) for _ in range(2))
            state["dh0"] = torch.empty(s, d, device=DEVICE) if case["initial"] else None
        return state
    r, k, z = case["rows"], case["k"], state["logits"]
    state["plan"] = B.Distillation(r, case["vocab"], z.dtype)
    if case["op"] == "top":
        state["out"] = state["plan"].alloc_top_logits(k)
    else:
        state["loss"] = torch.empty(r, device=DEVICE)
        state["dlogits"] = torch.empty(r, case["vocab"], dtype=z.dtype, device=DEVICE) if case["grad"] else None
    return state


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------
def run(state: dict):
    case = state["case"]
    if own:
        return _run_own(case, state)
    if case["op"] == "top":
        return _plain_top(case, state["logits"])
    if case["op"] == "distill":
        return _plain_distill(case, state)
    return _plain_scan(case, state)


def _run_own(case: dict, s: dict):
    plan = s["plan"]
    if case["op"] == "top":
        idx, val, lse = s["out"]
        plan.dgc_top_logits(s["logits"], idx, val, lse, temperature=case["temperature"])
        return idx, val, lse
    if case["op"] == "distill":
        plan.dgc_distill_loss(s["logits"], s["top_idx"], s["top_val"], s["loss"], s["dlogits"], top_lse=s["top_lse"],
                              labels=s["labels"], row_weight=s["row_weight"], temperature=case["temperature"],
                              hard_weight=case["hard"])
        return (s["loss"], s["dlogits"]) if case["grad"] else s["loss"]
    plan.dgc_gated_scan_forward(s["gate"], s["x"], s["h0"], s["h"], s["h_last"], s["states"])
    if not case["train"]:
        return s["h"], s["h_last"]
    plan.dgc_gated_scan_backward(s["gate"], s["x"], s["states"], s["dh"], s["dh_last"], s["dgate"], s["dx"], s["dh0"])
    out = [s["h"], s["h_last"], s["dgate"], s["dx"]]
    return out + [s["dh0"]] if case["initial"] else out


# --- plain forms, 32 bits ----------------------------------------------------
def _plain_top(case: dict, logits: torch.Tensor):
    z = logits.float()
    v, k = case["vocab"], case["k"]
    # a whole number for every element that orders by value and then by index, the lowest first
    bits = torch.where(torch.isnan(z), torch.full_like(z, float("-inf")), z + 0.0).view(torch.int32)
    key = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).to(torch.int64) * (1 << 32)
    key = key + ((1 << 32) - 1 - torch.arange(v, device=z.device))
    best = torch.topk(key, k, dim=1).values
    idx = ((1 << 32) - 1 - (best & 0xFFFFFFFF))
    val = z.gather(1, idx)
    taken = val > float("-inf")
    idx = torch.where(taken, idx, torch.full_like(idx, -1)).to(torch.int32)
    val = torch.where(taken, val, torch.full_like(val, float("-inf")))
    zt = z / case["temperature"]
    top = zt.amax(dim=1, keepdim=True)
    low = top == float("-inf")
    shift = torch.where(low, torch.zeros_like(top), top)
    lse = shift + torch.exp(zt - shift).sum(1, keepdim=True).log()
    return idx, val, lse[:, 0]


def _softmax(z: torch.Tensor):
    """Probabilities and log-sum-exp of every row; zeros and zero where a row is nothing but -inf."""
    top = z.amax(dim=1, keepdim=True)
    empty = top == float("-inf")
    top = torch.where(empty, torch.zeros_like(top), top)
    e = torch.exp(z - top)
    total = e.sum(1, keepdim=True)
    total = torch.where(empty, torch.ones_like(total), total)
    return e / total, (top + total.log())[:, 0], empty[:, 0]


def _plain_distill(case: dict, s: dict):
    z = s["logits"].float()
    tau, hard = case["temperature"], case["hard"]
    w = s["row_weight"]
    q, lse, empty = _softmax(z / tau)
    there = s["top_idx"] >= 0
    at = s["top_idx"].clamp_min(0).long()
    t = torch.where(there, s["top_val"] / tau, torch.full_like(s["top_val"], float("-inf")))
    if s["top_lse"] is None:
        p, c, none = _softmax(t)
    else:
        c, none = s["top_lse"], ~there.any(1)
        p = torch.where(there, torch.exp(t - c[:, None]), torch.zeros_like(t))
    log_q = z.gather(1, at) / tau - lse[:, None]
    terms = torch.where(p > 0, p * (t - c[:, None] - log_q), torch.zeros_like(p))
    kl = torch.where(none, torch.zeros_like(lse), terms.sum(1))
    loss = (1.0 - hard) * tau * tau * kl
    grad = None
    if case["grad"]:
        grad = (q * p.sum(1, keepdim=True)).scatter_add_(1, at, -p).mul_((1.0 - hard) * tau)
    del q
    if s["labels"] is not None:
        q1, lse1, _ = _softmax(z)
        known = s["labels"] >= 0
        y = s["labels"].clamp_min(0).long()[:, None]
        ce = torch.where(known, lse1 - z.gather(1, y)[:, 0], torch.zeros_like(lse1))
        loss = loss + hard * ce
        if case["grad"]:
            grad += hard * q1 * known[:, None]
            grad.scatter_add_(1, y, -hard * known[:, None].float())
    live = (w != 0) & ~empty
    loss = torch.where(live, w * loss, torch.zeros_like(loss))
    if not case["grad"]:
        return loss
    grad = torch.where(live[:, None], grad.mul_(w[:, None]), torch.zeros_like(grad))
    return loss, grad.to(s["logits"].dtype)


def _double(a: torch.Tensor, b: torch.Tensor, longest: int) -> torch.Tensor:
    """b_t + a_t (b_{t-1} + a_{t-1} (...)) for every row, by steps of 1, 2, 4, ... rows."""
    step = 1
    while step < longest and step < a.shape[0]:
        b = torch.cat((b[:step], torch.addcmul(b[step:], a[step:], b[:-step])))
        a = torch.cat((a[:step], a[step:] * a[:-step]))
        step *= 2
    return b


def _plain_scan(case: dict, s: dict):
    gate, x = s["gate"].float(), s["x"].float()
    n, d = gate.shape
    starts = s["starts"]
    live = [i for i in range(len(starts) - 1) if starts[i + 1] > starts[i]]
    first = torch.tensor([starts[i] for i in live], device=gate.device)
    last = torch.tensor([starts[i + 1] - 1 for i in live], device=gate.device)
    which = torch.tensor(live, device=gate.device)
    h0 = s["h0"] if s["h0"] is not None else torch.zeros(len(starts) - 1, d, device=gate.device)
    a = torch.sigmoid(gate)
    b = torch.ones_like(gate) if case["free"] else torch.sigmoid(-gate)
    drive = b * x
    drive[first] += a[first] * h0[which]
    carry = a.clone()
    carry[first] = 0.0
    h = _double(carry, drive, case["length"])
    h_last = h0.clone()
    h_last[which] = h[last]
    out_h = h.to(s["gate"].dtype)
    if not case["train"]:
        return out_h, h_last
    before = torch.cat((torch.zeros_like(h[:1]), h[:-1]))
    before[first] = h0[which]
    del h, drive
    dh = s["dh"].float().clone()                                      # a pass leaves its inputs as they are
    d_last = s["dh_last"] if s["dh_last"] is not None else torch.zeros_like(h0)
    dh[last] += d_last[which]
    # the gradient runs the other way: g_t = dh_t + a_{t+1} g_{t+1}
    after = torch.cat((a[1:], torch.zeros_like(a[:1])))
    after[last] = 0.0
    g = _double(after.flip(0), dh.flip(0), case["length"]).flip(0)
    dx = (b * g).to(s["x"].dtype)
    da = g * before if case["free"] else g * (before - x)
    dgate = (da * a * torch.sigmoid(-gate)).to(s["gate"].dtype)
    out = [out_h, h_last, dgate, dx]
    if case["initial"]:
        dh0 = d_last.clone()
        dh0[which] = a[first] * g[first]
        out.append(dh0)
    return out


# --- the definitions, 64 bits -------------------------------------------------
def exact(case: dict, seed: int):
    s = _inputs(case, seed)
    with torch.no_grad():
        if case["op"] == "top":
            return _exact_top(case, s)
        if case["op"] == "distill":
            return _exact_distill(case, s)
        if case["length"] > 70000:
            return None
        return _exact_scan(case, s)


def _pieces(rows: int, columns: int):
    step = max(1, (1 << 26) // columns)
    return [(i, min(rows, i + step)) for i in range(0, rows, step)]


def _exact_top(case: dict, s: dict):
    idx, val, lse = [], [], []
    for lo, hi in _pieces(case["rows"], case["vocab"]):
        z = s["logits"][lo:hi].double()
        order = torch.sort(torch.nan_to_num(z, nan=float("-inf"), posinf=float("inf"), neginf=float("-inf")), dim=1,
                           descending=True, stable=True)
        v, i = order.values[:, :case["k"]].clone(), order.indices[:, :case["k"]].clone()
        i[v == float("-inf")] = -1
        idx.append(i.to(torch.int32))
        val.append(v)
        lse.append(torch.logsumexp(z / case["temperature"], 1))
    return torch.cat(idx), torch.cat(val), torch.cat(lse)


def _exact_distill(case: dict, s: dict):
    tau, hard = case["temperature"], case["hard"]
    losses, grads = [], []
    for lo, hi in _pieces(case["rows"], case["vocab"]):
        z = s["logits"][lo:hi].double()
        dead = (s["row_weight"][lo:hi] == 0) | (z == float("-inf")).all(1)
        z[dead] = 0.0                                                  # such rows count as nothing; see the end
        log_q = torch.log_softmax(z / tau, 1)
        idx, val = s["top_idx"][lo:hi].long(), s["top_val"][lo:hi].double() / tau
        missing = idx < 0
        val = val.masked_fill(missing, float("-inf"))
        if s["top_lse"] is None:
            log_p = val - torch.logsumexp(val, 1, keepdim=True)
        else:
            log_p = val - s["top_lse"][lo:hi].double()[:, None]
        p = torch.where(missing, torch.zeros_like(val), log_p.exp())
        target = torch.zeros_like(z)
        target.scatter_add_(1, idx.clamp_min(0), p)
        entropy = torch.where(p > 0, p * log_p, torch.zeros_like(p)).sum(1)
        cross = torch.where(target > 0, target * log_q, torch.zeros_like(z)).sum(1)
        loss = (1.0 - hard) * tau ** 2 * (entropy - cross)
        grad = (1.0 - hard) * tau * (p.sum(1, keepdim=True) * log_q.exp() - target)
        if s["labels"] is not None:
            y = s["labels"][lo:hi].long()
            log_q1 = torch.log_softmax(z, 1)
            known = (y >= 0).double()
            picked = log_q1.gather(1, y.clamp_min(0)[:, None])[:, 0]
            loss -= hard * torch.where(y >= 0, picked, torch.zeros_like(picked))
            once = torch.zeros_like(z).scatter_(1, y.clamp_min(0)[:, None], 1.0)
            grad += hard * known[:, None] * (log_q1.exp() - once)
        w = s["row_weight"][lo:hi].double().masked_fill(dead, 0.0)
        losses.append(w * loss)
        if case["grad"]:
            grads.append(w[:, None] * grad)
    return (torch.cat(losses), torch.cat(grads)) if case["grad"] else torch.cat(losses)


def _exact_scan(case: dict, s: dict):
    """The recurrence as it is written, one step after the other for all sequences that are long enough."""
    starts = s["starts"]
    count = len(starts) - 1
    n, d = s["gate"].shape
    lengths = [starts[i + 1] - starts[i] for i in range(count)]
    device = s["gate"].device
    order = sorted(range(count), key=lambda i: -lengths[i])
    base = torch.tensor([starts[i] for i in order], device=device)
    which = torch.tensor(order, device=device)
    alive = [0] * (max(lengths) + 1)                                   # sequences longer than t, the longest first
    for t in range(max(lengths)):
        alive[t] = sum(1 for length in lengths if length > t) if t < 1 or alive[t - 1] > 1 else 1
    a = torch.sigmoid(s["gate"].double())
    b = torch.ones_like(a) if case["free"] else torch.sigmoid(-s["gate"].double())
    x = s["x"].double()
    drive = b * x
    state = torch.zeros(count, d, dtype=torch.float64, device=device)
    if s["h0"] is not None:
        state = s["h0"].double()[which]
    h = torch.empty(n, d, dtype=torch.float64, device=device)
    before = torch.empty_like(h) if case["train"] else None
    for t in range(max(lengths)):
        m = alive[t]
        rows = base[:m] + t
        if case["train"]:
            before[rows] = state[:m]
        state[:m] = a[rows] * state[:m] + drive[rows]
        h[rows] = state[:m]
    h_last = torch.empty_like(state)
    h_last[which] = state
    if not case["train"]:
        return h, h_last
    flow = torch.zeros(count, d, dtype=torch.float64, device=device)
    if s["dh_last"] is not None:
        flow = s["dh_last"].double()[which]
    dh = s["dh"].double()
    g = torch.empty_like(h)
    for t in reversed(range(max(lengths))):
        m = alive[t]
        rows = base[:m] + t
        step = dh[rows] + flow[:m]
        g[rows] = step
        flow[:m] = a[rows] * step
    dx = b * g
    dgate = g * (before if case["free"] else before - x) * a * torch.sigmoid(-s["gate"].double())
    out = [h, h_last, dgate, dx]
    if case["initial"]:
        dh0 = torch.empty_like(flow)
        dh0[which] = flow
        out.append(dh0)
    return out
