"""The operators of a recurrent language model with matrix states, as cases to measure.

A case is one pass through one operator:

  rotary     heads of queries and keys turned by their rows' positions, whole or in part, neighbouring elements or halves
             as pairs, frequencies as they are or scaled for long contexts; the gradient is the turn back
             (`Rotary.dgc_rotary`)
  attention  linear attention with a decay for each head, S_t = d S_{t-1} + k_t v_t^T, o_t = scale q_t^T S_t, over
             sequences of equal or of different lengths laid behind each other: forward alone, or forward and backward
             (`LinearAttention.dgc_linear_attention_forward`, `LinearAttention.dgc_linear_attention_backward`)
  loss       softmax cross entropy of the output layer, from its inputs and its matrix, without logits in memory: the loss
             and the rows' log-sum-exp alone, or the gradients of both too (`VocabularyLoss.dgc_vocab_loss_forward`,
             `VocabularyLoss.dgc_vocab_loss_backward`)

Where `own` is false, `run` computes the same from elementary torch operations in 32 bits (the angles in 64); `exact` in
64 bits.
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
def _rotary(**kw) -> dict:
    return dict(dict(op="rotary", rows=1, heads=1, key_heads=1, head_dim=64, rotary_dim=64, half=False, dtype="f32",
                     base=10000.0, factor=1.0, context=0, magnitude=1.0, far=0, scattered=False, joint=False,
                     inverse=False), **kw)


def _attention(**kw) -> dict:
    return dict(dict(op="attention", sequences=1, length=1, heads=1, key_dim=64, value_dim=64, dtype="f32", train=False,
                     packed=False, joint=False, initial=True, layout_seed=0), **kw)


def _loss(**kw) -> dict:
    return dict(dict(op="loss", rows=1, vocab=1, width=1, dtype="f32", train=True, masks=False, padding=0), **kw)


def listed() -> List[dict]:
    return [
        # one token for each of 64 streams that are far into their texts: latency
        _rotary(name="rotary_step", rows=64, heads=16, key_heads=16, head_dim=64, rotary_dim=64, half=True, dtype="bf16",
                far=1 << 20, scattered=True),
        # queries and keys of one projection, sequences of 512 steps, heads of 75 of which 50 are turned
        _rotary(name="rotary_odd", rows=10240, heads=20, key_heads=20, head_dim=75, rotary_dim=50, dtype="f16",
                joint=True),
        # a long document, context scaled by parts, the gradient's turn back
        _rotary(name="rotary_long", rows=65536, heads=16, key_heads=16, head_dim=128, rotary_dim=128, half=True,
                dtype="bf16", base=10000.0, factor=8.0, context=8192, magnitude=1.2, inverse=True),
        # one token for each of 64 streams: states in 32 bits read and written
        _attention(name="attention_step", sequences=64, length=1, heads=16, key_dim=64, value_dim=128, dtype="bf16"),
        # a training step of 20 sequences of 350 steps in 32 bits
        _attention(name="attention_lm", sequences=20, length=350, heads=12, key_dim=64, value_dim=64, dtype="f32",
                   train=True, initial=False),
        # prompts of very different lengths behind each other, 1200 channels as 12 heads of 100, one projection
        _attention(name="attention_packed", sequences=48, length=1500, heads=12, key_dim=50, value_dim=100, dtype="f16",
                   packed=True, joint=True, initial=False),
        # one long document, training
        _attention(name="attention_long", sequences=1, length=65536, heads=16, key_dim=128, value_dim=128, dtype="bf16",
                   train=True, joint=True),
        # one time step of the language model's batch, loss and gradients
        _loss(name="loss_small", rows=20, vocab=10000, width=1500, dtype="bf16"),
        # a batch of 20 x 35 tokens of the LSTM language model, in 32 bits
        _loss(name="loss_lm", rows=700, vocab=10000, width=1500, dtype="f32"),
        # validation over an odd vocabulary: the loss alone, some rows without a label
        _loss(name="loss_eval", rows=1111, vocab=50001, width=1200, dtype="f16", train=False, masks=True, padding=8),
        # the training step of a large vocabulary
        _loss(name="loss_large", rows=4096, vocab=131072, width=2048, dtype="bf16", masks=True),
    ]


def draw(rng) -> dict:
    """One more case of the ranges above: up to 65536 rows of up to 32 heads; sequences of 1 to 65536 steps, heads of 8 to
    256; vocabularies of 29 to 131072 for up to 4096 rows of 32 to 4096; odd sizes among them."""
    def spread(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    def dim(lo, hi):
        n = spread(lo, hi)
        return min(hi, (n + 7) // 8 * 8) if rng.random() < 0.6 else n

    dtype = rng.choice(("f32", "f16", "bf16", "bf16"))
    op = rng.choice(("rotary", "attention", "attention", "loss", "loss"))
    if op == "rotary":
        head_dim = max(2, dim(8, 256))
        rotary_dim = head_dim // 2 * 2 if rng.random() < 0.6 else 2 * rng.randint(1, head_dim // 2)
        heads = spread(1, 32)
        rows = max(1, min(spread(1, 65536), (1 << 26) // (heads * head_dim)))
        scaled = rng.random() < 0.4
        return _rotary(rows=rows, heads=heads, key_heads=rng.choice((heads, max(1, heads // 4))), head_dim=head_dim,
                       rotary_dim=rotary_dim, half=rng.random() < 0.5, dtype=dtype,
                       base=rng.choice((10000.0, 500000.0)), factor=rng.choice((2.0, 8.0)) if scaled else 1.0,
                       context=rng.choice((0, 4096, 8192)) if scaled else 0, magnitude=rng.choice((1.0, 1.2)),
                       far=rng.choice((0, spread(1, 1 << 20))), scattered=rng.random() < 0.3, joint=rng.random() < 0.5,
                       inverse=rng.random() < 0.4)
    if op == "attention":
        key_dim, value_dim = dim(8, 256), dim(8, 256)
        heads = spread(1, 32)
        length = spread(1, 65536)
        most = (1 << (26 if dtype == "bf16" else 25)) // (length * heads * max(key_dim, value_dim))
        sequences = max(1, min(spread(1, 256), most))
        return _attention(sequences=sequences, length=max(1, min(length, length * max(1, most))) if most else max(
                              1, (1 << 25) // (heads * max(key_dim, value_dim))), heads=heads, key_dim=key_dim,
                          value_dim=value_dim, dtype=dtype, train=rng.random() < 0.5, packed=rng.random() < 0.5,
                          joint=rng.random() < 0.5, initial=rng.random() < 0.6, layout_seed=rng.randrange(1 << 20))
    vocab, width = spread(29, 131072), dim(32, 4096)
    most = (1 << (39 if dtype == "bf16" else 37)) // (vocab * width)
    return _loss(rows=max(1, min(spread(1, 4096), most)), vocab=vocab, width=width, dtype=dtype,
                 train=rng.random() < 0.6, masks=rng.random() < 0.4, padding=rng.choice((0, 0, 8, 3)))


def work(case: dict) -> dict:
    b = BYTES[case["dtype"]]
    if case["op"] == "rotary":
        n = case["rows"] * (case["heads"] + case["key_heads"])
        # a turned element: two products and a sum
        return {"bytes": 2 * n * case["head_dim"] * b + 8 * case["rows"], "flops": 3 * n * case["rotary_dim"]}
    if case["op"] == "attention":
        lengths = _lengths(case)
        n, s, h, dk, dv = sum(lengths), len(lengths), case["heads"], case["key_dim"], case["value_dim"]
        states = s * h * dk * dv * 4 * (2 if case["initial"] else 1)   # first state read, last state written
        forward = n * h * (2 * dk + 2 * dv) * b + states
        if not case["train"]:
            return {"bytes": forward, "flops": 4 * n * h * dk * dv}
        # backward: q, k, v, do -> dq, dk, dv, and the gradients of the states
        return {"bytes": forward + n * h * (4 * dk + 3 * dv) * b + states, "flops": 14 * n * h * dk * dv}
    r, v, d = case["rows"], case["vocab"], case["width"]
    forward = (r * d + v * d) * b + 16 * r
    if not case["train"]:
        return {"bytes": forward, "flops": 2 * r * v * d}
    # logits once, and a product of the same size for either gradient
    return {"bytes": 3 * (r * d + v * d) * b + 28 * r, "flops": 6 * r * v * d}


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


def _normal(gen, *shape) -> torch.Tensor:
    return torch.randn(*shape, generator=gen, device=DEVICE)


def _inputs(case: dict, seed: int) -> dict:
    gen = _generator(seed, 29)
    dt = DTYPES[case["dtype"]]
    if case["op"] == "rotary":
        r, h, kh, d = case["rows"], case["heads"], case["key_heads"], case["head_dim"]
        if case["joint"]:                                              # q | k | v of one projection
            both = _normal(gen, r, h + 2 * kh, d).to(dt)
            q, k = both[:, :h], both[:, h:h + kh]
        else:
            q, k = _normal(gen, r, h, d).to(dt), _normal(gen, r, kh, d).to(dt)
        if case["scattered"]:
            positions = torch.randint(0, case["far"] + r, (r,), generator=gen, device=DEVICE)
        else:
            start = int(torch.randint(0, case["far"] + 1, (1,), generator=gen, device=DEVICE)) if case["far"] else 0
            positions = torch.arange(start, start + r, device=DEVICE)
        return dict(q=q, k=k, positions=positions)
    if case["op"] == "attention":
        lengths = _lengths(case)
        n, s, h, dk, dv = sum(lengths), len(lengths), case["heads"], case["key_dim"], case["value_dim"]
        starts = [0]
        for length in lengths:
            starts.append(starts[-1] + length)
        if case["joint"]:
            whole = torch.empty(n, h * (2 * dk + dv), dtype=dt, device=DEVICE)
            q, k, v = (x.view(n, h, -1) for x in whole.split((h * dk, h * dk, h * dv), dim=1))
        else:
            q, k = (torch.empty(n, h, dk, dtype=dt, device=DEVICE) for _ in range(2))
            v = torch.empty(n, h, dv, dtype=dt, device=DEVICE)
        q.copy_(_normal(gen, n, h, dk))
        k.copy_(_normal(gen, n, h, dk).mul_(dk ** -0.5))
        v.copy_(_normal(gen, n, h, dv))
        # heads that remember some 16 to some 2000 steps
        log_decay = torch.log1p(-torch.exp2(-4.0 - 7.0 * torch.arange(h, device=DEVICE) / h))
        state = dict(q=q, k=k, v=v, starts=starts, lengths=lengths, log_decay=log_decay, scale=dk ** -0.5, state0=None,
                     do=None, dstate_last=None)
        if case["initial"]:
            state["state0"] = _normal(gen, s, h, dk, dv).mul_(0.5)
        if case["train"]:
            state["do"] = _normal(gen, n, h, dv).to(dt)
            if case["initial"]:
                state["dstate_last"] = _normal(gen, s, h, dk, dv).mul_(0.1)
        return state
    r, v, d, pad = case["rows"], case["vocab"], case["width"], case["padding"]
    hidden = torch.empty(r, d + pad, dtype=dt, device=DEVICE)
    if pad:
        hidden[:, d:] = float("nan")                                   # nothing there may be read into a result
    hidden = hidden[:, :d]
    hidden.copy_(_normal(gen, r, d))
    weight = _normal(gen, v, d).mul_(2.0 * d ** -0.5).to(dt)           # logits of standard deviation 2
    labels = torch.randint(0, v, (r,), generator=gen, device=DEVICE, dtype=torch.int32)
    # the mean over the rows, times the loss scaling that gradients in 16 bits with 5 bits of exponent are kept with
    row_weight = torch.full((r,), (4096.0 if case["dtype"] == "f16" else 1.0) / r, device=DEVICE)
    if case["masks"]:
        labels[torch.rand(r, generator=gen, device=DEVICE) < 0.1] = -1
        row_weight[torch.rand(r, generator=gen, device=DEVICE) < 0.1] = 0.0
    return dict(hidden=hidden, weight=weight, labels=labels, row_weight=row_weight)


def prepare(case: dict, seed: int) -> dict:
    state = _inputs(case, seed)
    state["case"] = case
    if not own:
        return state
    from paper_1712_01887_amd import binding as B
    dt = DTYPES[case["dtype"]]
    if case["op"] == "rotary":
        state["plan"] = B.Rotary(case["head_dim"], dt, rotary_dim=case["rotary_dim"], base=case["base"],
                                 half=case["half"], factor=case["factor"], context=case["context"],
                                 magnitude=case["magnitude"])
        state["out"] = [torch.empty(x.shape, dtype=dt, device=DEVICE) for x in (state["q"], state["k"])]
    elif case["op"] == "attention":
        n, s = sum(state["lengths"]), len(state["lengths"])
        h, dk, dv = case["heads"], case["key_dim"], case["value_dim"]
        offsets = torch.tensor(state["starts"], dtype=torch.int64, device=DEVICE) if case["packed"] else None
        state["plan"] = B.LinearAttention(s, case["length"], h, dk, dv, dt, scale=state["scale"], row_offsets=offsets,
                                          rows=n)
        state["o"] = torch.empty(n, h, dv, dtype=dt, device=DEVICE)
        state["state_last"] = torch.empty(s, h, dk, dv, device=DEVICE)
        if case["train"]:
            if case["joint"]:
                whole = torch.empty(n, h * (2 * dk + dv), dtype=dt, device=DEVICE)
                state["grads"] = [x.view(n, h, -1) for x in whole.split((h * dk, h * dk, h * dv), dim=1)]
            else:
                state["grads"] = [torch.empty(n, h, d, dtype=dt, device=DEVICE) for d in (dk, dk, dv)]
            state["dstate0"] = torch.empty(s, h, dk, dv, device=DEVICE) if case["initial"] else None
    else:
        r, v, d = case["rows"], case["vocab"], case["width"]
        state["plan"] = B.VocabularyLoss(r, v, d, dt)
        state["loss"], state["lse"] = torch.empty(r, device=DEVICE), torch.empty(r, device=DEVICE)
        if case["train"]:
            state["dhidden"] = torch.empty(r, d, dtype=dt, device=DEVICE)
            state["dweight"] = torch.empty(v, d, dtype=dt, device=DEVICE)
    return state


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------
def run(state: dict):
    case = state["case"]
    if own:
        return _run_own(case, state)
    if case["op"] == "rotary":
        return _plain_rotary(case, state)
    if case["op"] == "attention":
        return _plain_attention(case, state)
    return _plain_loss(case, state)


def _run_own(case: dict, s: dict):
    plan = s["plan"]
    if case["op"] == "rotary":
        plan.dgc_rotary(s["positions"], [s["q"], s["k"]], s["out"], inverse=case["inverse"])
        return s["out"]
    if case["op"] == "attention":
        plan.dgc_linear_attention_forward(s["q"], s["k"], s["v"], s["log_decay"], s["state0"], s["o"], s["state_last"])
        if not case["train"]:
            return s["o"], s["state_last"]
        dq, dk, dv = s["grads"]
        plan.dgc_linear_attention_backward(s["q"], s["k"], s["v"], s["log_decay"], s["state0"], s["do"],
                                           s["dstate_last"], dq, dk, dv, s["dstate0"])
        out = [s["o"], s["state_last"], dq, dk, dv]
        return out + [s["dstate0"]] if case["initial"] else out
    plan.dgc_vocab_loss_forward(s["hidden"], s["weight"], s["labels"], s["loss"], s["lse"], row_weight=s["row_weight"])
    if not case["train"]:
        return s["loss"], s["lse"]
    plan.dgc_vocab_loss_backward(s["hidden"], s["weight"], s["labels"], s["lse"], s["dhidden"], s["dweight"],
                                 row_weight=s["row_weight"])
    return s["loss"], s["lse"], s["dhidden"], s["dweight"]


# --- plain forms, 32 bits ----------------------------------------------------
LOW_TURNS, HIGH_TURNS = 1.0, 32.0


def _frequencies(case: dict) -> torch.Tensor:
    """Radians a position, 64 bits: frequencies that turn often in the original context stay, slow ones are divided."""
    i = torch.arange(case["rotary_dim"] // 2, dtype=torch.float64, device=DEVICE)
    f = case["base"] ** (-2.0 * i / case["rotary_dim"])
    turns = f * case["context"] / (2.0 * math.pi)
    kept = ((turns - LOW_TURNS) / (HIGH_TURNS - LOW_TURNS)).clamp(0.0, 1.0)
    return (1.0 - kept) * f / case["factor"] + kept * f


def _plain_rotary(case: dict, s: dict):
    n = case["rotary_dim"]
    angle = s["positions"].double()[:, None] * _frequencies(case)
    if case["inverse"]:
        angle = -angle
    cos = (torch.cos(angle).float() * case["magnitude"])[:, None]
    sin = (torch.sin(angle).float() * case["magnitude"])[:, None]
    out = []
    for x in (s["q"], s["k"]):
        y = x.clone(memory_format=torch.contiguous_format)
        if case["half"]:
            first, second, to = x[..., :n // 2].float(), x[..., n // 2:n].float(), (y[..., :n // 2], y[..., n // 2:n])
        else:
            first, second, to = x[..., 0:n:2].float(), x[..., 1:n:2].float(), (y[..., 0:n:2], y[..., 1:n:2])
        to[0].copy_(first * cos - second * sin)
        to[1].copy_(first * sin + second * cos)
        out.append(y)
    return out


CHUNK = 128


def _padded(x: torch.Tensor, rows: torch.Tensor) -> torch.Tensor:
    """x's rows as [sequences, heads, chunks, CHUNK, dim] in 32 bits; zeros where `rows` names none."""
    x = torch.cat((x, torch.zeros_like(x[:1]))) if x.shape[0] else x.new_zeros(1, *x.shape[1:])
    x = x[rows].float()                                                # [sequences, steps, heads, dim]
    return x.permute(0, 2, 1, 3).reshape(x.shape[0], x.shape[2], -1, CHUNK, x.shape[3])


def _decayed(a, b, c, log_decay, first, out_scale, scale):
    """out_t = out_scale (sum over s <= t of d^(t-s) scale (a_t . b_s) c_s + d^(t+1) a_t . first), chunk by chunk."""
    heads, chunks = a.shape[1], a.shape[2]
    i = torch.arange(CHUNK, device=a.device)
    rate = log_decay[:, None, None]
    apart = (i[:, None] - i).float()
    inside = torch.where(apart >= 0, torch.exp(rate * apart.clamp_min(0.0)), torch.zeros_like(rate)) * scale
    out = (a @ b.transpose(-1, -2) * inside[None, :, None]) @ c
    left = torch.exp(log_decay[:, None] * (CHUNK - 1 - i).float()) * scale
    added = (b * left[None, :, None, :, None]).transpose(-1, -2) @ c  # what a chunk adds to the state
    j = torch.arange(chunks, device=a.device)
    apart = (j[:, None] - j - 1).float()
    between = torch.where(apart >= 0, torch.exp(rate * CHUNK * apart.clamp_min(0.0)), torch.zeros_like(rate))
    before = (between[None] @ added.flatten(3)).view(added.shape)      # the state in front of every chunk
    if first is not None:
        before = before + torch.exp(rate * CHUNK * j.float())[..., None].transpose(1, 2).view(
            1, heads, chunks, 1, 1) * first[:, :, None]
    out = out + (a @ before) * torch.exp(log_decay[:, None] * (i + 1).float())[None, :, None, :, None]
    return out * out_scale


def _last(b, c, log_decay, first, lengths, scale):
    """The state behind the last step of every sequence."""
    t = torch.arange(b.shape[2] * CHUNK, device=b.device)
    after = (lengths[:, None] - 1 - t).clamp_min(0).float()
    left = torch.exp(log_decay[None, :, None] * after[:, None]) * scale
    state = (b.flatten(2, 3) * left[..., None]).transpose(-1, -2) @ c.flatten(2, 3)
    if first is not None:
        state = state + torch.exp(log_decay * lengths[:, None].float())[..., None, None] * first
    return state


def _plain_attention(case: dict, s: dict):
    q, k, v, rate, scale = s["q"], s["k"], s["v"], s["log_decay"], s["scale"]
    n = q.shape[0]
    lengths = torch.tensor(s["lengths"], device=q.device)
    starts = torch.tensor(s["starts"][:-1], device=q.device)
    steps = (case["length"] + CHUNK - 1) // CHUNK * CHUNK
    t = torch.arange(steps, device=q.device)
    there = t < lengths[:, None]
    rows = torch.where(there, starts[:, None] + t, torch.full_like(there, n, dtype=torch.int64))
    back = torch.where(there, starts[:, None] + lengths[:, None] - 1 - t, torch.full_like(rows, n))

    def unpadded(x, at):
        x = x.flatten(2, 3).transpose(1, 2)                            # [sequences, steps, heads, dim]
        out = torch.empty(n, x.shape[2], x.shape[3], dtype=q.dtype, device=q.device)
        out[at[there]] = x[there].to(q.dtype)
        return out

    pq, pk, pv = _padded(q, rows), _padded(k, rows), _padded(v, rows)
    o = unpadded(_decayed(pq, pk, pv, rate, s["state0"], scale, 1.0), rows)
    state_last = _last(pk, pv, rate, s["state0"], lengths, 1.0)
    if not case["train"]:
        return o, state_last
    turned = None if s["state0"] is None else s["state0"].transpose(-1, -2).contiguous()
    dq = unpadded(_decayed(_padded(s["do"], rows), pv, pk, rate, turned, scale, 1.0), rows)
    pq, pk, pv, pdo = (_padded(x, back) for x in (q, k, v, s["do"]))
    # behind the last step the state's own gradient comes in without a decay
    flow = s["dstate_last"]
    if flow is not None:
        flow = flow * torch.exp(-rate)[None, :, None, None]
    turned = None if flow is None else flow.transpose(-1, -2).contiguous()
    dk = unpadded(_decayed(pv, pdo, pq, rate, turned, 1.0, scale), back)
    dv = unpadded(_decayed(pk, pq, pdo, rate, flow, 1.0, scale), back)
    out = [o, state_last, dq, dk, dv]
    if case["initial"]:
        out.append(_last(pq, pdo, rate, s["dstate_last"], lengths, scale * torch.exp(rate)[None, :, None]))
    return out


def _plain_loss(case: dict, s: dict):
    hidden, weight, labels, w = s["hidden"].float(), s["weight"].float(), s["labels"], s["row_weight"]
    z = hidden @ weight.t()
    top = z.amax(dim=1, keepdim=True)
    lse = top[:, 0] + torch.exp(z - top).sum(1).log()
    known = labels >= 0
    y = labels.clamp_min(0).long()[:, None]
    live = torch.where(known, w, torch.zeros_like(w))
    loss = live * (lse - z.gather(1, y)[:, 0])
    if not case["train"]:
        return loss, lse
    p = z.sub_(lse[:, None]).exp_()
    p.scatter_add_(1, y, torch.full_like(w, -1.0)[:, None])
    p.mul_(live[:, None])
    return loss, lse, (p @ weight).to(s["hidden"].dtype), (p.t() @ hidden).to(s["weight"].dtype)


# --- the definitions, 64 bits -------------------------------------------------
def exact(case: dict, seed: int):
    s = _inputs(case, seed)
    with torch.no_grad():
        if case["op"] == "rotary":
            return _exact_rotary(case, s)
        if case["op"] == "attention":
            return _exact_attention(case, s)
        return _exact_loss(case, s)


def _exact_rotary(case: dict, s: dict):
    n, out = case["rotary_dim"], []
    angles = []
    for i in range(n // 2):
        f = math.exp(-2.0 * i / n * math.log(case["base"]))
        turns = case["context"] * f / math.tau
        share = min(1.0, max(0.0, (turns - LOW_TURNS) / (HIGH_TURNS - LOW_TURNS)))
        angles.append(f * (share + (1.0 - share) / case["factor"]))
    angle = s["positions"].double()[:, None] * torch.tensor(angles, dtype=torch.float64, device=DEVICE)
    turn = torch.polar(torch.full_like(angle, case["magnitude"]), -angle if case["inverse"] else angle)[:, None]
    for x in (s["q"], s["k"]):
        y = x.double()
        z = y[..., :n].unflatten(-1, (2, n // 2)).transpose(-1, -2) if case["half"] else y[..., :n].unflatten(-1, (n // 2, 2))
        z = torch.view_as_real(torch.view_as_complex(z.contiguous()) * turn)
        z = z.transpose(-1, -2) if case["half"] else z
        out.append(torch.cat((z.flatten(-2), y[..., n:]), -1))
    return out


def _exact_attention(case: dict, s: dict):
    """The recurrence as it is written, one step after the other for all sequences that are long enough."""
    lengths, starts, scale = s["lengths"], s["starts"], s["scale"]
    count, n = len(lengths), s["q"].shape[0]
    h, dk, dv = case["heads"], case["key_dim"], case["value_dim"]
    order = sorted(range(count), key=lambda i: -lengths[i])            # the longest first
    base = torch.tensor([starts[i] for i in order], device=DEVICE)
    which = torch.tensor(order, device=DEVICE)
    longest = max(lengths)
    alive = [sum(1 for length in lengths if length > t) if count > 1 else 1 for t in range(longest)]
    d = torch.exp(s["log_decay"].double())[:, None, None]
    # a step's columns and rows, so that a step is products of matrices alone
    q, k, v = s["q"].double()[:, :, None], s["k"].double()[..., None], s["v"].double()[:, :, None]
    state = torch.zeros(count, h, dk, dv, dtype=torch.float64, device=DEVICE)
    if s["state0"] is not None:
        state = s["state0"].double()[which]
    o = torch.empty(n, h, 1, dv, dtype=torch.float64, device=DEVICE)
    if case["train"]:
        do = s["do"].double()[:, :, None]
        dq = torch.empty(n, h, dk, 1, dtype=torch.float64, device=DEVICE)
    for t in range(longest):
        now = state[:alive[t]]
        rows = base[:alive[t]] + t if count > 1 else slice(starts[0] + t, starts[0] + t + 1)
        now.mul_(d).add_(k[rows] * v[rows])
        o[rows] = q[rows] @ now
        if case["train"]:
            dq[rows] = now @ do[rows].transpose(-1, -2)
    state_last = torch.empty_like(state)
    state_last[which] = state
    o = o[:, :, 0] * scale
    if not case["train"]:
        return o, state_last
    flow = torch.zeros_like(state)
    if s["dstate_last"] is not None:
        flow = s["dstate_last"].double()[which]
    dk_, dv_ = torch.empty_like(dq), torch.empty_like(o[:, :, None])
    qs = q.transpose(-1, -2) * scale
    for t in reversed(range(longest)):
        now = flow[:alive[t]]
        rows = base[:alive[t]] + t if count > 1 else slice(starts[0] + t, starts[0] + t + 1)
        now.add_(qs[rows] * do[rows])
        dk_[rows] = now @ v[rows].transpose(-1, -2)
        dv_[rows] = k[rows].transpose(-1, -2) @ now
        now.mul_(d)
    out = [o, state_last, dq[..., 0] * scale, dk_[..., 0], dv_[:, :, 0]]
    if case["initial"]:
        dstate0 = torch.empty_like(flow)
        dstate0[which] = flow
        out.append(dstate0)
    return out


def _exact_loss(case: dict, s: dict):
    hidden, weight = s["hidden"].double(), s["weight"].double()
    w = torch.where(s["labels"] < 0, torch.zeros_like(s["row_weight"]), s["row_weight"]).double()
    y = s["labels"].clamp_min(0).long()
    losses, sums, dhidden = [], [], []
    dweight = torch.zeros_like(weight) if case["train"] else None
    step = max(1, (1 << 27) // case["vocab"])
    for i in range(0, case["rows"], step):
        part = slice(i, min(case["rows"], i + step))
        z = hidden[part] @ weight.t()
        sums.append(torch.logsumexp(z, 1))
        log_p = torch.log_softmax(z, 1)
        losses.append(-w[part] * log_p.gather(1, y[part, None])[:, 0])
        if case["train"]:
            g = log_p.exp_()
            g[torch.arange(g.shape[0], device=DEVICE), y[part]] -= 1.0
            g *= w[part, None]
            dhidden.append(g @ weight)
            dweight += g.t() @ hidden[part]
    out = [torch.cat(losses), torch.cat(sums)]
    return out + [torch.cat(dhidden), dweight] if case["train"] else out
