"""A language model with matrix states: trained on workers whose gradients are compressed, then asked for tokens.

    python examples/attention_lm.py [--steps 40] [--workers 4] [--density 0.05]

    x = embed[tokens],  q | k | v = x W_in          heads of one projection
    q, k turned by their positions                  Rotary.dgc_rotary
    o = linear attention, a decay for each head     LinearAttention.dgc_linear_attention_forward
    loss of x + o W_o against the next tokens       VocabularyLoss.dgc_vocab_loss_forward, no logits in memory

and back: VocabularyLoss.dgc_vocab_loss_backward, dgc_linear_attention_backward, dgc_rotary(inverse=True), into a flat
gradient for dgc_compress; one dgc_sparse_sgd_apply_regions of all workers' payloads steps the parameters.  For generating,
a prompt goes through in one call and every further token in a call of one step, the states in one array; the next token is
the largest of the logits (Distillation.dgc_top_logits).  The workers share one GPU here, one after the other, as
`num_workers` handles; the token streams are synthetic (a Markov chain)."""

from __future__ import annotations

import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch  # noqa: E402

from paper_1712_01887_amd import binding as B  # noqa: E402


class Model:
    """Parameters as views of one flat float32 tensor, in the order of their names.  The output layer is vocab x width."""

    def __init__(self, vocab: int, width: int, heads: int, seed: int):
        self.vocab, self.width, self.heads, self.dim = vocab, width, heads, width // heads
        self.shapes = {"embed": (vocab, width), "w_in": (width, 3 * width), "w_o": (width, width), "w_out": (vocab, width)}
        self.offsets = [0]
        for rows, columns in self.shapes.values():
            self.offsets.append(self.offsets[-1] + rows * columns)
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.theta = torch.empty(self.offsets[-1], device="cuda")
        for name in self.shapes:
            p = self.of(self.theta, name)
            p.copy_(torch.randn(p.shape, generator=gen, device="cuda") * (1.0 if name == "embed" else width ** -0.5))
        # heads that remember some 8 to some 500 steps
        self.log_decay = torch.log1p(-torch.exp2(-3.0 - 6.0 * torch.arange(heads, device="cuda") / heads))

    def of(self, flat: torch.Tensor, name: str) -> torch.Tensor:
        i = list(self.shapes).index(name)
        return flat[self.offsets[i]:self.offsets[i + 1]].view(self.shapes[name])


class Pass:
    """The buffers of a model's pass over `sequences` x `length` tokens, 16-bit activations."""

    def __init__(self, model: Model, sequences: int, length: int, train: bool = True):
        n, m, bf = sequences * length, model, torch.bfloat16
        self.model, self.n, self.sequences, self.length = model, n, sequences, length
        self.rotary = B.Rotary(m.dim, bf, half=True)
        self.attention = B.LinearAttention(sequences, length, m.heads, m.dim, m.dim, bf, scale=m.dim ** -0.5, backward=train)
        self.o = torch.empty(n, m.heads, m.dim, dtype=bf, device="cuda")
        self.state = torch.zeros(sequences, m.heads, m.dim, m.dim, device="cuda")
        if train:
            self.loss_plan = B.VocabularyLoss(n, m.vocab, m.width, bf)
            self.loss, self.lse = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
            self.d_projected = torch.empty(n, 3 * m.width, dtype=bf, device="cuda")
            self.d_hidden = torch.empty(n, m.width, dtype=bf, device="cuda")
            self.d_out = torch.empty(m.vocab, m.width, dtype=bf, device="cuda")

    def heads_of(self, projected: torch.Tensor):
        m = self.model
        return [x.view(self.n, m.heads, m.dim) for x in projected.split(m.width, dim=1)]

    def forward(self, tokens: torch.Tensor, first_position: int = 0, carry: bool = False) -> torch.Tensor:
        """The output layer's inputs; `carry`: the sequences go on from the states that the last call left."""
        m, bf = self.model, torch.bfloat16
        self.tokens, self.w = tokens, {name: m.of(m.theta, name).to(bf) for name in m.shapes}
        self.positions = (torch.arange(self.length, device="cuda") + first_position).repeat(self.sequences)
        self.x = self.w["embed"][tokens]
        self.projected = self.x @ self.w["w_in"]
        q, k, v = self.heads_of(self.projected)
        self.rotary.dgc_rotary(self.positions, [q, k], [q, k])
        state = self.state if carry else None
        self.attention.dgc_linear_attention_forward(q, k, v, m.log_decay, state, self.o, self.state)
        self.hidden = self.x + self.o.view(self.n, m.width) @ self.w["w_o"]
        return self.hidden

    def losses(self, labels: torch.Tensor, row_weight=None) -> torch.Tensor:
        self.labels, self.row_weight = labels, row_weight
        self.loss_plan.dgc_vocab_loss_forward(self.hidden, self.w["w_out"], labels, self.loss, self.lse, row_weight=row_weight)
        return self.loss

    def backward(self, grad: torch.Tensor) -> None:
        """Into the flat gradient `grad`."""
        m = self.model
        self.loss_plan.dgc_vocab_loss_backward(self.hidden, self.w["w_out"], self.labels, self.lse, self.d_hidden, self.d_out,
                                               row_weight=self.row_weight)
        m.of(grad, "w_out").copy_(self.d_out)
        do = (self.d_hidden @ self.w["w_o"].t().contiguous()).view(self.n, m.heads, m.dim)
        m.of(grad, "w_o").copy_(self.o.view(self.n, m.width).t().contiguous() @ self.d_hidden)
        q, k, v = self.heads_of(self.projected)
        dq, dk, dv = self.heads_of(self.d_projected)
        self.attention.dgc_linear_attention_backward(q, k, v, m.log_decay, None, do, None, dq, dk, dv)
        self.rotary.dgc_rotary(self.positions, [dq, dk], [dq, dk], inverse=True)
        m.of(grad, "w_in").copy_(self.x.t().contiguous() @ self.d_projected)
        dx = self.d_hidden.float() + (self.d_projected @ self.w["w_in"].t().contiguous()).float()
        m.of(grad, "embed").zero_().index_add_(0, self.tokens, dx)


def generate(model: Model, prompt: torch.Tensor, count: int) -> torch.Tensor:
    """`count` most likely tokens behind every row of `prompt`, [sequences, length]."""
    sequences, length = prompt.shape
    top = B.Distillation(sequences, model.vocab, torch.bfloat16)
    idx, val, _ = top.alloc_top_logits(1)
    run, step = Pass(model, sequences, length, train=False), Pass(model, sequences, 1, train=False)
    step.state = run.state
    hidden = run.forward(prompt.reshape(-1)).view(sequences, length, -1)[:, -1].contiguous()
    out = []
    for i in range(count):
        top.dgc_top_logits(hidden @ run.w["w_out"].t().contiguous(), idx, val)
        out.append(idx[:, 0].long())
        hidden = step.forward(out[-1], first_position=length + i, carry=True)
    return torch.stack(out, 1)


def train(steps: int = 40, workers: int = 4, vocab: int = 1000, width: int = 256, heads: int = 4, sequences: int = 20,
          length: int = 64, density: float = 0.05, lr: float = 5.0, momentum: float = 0.5, seed: int = 0, report=print):
    """The model, and the mean loss of every step."""
    gen = torch.Generator(device="cuda").manual_seed(seed + 1)
    chain = torch.softmax(torch.randn(vocab, vocab, generator=gen, device="cuda") * 2.5, 1)   # the language
    model = Model(vocab, width, heads, seed + 2)
    run = Pass(model, sequences, length)
    weight = torch.full((run.n,), 1.0 / (run.n * workers), device="cuda")        # the mean over all workers' tokens
    config = B.make_config(momentum=momentum, density=density, clip_threshold=0.25, num_workers=workers, seed=seed)
    handles = [B.Dgc(config, model.offsets) for _ in range(workers)]
    layout = handles[0].dgc_recommended_payload_layout(density)
    for handle in handles:
        handle.set_layout(layout)
    state = [(torch.zeros_like(model.theta), torch.zeros_like(model.theta)) for _ in handles]
    payloads = [handle.alloc_payload() for handle in handles]
    grad, losses = torch.empty_like(model.theta), []
    for step in range(steps):
        total = torch.zeros((), device="cuda")
        for worker, handle in enumerate(handles):
            tokens = torch.empty(sequences, length + 1, dtype=torch.int64, device="cuda")
            tokens[:, 0] = torch.randint(0, vocab, (sequences,), generator=gen, device="cuda")
            for t in range(length):
                tokens[:, t + 1] = torch.multinomial(chain[tokens[:, t]], 1, generator=gen)[:, 0]
            run.forward(tokens[:, :-1].reshape(-1))
            total += run.losses(tokens[:, 1:].reshape(-1).to(torch.int32), weight).sum()
            run.backward(grad)
            handle.dgc_compress(grad, *state[worker], *payloads[worker], step)
        handles[0].dgc_sparse_sgd_apply_regions(model.theta, lr, [p[0] for p in payloads], [p[1] for p in payloads],
                                                [p[2] for p in payloads])
        losses.append(float(total))
        if report and (step % 10 == 0 or step + 1 == steps):
            report(f"step {step}: loss {losses[-1]:.4f}")
    for handle in handles:
        handle.close()
    return model, losses


def main() -> None:
    parser = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    parser.add_argument("--steps", type=int, default=40)
    parser.add_argument("--workers", type=int, default=4)
    parser.add_argument("--density", type=float, default=0.05)
    args = parser.parse_args()
    model, _ = train(steps=args.steps, workers=args.workers, density=args.density)
    print("generated:", generate(model, torch.zeros(1, 4, dtype=torch.int64, device="cuda"), 16).tolist()[0])


if __name__ == "__main__":
    main()
