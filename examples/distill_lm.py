"""A recurrent language model distilled on several workers whose gradients are compressed.

    python examples/distill_lm.py [--steps 40] [--workers 4] [--density 0.05]

A student learns from a teacher's largest logits instead of its whole output, and the workers exchange 5 % of their
gradients instead of all of them.  Both models are an embedding, a gated linear recurrence and an output layer:

    p = embed[tokens] W_in          gate and candidate of every channel
    h = gated scan of p             GatedScan.dgc_gated_scan_forward
    z = h W_out                     logits

Per step and worker: the teacher's logits -> dgc_top_logits, k pairs a token -> dgc_distill_loss, loss and gradient of the
student's logits, in their place -> dgc_gated_scan_backward -> the flat gradient -> dgc_compress; then one
dgc_sparse_sgd_apply_regions of all workers' payloads steps the parameters.  The workers share one GPU here, one after the
other, as `num_workers` handles; the token streams are synthetic (a Markov chain that the teacher fits better than chance)."""

from __future__ import annotations

import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch  # noqa: E402

from paper_1712_01887_amd import binding as B  # noqa: E402


class Model:
    """Parameters as views of one flat float32 tensor, in the order of their names."""

    def __init__(self, vocab: int, width: int, seed: int):
        self.vocab, self.width = vocab, width
        self.shapes = {"embed": (vocab, width), "w_in": (width, 2 * width), "w_out": (width, vocab)}
        self.offsets = [0]
        for rows, columns in self.shapes.values():
            self.offsets.append(self.offsets[-1] + rows * columns)
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.theta = torch.empty(self.offsets[-1], device="cuda")
        for name, (rows, _) in self.shapes.items():
            scale = 1.0 if name == "embed" else rows ** -0.5
            p = self.of(self.theta, name)
            p.copy_(torch.randn(p.shape, generator=gen, device="cuda") * scale)

    def of(self, flat: torch.Tensor, name: str) -> torch.Tensor:
        i = list(self.shapes).index(name)
        return flat[self.offsets[i]:self.offsets[i + 1]].view(self.shapes[name])


class Pass:
    """The buffers of a model's pass over `sequences` x `length` tokens, 16-bit activations."""

    def __init__(self, model: Model, sequences: int, length: int):
        n, d, bf = sequences * length, model.width, torch.bfloat16
        self.model, self.scan = model, B.GatedScan(sequences, length, d, bf)
        self.h, self.states = torch.empty(n, d, dtype=bf, device="cuda"), self.scan.alloc_states()
        self.h0 = torch.zeros(sequences, d, device="cuda")
        self.d_projected = torch.empty(n, 2 * d, dtype=bf, device="cuda")

    def forward(self, tokens: torch.Tensor) -> torch.Tensor:
        m, bf, d = self.model, torch.bfloat16, self.model.width
        w = {name: m.of(m.theta, name).to(bf) for name in m.shapes}
        self.tokens, self.w = tokens, w
        self.x = w["embed"][tokens]
        self.projected = self.x @ w["w_in"]
        self.scan.dgc_gated_scan_forward(self.projected[:, :d], self.projected[:, d:], self.h0, self.h, None, self.states)
        return self.h @ w["w_out"]

    def backward(self, d_logits: torch.Tensor, grad: torch.Tensor) -> None:
        """Into the flat gradient `grad`."""
        m, d = self.model, self.model.width
        dh = d_logits @ self.w["w_out"].t().contiguous()
        m.of(grad, "w_out").copy_(self.h.t().contiguous() @ d_logits)
        self.scan.dgc_gated_scan_backward(self.projected[:, :d], self.projected[:, d:], self.states, dh, None,
                                          self.d_projected[:, :d], self.d_projected[:, d:])
        m.of(grad, "w_in").copy_(self.x.t().contiguous() @ self.d_projected)
        dx = self.d_projected @ self.w["w_in"].t().contiguous()
        m.of(grad, "embed").zero_().index_add_(0, self.tokens, dx.float())


def train(steps: int = 40, workers: int = 4, vocab: int = 1000, width: int = 256, sequences: int = 20, length: int = 35,
          k: int = 32, temperature: float = 2.0, hard_weight: float = 0.1, density: float = 0.05, lr: float = 20.0, momentum: float = 0.5,
          seed: int = 0, report=print):
    """The mean distillation loss of every step."""
    gen = torch.Generator(device="cuda").manual_seed(seed + 1)
    chain = torch.softmax(torch.randn(vocab, vocab, generator=gen, device="cuda") * 2.5, 1)   # the language
    teacher, student = Model(vocab, width, seed + 2), Model(vocab, width, seed + 3)
    # a teacher that knows the language: its output layer reads the last token from the state
    teacher.of(teacher.theta, "w_in").zero_()
    teacher.of(teacher.theta, "w_in")[:, width:].copy_(torch.eye(width, device="cuda"))
    embed = teacher.of(teacher.theta, "embed")
    teacher.of(teacher.theta, "w_out").copy_(torch.linalg.pinv(embed.cpu()).to("cuda") @ chain.log() * 0.5)
    rows = sequences * length
    teach, learn = Pass(teacher, sequences, length), Pass(student, sequences, length)
    plan = B.Distillation(rows, vocab, torch.bfloat16)
    top_idx, top_val, _ = plan.alloc_top_logits(k)
    loss = torch.empty(rows, device="cuda")
    weight = torch.full((rows,), 1.0 / (rows * workers), device="cuda")          # the mean over all workers' tokens
    config = B.make_config(momentum=momentum, density=density, clip_threshold=0.25, num_workers=workers, seed=seed)
    handles = [B.Dgc(config, student.offsets) for _ in range(workers)]
    layout = handles[0].dgc_recommended_payload_layout(density)
    for handle in handles:
        handle.set_layout(layout)
    state = [(torch.zeros_like(student.theta), torch.zeros_like(student.theta)) for _ in handles]
    payloads = [handle.alloc_payload() for handle in handles]
    grad = torch.empty_like(student.theta)
    losses = []
    for step in range(steps):
        total = torch.zeros((), device="cuda")
        for worker, handle in enumerate(handles):
            tokens = torch.empty(sequences, length + 1, dtype=torch.int64, device="cuda")
            tokens[:, 0] = torch.randint(0, vocab, (sequences,), generator=gen, device="cuda")
            for t in range(length):
                tokens[:, t + 1] = torch.multinomial(chain[tokens[:, t]], 1, generator=gen)[:, 0]
            inputs, labels = tokens[:, :-1].reshape(-1), tokens[:, 1:].reshape(-1).to(torch.int32)
            plan.dgc_top_logits(teach.forward(inputs), top_idx, top_val)
            logits = learn.forward(inputs)
            plan.dgc_distill_loss(logits, top_idx, top_val, loss, logits, labels=labels, row_weight=weight,
                                  temperature=temperature, hard_weight=hard_weight)
            learn.backward(logits, grad)
            handle.dgc_compress(grad, *state[worker], *payloads[worker], step)
            total += loss.sum()
        handles[0].dgc_sparse_sgd_apply_regions(student.theta, lr, [p[0] for p in payloads], [p[1] for p in payloads],
                                                [p[2] for p in payloads])
        losses.append(float(total))
        if report and (step % 10 == 0 or step + 1 == steps):
            sent = sum(int(p[2].sum()) for p in payloads) / workers
            report(f"step {step}: loss {losses[-1]:.4f}, {sent:.0f} of {student.theta.numel()} gradients sent a worker")
    for handle in handles:
        handle.close()
    return losses


def main() -> None:
    parser = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    parser.add_argument("--steps", type=int, default=40)
    parser.add_argument("--workers", type=int, default=4)
    parser.add_argument("--density", type=float, default=0.05)
    args = parser.parse_args()
    train(steps=args.steps, workers=args.workers, density=args.density)


if __name__ == "__main__":
    main()
