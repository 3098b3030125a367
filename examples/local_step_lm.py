"""K workers train a small feed-forward language model with Algorithm 1's loop: local steps on their
own text, a gossip-BMUF round every H steps, the average at the end.

Everything between the tokens and the new parameters runs through the library: the linear layers and
their gradients (``linear_forward``, ``linear_backward_input``, ``linear_backward_weight``), the loss
(``cross_entropy``, or ``linear_cross_entropy`` for the softmax layer and the loss in one), the gradient norm of each worker and clipping (``GradClip``), the Adagrad step
and the synchronisation round.  Weights are views into the workers' rows of theta and gradients are
written straight into the rows of the optimiser's gradient buffer.

    python examples/local_step_lm.py [--steps 200] [--workers 4] [--dtype bf16] [--no-scores]
"""
from __future__ import annotations

import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_1909_09010_b200 import binding                                       # noqa: E402


class Model:
    """Two context words -> embedding -> x + W2 gelu(W1 x + b1) + b2 -> scores of the next word."""

    def __init__(self, vocab, width, hidden):
        self.vocab, self.width, self.hidden = vocab, width, hidden
        d = 2 * width
        shapes = {"embedding": (vocab, width), "w1": (hidden, d), "b1": (hidden,), "w2": (d, hidden),
                  "b2": (d,), "ws": (vocab, d), "bs": (vocab,)}
        self.shapes, self.offsets, at = shapes, [0], 0
        for s in shapes.values():
            at += math.prod(s)
            self.offsets.append(at)
        self.n = at
        self.ld = (at + 31) // 32 * 32

    def views(self, row):
        """The tensors of a worker as views into its row of theta (or of the gradient buffer)."""
        return {name: row[a:b].view(shape) for (name, shape), a, b in
                zip(self.shapes.items(), self.offsets, self.offsets[1:])}

    def start(self, seed, dtype, device):
        g = torch.Generator(device="cpu")
        g.manual_seed(seed)
        flat = torch.zeros(self.n)
        for name, t in self.views(flat).items():
            if t.dim() == 2:
                t.copy_(torch.randn(t.shape, generator=g) * (0.5 if name == "embedding" else t.shape[1] ** -0.5))
        return flat.to(dtype).to(device)


def loss_and_gradients(ops, model, p, grad, words, targets, keep_scores=True):
    """Forward and backward pass of one worker: fills the views ``grad`` (float32), returns the losses
    of the batch's words (their mean is the objective).  Without ``keep_scores`` the softmax layer and
    its loss are one call, and the scores of the vocabulary are never in memory."""
    n = words.shape[0]
    x = p["embedding"][words].reshape(n, 2 * model.width)
    h, z = ops.linear_forward(x, p["w1"], bias=p["b1"], activation="gelu", keep_z=True)
    y = ops.linear_forward(h, p["w2"], bias=p["b2"], residual=x)
    if keep_scores:
        scores = ops.linear_forward(y, p["ws"], bias=p["bs"])
        loss, _, dscores = ops.cross_entropy(scores, targets, scale=1.0 / n, dlogits_out=scores)
        ops.linear_backward_weight(dscores, y, dw_out=grad["ws"], dbias_out=grad["bs"])
        dy = ops.linear_backward_input(dscores, p["ws"])
    else:
        loss, _, dy, _, _ = ops.linear_cross_entropy(y, p["ws"], targets, bias=p["bs"], scale=1.0 / n,
                                                     dw_out=grad["ws"], dbias_out=grad["bs"])
    ops.linear_backward_weight(dy, h, dw_out=grad["w2"], dbias_out=grad["b2"])
    dz = ops.linear_backward_input(dy, p["w2"], z_prev=z, activation="gelu")
    ops.linear_backward_weight(dz, x, dw_out=grad["w1"], dbias_out=grad["b1"])
    dx = ops.linear_backward_input(dz, p["w1"], residual=dy)
    grad["embedding"].zero_()
    grad["embedding"].index_add_(0, words.reshape(-1), dx.reshape(2 * n, model.width).float())
    return loss


def text(g, vocab, n, device):
    """Synthetic text: the next word is a fixed function of the word before it, with some noise."""
    words = torch.randint(0, vocab, (n, 2), generator=g, device=device)
    target = (words[:, 1] * 7 + 1) % vocab
    noise = torch.randint(0, vocab, (n,), generator=g, device=device)
    return words, torch.where(torch.rand(n, generator=g, device=device) < 0.1, noise, target)


def train(steps=200, workers=4, vocab=64, width=48, hidden=256, batch=512, period=4, lr=0.1, clip=1.0,
          dtype="f32", seed=0, keep_scores=True):
    """Returns the mean loss of all workers at every step, and the averaged model."""
    device = torch.device("cuda", torch.cuda.current_device())
    kind = {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]
    model, ops = Model(vocab, width, hidden), binding.local_ops()
    theta = torch.zeros((workers, model.ld), dtype=kind, device=device)
    omega, delta = torch.zeros((2, workers, model.ld), device=device).unbind(0)
    grad, accum = torch.zeros_like(omega), torch.full_like(omega, 0.1)
    p = max(1, (workers - 1) // 2) if workers > 1 else 0
    ctx = binding.Gbmuf(theta, omega, delta, K=workers, N=model.n, ld=model.ld, p=p, q=min(1, p), eta=0.5, zeta=1.0,
                        seed=seed, theta_dtype=binding.BF16 if dtype == "bf16" else binding.F32)
    ctx.set_partition(model.offsets)
    ctx.init(model.start(seed, kind, device))
    params = [model.views(theta[k]) for k in range(workers)]
    grads = [model.views(grad[k]) for k in range(workers)]
    clipping = binding.GradClip([(g, g, k) for k in range(workers) for g in grads[k].values()], groups=workers)
    streams = [torch.Generator(device=device) for _ in range(workers)]
    for k, g in enumerate(streams):
        g.manual_seed(1000 * seed + k)
    history = []
    for t in range(1, steps + 1):
        losses = [loss_and_gradients(ops, model, params[k], grads[k], *text(streams[k], vocab, batch, device), keep_scores)
                  for k in range(workers)]
        clipping.clip(clip)
        ctx.local_adagrad(grad, accum, lr, eps=1e-8)
        if t % period == 0:
            ctx.sync_round(t)
        history.append(torch.stack(losses).sum(1).mean())
    out = torch.zeros(model.n, dtype=kind, device=device)
    ctx.final_average(out)
    for word in (ops.device_status(), clipping.device_status()):
        if word != binding.GBMUF_OK:
            raise binding.GbmufError(word, "a kernel of the local steps reported a failure")
    clipping.destroy()
    ctx.destroy()
    return torch.stack(history).tolist(), out


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--workers", type=int, default=4)
    ap.add_argument("--dtype", choices=("f32", "bf16"), default="f32")
    ap.add_argument("--no-scores", action="store_true", help="never keep the vocabulary's scores in memory")
    a = ap.parse_args()
    history, _ = train(steps=a.steps, workers=a.workers, dtype=a.dtype, keep_scores=not a.no_scores)
    for t in sorted({0, *range(9, len(history), max(1, len(history) // 10)), len(history) - 1}):
        print(f"step {t + 1:5d}  loss {history[t]:.4f}")


if __name__ == "__main__":
    main()
