"""A trained language model teaches a narrower one: K workers train the teacher with gossip-BMUF rounds
(``local_step_lm``), their average is kept as lists of its likeliest words (``top_logits``), and the student
learns from these lists and from the text together (``distillation``).

    python examples/distil_lm.py [--steps 200] [--dtype bf16]
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import local_step_lm as lm                                                       # noqa: E402
from local_step_lm import binding                                               # noqa: E402


def scores_of(ops, model, p, words):
    """(hidden states for the backward pass, scores of the next word) of a model."""
    x = p["embedding"][words].reshape(words.shape[0], 2 * model.width)
    h, z = ops.linear_forward(x, p["w1"], bias=p["b1"], activation="gelu", keep_z=True)
    y = ops.linear_forward(h, p["w2"], bias=p["b2"], residual=x)
    return (x, h, z, y), ops.linear_forward(y, p["ws"], bias=p["bs"])


def lists_of(ops, model, p, words, k, temperature):
    """What is kept of a teacher: its k likeliest next words, their scores, its log-sum-exp."""
    return ops.top_logits(scores_of(ops, model, p, words)[1], k, temperature=temperature)


def distil_gradients(ops, model, p, grad, words, targets, lists, temperature, hard_weight):
    """Forward and backward pass of the student: fills the views ``grad`` (float32), returns the losses."""
    n = words.shape[0]
    (x, h, z, y), scores = scores_of(ops, model, p, words)
    values, index, lse = lists
    loss, _, d = ops.distillation(scores, values, index, teacher_lse=lse, temperature=temperature, targets=targets,
                                  hard_weight=hard_weight, scale=1.0 / n, dlogits_out=scores)
    ops.linear_backward_weight(d, y, dw_out=grad["ws"], dbias_out=grad["bs"])
    dy = ops.linear_backward_input(d, p["ws"])
    ops.linear_backward_weight(dy, h, dw_out=grad["w2"], dbias_out=grad["b2"])
    dz = ops.linear_backward_input(dy, p["w2"], z_prev=z, activation="gelu")
    ops.linear_backward_weight(dz, x, dw_out=grad["w1"], dbias_out=grad["b1"])
    dx = ops.linear_backward_input(dz, p["w1"], residual=dy)
    grad["embedding"].zero_()
    grad["embedding"].index_add_(0, words.reshape(-1), dx.reshape(2 * n, model.width).float())
    return loss


def distil(steps=200, vocab=64, batch=512, k=8, temperature=2.0, hard_weight=0.3, lr=0.05, dtype="f32", seed=0):
    """Returns the student's mean loss at every step, and its parameters."""
    _, average = lm.train(steps=steps, workers=4, vocab=vocab, dtype=dtype, seed=seed)
    device, ops = average.device, binding.local_ops()
    teacher, student = lm.Model(vocab, 48, 256), lm.Model(vocab, 16, 64)
    taught = teacher.views(average)
    flat = student.start(seed + 1, average.dtype, device)
    grad = torch.zeros(student.n, device=device)
    accum = torch.full_like(grad, 0.1)
    p, views = student.views(flat), student.views(grad)
    clipping = binding.GradClip([(g, g, 0) for g in views.values()], groups=1)
    g = torch.Generator(device=device)
    g.manual_seed(seed + 2)
    history = []
    for _ in range(steps):
        words, targets = lm.text(g, vocab, batch, device)
        lists = lists_of(ops, teacher, taught, words, k, temperature)
        loss = distil_gradients(ops, student, p, views, words, targets, lists, temperature, hard_weight)
        clipping.clip(1.0)
        accum.addcmul_(grad, grad)
        flat.sub_((lr * grad / (accum.sqrt() + 1e-8)).to(flat.dtype))
        history.append(loss.sum())
    for word in (ops.device_status(), clipping.device_status()):
        if word != binding.GBMUF_OK:
            raise binding.GbmufError(word, "a kernel of the distillation reported a failure")
    clipping.destroy()
    return torch.stack(history).tolist(), flat


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--dtype", choices=("f32", "bf16"), default="f32")
    a = ap.parse_args()
    history, _ = distil(steps=a.steps, dtype=a.dtype)
    for t in sorted({0, *range(9, len(history), max(1, len(history) // 10)), len(history) - 1}):
        print(f"step {t + 1:5d}  loss {history[t]:.4f}")


if __name__ == "__main__":
    main()
