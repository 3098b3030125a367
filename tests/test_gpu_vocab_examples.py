"""The vocabulary operators as the examples use them: gradients of whole models against automatic
differentiation in 64 bits, and short runs."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu


def forward64(model, p, words):
    x = p["embedding"][words].reshape(words.shape[0], 2 * model.width)
    y = torch.nn.functional.gelu(x @ p["w1"].t() + p["b1"]) @ p["w2"].t() + p["b2"] + x
    return y @ p["ws"].t() + p["bs"]


def small(seed, vocab=101, batch=77):
    import local_step_lm as lm
    from paper_1909_09010_b200 import binding
    model = lm.Model(vocab=vocab, width=24, hidden=72)
    flat = model.start(seed, torch.float32, torch.device("cuda:0"))
    g = torch.Generator(device="cuda:0")
    g.manual_seed(1)
    return lm, binding.local_ops(0), model, flat, torch.zeros_like(flat), *lm.text(g, vocab, batch, flat.device)


def agree(model, grad, ref):
    # fp32 throughout: products of parts to 2^-23, sums of a few hundred terms
    for name, got in model.views(grad).items():
        exact = model.views(ref.grad)[name]
        assert float((got.double() - exact).norm()) <= 2e-5 * float(exact.norm()), name


def test_gradients_of_the_whole_model_without_scores():
    lm, ops, model, flat, grad, words, targets = small(3)
    loss = lm.loss_and_gradients(ops, model, model.views(flat), model.views(grad), words, targets, keep_scores=False)
    ref = flat.double().requires_grad_()
    want = torch.nn.functional.cross_entropy(forward64(model, model.views(ref), words), targets)
    want.backward()
    assert abs(float(loss.double().sum()) - float(want.detach())) < 1e-5
    agree(model, grad, ref)


@pytest.mark.parametrize("temperature,hard", [(2.0, 0.3), (1.0, 0.0), (1.5, 0.5)])
def test_gradients_of_a_student(temperature, hard):
    import distil_lm
    lm, ops, model, flat, grad, words, targets = small(4)
    teacher = lm.Model(vocab=101, width=32, hidden=40)
    taught = teacher.start(5, torch.float32, flat.device)
    lists = distil_lm.lists_of(ops, teacher, teacher.views(taught), words, 12, temperature)
    loss = distil_lm.distil_gradients(ops, model, model.views(flat), model.views(grad), words, targets, lists, temperature, hard)
    ref = flat.double().requires_grad_()
    s = forward64(model, model.views(ref), words)
    index = lists[1]
    q = torch.exp(lists[0].double() / temperature - lists[2].double()[:, None])
    lp = torch.log_softmax(s / temperature, 1)
    rest = 1 - q.sum(1)
    soft = (q * (q.log() - lp.gather(1, index))).sum(1) + rest * (
        rest.log() - torch.logsumexp(lp.scatter(1, index, -float("inf")), 1))
    want = ((1 - hard) * temperature ** 2 * soft + hard * torch.nn.functional.cross_entropy(s, targets, reduction="none")).mean()
    want.backward()
    assert abs(float(loss.double().sum()) - float(want.detach())) < 1e-5
    agree(model, grad, ref)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_examples_run(dtype):
    import distil_lm
    import local_step_lm as lm
    history, out = lm.train(steps=12, workers=3, dtype=dtype, vocab=32, width=32, hidden=128, batch=256, keep_scores=False)
    assert len(history) == 12 and bool(torch.isfinite(out.float()).all())
    history, out = distil_lm.distil(steps=12, vocab=32, batch=128, dtype=dtype)
    assert len(history) == 12 and all(h == h for h in history) and bool(torch.isfinite(out.float()).all())
