"""The local-step operators together, as the example uses them: a worker's gradients against automatic
differentiation in 64 bits, and a short training run with gossip-BMUF rounds."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu


def test_gradients_of_the_whole_model():
    import local_step_lm as lm
    from paper_1909_09010_b200 import binding
    model = lm.Model(vocab=101, width=24, hidden=72)
    device = torch.device("cuda:0")
    flat = model.start(3, torch.float32, device)
    grad = torch.zeros_like(flat)
    g = torch.Generator(device=device)
    g.manual_seed(1)
    words, targets = lm.text(g, 101, 77, device)
    loss = lm.loss_and_gradients(binding.local_ops(0), model, model.views(flat), model.views(grad), words, targets)
    ref = flat.double().requires_grad_()
    p = model.views(ref)
    x = p["embedding"][words].reshape(77, 48)
    y = torch.nn.functional.gelu(x @ p["w1"].t() + p["b1"]) @ p["w2"].t() + p["b2"] + x
    want = torch.nn.functional.cross_entropy(y @ p["ws"].t() + p["bs"], targets)
    want.backward()
    assert abs(float(loss.double().sum()) - float(want.detach())) < 1e-5
    for name, got in model.views(grad).items():
        exact = model.views(ref.grad)[name]
        assert float((got.double() - exact).norm()) <= 2e-5 * float(exact.norm()), name


@pytest.mark.parametrize("dtype,workers", [("f32", 4), ("bf16", 3), ("f32", 1)])
def test_training_with_gossip_rounds_learns(dtype, workers):
    import local_step_lm as lm
    history, out = lm.train(steps=60, workers=workers, dtype=dtype, vocab=32, width=32, hidden=128, batch=256)
    assert bool(torch.isfinite(out.float()).all())
    first, last = sum(history[:5]) / 5, sum(history[-5:]) / 5
    assert last < 0.75 * first, (first, last)
