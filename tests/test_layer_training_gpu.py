"""GPU: the layer operators and the RelaySum round together, as
examples/train_layers.py runs them."""
import importlib.util
import math
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def example():
    spec = importlib.util.spec_from_file_location("train_layers", os.path.join(ROOT, "examples", "train_layers.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def announce(msg):
    sys.__stderr__.write(f"[gpu] {msg}\n")
    sys.__stderr__.flush()


def plain_gradients(model, x, tokens, targets):
    """The same model in 64 bits with torch's autograd, nothing in 8 bits."""
    x = x.double().requires_grad_()

    def view(name):
        return model.view(x, name)

    def norm(s, w):
        return s * torch.rsqrt(s.square().mean(-1, keepdim=True) + 1e-6) * w.unsqueeze(1)

    r = torch.gather(view("embedding"), 1, tokens.unsqueeze(-1).expand(-1, -1, model.width))
    for b in range(model.blocks):
        y = norm(r, view(f"norm{b}"))
        r = r + torch.relu(y @ view(f"up{b}").transpose(1, 2)) @ view(f"down{b}").transpose(1, 2)
    logits = norm(r, view("norm")) @ view("out").transpose(1, 2)
    loss = -torch.log_softmax(logits, -1).gather(2, targets.unsqueeze(-1))[..., 0].mean(1)
    loss.sum().backward()
    return loss.detach(), x.grad


def test_gradients_of_a_whole_model():
    """Every parameter's gradient against autograd in 64 bits without 8-bit
    rows.  A value held in 8 bits is off by up to half a quantum, 2^-7 of its
    group's largest entry, or about 2^-7 * 4 / sqrt(12) * 1.2 = 1% of a row's
    size for normal entries; a gradient passes some 10 such values and 10
    roundings to bfloat16 (0.2%), independent of one another: about 4% of its
    size.  A fifth is allowed, which a wrong or missing term would pass."""
    announce("gradients of a model of 5 workers")
    ex = example()
    model = ex.Model(37, 72, 136, 2)
    x = torch.empty(5, model.d, device="cuda")
    model.init(x, 3)
    x += 0.01 * torch.randn(x.shape, generator=torch.Generator(device="cuda").manual_seed(4), device="cuda")
    text = torch.randint(37, (5, 130), generator=torch.Generator(device="cuda").manual_seed(5), device="cuda")
    g = torch.full_like(x, 9.0)
    losses = model.gradients(x, g, text[:, :-1], text[:, 1:].contiguous())
    want_losses, want = plain_gradients(model, x, text[:, :-1], text[:, 1:])
    assert torch.allclose(losses.double(), want_losses, rtol=0.05)
    for name in model.at:
        a, b = model.view(g, name).double(), model.view(want, name)
        off = float((a - b).norm() / b.norm())
        assert off < 0.2, (name, off)


def test_training_lowers_the_loss():
    """From about log(vocab) to well below; workers' texts differ, so only the
    relayed models fit all of them."""
    announce("training 8 workers")
    losses = example().train(workers=8, rounds=80, tokens=128)
    assert all(math.isfinite(v) for v in losses)
    assert losses[0] > 0.8 * math.log(61)
    assert sum(losses[-10:]) / 10 < losses[0] - 0.5
