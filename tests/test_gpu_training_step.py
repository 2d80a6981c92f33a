"""The training step of examples/conditional_generator.py: its operators together, against
autograd on the same bf16 parameters, and the loss as it trains."""
import math
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                                "examples"))

pytestmark = pytest.mark.gpu


def _reference(gen, noise, labels, target):
    """Loss and gradients by autograd in 64 bits on the CPU."""
    leaf = [p.detach().cpu().double().requires_grad_() for p in
            gen.work + gen.gammas + gen.betas]
    k, n = len(gen.work), len(gen.norms)
    table, ws, gammas, betas = leaf[0], leaf[1:k], leaf[k:k + n], leaf[k + n:]
    F = torch.nn.functional
    x = (table[labels.cpu()] * math.sqrt(gen.dim) + noise.cpu().double())[..., None, None]
    for i, (w, c) in enumerate(zip(ws, gen.conv)):
        x = F.conv_transpose2d(x, w, None, c["stride"], c["padding"])
        if i < n:
            x = torch.relu(F.group_norm(x, gen.norms[i].desc.groups, gammas[i], betas[i], 1e-5))
    loss = ((torch.tanh(x) - target.cpu().double()) ** 2).mean()
    loss.backward()
    return float(loss.detach()), [p.grad for p in leaf]


def test_gradients_match_autograd():
    import conditional_generator as cg
    gen = cg.Generator(8, classes=5, dim=24, channels=(32, 16), groups=4)
    g = torch.Generator("cuda").manual_seed(1)
    labels = torch.tensor([0, 1, 2, 3, 3, 3, 1, 0], device="cuda")  # class 4 has none
    noise = (0.1 * torch.randn(8, 24, generator=g, device="cuda")).bfloat16()
    target = cg.class_images(5, 16)[labels]
    images, kept = gen.forward(noise, labels)
    diff = images.float() - target
    grads = gen.backward(diff * (2 / diff.numel()), images, kept, labels)
    loss, want = _reference(gen, noise, labels, target)
    assert abs(float((diff * diff).mean()) - loss) <= 2e-2 * loss
    assert float(grads[0][4].abs().max()) == 0
    for i, (a, b) in enumerate(zip(grads, want)):
        a = a.cpu().double()
        # some dozen bf16 roundings of 2^-9 on the way, independent of each other: 2% would be
        # 2^-9 ten times over; ReLUs whose sign they change add as much again
        assert float((a - b).norm()) <= 0.05 * float(b.norm()), i


@pytest.mark.parametrize("states", [32, 8])
def test_loss_falls(states):
    import conditional_generator as cg
    gen, losses = cg.train_generator(60, batch=32, states=states)
    print("loss", losses[0], losses[-1], flush=True)
    assert losses[-1] < 0.25 * losses[0] and math.isfinite(losses[-1])
    for work, param in zip(gen.work, gen.params):
        assert torch.equal(work, param.bfloat16())
