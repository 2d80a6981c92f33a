"""The training step of examples/conditional_generator.py with layer norms and Muon: its
operators together, against autograd on the same bf16 parameters and Muon's formulas."""
import math
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                                "examples"))
from test_gpu_muon import _model_error, _steps  # noqa: E402

pytestmark = pytest.mark.gpu


def _generator():
    import conditional_generator as cg
    gen = cg.Generator(8, classes=5, dim=24, channels=(32, 16), groups=4, norm="layer",
                       optimizer="muon")
    g = torch.Generator("cuda").manual_seed(1)
    labels = torch.tensor([0, 1, 2, 3, 3, 3, 1, 0], device="cuda")  # class 4 has none
    noise = (0.1 * torch.randn(8, 24, generator=g, device="cuda")).bfloat16()
    return gen, noise, labels, cg.class_images(5, 16)[labels]


def _reference(gen, noise, labels, target):
    """Loss and gradients by autograd in 64 bits on the CPU."""
    leaf = [p.detach().cpu().double().requires_grad_() for p in gen.work + gen.gammas + gen.betas]
    k, n = len(gen.work), len(gen.norms)
    table, ws, gammas, betas = leaf[0], leaf[1:k], leaf[k:k + n], leaf[k + n:]
    F = torch.nn.functional
    x = (table[labels.cpu()] * math.sqrt(gen.dim) + noise.cpu().double())[..., None, None]
    for i, (w, c) in enumerate(zip(ws, gen.conv)):
        x = F.conv_transpose2d(x, w, None, c["stride"], c["padding"])
        if i < n:
            x = x.movedim(1, -1)
            x = F.layer_norm(x, x.shape[-1:], gammas[i], betas[i], 1e-5)
            x = torch.relu(x).movedim(-1, 1)
    loss = ((torch.tanh(x) - target.cpu().double()) ** 2).mean()
    loss.backward()
    return float(loss.detach()), [p.grad for p in leaf]


def test_gradients_match_autograd():
    gen, noise, labels, target = _generator()
    images, kept = gen.forward(noise, labels)
    diff = images.float() - target
    grads = gen.backward(diff * (2 / diff.numel()), images, kept, labels)
    loss, want = _reference(gen, noise, labels, target)
    assert abs(float((diff * diff).mean()) - loss) <= 2e-2 * loss
    for i, (a, b) in enumerate(zip(grads, want)):
        a = a.cpu().double()
        # some dozen bf16 roundings of 2^-8 at most on the way, independent of each other (rms
        # 2^-9.8 each): 2% would be 2^-9.8 eighteen times over; ReLUs whose sign they change add
        # as much again
        assert float((a - b).norm()) <= 0.05 * float(b.norm()), i


def test_a_step_updates_every_parameter_once():
    """Matrices by Muon, the rest by AdamW, each with its bf16 copy."""
    gen, noise, labels, target = _generator()
    images, kept = gen.forward(noise, labels)
    diff = images.float() - target
    grads = [g.clone() for g in gen.backward(diff * (2 / diff.numel()), images, kept, labels)]
    before = [p.clone() for p in gen.params]
    loss = gen.step(noise, labels, target)
    torch.cuda.synchronize()
    assert math.isfinite(float(loss))
    assert sorted(gen.matrices + gen.others) == list(range(len(gen.params)))
    for i in gen.matrices:
        p, g = before[i].cpu().double(), grads[i].cpu().double()
        rows = p.shape[0]
        u = (0.1 * g + 0.9 * 0.1 * g).reshape(rows, -1)  # momentum 0.9 from nothing, Nesterov's
        scale = math.sqrt(max(1.0, rows / u.shape[1]))
        exact = _steps(u)
        want = p * (1 - 2e-2 * 0.01) - 2e-2 * scale * exact.reshape(p.shape)
        # A batch of 8 leaves gradients of rank 8 for 24 rows: what products of 11 bits leave in
        # the other directions grows as they do, by 3.44 a step.  Three times what the same
        # roundings leave in a model of them is allowed, and the parameter's own, 2^-24 twice.
        model = _model_error(u, exact, 1) * float(exact.norm())
        err = float((gen.params[i].cpu().double() - want).norm())
        print("matrix", i, tuple(u.shape), "off by %.1e of the update, model %.1e"
              % (err / (2e-2 * scale * float(exact.norm())), model / float(exact.norm())))
        assert err <= 2e-2 * scale * 3 * model + 2 ** -22 * float(p.norm()), i
        assert torch.equal(gen.work[i], gen.params[i].bfloat16())
    for i in gen.others:
        if float(grads[i].abs().max()) > 0:
            assert not torch.equal(gen.params[i], before[i]), i


@pytest.mark.parametrize("norm,optimizer", [("layer", "muon"), ("group", "muon"), ("layer", "adamw")])
def test_training_runs(norm, optimizer):
    import conditional_generator as cg
    gen, losses = cg.train_generator(5, batch=16, norm=norm, optimizer=optimizer)
    assert all(math.isfinite(v) for v in losses)
    for work, param in zip(gen.work, gen.params):
        assert torch.equal(work, param.bfloat16())
