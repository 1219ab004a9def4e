"""The layers together as they are used: the example trains a one-block classifier on padded
sequences. Its gradients are checked against torch's autograd in float32 on the same model."""
import math

import pytest
import torch

from examples import train_sequences as ex

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _device():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    torch.cuda.set_device(0)


def reference_step(model, ids, cls):
    p = {k: v.float().requires_grad_() for k, v in model.p.items()}
    H, D, C = model.H, model.D, model.C
    here = (ids >= 0).unsqueeze(-1)
    x = torch.where(here, p["emb"][ids.clamp(min=0)] * math.sqrt(C), 0.0)

    def heads(t):
        return t.view(*t.shape[:2], H, D).transpose(1, 2)

    def sdpa(q, k, v):
        return torch.softmax(q @ k.transpose(-1, -2) / math.sqrt(D), -1) @ v

    K, V, Kt, Vt = (heads(t) for t in (x @ p["W_in"].t()).split(C, -1))
    Q = sdpa(p["seeds"].unsqueeze(0), Kt, Vt)
    Y = sdpa(K, Q, sdpa(Q, K, V))
    h = x + Y.transpose(1, 2).reshape(*x.shape) @ p["Wo"].t()
    a = torch.nn.functional.gelu(h @ p["W1"].t() + p["b1"])
    y = h + a @ p["W2"].t() + p["b2"]
    pooled = (y * here).sum(1) / here.sum(1)
    loss = torch.nn.functional.cross_entropy(pooled @ p["Wc"].t() + p["bc"], cls)
    loss.backward()
    return float(loss.detach()), {k: v.grad for k, v in p.items()}


def test_gradients_of_the_whole_model():
    """bf16 activations against float32: every stage rounds to 2^-8, and some ten stages lie between a
    weight and the loss, so gradients agree to a few per cent of their norm, and the loss to 2e-2."""
    model = ex.Model(seed=3)
    gen = torch.Generator(device="cuda").manual_seed(4)
    ids, cls = ex.batch(gen, 4, 300, model.V, torch.device("cuda", 0))
    loss, _ = model.step(ids, cls)
    want, grads = reference_step(model, ids, cls)
    assert abs(float(loss) - want) <= 2e-2 * max(1.0, abs(want))
    for k, g in model.g.items():
        off = float((g.float() - grads[k]).norm() / grads[k].norm())
        assert off <= 6e-2, f"{k}: {off:.3g}"


@pytest.mark.parametrize("bits", [8, 32])
def test_it_learns(bits):
    losses, accuracy = ex.train(steps=60, state_bits=bits)
    assert all(math.isfinite(x) for x in losses)
    assert sum(losses[-5:]) / 5 < 0.5 * losses[0] and accuracy > 0.8, (losses[::10], accuracy)
