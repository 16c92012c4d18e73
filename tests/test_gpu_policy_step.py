"""The operators together, as examples/policy_step.py runs them."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("policy_step", os.path.join(ROOT, "examples", "policy_step.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("bits", [32, 8])
def test_loss_falls(gpu, example, bits):
    model = example.PolicyStep(state_bits=bits)
    losses = [model.step().item() for _ in range(25)]
    assert all(a == a for a in losses)
    assert losses[-1] < 0.7 * losses[0]


def test_gradients_against_differences(gpu, example):
    """In fp32, along random directions of every weight. The two losses are
    sums of some hundred fp32 terms around 8: each within 1e-5, so their
    difference over 2 h = 2e-2 times the direction within 2e-3 of the largest
    slope, besides the curvature of order h^2."""
    model = example.PolicyStep(T=96, d=64, F=32, E=6, K=2, V=301, dtype=torch.float32)
    f = model.forward()
    model.backward(f)
    h = 1e-2
    for w, dw in ((model.router, model.d_router), (model.gate_up, model.d_gate_up), (model.down, model.d_down),
                  (model.head, model.d_head)):
        u = torch.randn(w.shape, generator=torch.Generator(device=gpu).manual_seed(1), device=gpu)
        u = dw / dw.norm() + 0.3 * u / u.norm()
        slope = (dw.double() * u.double()).sum().item()
        w0 = w.clone()
        w.copy_(w0 + h * u)
        up = model.forward()["loss"].item()
        w.copy_(w0 - h * u)
        down = model.forward()["loss"].item()
        w.copy_(w0)
        assert abs((up - down) / (2 * h) - slope) <= 2e-3 + 0.02 * abs(slope)


def test_replay_keeps_the_routing(gpu, example):
    model = example.PolicyStep()
    first = model.forward()["routing"].ids
    model.router.add_(torch.randn_like(model.router))
    again = model.forward()["routing"]
    assert torch.equal(first, again.ids)
    assert torch.allclose(again.gates.sum(1), torch.ones(model.T, device=gpu), atol=1e-5)
