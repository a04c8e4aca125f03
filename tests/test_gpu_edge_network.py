"""The example network around the convolution, as a program runs it: its gradients from activations in
full against float64 automatic differentiation, from 8-bit checkpoints near them, and training."""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.fixture(scope="module")
def ex():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    import edge_network
    return edge_network


def _reference(net, basis, dh):
    """h and the gradients of <h, dh> in float64 on the host."""
    import torch
    p = {k: v.double().cpu().requires_grad_() for k, v in net.p.items()}
    silu = torch.nn.functional.silu
    a = silu(basis.double().cpu() @ p["W1"] + p["b1"])
    n = torch.nn.functional.layer_norm(a, a.shape[1:], p["gamma"], p["beta"], 1e-5)
    c = silu(n @ p["W2"] + p["b2"]) + n
    h = c @ p["W3"]
    (h * dh.double().cpu()).sum().backward()
    return h.detach(), {k: v.grad for k, v in p.items()}


@pytest.mark.parametrize("packed,bar", [(False, 5e-6), (True, 0.02)])
def test_gradients(ex, packed, bar):
    """In full: float32 sums through three layers.  From 8 bits: each saved value is off by up to 1/127 of
    its group's largest, 1/250 typically, at random over the rows (bar 0.02)."""
    import torch
    torch.manual_seed(3)
    net = ex.EdgeNetwork(packed=packed, seed=2)
    for k in ("b1", "gamma", "beta", "b2"):
        net.p[k] += 0.3 * torch.randn_like(net.p[k])
    basis = ex.bessel(0.8 + 4 * torch.rand(5000, device="cuda"), 8)
    dh = torch.randn(5000, 16, device="cuda")
    h = net.forward(basis)
    got = net.backward(dh)
    ref_h, ref = _reference(net, basis, dh)
    assert float((h.cpu() - ref_h).norm() / ref_h.norm()) < 2e-6
    for k, w in ref.items():
        assert float((got[k].cpu() - w).norm() / w.norm()) < bar, k


def test_training_lowers_the_loss_with_either(ex):
    full, net_f = ex.train(120, 8, packed=False, log=None)
    packed, net_p = ex.train(120, 8, packed=True, log=None)
    assert all(b < a for a, b in zip(full, full[1:])) and all(b < a for a, b in zip(packed, packed[1:]))
    assert abs(packed[0] - full[0]) < 1e-5 * full[0]        # the forward is the same
    # the drop over the steps differs by what the checkpoints' rounding moves the gradients
    assert abs((packed[0] - packed[-1]) - (full[0] - full[-1])) < 0.05 * (full[0] - full[-1])
    assert net_p.kept_bytes() < 0.45 * net_f.kept_bytes()


def test_command(ex):
    import subprocess
    r = subprocess.run([sys.executable, ex.__file__, "--atoms", "64", "--steps", "2"], capture_output=True, text=True,
                       timeout=110)
    assert r.returncode == 0, r.stderr
    assert "step 1: loss" in r.stdout and "MiB kept" in r.stdout
