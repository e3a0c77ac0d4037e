"""examples/expert_dense_part.py: inference and gradients against plain 64-bit evaluations of the same model, and the loop."""
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import expert_dense_part
    finally:
        sys.path.pop(0)
    return expert_dense_part


def model(features, A, B, gains, kinds):
    norm = lambda h, gain: h / torch.sqrt((h * h).mean(1, keepdim=True) + 1e-6) * gain
    u = torch.stack([A[k] @ v for k, v in zip(kinds, norm(features, gains[0]))])
    return torch.stack([B[k] @ v for k, v in zip(kinds, norm(u + features, gains[1]))])


def small(example):
    gen = torch.Generator(device="cuda").manual_seed(4)
    features = torch.randn(300, 72, device="cuda", generator=gen).to(torch.bfloat16)
    first = torch.tensor([0, 100, 100, 230, 300], dtype=torch.int32, device="cuda")
    d = example.ExpertDensePart(features, first, 64, max_norm=1e9)
    ids = torch.tensor([3, 50, 99, 100, 140, 141, 229, 299, 17, 250], dtype=torch.int32, device="cuda")
    return d, ids, torch.tensor([8], dtype=torch.int32, device="cuda"), [0, 0, 0, 2, 2, 2, 2, 3]      # the last two are not in use


def test_inference(example):
    """Each 8-bit factor is off by at most 2^-4, evenly spread: sums of 72 of them by about 2^-4 / sqrt(3) twice a layer, two
    layers.  0.15 of the result's norm."""
    d, ids, n, kinds = small(example)
    got = d.infer(ids, n, torch.float32)[:8].double()
    want = model(d.features[ids[:8].long()].double(), d.A.double(), d.B.double(), [t.double() for t in d.gain], kinds)
    assert (got - want).norm() < 0.15 * want.norm()


def test_gradients(example):
    """bf16 rounds weights and rows to 2^-8, four products deep: 0.05 of each gradient's norm."""
    d, ids, n, kinds = small(example)
    grads = torch.randn(10, 64, device="cuda", generator=torch.Generator(device="cuda").manual_seed(5))
    d.gradients(ids, grads, n)
    params = [t.double().cpu().requires_grad_() for t in (d.A, d.B, *d.gain)]
    out = model(d.features[ids[:8].long()].double().cpu(), params[0], params[1], params[2:], kinds)
    (out * grads[:8].double().cpu()).sum().backward()
    for got, p in zip(d.grads, params):
        assert (got.double().cpu() - p.grad).norm() < 0.05 * p.grad.norm()
    assert (d.grads[0][1] == 0).all() and (d.grads[1][1] == 0).all()      # a kind without images


def test_loop(example):
    st, dense, losses, norms = example.run(4, verbose=False)
    assert int(st.status.item()) == 0 and torch.isfinite(losses).all() and torch.isfinite(norms).all()
    assert int(dense.serve_A.status.item()) == 0 and int(dense.train_B.status.item()) == 0
    again = example.run(4, verbose=False)
    assert torch.equal(losses, again[2]) and torch.equal(norms, again[3])
