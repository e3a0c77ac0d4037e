"""examples/routed_dense_part.py: inference and gradients against plain 64-bit evaluations of the same model, and the loop."""
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
        import routed_dense_part
    finally:
        sys.path.pop(0)
    return routed_dense_part


def model(f, router, A, B, gain1, gain2, expert):
    """The model of the example's first lines; `expert` [rows x k]: the choice, held fixed."""
    norm = lambda h, gain: h / torch.sqrt((h * h).mean(1, keepdim=True) + 1e-6) * gain
    h = norm(f, gain1)
    s = torch.sigmoid(h @ router.t()).gather(1, expert)
    w = s / s.sum(1, keepdim=True)
    y = torch.stack([h @ a.t() for a in A], 1).gather(1, expert[:, :, None].expand(-1, -1, f.shape[1]))
    return norm(f + (w[:, :, None] * y).sum(1), gain2) @ B.t()


def small(example):
    gen = torch.Generator(device="cuda").manual_seed(4)
    features = torch.randn(300, 72, device="cuda", generator=gen).to(torch.bfloat16)
    d = example.RoutedDensePart(features, experts=8, k=3, dfv_dim=64, max_norm=1e9)
    d.bias.copy_(0.1 * torch.randn(8, device="cuda", generator=gen))
    ids = torch.randint(0, 300, (40,), device="cuda", generator=gen).to(torch.int32)
    return d, ids, torch.tensor([33], dtype=torch.int32, device="cuda")      # the last seven are not in use


def choice(d, ids, n):
    import paper_1806_03925_amd as g
    _, route = d.choose(g.gear_rmsnorm(d.rows_of(ids, n)[0], d.gain[0], 1e-6).y, n)
    assert (route.expert[33:] == -1).all() and (route.expert[:33] >= 0).all() and int(route.off[-1]) == 99
    return route.expert[:33].long().cpu()


def test_inference(example):
    """An integer is off by at most half a unit, 1/254 of the row's largest value (about 3 times its size): 0.7 % of the operands' size, evenly spread,
    for both operands of two products, and bf16 in between: 0.03 of the result's norm."""
    d, ids, n = small(example)
    got = d.infer(ids, n, torch.float32)[:33].double().cpu()
    want = model(d.features[ids[:33].long()].double().cpu(), *[p.double().cpu() for p in d.params], choice(d, ids, n))
    assert (got - want).norm() < 0.03 * want.norm()


def test_gradients(example):
    """bf16 rounds weights and rows to 2^-8, four products deep: 0.05 of each gradient's norm."""
    d, ids, n = small(example)
    grads = torch.randn(40, 64, device="cuda", generator=torch.Generator(device="cuda").manual_seed(5))
    d.gradients(ids, grads, n)
    params = [p.double().cpu().requires_grad_() for p in d.params]
    out = model(d.features[ids[:33].long()].double().cpu(), *params, choice(d, ids, n))
    (out * grads[:33].double().cpu()).sum().backward()
    for got, p in zip(d.grads, params):
        assert (got.double().cpu() - p.grad).norm() < 0.05 * p.grad.norm()


def test_loop(example):
    st, dense, losses, norms = example.run(4, verbose=False)
    assert int(st.status.item()) == 0 and torch.isfinite(losses).all() and torch.isfinite(norms).all()
    assert int(dense.serve_A.status.item()) == 0 and (dense.bias != 0).any()
    again = example.run(4, verbose=False)
    assert torch.equal(losses, again[2]) and torch.equal(norms, again[3])
