"""The loop of the method closed with a Dense Part whose images choose their experts: python examples/routed_dense_part.py [--steps N]

DFV(image) for an image with features f, its k experts e of `experts` and their weights w by the sigmoids of a learned router:

    h = norm(f),    u = f + sum_e w_e A_e h,    DFV = B norm(u)

Inference for the cache multiplies in 8-bit integers and adds up in fp32.  Back-propagation of a step's averaged gradients (Section 3, step 6) runs in
bf16 with fp32 weights: gradients of all layers and of the router through the weights, clipped together, one SGD step.  No loss
balances the experts: a bias that only the choice sees rises for those with fewer rows than their share and falls for the others.
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_1806_03925_amd as g  # noqa: E402
from gear_inputs import PageViewSource, get_workload  # noqa: E402

EPS = 1e-6


class RoutedDensePart:
    def __init__(self, features: torch.Tensor, experts: int, k: int, dfv_dim: int, max_norm: float, seed: int = 0):
        """features [n_images x dim] bf16."""
        gen = torch.Generator(device=features.device).manual_seed(seed)
        dim, dev = features.shape[1], features.device
        self.features, self.k, self.max_norm = features, k, max_norm
        self.router = torch.randn(experts, dim, device=dev, generator=gen) * dim ** -0.5
        self.A = torch.randn(experts, dim, dim, device=dev, generator=gen) * dim ** -0.5
        self.B = torch.randn(dfv_dim, dim, device=dev, generator=gen) * dim ** -0.5
        self.gain = [torch.ones(dim, device=dev) for _ in range(2)]
        self.bias = torch.zeros(experts, device=dev)
        self.params = [self.router, self.A, self.B, *self.gain]
        self.grads = [torch.zeros_like(p) for p in self.params]
        self.grad_list = g.GradList(self.grads)
        self.train = [g.ExpertWeights(w, operand=torch.bfloat16) for w in self.params[:3]]
        self.publish()

    def rows_of(self, ids: torch.Tensor, n: torch.Tensor):
        """Features of the first n[0] ids (n int32 on the device), and which rows those are."""
        used = torch.arange(ids.numel(), device=ids.device) < n
        return self.features[torch.where(used, ids, 0)], used

    def choose(self, h: torch.Tensor, n: torch.Tensor):
        logits = g.gear_expert_matmul(h, self.train[0], out_dtype=torch.float32)
        return logits, g.gear_route(logits, self.k, score="sigmoid", bias=self.bias, n=n)

    def infer(self, ids: torch.Tensor, n: torch.Tensor, dtype: torch.dtype) -> torch.Tensor:
        """DFV rows of the listed images for the cache; rows from n[0] on are of no image."""
        f, _ = self.rows_of(ids, n)
        h = g.gear_rmsnorm(f, self.gain[0], EPS).y
        _, route = self.choose(h, n)
        y = g.gear_matmul_i8(g.gear_expert_gather_i8(h, route), self.serve_A, route.off, out_dtype=torch.float32)
        u = g.gear_expert_combine(y, route, residual=f, out_dtype=f.dtype)       # one rounding, of the sum
        return g.gear_matmul_i8(g.gear_rows_i8(g.gear_rmsnorm(u, self.gain[1], EPS).y), self.serve_B, out_dtype=dtype)

    def gradients(self, ids: torch.Tensor, dfv_grads: torch.Tensor, n: torch.Tensor):
        """Gradients of sum over the first n[0] rows of dfv_grads[r] . DFV(ids[r]), left in self.grads; returns the route."""
        f, used = self.rows_of(ids, n)
        d = torch.where(used[:, None], dfv_grads, 0.0).to(torch.bfloat16)
        d_router, dA, dB, dgain1, dgain2 = self.grads
        w_router, w_A, w_B = self.train
        h = g.gear_rmsnorm(f, self.gain[0], EPS).y
        logits, route = self.choose(h, n)
        xs = g.gear_expert_gather(h, route)
        y = g.gear_expert_matmul(xs, w_A, route.off)
        u = g.gear_expert_combine(y, route, residual=f)
        v = g.gear_rmsnorm(u, self.gain[1], EPS).y
        g.gear_expert_wgrad(d, v, dw=dB)
        du, _ = g.gear_rmsnorm_backward(u, self.gain[1], g.gear_expert_dgrad(d, w_B), EPS, dgain=dgain2)
        dy, dweight = g.gear_expert_combine_backward(du, y, route)
        g.gear_expert_wgrad(dy, xs, route.off, dw=dA)
        dxs = g.gear_expert_dgrad(dy, w_A, route.off)
        dlogits = g.gear_route_backward(logits, route, dweight, score="sigmoid").to(torch.bfloat16)
        g.gear_expert_wgrad(dlogits, h, dw=d_router)
        dh = g.gear_expert_combine(dxs, route, weighted=False, residual=g.gear_expert_dgrad(dlogits, w_router))
        g.gear_rmsnorm_backward(f, self.gain[0], dh, EPS, dgain=dgain1)
        return route

    def backward(self, ids: torch.Tensor, dfv_grads: torch.Tensor, n: torch.Tensor, lr: float, bias_step: float = 1e-3) -> torch.Tensor:
        """One SGD step on a step's ready list, and one of the experts' balance; returns the gradients' norm before clipping."""
        route = self.gradients(ids, dfv_grads, n)
        norm = g.gear_clip_grads(self.grad_list, self.max_norm)
        for p, d in zip(self.params, self.grads):
            p.sub_(d, alpha=lr)
        for w, p in zip(self.train, self.params):
            w.update(p)
        rows = (route.off[1:] - route.off[:-1]).float()
        self.bias.add_(torch.sign(rows.mean() - rows), alpha=bias_step)
        return norm

    def publish(self) -> None:
        """The weights as they are now become those that inference uses."""
        self.serve_A, self.serve_B = g.gear_weights_i8(self.A), g.gear_weights_i8(self.B)


def run(steps: int, experts: int = 8, k: int = 2, dim: int = 72, expiry: int = 2, verbose: bool = True):
    wl = get_workload("tiny")
    st = g.GearState(g.config_for(wl))
    g.gear_init_tables(st)
    features = torch.empty(wl.n_images, dim, dtype=torch.bfloat16, device="cuda")
    g.gear_fill_normal(features, wl.n_images, dim, wl.seed, 40, 1.0)
    dense = RoutedDensePart(features, experts, k, wl.dfv_dim, max_norm=0.05)
    ids = torch.arange(wl.n_images, dtype=torch.int32, device="cuda")
    everything = torch.tensor([wl.n_images], dtype=torch.int32, device="cuda")
    g.gear_refresh_dfv(st, None, dense.infer(ids, everything, st.dfv_cache.dtype))
    stamp = torch.zeros(wl.n_images, dtype=torch.int32, device="cuda")
    src, losses, norms = PageViewSource(wl), [], []
    for step in range(1, steps + 1):
        batch = g.DeviceBatch.from_host(src.batch(step))
        old, n = g.gear_expired_ids(st, batch.img_id, stamp, step, expiry)
        rows = dense.infer(old, n, st.dfv_cache.dtype)
        g.gear_refresh_dfv_n(st, old, rows, n)
        g.gear_stamp_dfv_n(st, stamp, old, n, step)
        g.gear_step(st, batch, wl.M, wl.lr)
        norms.append(dense.backward(st.ready_ids, st.ready_grads, st.n_ready, lr=0.1))
        dense.publish()
        losses.append(st.loss.clone())
        if verbose:
            print(f"step {step}: loss {losses[-1].item():.6f}, averaged gradients {int(st.n_ready.item())}, their norm {norms[-1].item():.2e}", flush=True)
    if int(g.gear_expert_status().item()) != g.GEAR_OK:       # of all products and weight gradients above
        raise g.GearError(int(g.gear_expert_status().item()), "offsets of a list of images")
    return st, dense, torch.cat(losses), torch.stack(norms)


if __name__ == "__main__":
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--steps", type=int, default=8)
    run(p.parse_args().steps)
