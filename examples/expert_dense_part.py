"""The loop of the method closed with a Dense Part of experts: python examples/expert_dense_part.py [--steps N]

Images are of several kinds and numbered kind by kind, so that the ascending lists the framework works with (the ready list
of a step, the expired images of a batch) are already grouped by kind: where each kind's rows begin is one search in the
list, and nothing is sorted or copied to the host.  DFV(image) for an image with features f and kind e:

    u = A_e norm(f),    DFV = B_e norm(u + f)

Inference for the cache runs in 8 bits.  Back-propagation of a step's averaged gradients (Section 3, step 6) runs in bf16
with fp32 weights: both layers' gradients, clipped together by their global norm, one SGD step, and the weights laid out
again for either use.
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


class ExpertDensePart:
    def __init__(self, features: torch.Tensor, kind_first: torch.Tensor, dfv_dim: int, max_norm: float, seed: int = 0):
        """features [n_images x dim] bf16; kind_first [kinds + 1] int32: images of kind e are kind_first[e] .. kind_first[e + 1)."""
        gen = torch.Generator(device=features.device).manual_seed(seed)
        kinds, dim, dev = kind_first.numel() - 1, features.shape[1], features.device
        self.features, self.kind_first, self.max_norm = features, kind_first, max_norm
        self.A = torch.randn(kinds, dim, dim, device=dev, generator=gen) * dim ** -0.5
        self.B = torch.randn(kinds, dfv_dim, dim, device=dev, generator=gen) * dim ** -0.5
        self.gain = [torch.ones(dim, device=dev) for _ in range(2)]
        self.params = [self.A, self.B, *self.gain]
        self.grads = [torch.zeros_like(p) for p in self.params]
        self.grad_list = g.GradList(self.grads)
        self.train_A, self.train_B = (g.ExpertWeights(w, operand=torch.bfloat16) for w in (self.A, self.B))
        self.serve_A, self.serve_B = g.gear_weights8(self.A), g.gear_weights8(self.B)

    def rows_of(self, ids: torch.Tensor, n: torch.Tensor):
        """Features of the first n[0] ids (ascending; n on the device) and where each kind's rows begin among them."""
        used = torch.arange(ids.numel(), device=ids.device) < n
        ids = torch.where(used, ids, self.features.shape[0])            # behind every kind
        off = torch.searchsorted(ids, self.kind_first, out_int32=True)
        return self.features[ids.clamp(max=self.features.shape[0] - 1)], off, used

    def infer(self, ids: torch.Tensor, n: torch.Tensor, dtype: torch.dtype) -> torch.Tensor:
        """DFV rows of the listed images for the cache; rows from n[0] on are not written."""
        f, off, _ = self.rows_of(ids, n)
        y = g.gear_rmsnorm(f, self.gain[0], EPS, y=False, q8=True).rows8
        u = g.gear_matmul8(y, self.serve_A, off)
        y = g.gear_rmsnorm(u, self.gain[1], EPS, residual=f, y=False, q8=True).rows8
        return g.gear_matmul8(y, self.serve_B, off, out_dtype=dtype)

    def gradients(self, ids: torch.Tensor, dfv_grads: torch.Tensor, n: torch.Tensor) -> None:
        """Gradients of sum over the first n[0] rows of dfv_grads[r] . DFV(ids[r]), left in self.grads."""
        f, off, used = self.rows_of(ids, n)
        d = torch.where(used[:, None], dfv_grads, 0.0).to(torch.bfloat16)
        _, y1, _ = g.gear_rmsnorm(f, self.gain[0], EPS)
        u = g.gear_expert_matmul(y1, self.train_A, off, out=torch.zeros_like(f))      # rows of no kind stay zero
        h, y2, _ = g.gear_rmsnorm(u, self.gain[1], EPS, residual=f)
        dA, dB, dgain1, dgain2 = self.grads
        g.gear_expert_wgrad(d, y2, off, dw=dB)
        dy2 = g.gear_expert_dgrad(d, self.train_B, off, out=torch.zeros_like(f))
        du, _ = g.gear_rmsnorm_backward(h, self.gain[1], dy2, EPS, dgain=dgain2)
        g.gear_expert_wgrad(du, y1, off, dw=dA)
        dy1 = g.gear_expert_dgrad(du, self.train_A, off, out=torch.zeros_like(f))
        g.gear_rmsnorm_backward(f, self.gain[0], dy1, EPS, dgain=dgain1)

    def backward(self, ids: torch.Tensor, dfv_grads: torch.Tensor, n: torch.Tensor, lr: float) -> torch.Tensor:
        """One SGD step on a step's ready list; returns the gradients' norm before clipping."""
        self.gradients(ids, dfv_grads, n)
        norm = g.gear_clip_grads(self.grad_list, self.max_norm)
        for p, d in zip(self.params, self.grads):
            p.sub_(d, alpha=lr)
        self.train_A.update(self.A)
        self.train_B.update(self.B)
        return norm

    def publish(self) -> None:
        """The weights as they are now become those that inference uses."""
        self.serve_A, self.serve_B = g.gear_weights8(self.A), g.gear_weights8(self.B)


def run(steps: int, kinds: int = 5, dim: int = 72, expiry: int = 2, verbose: bool = True):
    wl = get_workload("tiny")
    st = g.GearState(g.config_for(wl))
    g.gear_init_tables(st)
    features = torch.empty(wl.n_images, dim, dtype=torch.bfloat16, device="cuda")
    g.gear_fill_normal(features, wl.n_images, dim, wl.seed, 40, 1.0)
    kind_first = torch.linspace(0, wl.n_images, kinds + 1, device="cuda").to(torch.int32)
    dense = ExpertDensePart(features, kind_first, wl.dfv_dim, max_norm=0.05)
    ids = torch.arange(wl.n_images, dtype=torch.int32, device="cuda")
    g.gear_refresh_dfv(st, None, dense.infer(ids, torch.tensor([wl.n_images], device="cuda"), st.dfv_cache.dtype))
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
