"""A radial network of a many-element model: trained, fine-tuned for two requests, and served.

Message passing takes the radial features `edge_radial` [E, C, L] as given. Here a small network makes
them from the 8 Gaussians of each edge's distance:

    hidden = silu(w1[pair of elements]^T g)                                    (grouped_layer)
    edge_radial = w2^T hidden + scale[request] b[request]^T (a[request]^T hidden)  (adapter_linear)

1. w1 and w2 learn given radial features (grouped_linear_grad, grouped_layer_grad, adamw with states in 8 bits).
2. w1 and w2 stay; every request learns its own change of them by its adapter
   (adapter_linear_grad, adamw with states in 32 bits).
3. One message pass serves all requests at once, and the atoms of none, which keep the base model.

    python examples/radial_network.py
"""
from __future__ import annotations

import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2605_15073_amd as cg  # noqa: E402
from paper_2605_15073_amd import inputs  # noqa: E402


class Model:
    """Weights and the orders of the rows (edges) of one batch of structures."""

    def __init__(self, n_atoms, elements, hidden, lmax, C, rank, seed):
        dev, rng = torch.device("cuda"), np.random.default_rng(seed)
        to = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(dev)
        d = inputs.mp_inputs(n_atoms, lmax, C, C, seed, r_cut=4.0)
        self.plan = cg.plan_create(lmax, C, C)
        self.call = {k: to(d[k]) for k in ("row_ptr", "col", "edge_unit", "edge_radial", "node_feat",
                                           "U_E", "U_I", "U_out_even", "U_out_odd")}
        E = d["n_edges"]
        self.width = C * (lmax + 1)
        self.target = self.call["edge_radial"].reshape(E, self.width)
        receiver = np.repeat(np.arange(n_atoms), np.diff(d["row_ptr"]))
        self.g = to(self._basis(n_atoms, seed, 4.0))
        # pairs of elements, and the request of the structure an atom belongs to (thirds: 0, 1, none)
        z = rng.integers(0, elements, n_atoms)
        lo, hi = np.minimum(z[receiver], z[d["col"]]), np.maximum(z[receiver], z[d["col"]])
        pairs = elements * (elements + 1) // 2
        request = np.where(3 * receiver // n_atoms == 2, -1, 3 * receiver // n_atoms)
        self.request = to(request.astype(np.int32))
        self.by_pair = cg.group_rows(to((hi * (hi + 1) // 2 + lo).astype(np.int32)), pairs)
        self.by_request = cg.group_rows(self.request, 2)
        self.all_rows = cg.group_rows(torch.zeros(E, dtype=torch.int32, device=dev), 1)
        normal = lambda *s, by=1.0: to((rng.standard_normal(s) * by).astype(np.float32))
        self.w1 = normal(pairs, 8, hidden, by=8 ** -0.5)
        self.w2 = normal(hidden, self.width, by=0.1 * hidden ** -0.5)
        self.a = normal(2, hidden, rank, by=hidden ** -0.5)
        self.b = torch.zeros(2, rank, self.width, device=dev)   # adapters start without effect
        self.scale = torch.tensor([1.0, 0.5], device=dev)

    @staticmethod
    def _basis(n_atoms, seed, r_cut):
        """The Gaussians of each edge's distance, of the positions that inputs.mp_inputs draws."""
        rng = np.random.default_rng(seed)
        box = (n_atoms / 0.1) ** (1.0 / 3.0)
        pos = rng.uniform(0.0, box, size=(n_atoms, 3))
        dist = inputs.periodic_neighbours(pos, box, r_cut)[3]
        return inputs.gaussian_radial(dist, r_cut).astype(np.float32)

    def hidden(self, z=False):
        """The hidden features; with z None (features, what the activation took)."""
        return cg.grouped_layer(self.g, self.w1, *self.by_pair, activation="silu", z=z)

    def radial(self, h):
        return cg.adapter_linear(h, self.w2, self.a, self.b, *self.by_request, scale=self.scale)

    def train(self, steps, lr):
        """w1 and w2 on the target, with no adapter's effect yet; returns the losses."""
        weights = [self.w1, self.w2]
        grads = [torch.empty_like(w) for w in weights]
        codes = lambda t: [torch.zeros(w.shape, dtype=t, device="cuda") for w in weights]
        scales = lambda: [torch.zeros(-(-w.numel() // cg.CGTP_ADAMW_BLOCK), device="cuda")
                          for w in weights]
        opt = cg.AdamWTensors(weights, grads, codes(torch.int8), codes(torch.uint8), scales(), scales())
        losses = []
        for step in range(1, steps + 1):
            h, z = self.hidden(z=None)
            err = self.radial(h) - self.target
            losses.append(err.square().mean())
            dy = err * (2.0 / err.numel())
            dh, _ = cg.grouped_linear_grad(h, self.w2[None], dy, *self.all_rows, dw=grads[1][None])
            cg.grouped_layer_grad(self.g, self.w1, dh, *self.by_pair, z=z, activation="silu", dx=False,
                                  dw=grads[0], dbias=False)
            cg.adamw(opt, step=step, lr=lr, weight_decay=0.0)
        return torch.stack(losses).tolist()

    def fine_tune(self, target, steps, lr):
        """The adapters alone, towards another target; returns the losses."""
        weights = [self.a, self.b]
        grads = [torch.empty_like(w) for w in weights]
        zeros = lambda: [torch.zeros_like(w) for w in weights]
        opt = cg.AdamWTensors(weights, grads, zeros(), zeros())
        h = self.hidden()
        losses = []
        for step in range(1, steps + 1):
            err = self.radial(h) - target
            losses.append(err.square().mean())
            dy = err * (2.0 / err.numel())
            cg.adapter_linear_grad(h, self.w2, self.a, self.b, dy, *self.by_request, scale=self.scale,
                                   dx=False, da=grads[0], db=grads[1])
            cg.adamw(opt, step=step, lr=lr, weight_decay=0.0)
        return torch.stack(losses).tolist()

    def serve(self):
        """One message pass over the whole batch: (radial features, out_even, out_odd)."""
        y = self.radial(self.hidden())
        t = dict(self.call, edge_radial=y.view_as(self.call["edge_radial"]))
        return y, *cg.message_pass(self.plan, *t.values())


def main(n_atoms=600, elements=4, hidden=32, lmax=2, C=16, rank=8, steps=120, seed=0):
    m = Model(n_atoms, elements, hidden, lmax, C, rank, seed)
    first = m.train(steps, 1e-2)
    base = m.serve()
    # each request's own data: the base features, bent in its own way; none for the other atoms
    bend = torch.zeros_like(base[0])
    for k in (0, 1):
        rows = m.request == k
        bend[rows] = 0.3 * torch.sin((2 + k) * base[0][rows])
    tuned = m.fine_tune(base[0] + bend, steps, 1e-2)
    served = m.serve()
    return m, dict(train=first, fine_tune=tuned), base, served


if __name__ == "__main__":
    _, losses, base, served = main()
    for name, v in losses.items():
        print(f"{name}: mean squared error {v[0]:.3e} -> {v[-1]:.3e} in {len(v)} steps")
    change = [(s - b).abs().max().item() for s, b in zip(served, base)]
    print("largest change by the adapters: radial features %.3f, out_even %.3f, out_odd %.3f"
          % tuple(change))
