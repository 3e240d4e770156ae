"""Layers of adapters whose routers learn, trained: a residual stack in which every sample goes to the experts that a
layer's router chooses for it, each of them a low-rank adapter beside the layer's shared projection.

  layer      h -> the router's choices and weights (router_forward) -> rows by expert (moe_dispatch; torch copies them
             first for more than one choice) -> projection with the expert's adapter (lora_forward) -> norm, gate by
             the weights, residual and the norm before the next layer (join_forward)
  gradients  of the mean of -ln p(tag) (token_logprob over a shared decoder) plus the routers' balance and z losses:
             token_logprob_backward, lora_backward, join_backward, router_backward, layer by layer; join_forward adds up
             what comes back to a layer's input
  step       orthogonalised updates (muon_step) of the adapters and the routers' rows, sgd_step for gains and biases

    python -m paper_1704_06363_amd.stack [--steps N] [--dtype bf16]

trains two layers on synthetic features whose tags depend on the cluster.
"""
from __future__ import annotations

import argparse

import torch

from . import hmoe
from . import workloads as W


class Stack:
    """`layers` layers of width d with E experts of which each sample takes top_k, on a shared decoder D [V, d].  Master
    weights are fp32; with bf16 the products take copies in bf16."""

    def __init__(self, layers: int, d: int, E: int, V: int, rank: int = 8, top_k: int = 1, dtype: str = "bf16", device="cuda",
                 seed: int = 0):
        self.dtype, self.top_k = W.torch_dtype(dtype), top_k
        g = torch.Generator(device=device)
        g.manual_seed(seed)
        rand = lambda *s, std: torch.randn(*s, generator=g, device=device) * std
        self.D = rand(V, d, std=d ** -0.5).to(self.dtype)
        self.w, self.fixed = {"gamma": torch.ones(d, device=device)}, []  # the first norm's gain
        for i in range(layers):
            self.w.update({f"R{i}": rand(E, d, std=d ** -0.5), f"bias{i}": torch.zeros(E, device=device),
                           f"A{i}": rand(E, rank, d, std=d ** -0.5), f"B{i}": rand(E, d, rank, std=0.1 * rank ** -0.5),
                           f"gamma_y{i}": torch.full((d,), 0.5, device=device), f"gamma_h{i}": torch.ones(d, device=device)})
            self.fixed.append(rand(d, d, std=d ** -0.5).to(self.dtype))
        # what the products take: biases stay fp32
        low = self.dtype != torch.float32
        self.low = {k: w.to(self.dtype) if low and not k.startswith("bias") else w for k, w in self.w.items()}
        self.v = {k: torch.zeros_like(w) for k, w in self.w.items()}
        none = torch.zeros(1, 8, d, device=device, dtype=self.dtype)
        self.head = {"W": self.D, "A": none, "B": torch.zeros(1, V, 8, device=device, dtype=self.dtype)}
        self.no_rows = torch.zeros(2, dtype=torch.int32, device=device)

    def _layer(self, i):
        p = self.low
        return {"W": self.fixed[i], "A": p[f"A{i}"], "B": p[f"B{i}"]}, {"R": p[f"R{i}"], "bias": p[f"bias{i}"]}

    def forward(self, X):
        """The last norm's rows, and what the gradients need of every layer."""
        p, k = self.low, self.top_k
        x, h = X, hmoe.join_forward(X, gamma_h=p["gamma"], want_x=False)["h"]
        kept = []
        for i in range(len(self.fixed)):
            lora, router = self._layer(i)
            r = hmoe.router_forward(router, h, top_k=k, renorm=k > 1)
            rows = h if k == 1 else h.repeat_interleave(k, 0)
            s = hmoe.moe_dispatch(r["expert"].view(-1), p[f"R{i}"].shape[0], rows=rows)
            f = hmoe.lora_forward(lora, s["rows_sorted"], s["offsets"], s["perm"])
            y = f["Y"].view(-1, k, f["Y"].shape[1])
            j = hmoe.join_forward(x, y, gate=r["weight"], gamma_y=p[f"gamma_y{i}"], gamma_h=p[f"gamma_h{i}"])
            kept.append({"h": h, "router": r, "sorted": s, "lora": f, "y": y, "x": j["x"]})
            x, h = j["x"], j["h"]
        return h, kept

    def gradients(self, X, tag, balance: float = 0.01, z: float = 0.001):
        """(log-probabilities of the tags [n], each layer's losses [2], gradients of every weight in fp32)."""
        n, p, k, g = X.shape[0], self.low, self.top_k, {}
        h, kept = self.forward(X)
        out = hmoe.lora_forward(self.head, h, self.no_rows)
        t = hmoe.token_logprob(out["Y"], tag)
        down = torch.full((n,), -1.0 / n, device=X.device)
        dY = hmoe.token_logprob_backward(out["Y"], tag, t["stat"], g_logp=down, out=out["Y"])
        dh = hmoe.lora_backward(self.head, h, self.no_rows, dY, out["U"], want_adapters=False)["dX"]
        dx = None
        for i in reversed(range(len(self.fixed))):
            lora, router = self._layer(i)
            c = kept[i]
            b = hmoe.join_backward(c["x"], c["y"], gate=c["router"]["weight"], gamma_y=p[f"gamma_y{i}"],
                                   gamma_h=p[f"gamma_h{i}"], dx_out=dx, dh=dh)
            s = c["sorted"]
            e = hmoe.lora_backward(lora, s["rows_sorted"], s["offsets"], b["dy"].view(n * k, -1), c["lora"]["U"], s["perm"])
            r = hmoe.router_backward(router, c["h"], c["router"], b["dgate"], balance, z, renorm=k > 1)
            g.update({f"A{i}": e["dA"], f"B{i}": e["dB"], f"R{i}": r["dR"], f"bias{i}": r["dbias"],
                      f"gamma_y{i}": b["dgamma_y"], f"gamma_h{i}": b["dgamma_h"]})
            # what comes back from the router and from every choice, in 32 bits and rounded once
            dx, dh = b["dx"], hmoe.join_forward(r["dX"], e["dX"].view(n, k, -1), norm_y=False, want_h=False)["x"]
        g["gamma"] = hmoe.join_backward(X, gamma_h=p["gamma"], dh=dh, want=("dgamma_h",))["dgamma_h"]
        return t["logp"], [c["router"]["loss"] for c in kept], g

    def step(self, X, tag, lr: float = 0.02, balance: float = 0.01, z: float = 0.001):
        """One step; returns the log-probabilities and the routers' losses before it."""
        logp, losses, g = self.gradients(X, tag, balance, z)
        for k, w in self.w.items():
            lo = None if self.low[k] is w else self.low[k]
            if w.dim() > 1:
                hmoe.muon_step(w, g[k], self.v[k], lr=lr, scale=max(1.0, w.shape[-2] / w.shape[-1]) ** 0.5, w_lo=lo)
            else:
                hmoe.sgd_step(w, g[k], lr, momentum=0.9, v=self.v[k], w_lo=lo)
        return logp, losses


def main(steps: int = 30, dtype: str = "bf16", n: int = 2048, seed: int = 0, show: bool = True):
    """Returns the mean log-probability of the tags at every step, and the last routers' losses."""
    c = W.CONFIGS["tiny"]
    dev = "cuda"
    X = W.gmm_features(n, c.d, c.extra["n_comp"], seed, dtype, dev)
    C = hmoe.kmeans_fit(X, c.K, 5, init_uniforms=W.uniforms(c.K, seed + 30))["C"]
    cluster, _ = hmoe.kmeans_assign(X, C.to(X.dtype))
    row_ptr, tag = W.zipf_labels(n, c.V, 1, seed + 10)  # one tag each: of a part of the vocabulary per cluster
    tag = (torch.tensor(tag, device=dev) % (c.V // c.K) + cluster * (c.V // c.K)).to(torch.int32)
    model = Stack(2, c.d, c.K, c.V, dtype=dtype, seed=seed + 40)
    means = []
    for s in range(steps):
        logp, losses = model.step(X, tag)
        means.append(logp.mean().item())
        if show and s % 10 == 0:
            print(f"step {s}: mean log-probability {means[-1]:.4f}, balance "
                  + ", ".join(f"{v[0].item():.3f}" for v in losses), flush=True)
    return means, losses


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=30)
    ap.add_argument("--dtype", choices=("bf16", "f32"), default="bf16")
    args = ap.parse_args()
    main(args.steps, args.dtype)
