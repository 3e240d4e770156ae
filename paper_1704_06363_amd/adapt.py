"""A hard mixture that answers a few samples at a time, and whose decoder is adapted per cluster.

The shared decoder of the paper's Section 2 gets a low-rank adapter for every cluster of the gater: decoders of
their own for the experts at a small part of the independent decoders' parameters.

  answer     features of a few samples -> gater and experts (moe_few) -> decoder with the cluster's
             adapter (lora_few) -> the most probable tags, with log-probabilities and the entropy (token_logprob);
             with bf16 parameters the logits between the two are plain bf16, good to 2^-9 of their size
  tune_step  one step of the adapters on samples with a tag each: rows by cluster (moe_dispatch), decoder with
             adapters (lora_forward), log-probabilities of the tags (token_logprob), their gradient back
             (token_logprob_backward, lora_backward), and the update (sgd_step)

    python -m paper_1704_06363_amd.adapt [--steps N] [--dtype bf16]

fits a gater on synthetic features, tunes the adapters on tags that depend on the cluster, and answers.
"""
from __future__ import annotations

import argparse

import torch

from . import hmoe
from . import workloads as W


class Adapted:
    """A gater's centres C [K, d] (fp32), the experts and shared decoder of a parameter dict (workloads.moe_params),
    and one adapter per cluster beside the decoder."""

    def __init__(self, C, params: dict, rank: int = 8, scale: float = 1.0, seed: int = 0):
        self.dtype = params["W1"].dtype
        K, V, o = params["W1"].shape[0], params["D"].shape[0], params["D"].shape[1]
        dev = C.device
        R = C.to(self.dtype)
        # Eq. 2 as scores: the nearest centre has the largest x . c - |c|^2 / 2
        self.experts = {k: params.get(k) for k in ("W1", "b1", "W2", "b2")}
        self.experts.update(R=R, r_bias=-0.5 * R.double().pow(2).sum(1).float())
        g = torch.Generator(device=dev)
        g.manual_seed(seed)
        self.A = torch.randn(K, rank, o, generator=g, device=dev) * o ** -0.5  # fp32 master weights
        self.B = torch.zeros(K, V, rank, device=dev)
        low = self.dtype != torch.float32
        self.decoder = {"W": params["D"], "b": params.get("bD"), "A": self.A.to(self.dtype) if low else self.A,
                        "B": self.B.to(self.dtype) if low else self.B,
                        "scale": torch.full((K,), scale, device=dev)}

    def answer(self, X, m: int = 5, temperature: float = 1.0):
        """For up to hmoe.FEW_ROWS samples: the cluster of each, its m most probable tags with their
        log-probabilities, and the entropy of its distribution."""
        f = hmoe.moe_few(self.experts, X)
        cluster = f["expert"][:, 0].contiguous()
        logits = hmoe.lora_few(self.decoder, f["Y"], cluster)
        t = hmoe.token_logprob(logits, m=m, scale=1.0 / temperature)
        return {"cluster": cluster, "tag": t["top_idx"], "logp": t["top_logp"], "entropy": t["entropy"]}

    def tune_step(self, H, cluster, tag, lr: float, entropy_weight: float = 0.0):
        """One step that raises the mean of the tags' log-probabilities (plus entropy_weight times the entropies) of
        samples with the experts' outputs H [n, o].  Returns the log-probabilities before it."""
        n, K = H.shape[0], self.A.shape[0]
        d = hmoe.moe_dispatch(cluster, K, rows=H)
        f = hmoe.lora_forward(self.decoder, d["rows_sorted"], d["offsets"], d["perm"])
        t = hmoe.token_logprob(f["Y"], tag)
        down = torch.full((n,), -1.0 / n, device=H.device)
        dY = hmoe.token_logprob_backward(f["Y"], tag, t["stat"], t["entropy"], down,
                                         down * entropy_weight if entropy_weight else None, out=f["Y"])
        g = hmoe.lora_backward(self.decoder, d["rows_sorted"], d["offsets"], dY, f["U"], d["perm"], want_dX=False)
        for w, grad, k in ((self.A, g["dA"], "A"), (self.B, g["dB"], "B")):
            low = self.decoder[k]
            hmoe.sgd_step(w, grad, lr, w_lo=None if low is w else low)
        return t["logp"]


def main(steps: int = 30, dtype: str = "bf16", n: int = 2048, lr: float = 0.5, seed: int = 0, show: bool = True):
    """Returns the mean log-probability of the tags at every step, and the answers at the end."""
    c = W.CONFIGS["tiny"]
    dev, dt = "cuda", W.torch_dtype(dtype)
    X = W.gmm_features(n, c.d, c.extra["n_comp"], seed, dtype, dev)
    params = W.moe_params(c.K, c.d, c.h, c.o, c.V, seed + 20, dtype, dev, bias=True)
    C = hmoe.kmeans_fit(X, c.K, 5, init_uniforms=W.uniforms(c.K, seed + 30))["C"]
    model = Adapted(C, params, rank=8, seed=seed + 40)
    cluster, _ = hmoe.kmeans_assign(X, C.to(dt))
    d = hmoe.moe_dispatch(cluster, c.K, rows=X)
    row_ptr, tag = W.zipf_labels(n, c.V, 1, seed + 10)  # one tag each: of a part of the vocabulary per cluster
    tag = (torch.tensor(tag, device=dev) % (c.V // c.K) + cluster * (c.V // c.K)).to(torch.int32)
    H = hmoe.moe_forward(params, d["rows_sorted"], d["offsets"], d["perm"], torch.tensor(row_ptr, device=dev), tag)["H"]
    means = []
    for s in range(steps):
        means.append(model.tune_step(H, cluster, tag, lr).mean().item())
        if show and s % 10 == 0:
            print(f"step {s}: mean log-probability {means[-1]:.4f}", flush=True)
    a = model.answer(X[:8])
    if show:
        for i in range(8):
            tags = ", ".join(f"{t} ({p:.2f})" for t, p in zip(a["tag"][i].tolist(), a["logp"][i].tolist()))
            print(f"sample {i}, cluster {a['cluster'][i].item()}, entropy {a['entropy'][i].item():.2f}: {tags}")
    return means, a


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=30)
    ap.add_argument("--dtype", choices=("bf16", "f32"), default="bf16")
    args = ap.parse_args()
    main(args.steps, args.dtype)
