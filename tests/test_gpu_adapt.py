"""The operators together: adapters of the decoder tuned by the tags' log-probabilities, and answers for a few
samples."""
import numpy as np
import pytest
import torch

from paper_1704_06363_amd import adapt, hmoe
from paper_1704_06363_amd import workloads as W
from tests.parity import np64, npi

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_tuning_raises_the_log_probabilities(dtype):
    means, a = adapt.main(steps=12, dtype=dtype, n=1000, show=False)
    assert len(means) == 12 and all(np.isfinite(means))
    assert means[-1] > means[0] + 0.5  # a bias per cluster alone is worth ln 8 nats
    assert (np.diff(npi(a["logp"].float()), axis=1) <= 0).all()


def test_the_first_step_is_the_gradient_of_the_mean():
    """A step of rate lr moves the mean by lr |gradient|^2 to first order; B starts at zero, so the first step moves B
    alone, and the mean by lr |dB|^2: against the plain change of the mean in 64 bits, to the second order's 5%."""
    n, lr = 300, 1e-2
    c = W.CONFIGS["tiny"]
    g = torch.Generator(device="cuda").manual_seed(1)
    p = W.moe_params(c.K, c.d, c.h, c.o, c.V, 2, "f32", "cuda", bias=True)
    m = adapt.Adapted(torch.randn(c.K, c.d, generator=g, device="cuda"), p, rank=8, seed=3)
    H = torch.randn(n, c.o, generator=g, device="cuda")
    cluster = torch.randint(0, c.K, (n,), generator=g, device="cuda", dtype=torch.int32)
    tag = torch.randint(0, c.V, (n,), generator=g, device="cuda", dtype=torch.int32)

    def mean():
        h, A, B = np64(H), np64(m.A), np64(m.B)
        z = h @ np64(p["D"]).T + np64(p["bD"])
        for i, e in enumerate(npi(cluster)):
            z[i] += B[e] @ (A[e] @ h[i])
        z -= z.max(1, keepdims=True)
        return (z[np.arange(n), npi(tag)] - np.log(np.exp(z).sum(1))).mean()

    before = mean()
    logp = m.tune_step(H, cluster, tag, lr)
    assert abs(logp.mean().item() - before) <= 1e-5 * abs(before) + 1e-5
    moved = (np64(m.B) / lr) ** 2
    assert mean() - before == pytest.approx(lr * moved.sum(), rel=0.05)


def test_answers_are_those_of_the_parts():
    c = W.CONFIGS["tiny"]
    p = W.moe_params(c.K, c.d, c.h, c.o, c.V, 2, "f32", "cuda", bias=True)
    C = W.gmm_means(c.K, c.d, 5, "cuda")
    m = adapt.Adapted(C, p, rank=16, seed=3)
    m.B.normal_(generator=torch.Generator(device="cuda").manual_seed(4))
    X = C[torch.arange(30, device="cuda") % c.K] + 0.1
    a = m.answer(X, m=4)
    assert torch.equal(a["cluster"], hmoe.kmeans_assign(X, C)[0])
    x, e = np64(X), npi(a["cluster"])
    for i in range(30):
        h = np.maximum(np64(p["W1"])[e[i]] @ x[i] + np64(p["b1"])[e[i]], 0)
        y = np64(p["W2"])[e[i]] @ h + np64(p["b2"])[e[i]]
        z = np64(p["D"]) @ y + np64(p["bD"]) + np64(m.B)[e[i]] @ (np64(m.A)[e[i]] @ y)
        lp = z - z.max() - np.log(np.exp(z - z.max()).sum())
        order = np.argsort(-lp, kind="stable")[:4]
        gaps = -np.diff(lp[np.argsort(-lp)[:5]])
        if gaps.min() > 1e-4:
            assert np.array_equal(npi(a["tag"])[i], order)
        assert np.abs(np64(a["logp"])[i] - lp[order]).max() <= 1e-3
        assert abs(a["entropy"][i].item() + (np.exp(lp) * lp).sum()) <= 1e-3
