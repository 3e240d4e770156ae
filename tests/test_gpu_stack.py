"""The operators of hmoe_train.h together with the dispatch, the adapters and the log-probabilities: a stack of layers
whose routers learn, its gradients against automatic differentiation of the formulas in 64 bits."""
import numpy as np
import pytest
import torch

from paper_1704_06363_amd import stack

pytestmark = pytest.mark.gpu


def loss64(m, w, X, tag, choices, counts, balance, z, top_k):
    """The loss in 64 bits on the CPU with the choices and counts that the routers made."""
    def unit(t):
        return t / torch.sqrt(t.pow(2).mean(-1, keepdim=True) + 1e-6)

    n = X.shape[0]
    x, total = X, 0.0
    h = unit(x) * w["gamma"]
    for i, W in enumerate(m.fixed):
        s = h @ w[f"R{i}"].t() + w[f"bias{i}"]
        p = torch.softmax(s, 1)
        e = choices[i]
        weight = p.gather(1, e)
        if top_k > 1:
            weight = weight / weight.sum(1, keepdim=True)
        E = s.shape[1]
        total = total + balance * E * (counts[i] / (n * top_k) * p.mean(0)).sum() + z * torch.logsumexp(s, 1).pow(2).mean()
        base = h @ W.double().cpu().t()
        y = torch.stack([base + torch.einsum("nor,nri,ni->no", w[f"B{i}"][e[:, j]], w[f"A{i}"][e[:, j]], h)
                         for j in range(top_k)], 1)
        x = x + (weight[:, :, None] * unit(y) * w[f"gamma_y{i}"]).sum(1)
        h = unit(x) * w[f"gamma_h{i}"]
    logp = torch.log_softmax(h @ m.D.double().cpu().t(), 1)
    return total - logp[torch.arange(n), tag.long().cpu()].mean()


@pytest.mark.parametrize("top_k", [1, 2])
def test_gradients(top_k):
    """fp32.  A gradient is a sum of products through two layers, each value good to some dozens of 2^-24; relative to
    its largest entry 1e-4 leaves a factor of ten for sums that cancel."""
    n, d, E, V = 300, 64, 6, 200
    m = stack.Stack(2, d, E, V, rank=8, top_k=top_k, dtype="f32", seed=1)
    g = torch.Generator(device="cuda").manual_seed(2)
    X = torch.randn(n, d, generator=g, device="cuda")
    tag = torch.randint(0, V, (n,), generator=g, device="cuda", dtype=torch.int32)
    balance, z = 0.5, 0.1
    logp, losses, got = m.gradients(X, tag, balance, z)
    kept = m.forward(X)[1]
    choices = [c["router"]["expert"].long().cpu() for c in kept]
    counts = [c["router"]["counts"].double().cpu() for c in kept]
    w = {k: v.detach().double().cpu().requires_grad_() for k, v in m.w.items()}
    loss = loss64(m, w, X.double().cpu(), tag, choices, counts, balance, z, top_k)
    ours = -logp.double().mean().item() + sum((balance * v[0] + z * v[1]).item() for v in losses)
    assert abs(ours - loss.item()) <= 1e-5 * abs(loss.item())
    want = torch.autograd.grad(loss, list(w.values()))
    for (k, _), ref in zip(w.items(), want):
        ref = ref.numpy()
        err = np.abs(got[k].double().cpu().numpy() - ref).max()
        assert err <= 1e-4 * np.abs(ref).max(), (k, err, np.abs(ref).max())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_runs(dtype):
    means, losses = stack.main(steps=4, dtype=dtype, n=1000, show=False)
    assert len(means) == 4 and all(np.isfinite(means)) and len(losses) == 2
    assert all(torch.isfinite(v).all() for v in losses)


def test_the_step_is_the_update_of_the_gradients():
    n, d, E, V = 128, 64, 4, 96
    a, b = (stack.Stack(1, d, E, V, top_k=2, dtype="bf16", seed=3) for _ in range(2))
    g = torch.Generator(device="cuda").manual_seed(4)
    X = torch.randn(n, d, generator=g, device="cuda").bfloat16()
    tag = torch.randint(0, V, (n,), generator=g, device="cuda", dtype=torch.int32)
    _, _, grad = a.gradients(X, tag)
    before = {k: v.clone() for k, v in a.w.items()}
    b.step(X, tag, lr=0.05)
    for k in a.w:
        moved = b.w[k] - before[k]
        assert torch.isfinite(moved).all()
        if a.w[k].dim() == 1:
            assert torch.allclose(moved, -0.05 * grad[k], rtol=1e-4, atol=1e-7), k
        else:  # an update against the gradient, and as large in every direction as the coefficients leave it
            assert (moved * grad[k]).sum() < 0, k
        if b.low[k] is not b.w[k]:
            assert torch.equal(b.low[k], b.w[k].to(b.low[k].dtype)), k
