"""Each kind of tile that the products of orthogonalised updates choose, for iterations and for the step with momentum,
wide and tall, against the formulas in 64 bits.  The launches' labels say that a case runs what it is here for.

Bounds.  Iterates are off by 8 2^-22 |a|^steps / sqrt(rank) of the result's norm, or by 8 2^-22 steps: two fp16 numbers hold
22 bits, a step rounds A, b A + c A^2 and X and drops the products of the low parts, and a small singular value grows
by a at most.  The update's U = g + momentum v is rounded in fp32, 2^-23 of it at most, which grows as much.  An entry
of w is rounded twice, 2^-24 of what is kept of it and of the result; momentum, rate and decay are such that nothing else
is."""
import pytest
import torch

from paper_1704_06363_amd import hmoe

pytestmark = pytest.mark.gpu

A, B, C = hmoe.COEF
U = 2.0 ** -24

# K, rows, cols, and the height of the tiles of X X^T, of the squares, and of the products with X on 256 CUs
CASES = [(3, 200, 136, (64, 64, 64)), (1, 272, 1504, (64, 64, 64)), (2, 64, 8200, (64, 64, 64)),
         (24, 264, 200, (128, 64, 128)), (70, 100, 504, (128, 64, 128)), (2, 700, 1032, (128, 64, 128)),
         (1, 2500, 640, (128, 64, 128)), (5, 600, 640, (128, 128, 128)), (16, 1024, 512, (128, 128, 128)),
         (1, 2048, 2056, (128, 128, 256)), (3, 1000, 5000, (256, 128, 256)), (2, 2048, 4096, (256, 256, 256)),
         (2, 4096, 2048, (256, 256, 256)), (2, 2056, 4104, (256, 256, 256)), (2, 4100, 1992, (256, 256, 256))]


def rand(*shape, seed=0):
    return torch.randn(*shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda")


def launched(call):
    """What `call` returns, and the labels of the products that it launched."""
    hmoe.timer_enable(True)
    try:
        out = call()
        labels = hmoe.timer_report()
    finally:
        hmoe.timer_enable(False)
    return out, {k for k in labels if k.split()[-1].isdigit()}


def names(tiles):
    return {f"ortho {what} {height}" for what, height in zip(("gram", "square", "apply"), tiles)}


def iterate64(u, steps=5):
    x = u / u.norm()
    if u.shape[0] > u.shape[1]:
        x = x.t().contiguous()
    for _ in range(steps):
        s = x @ x.t()
        x = A * x + (B * s + C * (s @ s)) @ x
    return x.t() if u.shape[0] > u.shape[1] else x


def tol(rows, cols, steps=5):
    return 8 * 2.0 ** -22 * max(A ** steps / min(rows, cols) ** 0.5, steps)


@pytest.mark.parametrize("K,rows,cols,tiles", CASES)
def test_iterations(K, rows, cols, tiles):
    G = rand(K, rows, cols, seed=rows + cols)
    for steps in (2, 5):
        O, labels = launched(lambda: hmoe.orthogonalise(G, steps=steps))
        assert labels == names(tiles)
        for k in {0, K // 2, K - 1}:
            ref = iterate64(G[k].double(), steps)
            off = ((O[k].double() - ref).norm() / ref.norm()).item()
            assert off <= tol(rows, cols, steps), (steps, k, off)
    low, labels = launched(lambda: hmoe.orthogonalise(G.bfloat16()))
    assert labels == names(tiles)
    assert torch.equal(low, hmoe.orthogonalise(G.bfloat16().float()).bfloat16())


@pytest.mark.parametrize("nesterov,lo", [(True, torch.bfloat16), (False, torch.float32)])
@pytest.mark.parametrize("K,rows,cols,tiles", CASES)
def test_step(K, rows, cols, tiles, nesterov, lo):
    mu, lr, decay, scale = 0.9375, 2.0 ** -5, 0.25, 1.5
    keep, rate = 1 - lr * decay, lr * scale
    w, v = rand(K, rows, cols, seed=1) * 0.01, rand(K, rows, cols, seed=2) * 1e-3
    w_lo = torch.zeros(K, rows, cols, dtype=lo, device="cuda")
    for i in range(2):
        g = rand(K, rows, cols, seed=3 + i) * 1e-3
        w0, v0, g0 = w.clone(), v.clone(), g.clone()
        _, labels = launched(lambda: hmoe.muon_step(w, g, v, lr, decay, mu, nesterov, scale, w_lo=w_lo))
        assert labels == names(tiles)
        assert torch.equal(g, g0) and torch.equal(w_lo, w.to(lo))
        new_v = mu * v0.double() + g0.double()
        assert ((v.double() - new_v).abs() <= U * new_v.abs() + 1e-40).all()
        for k in {0, K - 1}:
            u = g0[k].double() + mu * v[k].double() if nesterov else v[k].double()
            O = iterate64(u)
            ref = keep * w0[k].double() - rate * O
            most = rate * O.norm() * (tol(rows, cols) + 2.0 ** -23 * A ** 5) + U * (keep * w0[k].double().norm() + ref.norm())
            off = (w[k].double() - ref).norm()
            assert off <= most, (i, k, off.item(), most.item())
