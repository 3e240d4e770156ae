"""Newton-Schulz iterations and the step made of them against the formulas in 64 bits.

Bounds.  An iterate's entry is two fp16 numbers, good to 2^-22 of it, and the products drop lo lo, 2^-22 of theirs; a step
rounds A, b A + c A^2 and X, and sums in fp32: at most 8 2^-22 |X| of noise a step, |X| the Frobenius norm, which later
steps amplify by their derivative, a at most where the singular values are small.  The result of rank q has a norm of
about sqrt(q) and |X| is 1 at the start: relative to it at most 8 2^-22 |a|^steps / sqrt(q), and 8 2^-22 steps where the
last rounding counts."""
import numpy as np
import pytest
import torch

from paper_1704_06363_amd import hmoe
from tests.parity import np64

pytestmark = pytest.mark.gpu

COEF = hmoe.COEF


def iterate64(u, steps=5, coef=COEF):
    a, b, c = coef
    x = u / max(np.linalg.norm(u), 1e-300)
    tall = x.shape[0] > x.shape[1]
    if tall:
        x = x.T
    for _ in range(steps):
        s = x @ x.T
        x = a * x + (b * s + c * (s @ s)) @ x
    return x.T if tall else x


def tol(rank, steps=5):
    return 8 * 2.0 ** -22 * max(COEF[0] ** steps / rank ** 0.5, steps)


def off(got, ref):
    return np.linalg.norm(got - ref) / np.linalg.norm(ref)


def rand(*shape, seed=0):
    return torch.randn(*shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda")


SHAPES = [(1, 1, 8), (3, 8, 8), (2, 5, 40), (2, 33, 32), (1, 64, 64), (2, 100, 328), (1, 129, 128), (2, 130, 264),
          (1, 257, 200), (3, 1000, 64), (1, 40, 3000), (1, 300, 304), (1, 520, 1032), (1, 777, 512), (40, 64, 128),
          # short sides of up to 32, 64 and 128, one workgroup's columns and several's
          (9, 16, 16), (2, 31, 136), (3, 17, 704), (2, 32, 776), (1, 30, 5000), (2, 5000, 24), (1, 9, 49160), (2, 64, 384),
          (3, 60, 392), (1, 3000, 56), (1, 64, 6152), (2, 128, 128), (2, 120, 136), (1, 128, 2056), (2, 900, 128), (1, 65, 1024)]


@pytest.mark.parametrize("K,rows,cols", SHAPES)
@pytest.mark.parametrize("steps", [1, 5])
def test_shapes(K, rows, cols, steps):
    G = rand(K, rows, cols, seed=rows) * torch.logspace(-3, 3, K, device="cuda")[:, None, None]
    keep = G.clone()
    O = hmoe.orthogonalise(G, steps=steps)
    assert torch.equal(G, keep)
    for k in range(K):
        ref = iterate64(np64(G[k]), steps)
        assert off(np64(O[k]), ref) <= tol(min(rows, cols), steps), k


@pytest.mark.parametrize("K,rows,cols", [(16, 1024, 512), (5, 512, 2048), (1, 2048, 2056)])
def test_large_tiles(K, rows, cols):
    """Enough tiles of 256 x 256 for the larger ones."""
    G = rand(K, rows, cols, seed=cols)
    O = hmoe.orthogonalise(G)
    for k in (0, K - 1):
        u = G[k].double()
        u = u / u.norm()
        x = u if rows <= cols else u.t().contiguous()
        for _ in range(5):
            s = x @ x.t()
            x = COEF[0] * x + (COEF[1] * s + COEF[2] * (s @ s)) @ x
        assert off(np64(O[k]), np64(x if rows <= cols else x.t())) <= tol(min(rows, cols))


@pytest.mark.parametrize("rows,cols", [(64, 128), (300, 96)])
def test_bf16(rows, cols):
    G = rand(2, rows, cols).bfloat16()
    O = hmoe.orthogonalise(G)
    assert O.dtype == torch.bfloat16
    for k in range(2):
        ref = iterate64(np64(G[k]))
        far = np.abs(np64(O[k]) - ref) - 2.0 ** -8 * np.abs(ref)
        assert far.max() <= tol(min(rows, cols)) * np.linalg.norm(ref)
    same = G.clone()
    assert torch.equal(hmoe.orthogonalise(same, out=same), O)
    assert torch.equal(hmoe.orthogonalise(G[0].contiguous()), O[0])  # one matrix, in two dimensions


@pytest.mark.parametrize("rank", [1, 3])
def test_low_rank(rank):
    G = rand(200, rank, seed=1) @ rand(rank, 360, seed=2)
    ref = iterate64(np64(G))
    assert off(np64(hmoe.orthogonalise(G)), ref) <= tol(rank)


@pytest.mark.parametrize("K,rows,cols", [(2, 72, 96), (1, 200, 1504), (3, 900, 136)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_numbers_of_steps(K, rows, cols, dtype):
    """bf16: the last step, but where it is the first, takes fp16 numbers alone: eight roundings of 2^-11 of 1 or more
    that no later step amplifies, relative to a result of norm sqrt(q) at most 8 2^-11 |X| |a| / sqrt(q) with |X| <= sqrt(q)
    as the steps leave it, and the result's own 2^-8."""
    G = rand(K, rows, cols, seed=9).to(dtype)
    for steps in range(1, 8):
        O = hmoe.orthogonalise(G, steps=steps)
        for k in range(K):
            ref = iterate64(np64(G[k]), steps)
            most = tol(min(rows, cols), steps)
            if dtype == torch.bfloat16:
                most += 2.0 ** -8 + (8 * 2.0 ** -11 * COEF[0] if steps > 1 else 0)
            assert off(np64(O[k]), ref) <= most, (steps, k)


def test_sizes_of_entries():
    """The norm is taken in 64 bits: matrices of very small and very large entries have the same result."""
    G = rand(64, 96)
    O = hmoe.orthogonalise(G)
    for p in (-100, -60, 60, 100):
        assert torch.equal(hmoe.orthogonalise(G * 2.0 ** p), O)


def test_one_large_entry():
    G = torch.zeros(72, 40, device="cuda")
    G[3, 5] = 2.5
    O = np64(hmoe.orthogonalise(G))
    s = 1.0
    for _ in range(5):
        s = COEF[0] * s + COEF[1] * s ** 3 + COEF[2] * s ** 5
    assert abs(O[3, 5] - s) <= tol(1) * s
    O[3, 5] = 0
    assert not O.any()


@pytest.mark.parametrize("K,rows,cols", [(5, 48, 200), (5, 40, 2000), (5, 152, 304), (24, 264, 200), (5, 600, 640)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_zeros_and_not_numbers_stay_in_their_matrices(K, rows, cols, dtype):
    G = rand(K, rows, cols).to(dtype)
    clean = hmoe.orthogonalise(G)
    G[1] = 0
    G[2, 3, 4] = float("nan")
    G[3, 0, 0] = float("inf")
    O = hmoe.orthogonalise(G)
    keep = [k for k in range(K) if k not in (1, 2, 3)]
    assert torch.equal(O[keep], clean[keep])
    assert not O[1].any()
    assert torch.isnan(O[2].float()).all() and torch.isnan(O[3].float()).all()


def test_other_coefficients():
    coef = (1.875, -1.25, 0.375)  # the classical quintic: towards singular values of 1 from below
    G = rand(1, 96, 160)
    O = np64(hmoe.orthogonalise(G, steps=12, coef=coef)[0])
    assert off(O, iterate64(np64(G[0]), 12, coef)) <= 8 * 2.0 ** -22 * 12 * 8
    assert np.abs(O @ O.T - np.eye(96)).max() <= 1e-4


@pytest.mark.parametrize("K,rows,cols,nesterov,decay,momentum,lo", [
    (3, 40, 72, True, 0.01, 0.95, torch.bfloat16), (2, 129, 64, False, 0.0, 0.9, torch.float32),
    (1, 1000, 200, True, 0.1, 0.0, None), (1, 16, 16, False, 0.01, 0.0, torch.bfloat16),
    (2, 64, 520, True, 0.0, 0.5, torch.bfloat16), (2, 600, 64, True, 0.02, 0.95, torch.bfloat16)])
def test_step(K, rows, cols, nesterov, decay, momentum, lo):
    w, g = rand(K, rows, cols, seed=1) * 0.1, rand(K, rows, cols, seed=2) * 1e-3
    v = rand(K, rows, cols, seed=3) * 1e-3 if momentum else None
    w0, g0, v0 = np64(w), np64(g), np64(v) if momentum else 0.0
    w_lo = torch.empty_like(w, dtype=lo) if lo else None
    lr, scale = 0.03, 1.7
    for _ in range(2):
        hmoe.muon_step(w, g, v, lr, decay, momentum, nesterov, scale, w_lo=w_lo)
        v0 = momentum * v0 + g0
        u = g0 + momentum * v0 if nesterov else v0
        O = np.stack([iterate64(m) for m in u])
        w0 = (1 - lr * decay) * w0 - lr * scale * O
    if momentum:
        assert np.abs(np64(v) - v0).max() <= 4 * 2.0 ** -24 * np.abs(v0).max() + 1e-12
    # two steps, each off by the tolerance of O and three roundings of w
    size = np.linalg.norm(O, axis=(1, 2)).max()
    assert np.linalg.norm(np64(w) - w0) <= 2 * lr * scale * size * K * (tol(min(rows, cols)) + 4 * 2.0 ** -24) \
        + 8 * 2.0 ** -24 * np.linalg.norm(w0)
    if lo:
        assert torch.equal(w_lo, w.to(lo))


def test_one_matrix_in_two_dimensions():
    w, g, v = rand(24, 48, seed=1), rand(24, 48, seed=2), rand(24, 48, seed=3)
    w3, v3 = w[None].clone(), v[None].clone()
    hmoe.muon_step(w, g, v)
    hmoe.muon_step(w3, g[None].clone(), v3)
    assert torch.equal(w, w3[0]) and torch.equal(v, v3[0])


@pytest.mark.parametrize("K,rows,cols", [(3, 200, 136), (4, 60, 96), (2, 48, 3000), (30, 256, 264), (2, 700, 1032)])
def test_captured_and_replayed(K, rows, cols):
    w, g, v = rand(K, rows, cols, seed=1), rand(K, rows, cols, seed=2), rand(K, rows, cols, seed=3)
    lo = torch.empty_like(w, dtype=torch.bfloat16)
    ew, ev, elo = w.clone(), v.clone(), lo.clone()
    ws = torch.empty(hmoe.muon_workspace(K, rows, cols), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        hmoe.muon_step(w, g, v, w_lo=lo, ws=ws)
    for _ in range(3):
        ws.fill_(255)
        graph.replay()
        hmoe.muon_step(ew, g, ev, w_lo=elo)
        torch.cuda.synchronize()
        assert torch.equal(w, ew) and torch.equal(v, ev) and torch.equal(lo, elo)
