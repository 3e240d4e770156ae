"""Iterations of bf16 matrices have the accuracy of fp32 ones, whatever their size: the result is that of the same numbers
in fp32, rounded once.

Against 64 bits: an entry that rounds another way than the exact one is off, before its rounding, by at least the distance
of the exact value from the interval of numbers that round to it.  The norm of these distances is therefore at most
that of the errors before rounding, for which 8 2^-22 |a|^steps / sqrt(rank), or 8 2^-22 steps, of the result's norm
is the bound of fp32 results."""
import pytest
import torch

from paper_1704_06363_amd import hmoe

pytestmark = pytest.mark.gpu

A, B, C = hmoe.COEF
# one workgroup to a matrix, a launch to a step, and tiles of 64 x 64, 128 x 128 and 256 x 256
SHAPES = [(3, 17, 704), (2, 100, 328), (3, 777, 120), (2, 200, 1504), (3, 900, 136), (24, 264, 200), (5, 600, 640), (3, 513, 528),
          (23, 130, 264), (1, 2500, 640), (2, 2048, 4096), (1, 4104, 1000)]


def rand(*shape, seed=0):
    return torch.randn(*shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").bfloat16()


@pytest.mark.parametrize("K,rows,cols", SHAPES)
def test_the_same_numbers_as_of_fp32(K, rows, cols):
    G = rand(K, rows, cols, seed=rows)
    for steps in (1, 2, 3, 5, 6):
        got, want = hmoe.orthogonalise(G, steps=steps), hmoe.orthogonalise(G.float(), steps=steps)
        assert torch.equal(got, want.bfloat16()), (steps, (got != want.bfloat16()).float().mean().item())


def iterate64(u, steps):
    x = u / u.norm()
    if u.shape[0] > u.shape[1]:
        x = x.t().contiguous()
    for _ in range(steps):
        s = x @ x.t()
        x = A * x + (B * s + C * (s @ s)) @ x
    return x.t() if u.shape[0] > u.shape[1] else x


def outside(got, ref):
    """How far each of `ref` is outside the numbers that round to `got` in bf16."""
    bits = got.contiguous().view(torch.int16)
    away = (bits + 1).view(torch.bfloat16).double()  # the next number away from zero, and the one towards it
    near = torch.where(got == 0, -away, (bits - 1).view(torch.bfloat16).double())
    g = got.double()
    one, two = (g + away) / 2, (g + near) / 2
    lo, hi = torch.minimum(one, two), torch.maximum(one, two)
    return (lo - ref).clamp(min=0) + (ref - hi).clamp(min=0)


@pytest.mark.parametrize("K,rows,cols", SHAPES)
@pytest.mark.parametrize("steps", [1, 2, 5])
def test_against_64_bits(K, rows, cols, steps):
    G = rand(K, rows, cols, seed=cols)
    O = hmoe.orthogonalise(G, steps=steps)
    most = 8 * 2.0 ** -22 * max(A ** steps / min(rows, cols) ** 0.5, steps)
    for k in {0, K - 1}:
        ref = iterate64(G[k].double(), steps)
        off = (outside(O[k], ref).norm() / ref.norm()).item()
        assert off <= most, (k, off, most)


@pytest.mark.parametrize("rank", [1, 3])
def test_low_rank(rank):
    G = (rand(1100, rank, seed=1).float() @ rand(rank, 1400, seed=2).float()).bfloat16()
    ref = iterate64(G.double(), 5)
    off = (outside(hmoe.orthogonalise(G), ref).norm() / ref.norm()).item()
    assert off <= 8 * 2.0 ** -22 * A ** 5 / rank ** 0.5, off
