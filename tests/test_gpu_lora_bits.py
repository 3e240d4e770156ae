"""The adapters' gradients take all bits of the narrow products.  Integers: U = A x and V = B^T dY of up to 21 bits,
which fp32 sums hold exactly and two bf16 numbers do not, times -1, 0 and 1 over a few rows: dA and dB are
exact integers."""
import numpy as np
import pytest
import torch

from paper_1704_06363_amd import hmoe
from tests.parity import np64
from tests.test_gpu_lora import grouped

pytestmark = pytest.mark.gpu


def two_parts(v):
    """v as two bf16 numbers, the first cut off and the second rounded."""
    f = v.astype(np.float32)
    hi = (f.view(np.uint32) & np.uint32(0xFFFF0000)).view(np.float32)
    return hi.astype(np.float64) + np64(torch.tensor(f - hi).bfloat16())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,E,r", [(3, 1, 8), (9, 2, 16), (40, 3, 24), (16, 1, 104)])
def test_gradients_hold_every_bit_of_the_narrow_products(dtype, n, E, r):
    d = o = 72
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    g = torch.Generator().manual_seed(n + r)
    wide = lambda *s: torch.randint(-127, 128, s, generator=g).to(dt).cuda()  # 72 products of them: below 2^21
    unit = lambda *s: torch.randint(-1, 2, s, generator=g).to(dt).cuda()
    p = {"W": unit(o, d), "b": None, "A": wide(E, r, d), "B": wide(E, o, r), "scale": None}
    ids = (np.arange(n) % E).astype(np.int32)
    for X, dY, k in ((wide(n, d), unit(n, o), "dB"), (unit(n, d), wide(n, o), "dA")):
        got = np64(grouped(p, X, ids, dY)[k])
        x, dy, A, B = (np64(t) for t in (X, dY, p["A"], p["B"]))
        for e in range(E):
            i = ids == e
            if k == "dB":
                q = x[i] @ A[e].T
                ref, less = dy[i].T @ q, dy[i].T @ two_parts(q)
            else:
                q = dy[i] @ B[e]
                ref, less = q.T @ x[i], two_parts(q).T @ x[i]
            assert np.abs(ref).max() < 2 ** 24  # n of them, so every sum is exact
            assert (ref != less).any()  # and two numbers are not enough
            # (a product of one bf16 number has remainders of 2^-126)
            assert np.abs(got[e] - ref).max() <= 1e-30, (k, e)
