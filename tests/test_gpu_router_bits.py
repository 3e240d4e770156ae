"""The gradient of a batch's rows takes every bit of the scores' gradient.

Scores of zero give all `on` experts that are on, a power of two, the same probability 1 / on without rounding, and two
choices with gradients a and -a of their weights leave a / on and -a / on as the scores' gradients, again without
rounding.  Rows of R with one power of two in a column then make every entry of dX one such number, or zero: it is
that number rounded once, bit for bit.  Half of the numbers lie next to the middle between two of bf16, so that
their last bits decide."""
import pytest
import torch

from paper_1704_06363_amd import hmoe

pytestmark = pytest.mark.gpu

# up to 32 experts; more, and few rows; more, and many, on tiles of the engine: of experts that fill them and do not
CASES = [(40, 8, 8, 64), (333, 16, 16, 200), (70, 24, 16, 72), (600, 32, 32, 64), (200, 64, 64, 136), (300, 48, 32, 104),
         (300, 64, 64, 64), (515, 128, 128, 264), (1030, 130, 128, 136), (290, 600, 512, 1200)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,K,on,d", CASES)
def test_every_bit_counts(n, K, on, d, dtype):
    g = torch.Generator(device="cuda").manual_seed(n + K)
    e = torch.arange(K, device="cuda")
    bias = torch.zeros(K, device="cuda")
    live = torch.randperm(K, generator=g, device="cuda")[:on].sort()[0]
    bias[torch.isin(e, live, invert=True)] = float("-inf")
    c = torch.arange(d, device="cuda")
    R = torch.where(c[None] % K == e[:, None], 2.0 ** (e % 3)[:, None], 0.0)
    X = torch.zeros(n, d, device="cuda", dtype=dtype)
    p = {"R": R.to(dtype), "bias": bias}
    f = hmoe.router_forward(p, X, top_k=2)
    pick = torch.rand(n, on, generator=g, device="cuda").topk(2, 1)[1]
    f["expert"] = live[pick].to(torch.int32)

    a = torch.randn(n, generator=g, device="cuda")
    i = lambda lo, hi: torch.randint(lo, hi, (n,), generator=g, device="cuda")
    middle = (1 + (2 * i(0, 128) + 1) * 2.0 ** -8 + (2 * i(0, 2) - 1) * 2.0 ** -(17 + i(0, 7)).double())
    near = ((2 * i(0, 2) - 1) * middle * 2.0 ** i(-8, 8)).float()
    a = torch.where(torch.arange(n, device="cuda") % 2 == 0, a, near)
    gw = torch.stack([a, -a], 1)
    dX = hmoe.router_backward(p, X, f, gw)["dX"]
    want = torch.zeros(n, K, device="cuda").scatter_(1, f["expert"].long(), gw / on) * 2.0 ** (e % 3)
    want = want[:, c % K].to(dtype)
    wrong = dX != want
    assert not wrong.any(), (wrong.any(1).float().mean().item(), dX[wrong][:4], want[wrong][:4])
