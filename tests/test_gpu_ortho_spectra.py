"""GPU: orthogonalisation of matrices with a few strong directions, with one half and with two, against the same iteration in 64 bits.

Tolerance.  A stored operand is off by u = 2^-11 (one half) or 2^-22 (two) of an entry at most, evenly spread: u / sqrt(3) root mean
square.  With two halves the sums count as well: sums of 3 K / 16 products of 16 each, in fp32, sqrt(3 K / 16) 2^-24.  Rounding X lies
in all directions.  Where X has singular values near zero the following steps multiply it by a = 3.4445 each, whatever the
strong ones do, and ||X|| in step k is at most min(3.4445^k, 1.21 sqrt(rank)); so the last X is off by
  sum over k < 5 of 3.4445^(5 - k) min(3.4445^k, 1.21 sqrt(rank)) u / sqrt(3).
Roundings of G and B act on the left of X, hence only in its own row space, where the steps lead to one and not beyond: what the
other tests allow, 16 u a step."""
import math

import pytest
import torch

import paper_1905_05957_amd as P

pytestmark = pytest.mark.gpu
A, B, C = 3.4445, -4.7750, 2.0315


def reference(u):
    x = u.double() / u.double().norm()
    x = x.t().contiguous() if u.shape[0] > u.shape[1] else x
    for _ in range(5):
        g = x @ x.t()
        x = A * x + (B * g + C * (g @ g)) @ x
    return x.t() if u.shape[0] > u.shape[1] else x


def matrix(m, n, spectrum, dev):
    gen = torch.Generator()
    gen.manual_seed(17)
    if isinstance(spectrum, int):
        return (torch.randn(m, spectrum, generator=gen) @ torch.randn(spectrum, n, generator=gen)).to(dev), spectrum
    left = torch.linalg.qr(torch.randn(m, m, generator=gen, dtype=torch.float64))[0]
    right = torch.linalg.qr(torch.randn(n, m, generator=gen, dtype=torch.float64))[0]
    s = torch.arange(1, m + 1, dtype=torch.float64) ** -spectrum
    return ((left * s) @ right.t()).float().to(dev), m


def allowed(m, n, rank, half):
    u = 2.0 ** -11 if half else 2.0 ** -22 + math.sqrt(3 * n / 16) * 2.0 ** -24
    weak = sum(A ** (5 - k) * min(A ** k, 1.21 * math.sqrt(rank)) for k in range(5)) * u / math.sqrt(3)
    return weak, 5 * (16 * (2.0 ** -11 if half else 2.0 ** -22) + 4 * math.sqrt(n) * 2.0 ** -24)


@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("half", [False, True])
@pytest.mark.parametrize("spectrum", [1, 2, 16, 1.0, 1.5], ids=["rank 1", "rank 2", "rank 16", "1 / k", "1 / k^1.5"])
@pytest.mark.parametrize("m,n,tall", [(64, 128, False), (100, 120, True), (256, 512, False), (300, 700, True), (768, 2048, False)])
def test_few_strong_directions(gpu_device, m, n, tall, spectrum, half, out):
    w, rank = matrix(m, n, spectrum, gpu_device)
    w = w.t().contiguous() if tall else w
    plan = P.OrthoPlan(m * n, [(0, *w.shape)], half=half)
    dst = torch.empty(m * n, dtype=out, device=gpu_device)
    plan.orthogonalize(w.reshape(-1), dst)
    want = reference(w)
    weak, rest = allowed(m, n, rank, half)
    rounding = 2.0 ** -8 if out == torch.bfloat16 else 2.0 ** -24
    off = float((dst.view(w.shape).double() - want).norm())
    assert off <= weak + (rest + rounding) * float(want.norm()), (off / float(want.norm()), weak / float(want.norm()), rest)
    plan.close()
