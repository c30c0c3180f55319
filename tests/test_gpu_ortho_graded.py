"""GPU: orthogonalisation of matrices whose rows or columns differ in size, against the same iteration in 64 bits.

Tolerance.  Every other row of W = U / ||U|| is smaller by `grade`; rho is the norm of those mw rows together.  Held as halves,
an entry of X is off by at most 2^-39 (half of 2^-24, the spacing of the smallest halves, over 2^14), one of G by 2^-38 and one of B by
2^-37, evenly spread: 1 / sqrt(3) of that root mean square.  In step k that puts into those rows sqrt(mw n) 2^-39 through X, and through
G (times |b| + 2 |c| < 9) and B sqrt(mw) (9 2^-38 + 2^-37) ||X||, ||X|| at most 1.21 sqrt(m) and 3.4445^k.  The rows
themselves grow 3.4445 times a step except along the larger rows, which span half of the m directions at most: 0.7 of them at least is left.
That, relative to the rows, and what the other tests allow for roundings relative to the value, 16 2^-22 a step and sums in fp32."""
import math

import pytest
import torch

import paper_1905_05957_amd as P

pytestmark = pytest.mark.gpu
A, B, C = 3.4445, -4.7750, 2.0315


def reference(x, steps):
    x = x.double() / x.double().norm()
    for _ in range(steps):
        g = x @ x.t()
        x = A * x + (B * g + C * (g @ g)) @ x
    return x


def tolerance(w, steps):
    m, n = w.shape
    mw, rho = (m + 1) // 2, float(w[::2].norm() / w.norm())
    floor = 0.0
    for k in range(steps):
        grown = A ** k
        floor += (math.sqrt(mw * n) * 2.0 ** -39 + math.sqrt(mw) * (9 * 2.0 ** -38 + 2.0 ** -37) * min(grown, 1.21 * math.sqrt(m))) / \
            math.sqrt(3) / (0.7 * rho * grown)
    return floor + steps * (16 * 2.0 ** -22 + 4 * math.sqrt(n) * 2.0 ** -24)


@pytest.mark.parametrize("tall", [False, True])
@pytest.mark.parametrize("steps", [5, 12])
@pytest.mark.parametrize("grade", [1e-3, 1e-5, 1e-6])
@pytest.mark.parametrize("m,n", [(48, 64), (128, 144), (192, 256), (300, 700), (520, 530)])
def test_rows_of_different_size(gpu_device, m, n, grade, steps, tall):
    gen = torch.Generator(device=gpu_device)
    gen.manual_seed(91)
    w = torch.randn(m, n, generator=gen, device=gpu_device)
    w[::2] *= grade
    src = (w.t() if tall else w).contiguous().reshape(-1)
    plan = P.OrthoPlan(m * n, [(0, n, m) if tall else (0, m, n)], steps=steps)
    dst = torch.empty_like(src)
    plan.orthogonalize(src, dst)
    got = dst.view(n, m).t() if tall else dst.view(m, n)
    want = reference(w, steps)
    off = float((got.double() - want)[::2].norm() / want[::2].norm())
    assert off <= tolerance(w, steps), (off, tolerance(w, steps))
    plan.close()
