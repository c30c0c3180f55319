"""Lists of coefficients against the range in which the orthogonalisation holds its operands, without a GPU.

What a plan accepts may not end in NaN for any matrix.  `held` is the iteration with operands stored as the kernels store them
(halves, G times 2^13, B times 2^12), in plain torch; two singular values, s and sqrt(1 - s^2), take every place in [0, 1]."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_1905_05957_amd as P
from paper_1905_05957_amd import binding as B

CONFIG, DEVICE, HALF = 3, 6, 2

LEAVES = {
    # converges for [0, 1]: 3 s, then back to 1; G = 9 in between
    "three times": [(3.0, 0.0, 0.0), (0.5, -0.5 / 27, 0.0), (1.5, -0.5, 0.0), (1.5, -0.5, 0.0), (1.5, -0.5, 0.0)],
    "slowly": [(1.25, 0.0, 0.0)] * 6,
    "B in the second step": [(2.0, 0.0, 0.0), (3.0, -5.0, 0.0)],
    "largest between the ends": [(8.0, -8.0, 0.0), (1.5, -0.5, 0.0)],
    "the standard's first and its negative, enlarged": [(3.4445, -4.775, 2.0315), (-10.0, 6.0, 0.0), (1.0, 0.0, 0.0)],
}
STAYS = {
    "standard": [(3.4445, -4.775, 2.0315)] * 32,
    "cubic": [(1.5, -0.5, 0.0)] * 32,
    "quintic": [(1.875, -1.25, 0.375)] * 32,
    "the last step may lead anywhere": [(1.5, -0.5, 0.0), (9.0, 0.0, 0.0)],
    "up to 2.79": [(2.79, 0.0, 0.0), (0.5, 0.0, 0.0)],
    "zeros": [(0.0, 0.0, 0.0), (1.0, 0.0, 0.0)],
    "negative": [(-1.5, 0.5, 0.0), (-1.875, 1.25, -0.375)],
}
# comes back from close to 2, where its polynomials are steep: roundings to one half carry a singular value of 1 out of range
NEAR_TWO = [(8.2872, -23.5959, 17.3004), (4.1071, -2.9478, 0.5448), (3.9487, -2.9089, 0.5518), (3.3184, -2.4885, 0.5100),
            (2.3007, -1.6689, 0.4188), (1.8913, -1.2680, 0.3768), (1.8750, -1.2500, 0.3750)]
# the same for singular values up to 1.01
NEAR_TWO_WITH_ROOM = [(a / 1.01, b / 1.01 ** 3, c / 1.01 ** 5) for a, b, c in NEAR_TWO]


def create(coef, half):
    cfg = B.ds_ortho_config_t()
    mats = (B.ds_matrix_t * 1)(B.ds_matrix_t(0, 0, 4, 4))
    c = np.ascontiguousarray(np.asarray(coef, dtype=np.float32))
    cfg.d, cfg.mats, cfg.n_mats, cfg.steps, cfg.eps, cfg.flags = 100, mats, 1, len(coef), 1e-7, HALF if half else 0
    cfg.coef = c.ctypes.data_as(C.POINTER(C.c_float))
    h = C.c_void_p()
    rc = P.load_library().ds_ortho_create(C.byref(cfg), C.byref(h))
    P.load_library().ds_ortho_destroy(h)
    return rc


def held(x, coef, half, scale=1024.0):
    """The iteration on x (fp32, norm 1, wide) with stored operands rounded to one or two halves."""
    def store(v):
        hi = v.half()
        return (hi.float(),) if half else (hi.float(), (v - hi.float()).half().float())

    def product(p, q):
        return p[0] @ q[0] if half else p[1] @ q[0] + p[0] @ q[1] + p[0] @ q[0]

    eye = torch.eye(x.shape[0])
    x = store(x * scale)
    for k, (a, b, c) in enumerate(coef):
        g = store(product(x, tuple(v.t() for v in x)) * (8192.0 / scale ** 2))
        poly = store(sum(g) * (b / 2) + product(g, g) * (c * 4096.0 / 8192.0 ** 2) + eye * (a * 4096.0))
        y = product(poly, x) / 4096.0
        x = store(y)
    return y / scale


def finite_for_every_singular_value(coef, half):
    s = torch.linspace(0.0, 1.0, 101, dtype=torch.float64)
    return all(torch.isfinite(held(torch.diag(torch.stack([v, (1 - v * v).sqrt()])).float(), coef, half)).all() for v in s)


@pytest.mark.parametrize("half", [False, True])
@pytest.mark.parametrize("name", list(LEAVES))
def test_lists_that_leave_the_range_are_refused(name, half):
    assert create(LEAVES[name], half) == CONFIG


@pytest.mark.parametrize("half", [False, True])
def test_a_list_that_converges_and_ends_in_nan(half):
    coef = LEAVES["three times"]
    s = torch.linspace(0.0, 1.0, 101, dtype=torch.float64)
    for a, b, c in coef:
        s = a * s + b * s ** 3 + c * s ** 5
    assert s[1:].max() < 1.0001 and s[50:].min() > 0.8        # in exact arithmetic
    assert not finite_for_every_singular_value(coef, half)    # as it is held


@pytest.mark.parametrize("half", [False, True])
@pytest.mark.parametrize("name", list(STAYS))
def test_lists_that_stay_are_taken(name, half):
    assert create(STAYS[name], half) in (0, DEVICE)
    assert finite_for_every_singular_value(STAYS[name], half)


def test_a_list_that_comes_back_from_near_two():
    assert create(NEAR_TWO, False) in (0, DEVICE) and finite_for_every_singular_value(NEAR_TWO, False)
    assert create(NEAR_TWO, True) == CONFIG and not finite_for_every_singular_value(NEAR_TWO, True)
    for half in (False, True):
        assert create(NEAR_TWO_WITH_ROOM, half) in (0, DEVICE) and finite_for_every_singular_value(NEAR_TWO_WITH_ROOM, half)


@pytest.mark.parametrize("half", [False, True])
def test_what_is_accepted_stays_finite(half):
    """Lists drawn around usable ones: each that a plan takes gives finite results for all singular values."""
    gen = torch.Generator()
    gen.manual_seed(1)
    steps = NEAR_TWO + [(3.4445, -4.775, 2.0315), (1.5, -0.5, 0.0), (4.0, -6.5, 2.9)]
    taken = refused = 0
    for _ in range(60):
        coef = []
        for _ in range(int(torch.randint(2, 6, (1,), generator=gen))):
            a, b, c = steps[int(torch.randint(0, len(steps), (1,), generator=gen))]
            f = 1.0 + 0.2 * float(torch.rand(1, generator=gen) - 0.5)
            coef.append((a * f, b * f ** 3, c * f ** 5))
        if create(coef, half) == CONFIG:
            refused += 1
        else:
            taken += 1
            assert finite_for_every_singular_value(coef, half), coef
    assert taken >= 5 and refused >= 5
