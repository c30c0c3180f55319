"""Refusals of the orthogonalisation plan and of the update calls that need no GPU: all of them come before any device work."""
import ctypes as C

import numpy as np
import pytest

import paper_1905_05957_amd as P
from paper_1905_05957_amd import binding as B

NULL, SHAPE, CONFIG, DEVICE = 1, 2, 3, 6


def _create(d=1000, mats=((0, 0, 10, 20),), n=None, steps=5, coef=None, eps=1e-7, factor=0, flags=0, no_mats=False):
    cfg = B.ds_ortho_config_t()
    arr = (B.ds_matrix_t * max(1, len(mats)))(*[B.ds_matrix_t(*m) for m in mats])       # offset, ld, rows, cols
    cfg.d, cfg.n_mats, cfg.steps, cfg.eps, cfg.factor, cfg.flags = d, len(mats) if n is None else n, steps, eps, factor, flags
    if not no_mats:
        cfg.mats = arr
    if coef is not None:
        c = np.asarray(coef, dtype=np.float32)
        cfg.coef = c.ctypes.data_as(C.POINTER(C.c_float))
    h = C.c_void_p()
    rc = P.load_library().ds_ortho_create(C.byref(cfg), C.byref(h))
    if rc == 0:
        P.load_library().ds_ortho_destroy(h)
    else:
        assert not h.value
    return rc


def test_create_refuses_what_it_cannot_take():
    lib = P.load_library()
    h = C.c_void_p()
    assert lib.ds_ortho_create(None, C.byref(h)) == NULL
    assert lib.ds_ortho_create(C.byref(B.ds_ortho_config_t()), None) == NULL
    assert _create(no_mats=True) == NULL
    assert _create(d=0) == SHAPE and _create(d=1 << 31) == SHAPE
    assert _create(n=0) == SHAPE and _create(n=-1) == SHAPE and _create(n=(1 << 20) + 1) == SHAPE
    assert _create(steps=0) == SHAPE and _create(steps=33) == SHAPE
    for bad in (-1.0, float("nan"), float("inf")):
        assert _create(eps=bad) == CONFIG
    assert _create(factor=-1) == CONFIG and _create(factor=3) == CONFIG
    assert _create(flags=4) == CONFIG and _create(flags=-1) == CONFIG
    assert _create(steps=1, coef=[1.5, float("nan"), 0.0]) == CONFIG
    # the polynomial leaves the range in which B is held: at an end, in between, in the second step
    assert _create(steps=1, coef=[16.0, 0.0, 0.0]) == CONFIG and _create(steps=1, coef=[1.0, 20.0, 0.0]) == CONFIG
    assert _create(steps=1, coef=[1.0, 70.0, -70.0]) == CONFIG
    assert _create(steps=2, coef=[1.5, -0.5, 0.0, 1.0, -17.0, 0.0]) == CONFIG
    assert _create(steps=1, coef=[8.2872, -23.5959, 17.3004]) in (0, DEVICE)


@pytest.mark.parametrize("mat", [
    (0, 0, 0, 5), (0, 0, 5, 0), (0, 0, -1, 5), (-1, 0, 2, 2), (0, 4, 2, 5),     # empty, before the vector, rows into each other
    (990, 0, 1, 11), (901, 0, 10, 10), (0, 500, 3, 10), (1001, 0, 1, 1),        # past its end
    (0, 1 << 62, 2, 1), (1 << 62, 0, 1, 1), (0, -20, 2, 20),
    (0, 0, 2 ** 31 - 1, 2 ** 31 - 1),
])
def test_matrices_outside_the_vector_are_refused(mat):
    assert _create(mats=(mat,)) == SHAPE


def test_sides_out_of_range_are_refused():
    big = 2 ** 31 - 1
    assert _create(d=big, mats=((0, 0, 1, (1 << 24) + 1),)) == SHAPE
    assert _create(d=big, mats=((0, 0, 32769, 32769),)) == SHAPE


@pytest.mark.parametrize("mats", [
    ((0, 0, 10, 20), (199, 0, 1, 1)),
    ((0, 0, 10, 20), (0, 0, 10, 20)),
    ((0, 30, 5, 10), (5, 30, 5, 10)),                     # column blocks that share five columns
    ((0, 30, 5, 10), (140, 0, 1, 1), (125, 0, 1, 1)),     # inside a row of the first
])
def test_matrices_that_share_an_element_are_refused(mats):
    assert _create(mats=mats) == CONFIG


def test_matrices_side_by_side_pass_the_checks():
    # without a GPU the first thing that fails is the device; with one the plan is made
    for mats in (((0, 30, 5, 10), (10, 30, 5, 10), (20, 30, 5, 10)), ((0, 0, 10, 20), (200, 0, 1, 1)), ((999, 0, 1, 1),),
                 ((0, 0, 1000, 1),)):
        assert _create(mats=mats) in (0, DEVICE)


def test_null_arguments():
    lib = P.load_library()
    assert lib.ds_ortho_destroy(None) == 0
    assert lib.ds_orthogonalize(None, None, 0, None, 0, None) == NULL
    assert lib.ds_apply_update_ortho(None, None, None, None, None, 0.1, 0.9, 0.0, None) == NULL
    assert lib.ds_apply_update_adamw(None, None, None, 0, None, None, None, 0.1, 0.9, 0.999, 1e-8, 0.0, None) == NULL


def test_the_binding_checks_what_ctypes_would_cut():
    for bad in (dict(mats=[(0, 1)]), dict(mats=[(0, 1, 2, 3, 4)]), dict(mats=[(0, 2 ** 32 + 1, 1)]),
                dict(mats=[(0, 2, 2)], coef=[1.0, 2.0]), dict(mats=[(0, 2, 2)], coef=[[1.0, 2.0, 3.0]] * 4)):
        with pytest.raises(ValueError):
            P.OrthoPlan(100, **bad)
    with pytest.raises(KeyError):
        P.OrthoPlan(100, [(0, 2, 2)], scale="max")
    with pytest.raises(P.DsError):
        P.OrthoPlan(100, [])


def test_more_workspace_than_the_card_has_is_refused_at_once():
    # a row of 2^24 elements is worked on as 64 rows: 100 of them would take 860 GB, and tables of gigabytes
    assert _create(d=2 ** 31 - 1, mats=[(k << 24, 0, 1, 1 << 24) for k in range(100)]) == DEVICE
