"""GPU: AdamW from the server's message against the same update in 64 bits.

Tolerance, with h = 2^-24 (half a step of fp32): m and v are fma(beta, old, rest * q (* q)) with beta and rest rounded to
fp32, so 4 h of |beta old| + |rest q| and 5 h of v (its terms have one sign).  x: keep, its product and the final fma
3 h |x|; the step's factor m / (sqrt(v) root + eps) rate: m's error, and relative to it half of v's, the root, root,
the sum, the quotient, rate: less than 4 h of the terms' sizes + 8 h."""
import pytest
import torch

import paper_1905_05957_amd as P
from test_gpu_ortho import BOTH, COMPRESSORS, D, MATS, message, random_flat, state, view

pytestmark = pytest.mark.gpu
H = 2.0 ** -24


def check_step(q, old, new, step, gamma, b1, b2, eps, decay, inside=None):
    x, m, v = (t.double() for t in old)
    q = q.double()
    wm, wv = b1 * m + (1 - b1) * q, b2 * v + (1 - b2) * q * q
    size = (wv / (1 - b2 ** (step + 1))).sqrt() + eps
    rate = gamma / (1 - b1 ** (step + 1))
    wx = (1 - gamma * decay) * x - rate * wm / size
    terms = (b1 * m).abs() + ((1 - b1) * q).abs()
    tol = (3 * H * (x.abs() + wx.abs()) + (4 * terms + 8 * wm.abs()) * H * rate / size, 4 * H * terms, 5 * H * wv)
    touched = torch.ones_like(q, dtype=torch.bool) if inside is None else ~inside
    for name, got, was, want, t in zip("xmv", new, old, (wx, wm, wv), tol):
        err = (got.double() - want).abs()
        assert (err <= t)[touched].all(), (name, float((err / t.clamp_min(1e-300))[touched].max()))
        assert torch.equal(got[~touched], was[~touched]), name


@pytest.mark.parametrize("skip", [False, True])
@pytest.mark.parametrize("comp,kw,flags", COMPRESSORS, ids=lambda v: v if isinstance(v, str) else None)
def test_every_message(gpu_device, comp, kw, flags, skip):
    ctx, ps, q = message(comp, kw, flags, gpu_device)
    x, m = state(gpu_device)
    v = random_flat(D, gpu_device, 60).square() * 1e-4
    plan = P.OrthoPlan(D, MATS) if skip else None
    inside = torch.zeros(D, dtype=torch.bool, device=gpu_device)
    for mat in MATS if skip else ():
        view(inside, mat).fill_(True)
    old = [t.clone() for t in (x, m, v)]
    ctx.apply_update_adamw(ps, 4, x, m, v, 1e-3, 0.9, 0.999, 1e-8, 0.1, skip=plan)
    check_step(q, old, (x, m, v), 4, 1e-3, 0.9, 0.999, 1e-8, 0.1, inside)
    ctx.close()


@pytest.mark.parametrize("d", [1, 2, 3, 4, 5, 63, 64, 65, 2047, 2049, 100003])
def test_lengths_and_first_step(gpu_device, d):
    ctx = P.Context("identity", 1, d)
    ps = ctx.alloc_payload(1)
    q = random_flat(d, gpu_device, d)
    ps.dense.copy_(q.view(1, d))
    x, m, v = random_flat(d, gpu_device, 2), torch.zeros(d, device=gpu_device), torch.zeros(d, device=gpu_device)
    for step in range(3):
        old = [t.clone() for t in (x, m, v)]
        ctx.apply_update_adamw(ps, step, x, m, v, 1e-2, 0.9, 0.95)
        check_step(q, old, (x, m, v), step, 1e-2, 0.9, 0.95, 1e-8, 0.0)
    ctx.close()


def test_late_steps_and_extreme_constants(gpu_device):
    d = 5000
    ctx = P.Context("identity", 1, d)
    ps = ctx.alloc_payload(1)
    q = random_flat(d, gpu_device, 1)
    ps.dense.copy_(q.view(1, d))
    for step, b1, b2, eps, decay in ((10 ** 7, 0.9, 0.999, 1e-8, 0.0), (2 ** 40, 0.9, 0.9999, 1e-6, 0.1), (0, 0.0, 0.0, 1e-8, 0.0),
                                     (0, 0.0, 0.999, 1.0, 1.0)):
        x, m, v = (random_flat(d, gpu_device, s) for s in (2, 3, 4))
        v = v.square()
        old = [t.clone() for t in (x, m, v)]
        ctx.apply_update_adamw(ps, step, x, m, v, 1e-2, b1, b2, eps, decay)
        check_step(q, old, (x, m, v), step, 1e-2, b1, b2, eps, decay)
    ctx.close()


def test_a_plan_that_covers_everything_leaves_nothing_to_do(gpu_device):
    d = 64 * 50
    ctx = P.Context("sign", 1, d)
    ps = ctx.alloc_payload(1)
    ps.scales.fill_(1.0)
    plan = P.OrthoPlan(d, [(0, 64, 50)])
    x, m, v = (random_flat(d, gpu_device, s) for s in (2, 3, 4))
    old = [t.clone() for t in (x, m, v)]
    ctx.apply_update_adamw(ps, 0, x, m, v, 1.0, skip=plan)
    assert all(torch.equal(a, b) for a, b in zip(old, (x, m, v)))
    ctx.close()
    plan.close()


def test_a_step_of_training_with_both_updates(gpu_device):
    """Four steps of the whole path: the matrices through their orthogonalisation, the rest through AdamW, each element by
    exactly one of the two."""
    from test_gpu_ortho import expected
    dev = gpu_device
    ctx = P.Context("topk", 2, D, k=2000)
    plan = P.OrthoPlan(D, MATS, nesterov=True, scale="rms")
    x, m = state(dev)
    v = torch.zeros(D, device=dev)
    delta, delta_s = torch.zeros(2, D, device=dev), torch.zeros(D, device=dev)
    pw, ps, q = ctx.alloc_payload(2), ctx.alloc_payload(1), torch.empty(D, device=dev)
    inside = torch.zeros(D, dtype=torch.bool, device=dev)
    for mat in MATS:
        view(inside, mat).fill_(True)
    for step in range(4):
        g = random_flat(2 * D, dev, 100 + step).view(2, D) * 1e-2
        ctx.worker_compress(step, g, delta, pw)
        ctx.server_aggregate_compress(step, pw, delta_s, ps)
        ctx.decompress(ps, 0, q)
        old = [t.clone() for t in (x, m, v)]
        want_x, want_m, off = expected(dict(nesterov=True, scale="rms"), q, x, m, 0.03125, 0.9375, 0.25)
        ctx.apply_update_ortho(plan, ps, x, m, 0.03125, 0.9375, 0.25)
        ctx.apply_update_adamw(ps, step, x, m, v, 1e-3, 0.9, 0.95, 1e-8, 0.1, skip=plan)
        assert ((x.double() - want_x).abs() <= off)[inside].all()
        assert ((m.double() - want_m).abs() <= 2.0 ** -24 * want_m.abs() * 1.0001)[inside].all()
        new = [torch.where(inside, o, n) for o, n in zip(old, (x, m, v))]
        check_step(q, old, new, step, 1e-3, 0.9, 0.95, 1e-8, 0.1, inside)
        assert not v[inside].any()
    ctx.close()
    plan.close()


class _Sub(torch.Tensor):
    pass


@pytest.mark.parametrize("comp,kw,flags", [("sign", dict(scale_mode="chunk", chunk=1024), 0), ("topk", dict(k=50), 0),
                                           ("ternary", {}, BOTH)])
def test_extension_and_python_route_agree(gpu_device, comp, kw, flags):
    """Plain arguments go through the extension module, a tensor subclass through the checks in Python and ctypes: the same bytes."""
    outs = []
    for plain in (True, False):
        wrap = (lambda t: t) if plain else (lambda t: t.as_subclass(_Sub))
        ctx, ps, _ = message(comp, kw, flags, gpu_device)
        plan = P.OrthoPlan(D, MATS)
        x, m = state(gpu_device)
        v = torch.zeros(D, device=gpu_device)
        address = plan._h.value
        want = 0 if plain else -1
        assert ctx._calls.ortho(address, ps, wrap(x.clone()), None, 0.1, 0, 0.0, None) == want
        assert ctx._calls.adamw(0, ps, 0, wrap(x.clone()), wrap(m.clone()), wrap(v.clone()), 1, 0.9, 0.99, 1e-8, 0, None) == want
        ctx.apply_update_ortho(plan, ps, wrap(x), wrap(m), 0.1, 0.9, 0.1)
        ctx.apply_update_adamw(ps, 1, wrap(x), wrap(m), wrap(v), 1e-3, 0.9, 0.99, 1e-8, 0.1, plan)
        ctx.apply_update_adamw(ps, 2, wrap(x), wrap(m), wrap(v), 1e-3, stream=torch.cuda.current_stream())
        torch.cuda.synchronize()
        outs.append([t.clone() for t in (x, m, v)])
        ctx.close()
        plan.close()
        assert ctx._calls.adamw(0, ps, 0, x, m, v, 1.0, 0.9, 0.99, 1e-8, 0.0, None) == -1        # closed
    for a, b in zip(*outs):
        assert torch.equal(a, b)
