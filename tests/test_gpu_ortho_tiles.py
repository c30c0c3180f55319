"""GPU: what the orthogonalisation's tiles of every size compute, whole and in parts, into fp32, bf16 and the model, against the
same iteration in 64 bits; tolerances as in test_gpu_ortho.py."""
import pytest
import torch

import paper_1905_05957_amd as P
from ortho_plans import PLANS, layout, name
from test_gpu_ortho import bound, check, random_flat, reference, view

pytestmark = pytest.mark.gpu
GAMMA, DECAY = 0.03125, 0.25                              # exact in fp32


@pytest.mark.parametrize("plan", PLANS, ids=name)
def test_plans_that_reach_every_kernel(gpu_device, plan):
    half, shapes, _ = plan
    mats, d = layout(shapes, PLANS.index(plan) % 2)
    src = random_flat(d, gpu_device, 60, torch.bfloat16)
    inside = torch.zeros(d, dtype=torch.bool, device=gpu_device)
    for m in mats:
        view(inside, m).fill_(True)
    src[~inside] = float("nan")                           # not read
    wide = src.float()
    o = P.OrthoPlan(d, mats, half=half)
    f32, bf16 = torch.full((d,), 3.25, device=gpu_device), torch.full((d,), 3.25, device=gpu_device, dtype=torch.bfloat16)
    o.orthogonalize(wide, f32)
    o.orthogonalize(src, bf16)
    x = random_flat(d, gpu_device, 61) * 0.02
    before = x.clone()
    ctx = P.Context("identity", 1, d)
    srv = ctx.alloc_payload(1)
    srv.dense.copy_(wide.view(1, d))
    ctx.apply_update_ortho(o, srv, x, None, GAMMA, 0.0, DECAY)
    for m in mats:
        want = reference(view(wide, m))
        check(view(f32, m), want, half)
        check(view(bf16, m), want, half)
        old = view(before, m).double()
        off = 3 * 2.0 ** -24 * (old.abs() + GAMMA * want.abs()) + 6 * GAMMA * bound(want.shape, half) * want.square().mean().sqrt()
        assert ((view(x, m).double() - ((1.0 - GAMMA * DECAY) * old - GAMMA * want)).abs() <= off).all()
    for t in (f32, bf16):
        assert (t[~inside] == 3.25).all()
    assert torch.equal(x[~inside], before[~inside])
    o.orthogonalize(wide, wide)                           # in place, and the same bits every time
    assert torch.equal(wide[inside], f32[inside])
    o.close()
    ctx.close()
