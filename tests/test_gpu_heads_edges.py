"""Operators of a multi-class head at the edges of their inputs' ranges, against plain implementations in 64 bits.  Bounds as in
test_gpu_heads.py."""
import math

import pytest

import paper_2008_03433_amd as tron
from test_gpu_heads import E, TINY, U, _distill_bounds, _distill_plain, _dt, _gen, _randn, _within
from util import torch_mod

pytestmark = pytest.mark.gpu


# --------------------------------------------------------------------------- a teacher's masks
@pytest.mark.parametrize("low", ["f32", "bf16"])
@pytest.mark.parametrize("T", [2.0, 1.0, 0.5, 2.0 ** -20])
@pytest.mark.parametrize("m,V", [(5, 300), (2, 40_000)])
def test_distill_teacher_of_the_lowest_value(m, V, T, low):
    """Entries of t that are masked with a float's lowest value have no mass beside others, whatever the temperature; rows of whole
    workgroups and rows in parts."""
    torch = torch_mod()
    g = _gen(V)
    K, scale = 6, min(T, 1.0)
    z, t, weight = (3 * scale * _randn(g, m, V)).float(), (3 * scale * _randn(g, m, K)).float(), torch.rand(m, generator=g) + 0.5
    ids = torch.stack([torch.randperm(V, generator=g)[:K] for _ in range(m)])
    t[:, 2:4] = torch.finfo(_dt(low)).min
    t[1] = torch.finfo(_dt(low)).min   # nothing but masks: all alike
    loss, lse, dz, p, q, w = _distill_plain(z, ids, t, T, weight)
    assert torch.isfinite(loss).all() and float(q.sum()) == pytest.approx(m)
    lse_b, off, dz_b = _distill_bounds("f32", z, lse, p, q, w, T, V)
    got_loss, got_lse, got = torch.empty(m, device="cuda"), torch.empty(m, device="cuda"), torch.empty(m, V, device="cuda")
    args = (z.cuda(), ids.cuda(), t.cuda())
    tron.tron_distill(*args, got_loss, got_lse, temperature=T, weight=weight.cuda(), dz=got)
    _within(got_loss, loss, w[:, 0] * T * T * (off + 1e-12 * lse.abs()) + 2 * E * loss.abs(), "loss")
    _within(got_lse, lse, lse_b, "lse")
    bound = (U["f32"] + 4 * E) * dz.abs() + w * T * dz_b * (1 + E) + TINY["f32"]
    _within(got, dz, bound, "dz")
    only = torch.empty(m, device="cuda")
    tron.tron_distill(*args, only, temperature=T, weight=weight.cuda())
    assert torch.equal(only, got_loss)
    got.fill_(7.0)
    tron.tron_distill_grad(args[0], got_lse, *args[1:], got, temperature=T, weight=weight.cuda())
    _within(got, dz, bound, "dz from lse")
