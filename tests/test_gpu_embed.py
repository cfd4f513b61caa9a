"""Embeddings and the gradient of their table against indexing in 64 bits.

Bounds: a value is rounded twice in 32 bits (the product of the scales, the product with it) and once to its type; a sum of n rows loses n E of the sizes of its
terms, in any order.  E = 2^-24; U: half a step of the output's type."""
import math

import pytest

import paper_2008_03433_amd as tron
from test_gpu_heads import E, TINY, U, _dt, _gen, _randn, _strided, _surround_untouched, _within
from util import torch_mod

pytestmark = pytest.mark.gpu

SIZES = [(1, 1, 1), (3, 7, 5), (1, 4096, 100), (17, 511, 40), (40, 513, 1000), (9, 1024, 3), (300, 65, 70), (5, 9000, 11)]


def _ids(g, m, V, wide, frequent=False):
    torch = torch_mod()
    ids = torch.randint(0, V, (m,), generator=g)
    if frequent:
        ids[torch.rand(m, generator=g) < 0.5] = V // 2
    if m > 2:
        ids[torch.rand(m, generator=g) < 0.1] = -1
        ids[1] = V
        if wide:
            ids[2] = 2 ** 40 + 1
    return ids if wide else ids.to(torch.int32)


def _tables(g, V, d, kind):
    """The table as it is held, its scales, and its values in 64 bits."""
    torch = torch_mod()
    t = _randn(g, V, d)
    if kind == "i8":
        held, scale = torch.randint(-128, 128, (V, d), generator=g, dtype=torch.int8), (torch.rand(V, generator=g) + 0.1)
    elif kind == "e4m3":
        held, scale = (50.0 * t).float().to(torch.float8_e4m3fn), (torch.rand(V, generator=g) + 0.1)
    else:
        return t.to(_dt(kind)), None, t.to(_dt(kind)).double()
    return held, scale, held.float().double() * scale.double()[:, None]


@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("kind,out", [("f32", "f32"), ("bf16", "bf16"), ("f16", "f16"), ("e4m3", "bf16"), ("i8", "f32"), ("i8", "f16"), ("f32", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("m,d,V", SIZES)
def test_embed(m, d, V, kind, out, wide):
    torch = torch_mod()
    g = _gen(m + d + V)
    ids = _ids(g, m, V, wide)
    held, scale, table = _tables(g, V, d, kind)
    there = (ids >= 0) & (ids < V)
    want = torch.where(there[:, None], 1.7 * table[torch.where(there, ids, 0).long()], 0.0)
    pad = 3 if m > 1 else 0
    y = _strided(torch.zeros((m, d), dtype=_dt(out)), pad, 1)
    tv = _strided(held, 5 if V > 1 else 0, 3) if kind not in ("i8",) else held.cuda()
    tron.tron_embed(ids.cuda(), tv, y, scale=1.7, row_scale=None if scale is None else scale.cuda())
    _within(y, want, (U[out] + 4 * E) * want.abs() + TINY[out], "y")
    assert _surround_untouched(y, pad, 1)


def test_embed_of_rows_that_are_not_finite_and_of_one_row_for_all():
    torch = torch_mod()
    table = torch.randn(4, 600, device="cuda")
    table[1], table[2] = math.nan, math.inf
    ids = torch.tensor([0, 1, 2, 9, 3], device="cuda")
    y = torch.empty((5, 600), device="cuda")
    tron.tron_embed(ids, table, y)
    assert torch.equal(y[[0, 4]], table[[0, 3]]) and torch.isnan(y[1]).all() and torch.isinf(y[2]).all() and (y[3] == 0).all()
    tron.tron_embed(ids, table[:1].expand(4, 600), y, scale=2.0)
    assert torch.equal(y[[0, 1, 2, 4]], 2.0 * table[:1].expand(4, 600)) and (y[3] == 0).all()
    tron.tron_embed(ids[:0], table, y[:0])


@pytest.mark.parametrize("add", [False, True])
@pytest.mark.parametrize("kind,out", [("f32", "f32"), ("bf16", "f32"), ("f16", "f16"), ("bf16", "bf16"), ("f16", "f32")])
@pytest.mark.parametrize("m,d,V", SIZES + [(5000, 40, 30), (3000, 700, 5000), (700, 513, 70000), (20000, 8, 257), (4097, 1024, 2)])
def test_embed_grad(m, d, V, kind, out, add):
    torch = torch_mod()
    g = _gen(3 * m + d + V)
    wide = (m + d) % 2 == 0
    ids, dy = _ids(g, m, V, wide, frequent=m % 2 == 0), _randn(g, m, d).to(_dt(kind))
    there = (ids >= 0) & (ids < V)
    was = _randn(g, V, d).to(_dt(out))
    at = ids[there].long()
    want = torch.zeros(V, d, dtype=torch.float64).index_add_(0, at, dy[there].double()) * 0.3
    size = torch.zeros(V, d, dtype=torch.float64).index_add_(0, at, dy[there].double().abs()) * 0.3
    number = torch.zeros(V, dtype=torch.float64).index_add_(0, at, torch.ones(at.numel(), dtype=torch.float64))[:, None]
    if add:
        want = want + was.double()
    pad = 3 if V > 1 else 0
    table = _strided(was, pad, 1)
    dv, iv = _strided(dy, 5 if m > 1 else 0, 3), ids.cuda()
    tron.tron_embed_grad(iv, dv, table, scale=0.3, add=add)
    # the scale's own rounding, its product, and the addition
    off = (number + 4) * E * size + 2 * E * want.abs()
    _within(table, want, U[out] * want.abs() + (1 + U[out]) * off + TINY[out], "dtable")
    assert _surround_untouched(table, pad, 1)
    if add:
        rest = (number[:, 0] == 0)
        assert torch.equal(table.cpu()[rest], was[rest])
    again = _strided(was, pad, 1)
    tron.tron_embed_grad(iv, dv, again, scale=0.3, add=add)
    assert torch.equal(again, table)


def test_embed_grad_of_one_token_and_of_none():
    torch = torch_mod()
    m, d, V = 10000, 600, 50000
    dy = torch.randn(m, d, generator=_gen(2)).bfloat16()
    for ids in (torch.full((m,), V - 1), torch.full((m,), 0), torch.full((m,), -5)):
        table = torch.full((V, d), math.nan, device="cuda")
        tron.tron_embed_grad(ids.cuda(), dy.cuda(), table)
        at = int(ids[0])
        rest = torch.ones(V, dtype=torch.bool)
        if at >= 0:
            _within(table[at], dy.double().sum(0), m * E * dy.double().abs().sum(0), "sum")
            rest[at] = False
        assert (table.cpu()[rest] == 0).all()
    table = torch.full((V, d), math.nan, device="cuda")
    tron.tron_embed_grad(ids[:0].cuda(), dy[:0].cuda(), table)
    assert (table == 0).all()
    tron.tron_embed_grad(ids[:0].cuda(), dy[:0].cuda(), table, add=True)
    assert (table == 0).all()
    # one row for all: the gradient of a broadcast input
    ids = torch.randint(0, 7, (m,), generator=_gen(3))
    small, twice = torch.empty((7, d), device="cuda"), torch.empty((7, d), device="cuda")
    tron.tron_embed_grad(ids.cuda(), dy[:1].cuda().expand(m, d), small)
    tron.tron_embed_grad(ids.cuda(), dy[:1].cuda().repeat(m, 1), twice)
    assert torch.equal(small, twice)


def test_embed_grad_is_the_gradient():
    """The lookup is linear in its table: <dtable, direction> = <dy, lookup of the direction>, in products of 32 bits that lose (m d)^(1/2) E or less."""
    torch = torch_mod()
    g = _gen(12)
    m, d, V = 500, 200, 90
    ids, dy, direction = _ids(g, m, V, True, True).cuda(), _randn(g, m, d).float().cuda(), _randn(g, V, d).float().cuda()
    dtable, y = torch.empty((V, d), device="cuda"), torch.empty((m, d), device="cuda")
    tron.tron_embed_grad(ids, dy, dtable, scale=1.3)
    tron.tron_embed(ids, direction, y, scale=1.3)
    left, right = (dtable.double() * direction.double()).sum(), (y.double() * dy.double()).sum()
    assert abs(float(left - right)) <= (m + 8) * E * float((y.double() * dy.double()).abs().sum())


@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("m,d,V,frequent", [(20000, 24, 70000, (5, 261, 517)), (20000, 24, 70000, (255, 69887, 511, 5)), (65536, 9, 100, ()), (65536, 9, 700, (3, 259, 515)),
                                            (30000, 5, 1500000, (7, 4103, 1499999)), (300, 8, 262144, ()), (300, 8, 262143, (262142,))])
def test_embed_grad_of_several_frequent_tokens_of_a_workgroup(m, d, V, frequent, wide):
    """Tokens of which one workgroup of the sort has several (equal modulo the number of workgroups), more often in a wavefront's ids than LDS keeps, one among the
    other; and vocabularies of more workgroups than 256."""
    torch = torch_mod()
    g = _gen(m + V + len(frequent))
    ids = torch.randint(0, V, (m,), generator=g)
    if frequent:
        often = torch.rand(m, generator=g) < 0.7
        ids[often] = torch.tensor(frequent)[torch.randint(0, len(frequent), (m,), generator=g)][often]
    ids[torch.rand(m, generator=g) < 0.05] = -1
    if not wide:
        ids = ids.to(torch.int32)
    dy = _randn(g, m, d).float()
    there = ids >= 0
    at = ids[there].long()
    want = torch.zeros(V, d, dtype=torch.float64).index_add_(0, at, dy[there].double())
    size = torch.zeros(V, d, dtype=torch.float64).index_add_(0, at, dy[there].double().abs())
    number = torch.bincount(at, minlength=V).double()[:, None]
    table, again = torch.full((V, d), math.nan, device="cuda"), torch.empty((V, d), device="cuda")
    tron.tron_embed_grad(ids.cuda(), dy.cuda(), table)
    _within(table, want, (number + 2) * E * size + TINY["f32"], "dtable")
    tron.tron_embed_grad(ids.cuda(), dy.cuda(), again)
    assert torch.equal(again, table)
    # rows that hold their own place: sums of whole numbers, exact in any order, which a wrong place would change
    whole = torch.stack([torch.arange(m) % 1021, torch.arange(m) // 1021], 1).float()
    table = torch.empty((V, 2), device="cuda")
    tron.tron_embed_grad(ids.cuda(), whole.cuda(), table)
    assert torch.equal(table.cpu().double(), torch.zeros(V, 2, dtype=torch.float64).index_add_(0, at, whole[there].double()))
