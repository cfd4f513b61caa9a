"""Layer norm and its gradient against plain implementations in 64 bits, and the norms' outputs in whole numbers of 8 bits.

Bounds, from the rounding of each step: U is the unit roundoff of the output's type, E = 2^-24 that of 32-bit sums.  A row's sums have at most 32 terms a
thread, and are joined by 6 steps in a wavefront and 16 in a workgroup: 64 roundings of E each cover them (LOST), relative to the sum of the terms' sizes."""
import math

import pytest

import paper_2008_03433_amd as tron
from test_gpu_heads import E, NORM_SIZES, TINY, U, _dt, _gen, _randn, _same, _strided, _surround_untouched, _within
from util import torch_mod

pytestmark = pytest.mark.gpu

LOST = 64 * E


def _plain(x, r, gain, shift, eps):
    """s, mean, rstd, y of the formula, and bounds of the errors of the last three."""
    s = x.double() if r is None else x.double() + r.double()
    mean = s.mean(1, keepdim=True)
    c = s - mean
    rstd = ((c * c).mean(1, keepdim=True) + eps) ** -0.5
    h = c * rstd
    g = 1.0 if gain is None else gain.double()
    b = torch_mod().zeros(s.shape[1], dtype=s.dtype) if shift is None else shift.double()
    # s is rounded once (E |s|), and so is c; the sum of c, which mends the mean, loses LOST of the sizes of its terms
    off_c = E * (s.abs() + s.abs().mean(1, keepdim=True)) + LOST * c.abs().mean(1, keepdim=True) + 2 * E * c.abs()
    # squares: LOST of their sum, and what the roundings of s do to them; half of that in the root, and a few of its own
    off_r = LOST + 2 * E * (s * s).mean(1, keepdim=True).sqrt() * rstd
    off_h = off_c * rstd + 1.01 * h.abs() * off_r
    y = h * g + b
    off_y = abs(g) * off_h + 4 * E * ((h * g).abs() + b.abs())
    off_mean = 2 * E * mean.abs() + E * s.abs().mean(1, keepdim=True) + LOST * c.abs().mean(1, keepdim=True)
    return s, mean[:, 0], rstd[:, 0], y, off_mean[:, 0], (off_r * rstd)[:, 0], off_y


def _cuda(t):
    return None if t is None else t.cuda()


@pytest.mark.parametrize("out", ["same", "e4m3", "i8"])
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("m,d", NORM_SIZES + [(70, 128), (33, 127), (19, 8), (21, 6), (9, 129)])
def test_layer_norm(m, d, kind, out):
    torch = torch_mod()
    g = _gen(7000 * m + d)
    dt, eps = _dt(kind), 1e-5
    with_r, with_gain, with_shift = (m + d) % 3 != 0, d % 2 == 1 or m == 1, d % 4 != 2
    # rows far from 0, too
    x = (_randn(g, m, d) + 20.0 * _randn(g, m, 1)).to(dt)
    r = _randn(g, m, d).to(dt) if with_r else None
    gain = (1.0 + 0.2 * _randn(g, d)).float() if with_gain else None
    shift = (0.2 * _randn(g, d)).float() if with_shift else None
    s, mean, rstd, y, off_mean, off_rstd, off_y = _plain(x, r, gain, shift, eps)
    pad = 3 if m > 1 else 0
    kind8 = {"e4m3": torch.float8_e4m3fn, "i8": torch.int8}.get(out)
    if out == "i8":
        room = torch.full((m, d + pad), 77, dtype=torch.int8, device="cuda")
        yv = room[:, :d]
    else:
        yv = _strided(torch.zeros((m, d)).to(dt if out == "same" else kind8), pad, 1)
    tv = _strided(torch.zeros((m, d), dtype=dt), pad, 1)
    ms, rs, scale = torch.empty(m, device="cuda"), torch.empty(m, device="cuda"), torch.empty(m, device="cuda") if kind8 else None
    tron.tron_layer_norm(_strided(x, pad, 1), yv, gain=_cuda(gain), shift=_cuda(shift), eps=eps, residual=None if r is None else _strided(r, pad + 2, 3), total=tv,
                         scale=scale, mean=ms, rstd=rs)
    _within(ms, mean, off_mean, "mean")
    _within(rs, rstd, off_rstd, "rstd")
    _within(tv, s, (U[kind] + E) * s.abs() + TINY[kind], "total")
    assert _surround_untouched(tv, pad, 1)
    if out == "same":
        _within(yv, y, U[kind] * y.abs() + (1 + U[kind]) * off_y + TINY[kind], "y")
        assert _surround_untouched(yv, pad, 1)
        return
    most = 448.0 if out == "e4m3" else 127.0
    want = y.abs().amax(1) / most
    want = torch.where(want > 0, want, 1.0)
    _within(scale, want, 4 * E * want + off_y.amax(1) / most, "scale")
    held = yv.float().double().cpu() * scale.double().cpu()[:, None]
    if out == "e4m3":   # four bits with the hidden one: half of 2^-3; below 2^-6: half of 2^-9
        _within(held, y, (2.0 ** -4 + 8 * E) * y.abs() + 1.1 * off_y + 2.0 ** -10 * 1.01 * want[:, None], "y")
    else:
        _within(held, y, 0.5 * 1.0001 * want[:, None] + 8 * E * y.abs() + 1.1 * off_y, "y")
        assert int(yv.max().abs()) <= 127 and int(yv.min()) >= -127
        assert (room[:, d:] == 77).all()


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("m,d", NORM_SIZES)
def test_rms_norm_to_whole_numbers(m, d, kind):
    torch = torch_mod()
    g = _gen(9000 * m + d)
    dt, eps = _dt(kind), 1e-6
    x, gain = _randn(g, m, d).to(dt), (1.0 + 0.2 * _randn(g, d)).float()
    rstd = ((x.double() ** 2).mean(1) + eps) ** -0.5
    y = x.double() * rstd[:, None] * gain.double()
    room = torch.full((m, d + 5), 77, dtype=torch.int8, device="cuda")
    scale = torch.empty(m, device="cuda")
    tron.tron_rms_norm(x.cuda(), room[:, :d], gain=gain.cuda(), eps=eps, scale=scale)
    want = y.abs().amax(1) / 127
    _within(scale, want, 2 * LOST * want, "scale")
    _within(room[:, :d].double().cpu() * scale.double().cpu()[:, None], y, 0.5 * (1 + 4 * LOST) * want[:, None] + 4 * LOST * y.abs(), "y")
    assert (room[:, d:] == 77).all()


def test_whole_numbers_of_rows_that_are_not_finite():
    torch = torch_mod()
    x = torch.randn(5, 1500, device="cuda")
    x[1], x[2, 17], x[3, 1499] = 0.0, math.nan, math.inf
    for norm in (tron.tron_rms_norm, tron.tron_layer_norm):
        y, scale = torch.full((5, 1500), 9, dtype=torch.int8, device="cuda"), torch.empty(5, device="cuda")
        norm(x, y, eps=1e-6, scale=scale)
        assert float(scale[1]) == 1.0 and (y[1] == 0).all()
        assert torch.isnan(scale[[2, 3]]).all() and (y[[2, 3]] == 0).all()
        assert torch.isfinite(scale[[0, 4]]).all() and (y[[0, 4]].abs().amax(1) == 127).all()
        norm(x[:, :40], y[:, :40], eps=0.0, scale=scale)   # no variance and no eps: 1/0 and 0 * inf
        assert math.isnan(float(scale[1])) and (y[1, :40] == 0).all()
    # a gain that is not finite
    gain = torch.ones(1500, device="cuda")
    gain[7] = math.inf
    for norm in (tron.tron_rms_norm, tron.tron_layer_norm):
        norm(x, y, eps=1e-6, scale=scale, gain=gain)
        assert torch.isnan(scale).all() and (y == 0).all()


@pytest.mark.parametrize("d", [40, 1500, 20000, 40000])
def test_layer_norm_of_rows_that_are_not_finite_or_do_not_vary(d):
    torch = torch_mod()
    x = torch.randn(6, d, device="cuda")
    x[1], x[2, d // 2], x[3, d - 1], x[4] = 0.0, math.nan, math.inf, 12345.678
    shift = torch.randn(d, device="cuda")
    y, mean, rstd = torch.empty_like(x), torch.empty(6, device="cuda"), torch.empty(6, device="cuda")
    tron.tron_layer_norm(x, y, shift=shift, eps=1e-5, mean=mean, rstd=rstd)
    assert torch.equal(y[1], shift) and float(mean[1]) == 0.0
    assert torch.isnan(y[[2, 3]]).all() and torch.isnan(rstd[[2, 3]]).all()
    # a row of one number: the rest of its mean is at most a unit of its last place (2^-10)
    assert float((y[4] - shift).abs().max()) <= 2.0 ** -9 * 1e-5 ** -0.5 * 2 ** -13
    assert float(mean[4]) == float(x[4, 0])
    assert torch.isfinite(y[[0, 5]]).all()
    tron.tron_layer_norm(x, y, eps=0.0, rstd=rstd)
    assert torch.isnan(y[1]).all() and math.isinf(float(rstd[1]))


@pytest.mark.parametrize("size", [1e30, 1e-30])
@pytest.mark.parametrize("d", [3, 700, 5000, 40000])
def test_layer_norm_of_rows_of_any_size(size, d):
    """Squares that 32 bits do not hold: with eps = 0 the output is that of the row at its ordinary size."""
    torch = torch_mod()
    x = (torch.randn(3, d, generator=_gen(d), dtype=torch.float64) * size).float()
    s, mean, rstd, y, off_mean, off_rstd, off_y = _plain(x, None, None, None, 0.0)
    yv, ms, rs = torch.empty_like(x, device="cuda"), torch.empty(3, device="cuda"), torch.empty(3, device="cuda")
    tron.tron_layer_norm(x.cuda(), yv, eps=0.0, mean=ms, rstd=rs)
    _within(yv, y, off_y + U["f32"] * y.abs() + TINY["f32"], "y")
    _within(rs, rstd, off_rstd + TINY["f32"], "rstd")
    _within(ms, mean, off_mean + TINY["f32"], "mean")


def test_layer_norm_in_place_and_of_one_row_for_all():
    torch = torch_mod()
    x, r = torch.randn(9, 300, device="cuda").bfloat16(), torch.randn(300, device="cuda").bfloat16().expand(9, 300)
    y, total = torch.empty_like(x), torch.empty_like(x)
    tron.tron_layer_norm(x, y, residual=r, total=total)
    again = torch.empty_like(x)
    own = x.clone()
    tron.tron_layer_norm(own, again, residual=r, total=own)   # the sum over x
    assert _same(again, y) and _same(own, total)
    tron.tron_layer_norm(x[:0], y[:0], residual=r[:0])
    assert _same(again, y)


@pytest.mark.parametrize("d", [1027, 1032, 1537, 8195, 20483])
def test_layer_norm_with_its_sum_over_x_or_the_residual(d):
    """Rows whose last chunk is another wavefront's than the one before it."""
    torch = torch_mod()
    x, r = torch.randn(700, d, device="cuda").bfloat16(), torch.randn(700, d, device="cuda").bfloat16()
    y, total, again = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x)
    tron.tron_layer_norm(x, y, residual=r, total=total)
    for over in ("x", "residual"):
        a, b = x.clone(), r.clone()
        tron.tron_layer_norm(a, again, residual=b, total=a if over == "x" else b)
        assert torch.equal(again, y) and torch.equal(a if over == "x" else b, total)


# --------------------------------------------------------------------------- gradient
def _plain_grad(total, mean, rstd, gain, dy, dtotal):
    s, dy, mean, rstd = total.double(), dy.double(), mean.double()[:, None], rstd.double()[:, None]
    g = torch_mod().ones(s.shape[1], dtype=s.dtype) if gain is None else gain.double()
    h, a = (s - mean) * rstd, dy * g
    level, along = a.mean(1, keepdim=True), (a * h).mean(1, keepdim=True)
    dx = rstd * (a - level - h * along)
    off = rstd.abs() * (6 * E * (a.abs() + level.abs() + (h * along).abs()) + LOST * (a.abs().mean(1, keepdim=True) + h.abs() * (a * h).abs().mean(1, keepdim=True)))
    if dtotal is not None:
        dx = dx + dtotal.double()
        off = off + E * dx.abs()
    n = s.shape[0]
    return dx, off, (dy * h).sum(0), (n + 8) * 2 * E * (dy * h).abs().sum(0), dy.sum(0), (n + 8) * 2 * E * dy.abs().sum(0)


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("m,d", NORM_SIZES + [(1500, 40), (700, 128), (333, 121), (50, 8), (37, 129), (700, 1030), (41, 700), (300, 9000), (70, 17000)])
def test_layer_norm_grad(m, d, kind):
    torch = torch_mod()
    g = _gen(11 * m + d)
    dt = _dt(kind)
    with_t, with_gain = (m + d) % 3 != 0, d % 2 == 1 or m == 1
    total = (_randn(g, m, d) + 3.0 * _randn(g, m, 1)).to(dt)
    dy, dtotal = _randn(g, m, d).to(dt), _randn(g, m, d).to(dt) if with_t else None
    gain = (1.0 + 0.2 * _randn(g, d)).float() if with_gain else None
    mean = total.double().mean(1).float()
    rstd = ((total.double() - mean.double()[:, None]).pow(2).mean(1) + 1e-5).rsqrt().float()
    dx, off, dgain, off_g, dshift, off_b = _plain_grad(total, mean, rstd, gain, dy, dtotal)
    pad = 3 if m > 1 else 0
    dxv, dg, db = _strided(torch.zeros((m, d), dtype=dt), pad, 1), torch.empty(d, device="cuda"), torch.empty(d, device="cuda")
    args = dict(gain=_cuda(gain), dtotal=None if dtotal is None else _strided(dtotal, pad, 2))
    tv, dyv = _strided(total, pad, 1), _strided(dy, pad + 1, 3)
    tron.tron_layer_norm_grad(tv, mean.cuda(), rstd.cuda(), dyv, dxv, dgain=dg, dshift=db, **args)
    _within(dxv, dx, U[kind] * dx.abs() + (1 + U[kind]) * off + TINY[kind], "dx")
    _within(dg, dgain, off_g, "dgain")
    _within(db, dshift, off_b, "dshift")
    assert _surround_untouched(dxv, pad, 1)
    # each alone: the same bits
    one, two, alone = torch.empty_like(dg), torch.empty_like(db), torch.empty((m, d), dtype=dt, device="cuda")
    tron.tron_layer_norm_grad(tv, mean.cuda(), rstd.cuda(), dyv, alone, dgain=one, **args)
    tron.tron_layer_norm_grad(tv, mean.cuda(), rstd.cuda(), dyv, alone, dshift=two, **args)
    assert torch.equal(one, dg) and torch.equal(two, db) and torch.equal(alone, dxv)
    # over dy, and over dtotal
    over = dyv.clone()
    tron.tron_layer_norm_grad(tv, mean.cuda(), rstd.cuda(), over, over, dgain=one, dshift=two, **args)
    assert torch.equal(over, alone) and torch.equal(one, dg) and torch.equal(two, db)
    if with_t:
        over = args["dtotal"].clone()
        tron.tron_layer_norm_grad(tv, mean.cuda(), rstd.cuda(), dyv, over, dgain=one, gain=args["gain"], dtotal=over)
        assert torch.equal(over, alone) and torch.equal(one, dg)


@pytest.mark.parametrize("m,d", [(4, 37), (3, 1300)])
def test_layer_norm_grad_against_differences(m, d):
    """Differences of the 64-bit formula: with steps of 1e-4 they are off by 1e-8 of the third derivative, which is below 100 here, and by 1e-11 of rounding."""
    torch = torch_mod()
    g = _gen(d)
    x, dy, v = _randn(g, m, d).float(), _randn(g, m, d).float(), _randn(g, m, d)
    gain, shift, u = (1.0 + 0.2 * _randn(g, d)).float(), _randn(g, d).float(), _randn(g, d)

    def loss(x, gain, shift):
        return float((_plain(x, None, gain, shift, 1e-5)[3] * dy.double()).sum())

    y, mean, rstd = torch.empty_like(x, device="cuda"), torch.empty(m, device="cuda"), torch.empty(m, device="cuda")
    tron.tron_layer_norm(x.cuda(), y, gain=gain.cuda(), shift=shift.cuda(), mean=mean, rstd=rstd)
    dx, dg, db = torch.empty_like(y), torch.empty(d, device="cuda"), torch.empty(d, device="cuda")
    tron.tron_layer_norm_grad(x.cuda(), mean, rstd, dy.cuda(), dx, gain=gain.cuda(), dgain=dg, dshift=db)
    h, (x, gain, shift) = 1e-4, (x.double(), gain.double(), shift.double())
    # 32-bit gradients: LOST of the sizes of what they sum
    for got, direction, plus, minus in ((dx, v, (x + h * v, gain, shift), (x - h * v, gain, shift)), (dg, u, (x, gain + h * u, shift), (x, gain - h * u, shift)),
                                        (db, u, (x, gain, shift + h * u), (x, gain, shift - h * u))):
        got = got.double().cpu()
        want, have = (loss(*plus) - loss(*minus)) / (2 * h), float((got * direction).sum())
        assert abs(have - want) <= 4 * LOST * float((got * direction).abs().sum()) + LOST * float(dy.abs().sum()) + 1e-5


def test_layer_norm_grad_of_broadcast_rows_and_of_no_rows():
    torch = torch_mod()
    m, d = 50, 600
    total, dy = torch.randn(m, d, device="cuda").bfloat16(), torch.randn(d, device="cuda").bfloat16()
    mean, rstd = torch.randn(m, device="cuda"), torch.rand(m, device="cuda")
    dx, dg, db = torch.empty_like(total), torch.empty(d, device="cuda"), torch.empty(d, device="cuda")
    tron.tron_layer_norm_grad(total, mean, rstd, dy.expand(m, d), dx, dgain=dg, dshift=db)
    dx2, dg2, db2 = torch.empty_like(total), torch.empty(d, device="cuda"), torch.empty(d, device="cuda")
    tron.tron_layer_norm_grad(total, mean, rstd, dy.repeat(m, 1), dx2, dgain=dg2, dshift=db2)
    assert torch.equal(dx, dx2) and torch.equal(dg, dg2) and torch.equal(db, db2)
    tron.tron_layer_norm_grad(total[:0], mean[:0], rstd[:0], dx2[:0], dx[:0], dgain=dg, dshift=db)
    assert (dg == 0).all() and (db == 0).all()
    tron.tron_layer_norm_grad(total[:0], mean[:0], rstd[:0], dx2[:0], dx[:0], dshift=dg2)
    assert (dg2 == 0).all()


@pytest.mark.parametrize("with_gain", [False, True])
@pytest.mark.parametrize("kind,value", [("f32", "lowest"), ("bf16", "lowest"), ("f32", 1e37), ("bf16", 1e37), ("f16", "lowest")])
@pytest.mark.parametrize("d", [1, 5, 8, 40, 43, 127, 700, 705, 1024, 1280, 5000, 9001, 16384, 17001, 17008])
def test_layer_norm_grad_of_rows_of_one_large_number(d, kind, value, with_gain):
    """mean * rstd passes 32 bits, and h is 0: dx = rstd (a - mean a).  Rows of many lengths, so that lanes and elements have no column."""
    torch = torch_mod()
    m, dt, g = 7, _dt(kind), _gen(d)
    total, dy, dtotal = _randn(g, m, d).to(dt), _randn(g, m, d).to(dt), _randn(g, m, d).to(dt)
    total[1:6] = torch.finfo(dt).min if value == "lowest" else value
    gain = (1.0 + 0.2 * _randn(g, d)).float() if with_gain else None
    mean = total.double().mean(1)
    rstd = ((total.double() - mean[:, None]).pow(2).mean(1) + 1e-5).rsqrt()
    mean, rstd = mean.float(), rstd.float()
    mean[1:6], rstd[1:6] = total[1:6, 0].float(), 1e-5 ** -0.5   # without the roundings of sums of such numbers
    dx, off, dgain, off_g, dshift, off_b = _plain_grad(total, mean, rstd, gain, dy, dtotal)
    got, dg, db = torch.empty((m, d), dtype=dt, device="cuda"), torch.empty(d, device="cuda"), torch.empty(d, device="cuda")
    tron.tron_layer_norm_grad(total.cuda(), mean.cuda(), rstd.cuda(), dy.cuda(), got, gain=_cuda(gain), dtotal=dtotal.cuda(), dgain=dg, dshift=db)
    _within(got, dx, U[kind] * dx.abs() + (1 + U[kind]) * off + TINY[kind], "dx")
    _within(dg, dgain, off_g + TINY["f32"], "dgain")
    _within(db, dshift, off_b, "dshift")


@pytest.mark.parametrize("value", [1e5, 3e8, 1e9, -3.3e12, 1e20, 1e26, 1e30, "lowest"])
@pytest.mark.parametrize("d", [1, 5, 41, 47, 55, 61, 82, 83, 97, 115, 128, 249, 509, 700, 1019, 1033, 1311, 4093, 8189, 8201, 32003, 33001])
def test_layer_norm_of_rows_of_one_number_or_nearly(d, value):
    """A row of one number has no variance, whatever its size and however its sum is rounded, and one of few numbers a unit of the last place apart has theirs.

    The squares' sum is taken in 32 bits only where at least half of it is the variance: a relative error of 2 LOST each of the two parts that are subtracted, 6 LOST of the
    variance, 3 LOST of the root.  Its mean is mended by the mean of c, off by 1.5 LOST sigma there, and by three roundings of |c| and of the first mean's error, 66 E |s|."""
    torch = torch_mod()
    value = torch.finfo(torch.float32).min if value == "lowest" else value
    x = torch.full((6, d), value, dtype=torch.float32)
    if d > 1:   # towards 0, so that the lowest one stays finite
        one = torch.nextafter(x[0, 0], torch.tensor(0.0))
        x[1, d // 2] = one
        x[2, 0] = one
        x[3, ::2] = one
        x[4, : d - d // 3] = one
    x[5] = torch.randn(d, generator=_gen(d))
    shift = torch.randn(d, generator=_gen(d + 1))
    s = x.double()
    mean = s.mean(1, keepdim=True)
    sigma = (s - mean).pow(2).mean(1, keepdim=True).sqrt()
    rstd = (sigma * sigma + 1e-5) ** -0.5
    h = (s - mean) * rstd
    off_h = rstd * (1.5 * LOST * sigma + 3 * E * ((s - mean).abs() + 2 * 66 * E * s.abs())) + 3 * LOST * h.abs()
    y, ms, rs = torch.empty((6, d), device="cuda"), torch.empty(6, device="cuda"), torch.empty(6, device="cuda")
    tron.tron_layer_norm(x.cuda(), y, shift=shift.cuda(), eps=1e-5, mean=ms, rstd=rs)
    _within(rs, rstd[:, 0], (3 * LOST + 4 * E) * rstd[:, 0], "rstd")
    _within(y, h + shift.double(), off_h + 4 * E * (h.abs() + shift.double().abs()), "y")
    assert torch.equal(y[0].cpu(), shift) and float(ms[0]) == float(x[0, 0])
    _within(ms, mean[:, 0], 2 * E * mean[:, 0].abs() + 2 * LOST * sigma[:, 0], "mean")
