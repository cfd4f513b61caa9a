"""Operators of a multi-class head against plain implementations in 64 bits.

Bounds, from the rounding of each step: U is the unit roundoff of the output's type, E = 2^-24 that of 32-bit sums.  A result is rounded once to its type; before that a sum of n terms in 32 bits, in any order and
truncated at worst, is off by at most (n + 8) 2 E times the sum of its terms' sizes."""
import math

import pytest

import paper_2008_03433_amd as tron
from util import torch_mod

pytestmark = pytest.mark.gpu

E = 2.0 ** -24
U = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}   # |round(x) - x| <= U |x| (bf16: 8 bits with the hidden one: half of 2^-7)
TINY = {"f32": 2.0 ** -149, "f16": 2.0 ** -25, "bf16": 2.0 ** -133}   # half the spacing of the smallest numbers, or more


def _dt(name):
    torch = torch_mod()
    return {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn}[name]


def _gen(seed):
    torch = torch_mod()
    return torch.Generator().manual_seed(seed)


def _randn(g, *shape):
    torch = torch_mod()
    return torch.randn(*shape, generator=g, dtype=torch.float64)


def _strided(t, pad, offset=0):
    """The same values in rows that lie `pad` elements further apart, `offset` elements into a buffer, with NaN around them."""
    torch = torch_mod()
    m, d = t.shape
    ld = d + pad
    buf = torch.full((m * ld + offset + 16,), math.nan, dtype=torch.float32).to(t.dtype).to("cuda")
    view = buf[offset:offset + m * ld].view(m, ld)[:, :d]
    view.copy_(t)
    return view


def _surround_untouched(view, pad, offset):
    """Whether nothing was written beside a view that _strided made."""
    torch = torch_mod()
    m, d = view.shape
    whole = view.new_empty(0).set_(view.untyped_storage())
    keep = torch.zeros(whole.numel(), dtype=torch.bool, device="cuda")
    keep[offset:offset + m * (d + pad)].view(m, d + pad)[:, :d] = True
    rest = whole[~keep]
    return bool(torch.isnan(rest.float()).all())


def _within(got, want, bound, what=""):
    torch = torch_mod()
    got, want, bound = got.double().cpu(), want.double().cpu(), bound.double().cpu()
    assert got.shape == want.shape, what
    nan = torch.isnan(want)
    assert torch.equal(torch.isnan(got), nan), what
    got, want, bound = got[~nan], want[~nan], bound[~nan]
    if not got.numel():
        return
    assert torch.isfinite(got).all(), what
    over = (got - want).abs() - bound
    at = int(over.argmax())
    assert float(over.max()) <= 0.0, f"{what}: off by {float((got - want).abs().flatten()[at]):.3e} where {float(bound.flatten()[at]):.3e} is allowed"


def _same(a, b):
    """Equal values, NaN in the same places."""
    torch = torch_mod()
    return torch.equal(torch.isnan(a), torch.isnan(b)) and torch.equal(a.float().nan_to_num(nan=0.0), b.float().nan_to_num(nan=0.0))


# --------------------------------------------------------------------------- norm
NORM_SIZES = [(1, 1), (3, 7), (1, 64), (5, 511), (9, 513), (2, 1024), (7, 1025), (6, 2048), (3, 2049), (4, 4096), (2, 8192), (3, 8195), (2, 16385), (2, 32768), (1, 32771)]


def _norm_plain(x, r, gain, eps):
    s = x.double() if r is None else x.double() + r.double()
    rstd = ((s * s).mean(1) + eps) ** -0.5
    y = s * rstd[:, None]
    return s, rstd, y if gain is None else y * gain.double()


@pytest.mark.parametrize("out", ["same", "e4m3"])
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("m,d", NORM_SIZES)
def test_norm(m, d, kind, out):
    torch = torch_mod()
    g = _gen(1000 * m + d)
    dt, eps, u = _dt(kind), 1e-5, U[kind]
    with_r, with_gain = (m + d) % 3 != 0, d % 2 == 1 or m == 1
    x, r = _randn(g, m, d).to(dt), _randn(g, m, d).to(dt) if with_r else None
    gain = (1.0 + 0.2 * _randn(g, d)).float() if with_gain else None
    s, rstd, y = _norm_plain(x, r, gain, eps)
    pad = 3 if m > 1 else 0
    yv = _strided(torch.zeros((m, d)).to(dt if out == "same" else _dt("e4m3")), pad, 1)
    tv = _strided(torch.zeros((m, d), dtype=dt), pad, 1)
    rs, scale = torch.empty(m, device="cuda"), torch.empty(m, device="cuda") if out == "e4m3" else None
    tron.tron_rms_norm(_strided(x, pad, 1), yv, gain=None if gain is None else gain.cuda(), eps=eps, residual=None if r is None else _strided(r, pad + 2, 3), total=tv,
                       scale=scale, rstd=rs)
    # the sum of squares, its root and the products with rstd and gain: 64 roundings cover sums of up to 32 squares a thread and their joining
    lost = 64 * E
    _within(rs, rstd, lost * rstd, "rstd")
    _within(tv, s, (u + E) * s.abs() + TINY[kind], "total")
    if out == "same":
        _within(yv, y, (u + 2 * lost) * y.abs() + TINY[kind], "y")
        assert _surround_untouched(yv, pad, 1)
    else:
        want = y.abs().amax(1) / 448
        want = torch.where(want > 0, want, 1.0)
        _within(scale, want, 2 * lost * want, "scale")
        # four bits with the hidden one: half of 2^-3; below 2^-6: half of 2^-9
        _within(yv.float().double().cpu() * scale.double().cpu()[:, None], y, (2.0 ** -4 + 4 * lost) * y.abs() + 2.0 ** -10 * (1 + lost) * want[:, None], "y")
    assert _surround_untouched(tv, pad, 1)


def test_norm_rows_of_zeros_and_of_what_is_not_finite():
    torch = torch_mod()
    x = torch.randn(5, 100, device="cuda").bfloat16()
    x[1] = 0.0
    x[2, 17] = math.nan
    x[3, 5] = math.inf
    y, scale, rstd = torch.empty_like(x, dtype=_dt("e4m3")), torch.empty(5, device="cuda"), torch.empty(5, device="cuda")
    tron.tron_rms_norm(x, y, eps=0.0, scale=scale, rstd=rstd)
    f = y.float()
    # no variance and no eps: 1/0 and 0 * inf
    assert torch.isnan(f[1]).all() and math.isinf(float(rstd[1]))
    assert torch.isnan(f[2]).all() and math.isnan(float(rstd[2]))
    assert math.isnan(float(f[3, 5])) and float(rstd[3]) == 0.0
    assert torch.isfinite(f[[0, 4]]).all() and (scale[[0, 4]] > 0).all()
    tron.tron_rms_norm(x, y, eps=1e-6, scale=scale)
    assert (y.float()[1] == 0).all() and float(scale[1]) == 1.0
    # values whose scale would be no normal number
    x[1] = 1e-39
    tron.tron_rms_norm(x.float(), y, eps=1e-6, scale=scale)
    assert torch.isfinite(y.float()[1]).all() and float(scale[1]) > 0


def test_norm_in_place_broadcast_and_empty():
    torch = torch_mod()
    x, r = torch.randn(6, 300, device="cuda"), torch.randn(1, 300, device="cuda")
    s = x.double() + r.double()
    y, y2 = torch.empty_like(x), torch.empty_like(x)
    tron.tron_rms_norm(x, y, residual=r.expand(6, 300), total=x)
    _within(x, s, E * s.abs() + 1e-45, "total in place of x")
    tron.tron_rms_norm(x, y2)
    _within(y2, y.double().cpu(), 256 * E * y.double().cpu().abs() + 1e-7, "of the stored sum")
    e = torch.empty((0, 300), device="cuda")
    tron.tron_rms_norm(e, e.clone())
    dgain = torch.full((300,), 7.0, device="cuda")
    tron.tron_rms_norm_grad(e, torch.empty(0, device="cuda"), e, e.clone(), dgain=dgain)
    assert (dgain == 0).all()


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("m,d", NORM_SIZES + [(40, 33), (5000, 24), (2100, 2056), (1100, 2500)])
def test_norm_gradient(m, d, kind):
    torch = torch_mod()
    g = _gen(2000 * m + d)
    dt, u = _dt(kind), U[kind]
    s, dy = _randn(g, m, d).to(dt), _randn(g, m, d).to(dt)
    dtotal = _randn(g, m, d).to(dt) if m % 2 else None
    gain = (1.0 + 0.2 * _randn(g, d)).float() if d % 2 or m > 4 else None
    rstd = ((s.double() ** 2).mean(1) + 1e-5).rsqrt().float()
    pad = 5 if m > 1 else 0
    dx = _strided(torch.zeros((m, d), dtype=dt), pad, 1)
    dgain = torch.empty(d, device="cuda")
    tron.tron_rms_norm_grad(_strided(s, pad, 1), rstd.cuda(), _strided(dy, pad, 3), dx, gain=None if gain is None else gain.cuda(),
                            dtotal=None if dtotal is None else _strided(dtotal, pad, 1), dgain=dgain)
    S, R, A = s.double(), rstd.double()[:, None], dy.double() * (1.0 if gain is None else gain.double())
    back = R * R * (A * S).mean(1, keepdim=True)
    want = R * (A - S * back) + (0.0 if dtotal is None else dtotal.double())
    # the mean's error, 64 roundings of its terms' sizes; the other factors' roundings
    size = R * (A.abs() + S.abs() * R * R * (A * S).abs().mean(1, keepdim=True)) + (0.0 if dtotal is None else dtotal.double().abs())
    _within(dx, want, u * want.abs() + 80 * E * size + TINY[kind], "dx")
    assert _surround_untouched(dx, pad, 1)
    terms = dy.double() * S * R
    _within(dgain, terms.sum(0), (m + 8) * 2 * E * terms.abs().sum(0), "dgain")


def test_norm_gradient_against_differences():
    torch = torch_mod()
    g = _gen(7)
    m, d, eps, h = 3, 70, 1e-3, 2.0 ** -8
    x, dy, gain = (_randn(g, m, d).float().cuda(), _randn(g, m, d).float().cuda(), (1 + 0.2 * _randn(g, d)).float().cuda())
    y, rstd, dx, dgain = torch.empty_like(x), torch.empty(m, device="cuda"), torch.empty_like(x), torch.empty(d, device="cuda")
    tron.tron_rms_norm(x, y, gain=gain, eps=eps, rstd=rstd)
    tron.tron_rms_norm_grad(x, rstd, dy, dx, gain=gain, dgain=dgain)

    def f(a, b):
        out = torch.empty_like(x)
        tron.tron_rms_norm(a, out, gain=b, eps=eps)
        return float((out.double() * dy.double()).sum())

    # the quotient is off by h^2 / 6 of a third derivative of size about 1, and by the values' roundings, sqrt(210) E a sum of about 200 / 2h
    for j in (0, 33, 69):
        e = torch.zeros_like(x)
        e[1, j] = h
        assert abs((f(x + e, gain) - f(x - e, gain)) / (2 * h) - float(dx[1, j])) < 1e-3
        e = torch.zeros_like(gain)
        e[j] = h
        assert abs((f(x, gain + e) - f(x, gain - e)) / (2 * h) - float(dgain[j])) < 1e-3


# --------------------------------------------------------------------------- matrix product
def _act64(a, act):
    torch = torch_mod()
    return [lambda v: v, torch.relu, torch.nn.functional.gelu, torch.nn.functional.silu][act](a)


def _operand(g, rows, k, kind, std=1.0):
    """(tensor, scale or None, values in 64 bits)"""
    torch = torch_mod()
    a = _randn(g, rows, k) * std
    if kind != "e4m3":
        a = a.to(_dt(kind))
        return a, None, a.double()
    scale = (a.abs().amax(1) / 448).float()
    q = (a.float() / scale[:, None]).to(torch.float8_e4m3fn)
    return q, scale, q.float().double() * scale.double()[:, None]


LINEAR_SIZES = [(1, 1, 1), (1, 16, 32), (2, 65, 129), (16, 64, 64), (17, 130, 200), (33, 48, 1000), (64, 257, 513), (65, 64, 8), (100, 100, 100), (128, 128, 128),
                (129, 127, 65), (130, 300, 1030), (70, 20, 4100), (1, 200, 5000), (300, 513, 72)]


def _check_linear(m, n, k, kind, out, act, bias, residual, pre, pads=(0, 0), seed=0):
    torch = torch_mod()
    g = _gen(seed + 31 * m + 7 * n + k)
    x, xs, X = _operand(g, m, k, kind)
    w, ws, W = _operand(g, n, k, kind, k ** -0.5)
    b = _randn(g, n).float() if bias else None
    r = _randn(g, m, n).to(_dt(out)) if residual else None
    y = _strided(torch.zeros((m, n), dtype=_dt(out)), 3, 1)
    p = _strided(torch.zeros((m, n), dtype=_dt(out)), 1, 1) if pre else None
    tron.tron_linear(_strided(x, *pads), _strided(w, *pads), y, bias=None if b is None else b.cuda(), act=act, residual=None if r is None else _strided(r, 2, 1), pre=p,
                     x_scale=None if xs is None else xs.cuda(), w_scale=None if ws is None else ws.cuda())
    a = X @ W.T + (0.0 if b is None else b.double())
    size = X.abs() @ W.abs().T + (0.0 if b is None else b.double().abs())
    off = (k + 8) * 2 * E * size
    u, tiny = U[out], TINY[out]
    if pre:
        _within(p, a, u * a.abs() + off + tiny, "pre")
        assert _surround_untouched(p, 1, 1)
    want = _act64(a, act)
    # slopes of the activations are at most 1.13, their own roundings a few of 32 bits of |a|
    bound = 1.13 * off + 16 * E * (want.abs() + a.abs())
    if residual:
        want = want + r.double()
    _within(y, want, u * want.abs() + bound * (1 + u) + E * want.abs() + tiny, "y")
    assert _surround_untouched(y, 3, 1)


@pytest.mark.parametrize("kind,out", [("bf16", "bf16"), ("bf16", "f32"), ("f16", "f16"), ("e4m3", "bf16"), ("e4m3", "f32")])
@pytest.mark.parametrize("m,n,k", LINEAR_SIZES)
def test_linear(m, n, k, kind, out):
    _check_linear(m, n, k, kind, out, act=(m + n) % 4, bias=n % 2 == 1, residual=k % 2 == 0, pre=m % 2 == 1)


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("m,n,k", [(3, 40, 96), (80, 150, 260), (150, 140, 512)])
@pytest.mark.parametrize("pads", [(1, 0), (0, 1), (16, 16), (7, 3)])
def test_linear_rows_anywhere(m, n, k, kind, pads):
    _check_linear(m, n, k, kind, "bf16", act=tron.ACT_GELU, bias=True, residual=True, pre=True, pads=pads)


# the tiles of many rows: several of both kinds, ragged at both ends, an inner length that ends inside a step and inside a chunk
@pytest.mark.parametrize("kind", ["bf16", "f16", "e4m3"])
@pytest.mark.parametrize("m,n,k", [(4096, 4096, 144), (4000, 4200, 200), (4100, 4099, 77), (1000, 1500, 320), (257, 300, 8200)])
def test_linear_large(m, n, k, kind):
    torch = torch_mod()
    g = torch.Generator(device="cuda").manual_seed(m + n + k)
    x = torch.randn(m, k, generator=g, device="cuda")
    w = torch.randn(n, k, generator=g, device="cuda") * k ** -0.5
    xs = ws = None
    if kind == "e4m3":
        xs, ws = x.abs().amax(1) / 448, w.abs().amax(1) / 448
        x, w = (x / xs[:, None]).to(_dt(kind)), (w / ws[:, None]).to(_dt(kind))
        X, W = x.float().double() * xs.double()[:, None], w.float().double() * ws.double()[:, None]
    else:
        x, w = x.to(_dt(kind)), w.to(_dt(kind))
        X, W = x.double(), w.double()
    y = torch.empty((m, n), device="cuda")
    tron.tron_linear(x, w, y, x_scale=xs, w_scale=ws)
    want, size = X @ W.T, X.abs() @ W.abs().T
    _within(y, want, (k + 8) * 2 * E * size + E * want.abs(), "y")
    again = torch.empty_like(y)
    tron.tron_linear(x, w, again, x_scale=xs, w_scale=ws)
    assert torch.equal(y, again)


def test_linear_residual_in_place_of_the_output_broadcast_rows_and_no_rows():
    torch = torch_mod()
    for m, n, k in ((5, 70, 64), (200, 150, 128)):
        x, w = torch.randn(m, k, device="cuda").bfloat16(), (torch.randn(n, k, device="cuda") / 8).bfloat16()
        y, r = torch.empty(m, n, device="cuda"), torch.randn(m, n, device="cuda")
        tron.tron_linear(x, w, y, residual=r)
        tron.tron_linear(x, w, r, residual=r)
        assert torch.equal(y, r)
        one, y2 = x[:1].expand(m, k), torch.empty_like(y)
        tron.tron_linear(one, w, y2)
        tron.tron_linear(one.contiguous(), w, y)
        assert torch.equal(y, y2)
    e = torch.empty(0, 64, device="cuda").bfloat16()
    dw, db = torch.full((70, 64), 3.0, device="cuda"), torch.full((70,), 3.0, device="cuda")
    tron.tron_linear(e, torch.zeros(70, 64, device="cuda").bfloat16(), torch.empty(0, 70, device="cuda"))
    tron.tron_linear_grad(e, None, torch.empty(0, 70, device="cuda").bfloat16(), dw=dw, dbias=db)
    assert (dw == 0).all() and (db == 0).all()


def test_linear_what_is_not_finite_stays_in_its_row_and_column():
    torch = torch_mod()
    for m in (7, 140):
        n, k = 130, 72
        x, w = torch.randn(m, k, device="cuda").bfloat16(), torch.randn(n, k, device="cuda").bfloat16()
        x[3, 70], w[100, 5] = math.nan, math.inf
        y = torch.empty(m, n, device="cuda")
        tron.tron_linear(x, w, y)
        bad = torch.zeros(m, n, dtype=torch.bool, device="cuda")
        bad[3], bad[:, 100] = True, True
        assert torch.equal(~torch.isfinite(y), bad)
        tron.tron_linear(x, w, y, act=tron.ACT_RELU)
        assert torch.isnan(y[3]).all() and torch.isfinite(y[~bad]).all()


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("m,n,k", [(1, 1, 1), (1, 40, 70), (5, 64, 64), (65, 33, 129), (64, 200, 72), (130, 70, 257), (300, 140, 90), (700, 24, 16), (513, 300, 264)])
def test_linear_gradients(m, n, k, kind):
    torch = torch_mod()
    g = _gen(m + 3 * n + 5 * k)
    dt, u = _dt(kind), U[kind]
    act = (m + n + k) % 4
    x, w, dy, pre = (a.to(dt) for a in (_randn(g, m, k), _randn(g, n, k) * k ** -0.5, _randn(g, m, n), _randn(g, m, n)))
    dw_kind = "f32" if k % 2 else kind
    dx, dw, db = _strided(torch.zeros((m, k), dtype=dt), 3, 1), _strided(torch.zeros((n, k)).to(_dt(dw_kind)), 1, 1), torch.empty(n, device="cuda")
    tron.tron_linear_grad(_strided(x, 1, 1), _strided(w, 2, 1), _strided(dy, 3, 1), dx=dx, dw=dw, dbias=db, act=act, pre=_strided(pre, 5, 1) if act else None)
    a = pre.double().requires_grad_()
    (d,) = torch.autograd.grad(_act64(a, act), a, dy.double())
    # dpre is rounded to the operands' type where there is an activation, after roundings of 32 bits of its factors (slopes up to 1.13)
    off = (u * d.abs() if act else 0.0) + 32 * E * dy.double().abs()
    X, W = x.double(), w.double()
    want = d @ W
    _within(dx, want, u * want.abs() * (1 + u) + (off + (n + 8) * 2 * E * d.abs()) @ W.abs() * (1 + u) + TINY[kind] * (1 + W.abs().sum(0)), "dx")
    want = d.T @ X
    ud = U[dw_kind]
    _within(dw, want, ud * want.abs() * (1 + u) + (off + (m + 8) * 2 * E * d.abs()).T @ X.abs() * (1 + u) + TINY[kind] * (1 + X.abs().sum(0)), "dw")
    _within(db, d.sum(0), ((m + 8) * 2 * E * d.abs() + 32 * E * dy.double().abs()).sum(0), "dbias")
    assert _surround_untouched(dx, 3, 1) and _surround_untouched(dw, 1, 1)
    # one at a time: the same bits
    for want_dx, want_dw, want_db in ((1, 0, 0), (0, 1, 0), (0, 0, 1)):
        o = [torch.empty_like(t) if f else None for t, f in ((dx.contiguous(), want_dx), (dw.contiguous(), want_dw), (db, want_db))]
        tron.tron_linear_grad(x.cuda() if want_dw else None, w.cuda() if want_dx else None, dy.cuda(), dx=o[0], dw=o[1], dbias=o[2], act=act, pre=pre.cuda() if act else None)
        for got, all_at_once in zip(o, (dx, dw, db)):
            assert got is None or torch.equal(got, all_at_once)


# few rows, whose dx reads w as it lies: its ends inside a thread's columns, in one part and in many, either side of each bound on the rows
@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("m,n,k", [(2, 700, 600), (4, 1000, 513), (5, 257, 1030), (8, 63, 64), (9, 2100, 520), (16, 4100, 1025), (16, 40, 7), (17, 1500, 96), (12, 34000, 1001)])
def test_linear_gradients_of_few_rows(m, n, k, kind):
    test_linear_gradients(m, n, k, kind)


def test_linear_gradients_of_few_rows_keep_what_is_not_finite():
    torch = torch_mod()
    m, n, k = 6, 300, 530
    dy, w = torch.randn(m, n, device="cuda").bfloat16(), torch.randn(n, k, device="cuda").bfloat16()
    dy[2, 299], w[17, 529] = math.nan, math.inf
    dx = torch.empty(m, k, device="cuda").bfloat16()
    tron.tron_linear_grad(None, w, dy, dx=dx)
    bad = torch.zeros(m, k, dtype=torch.bool, device="cuda")
    bad[2], bad[:, 529] = True, True
    assert torch.equal(~torch.isfinite(dx), bad)


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("m,n,k", [(1, 60, 30000), (20, 9, 20001), (200, 100, 9000)])
def test_linear_cut_in_many(m, n, k, kind):
    _check_linear(m, n, k, kind, "f32", act=tron.ACT_SILU, bias=True, residual=True, pre=True)


def test_linear_gradients_against_differences():
    torch = torch_mod()
    g = _gen(3)
    m, n, k, h = 6, 5, 64, 2.0 ** -3
    for act in (tron.ACT_NONE, tron.ACT_GELU, tron.ACT_SILU):
        # multiples of 2^-3 and 2^-6: moved by h they are still numbers of the type, and the products are exact in 32 bits
        x = (torch.randint(-8, 9, (m, k), generator=g) / 8).bfloat16().cuda()
        w = (torch.randint(-8, 9, (n, k), generator=g) / 64).bfloat16().cuda()
        dy = (torch.randint(-8, 9, (m, n), generator=g) / 8).bfloat16().cuda()
        b = torch.zeros(n, device="cuda")
        y, pre = torch.empty(m, n, device="cuda"), torch.empty(m, n, device="cuda")

        def f(x, w, b):
            tron.tron_linear(x, w, y, bias=b, act=act, pre=pre)
            return float((y.double() * dy.double()).sum())

        f(x, w, b)
        dx, dw, db = torch.empty_like(x), torch.empty(n, k, device="cuda"), torch.empty(n, device="cuda")
        tron.tron_linear_grad(x, w, dy, dx=dx, dw=dw, dbias=db, act=act, pre=pre.bfloat16())
        # rounding of pre (|pre| < 4: up to 2^-7, times a curvature of at most 0.8) and of dpre, 2^-8 of it; the quotient's error h^2 / 6 times a third
        # derivative of at most 1, the moved input's factor cubed
        def near(quotient, got, factor):
            size = float((dy.double().abs() * 1.13).sum(1).max()) * factor
            assert abs(quotient - float(got)) <= size * (2.0 ** -7 * 0.8 + 2.0 ** -7) + m * n * (h * factor) ** 2 / 6 + 1e-5

        e = torch.zeros_like(x)
        e[2, 9] = h
        near((f(x + e, w, b) - f(x - e, w, b)) / (2 * h), dx[2, 9], float(w.abs().max()))
        e = torch.zeros_like(b)
        e[3] = h
        near((f(x, w, b + e) - f(x, w, b - e)) / (2 * h), db[3], m)
        e = torch.zeros_like(w)
        e[1, 30] = 2.0 ** -6
        near((f(x, w + e, b) - f(x, w - e, b)) / 2.0 ** -5, dw[1, 30], m)


# --------------------------------------------------------------------------- distillation
def _distill_plain(z, ids, t, T, weight):
    """loss, lse, dz, p and the weights that count, in 64 bits, entry by entry."""
    torch = torch_mod()
    m, V = z.shape
    z, t = z.double() / T, t.double() / T
    loss, lse, q = torch.zeros(m, dtype=torch.float64), torch.zeros(m, dtype=torch.float64), torch.zeros(m, V, dtype=torch.float64)
    w = weight.double().clone()
    for i in range(m):
        lse[i] = torch.logsumexp(z[i], 0)
        there = [(int(c), float(v)) for c, v in zip(ids[i], t[i]) if 0 <= int(c) < V]
        if any(math.isnan(v) for _, v in there):
            loss[i] = math.nan
            q[i, [c for c, _ in there]] = math.nan
            continue
        top = max((v for _, v in there), default=-math.inf)
        if top == -math.inf:
            w[i] = 0.0
            continue
        total = sum(math.exp(v - top) for _, v in there)
        for c, v in there:
            p = math.exp(v - top) / total
            if p > 0:
                q[i, c] += p
                loss[i] += p * (v - top - math.log(total) - (float(z[i, c]) - float(lse[i])))
        if float(lse[i]) == -math.inf:
            loss[i] = math.inf
    p = torch.where(lse[:, None] == -math.inf, 0.0, torch.exp(z - torch.where(lse == -math.inf, 0.0, lse)[:, None]))
    w = w[:, None]
    loss = torch.where(w[:, 0] == 0, 0.0, w[:, 0] * T * T * loss)
    return loss, lse, torch.where(w == 0, 0.0, w * T * (p - q)), p, q, w


DISTILL_SIZES = [(1, 1, 1), (2, 5, 3), (3, 100, 100), (1, 4097, 7), (4, 9001, 65), (5, 33000, 20), (2, 50021, 300), (1100, 130, 9), (1030, 4100, 4), (1025, 16500, 2), (1, 3, 0)]


def _distill_inputs(m, V, K, kind, seed):
    torch = torch_mod()
    g = _gen(seed + 17 * m + V + K)
    z = (3 * _randn(g, m, V)).to(_dt(kind))
    ids = torch.randint(0, V, (m, K), generator=g)
    t = (3 * _randn(g, m, K)).float()
    if K > 1:
        ids[::3, -1] = -1
        t[::3, -1] = math.nan          # a missing entry's value says nothing
        ids[::2, 1] = ids[::2, 0]      # listed twice
    if m > 2:
        ids[2] = -5
        ids[2, -1:] = V                # nothing that lies in the row
    weight = torch.rand(m, generator=g) + 0.5
    if m > 1:
        weight[1] = 0.0
        z[1, V // 2] = math.nan        # of a row that does not count
    if V > 20:
        z[0, 5:9] = -math.inf
        ids[0][(ids[0] >= 5) & (ids[0] < 9)] = 4
    return z, ids, t, weight


def _distill_bounds(kind, z, lse, p, q, w, T, V):
    """Errors of lse, of loss and of dz before and after rounding."""
    u = U[kind]
    # sums of V / 512 terms a thread at worst with their exponents' roundings (arguments up to 64: 64 E each, an instruction of two units)
    off = (V / 512 + 160) * E
    lse_b = E * lse.abs() + off
    # from the stored lse and z / T: three roundings of numbers of their size
    arg = (4 * lse.abs()[:, None] + 4 * abs(1 / T) * z.double().abs().nan_to_num(posinf=0.0, neginf=0.0, nan=0.0)) * E + off
    return lse_b, off, p * (arg + 8 * E) + q * 8 * E


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("m,V,K", DISTILL_SIZES)
def test_distill(m, V, K, kind):
    torch = torch_mod()
    z, ids, t, weight = _distill_inputs(m, V, K, kind, 5)
    T = (1.0, 2.0, 0.7)[(m + V) % 3]
    if m > 64:   # the plain implementation goes entry by entry: some rows of many
        some = torch.cat([torch.arange(40), torch.arange(m - 3, m)])
    else:
        some = torch.arange(m)
    loss, lse, dz, p, q, w = _distill_plain(z[some], ids[some], t[some], T, weight[some])
    lse_b, off, dz_b = _distill_bounds(kind, z[some], lse, p, q, w, T, V)
    dev_ids = (ids if V % 2 else ids.int()).cuda()
    got_loss, got_lse = torch.empty(m, device="cuda"), torch.empty(m, device="cuda")
    out = _strided(torch.zeros((m, V), dtype=_dt(kind)), 3, 1)
    zd, wd, td = _strided(z, 5, 1), weight.cuda(), t.cuda()
    tron.tron_distill(zd, dev_ids, td, got_loss, got_lse, temperature=T, weight=wd, dz=out)
    finite = ~torch.isnan(z[some]).any(1)
    assert torch.isnan(got_lse.cpu()[some][~finite]).all()
    _within(got_lse[some.cuda()][finite.cuda()], lse[finite], lse_b[finite], "lse")
    _within(got_loss[some.cuda()], loss, w[:, 0] * T * T * (off + 1e-12 * lse.abs().nan_to_num()) + 2 * E * loss.abs(), "loss")
    bound = lambda extra: U[kind] * dz.abs() + (w * T * torch.where(torch.isnan(dz_b), 0.0, dz_b)) * (1 + U[kind]) + extra + TINY[kind]  # noqa: E731
    _within(out[some.cuda()], dz, bound(4 * E * dz.abs()), "dz")
    assert _surround_untouched(out, 3, 1)
    assert (out[weight.cuda() == 0] == 0).all()

    only = torch.empty(m, device="cuda")
    tron.tron_distill(zd, dev_ids, td, only, temperature=T, weight=wd)
    assert _same(only, got_loss)

    after = _strided(torch.zeros((m, V), dtype=_dt(kind)), 3, 1)
    tron.tron_distill_grad(zd, got_lse, dev_ids, td, after, temperature=T, weight=wd)
    _within(after[some.cuda()], dz, bound(4 * E * dz.abs()), "dz from lse")
    assert _surround_untouched(after, 3, 1)

    # in place of the logits
    mine = z.cuda()
    tron.tron_distill(mine, dev_ids, td, got_loss, temperature=T, weight=wd, dz=mine)
    assert _same(mine, out)
    mine = z.cuda()
    tron.tron_distill_grad(mine, got_lse, dev_ids, td, mine, temperature=T, weight=wd)
    assert _same(mine, after)


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("m,V,K", DISTILL_SIZES)
def test_distill_hessian_vector_product(m, V, K, kind):
    torch = torch_mod()
    z, ids, t, weight = _distill_inputs(m, V, K, kind, 6)
    T = (1.0, 2.0, 0.7)[(m + V) % 3]
    some = torch.cat([torch.arange(40), torch.arange(m - 3, m)]) if m > 64 else torch.arange(m)
    u = _randn(_gen(m + V), m, V).to(_dt(kind))
    _, lse, _, p, _, w = _distill_plain(z[some], ids[some], t[some], T, weight[some])
    all_lse = torch.logsumexp(z.double() / T, 1).float()
    hu = _strided(torch.zeros((m, V), dtype=_dt(kind)), 1, 1)
    tron.tron_distill_hv(_strided(z, 1, 1), all_lse.cuda(), _strided(u, 3, 1), hu, ids=ids.cuda(), t=t.cuda(), temperature=T, weight=weight.cuda())
    U64 = u[some].double()
    P = torch.where(w == 0, 0.0, p)
    want = w * (P * U64 - P * (P * U64).sum(1, keepdim=True))
    _, _, off = _distill_bounds(kind, z[some], lse, P, torch.zeros_like(P), w, T, V)
    off = torch.where(w == 0, 0.0, off)
    rel = torch.where(P > 0, off / P, 0.0).amax(1, keepdim=True)   # of a probability
    size = P * (U64.abs() + (P * U64.abs()).sum(1, keepdim=True))
    _within(hu[some.cuda()], want, U[kind] * want.abs() + w * size * (2 * rel + (V / 512 + 40) * 2 * E) * (1 + U[kind]) + TINY[kind], "hu")
    assert _surround_untouched(hu, 1, 1)
    mine = u.cuda()
    tron.tron_distill_hv(z.cuda(), all_lse.cuda(), mine, mine, ids=ids.cuda(), t=t.cuda(), temperature=T, weight=weight.cuda())
    assert _same(mine, hu)
    if K:   # every row counts where there is no list
        tron.tron_distill_hv(z.cuda(), all_lse.cuda(), u.cuda(), mine, temperature=T)
        row = 2 if m > 2 else 0
        pr = torch.exp(z[row].double() / T - all_lse[row].double())
        full = pr * u[row].double() - pr * (pr * u[row].double()).sum()
        assert float((mine[row].double().cpu() - full).abs().max()) <= 2 * U[kind] * float(full.abs().max()) + 2.0 ** -14 * float(u.abs().max())


# either side of what decides whether rows are split: their length, and their number
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("m,V,K", [(3, 32768, 9), (3, 32769, 40), (1, 70000, 100), (128, 33001, 5), (129, 33000, 3)])
def test_distill_long_rows(m, V, K, kind):
    test_distill(m, V, K, kind)
    test_distill_hessian_vector_product(m, V, K, kind)


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("m,V", [(4, 6000), (1100, 200)])
def test_distill_masks(m, V, kind):
    """Rows of nothing but -inf, of the type's lowest value, with NaN, with +inf; a teacher of -inf."""
    torch = torch_mod()
    dt = _dt(kind)
    low = torch.finfo(dt).min
    z = torch.randn(m, V).to(dt)
    z[0] = -math.inf
    z[1] = low
    z[2, 3] = math.nan
    z[3, 4] = math.inf
    ids, t = torch.arange(4).repeat(m, 1), torch.zeros(m, 4)
    rows = [0, 1, 2, 3]
    loss, lse, dz = torch.empty(m, device="cuda"), torch.empty(m, device="cuda"), torch.empty(m, V, dtype=dt, device="cuda")
    tron.tron_distill(z.cuda(), ids.cuda(), t.cuda(), loss, lse, dz=dz)
    assert float(loss[0]) == math.inf and float(lse[0]) == -math.inf
    assert (dz[0, :4].float() == -0.25).all() and (dz[0, 4:] == 0).all()
    assert math.isfinite(float(lse[1])) and abs(float(loss[1]) - math.log(V / 4)) < 1e-4
    want = torch.full((V,), 1 / V, dtype=torch.float64)
    want[:4] -= 0.25
    _within(dz[1], want, 2 * U[kind] * want.abs() + 1e-6, "uniform row")
    assert math.isnan(float(lse[2])) and torch.isnan(dz[2].float()).all() and math.isnan(float(loss[2]))
    assert not math.isfinite(float(lse[3])) and math.isnan(float(dz[3, 4]))
    tron.tron_distill_grad(z.cuda(), lse, ids.cuda(), t.cuda(), dz)
    assert (dz[0, :4].float() == -0.25).all() and (dz[0, 4:] == 0).all()
    assert torch.isnan(dz[2].float()).all()
    # none of them counts: weight 0, no entry, entries of -inf
    weight = torch.ones(m)
    weight[rows] = 0.0
    for w, i, v in ((weight, ids, t), (None, torch.full_like(ids, -1), t), (None, ids, torch.full_like(t, -math.inf))):
        w = None if w is None else w.cuda()
        dz.fill_(7.0)
        tron.tron_distill(z.cuda(), i.cuda(), v.cuda(), loss, lse, weight=w, dz=dz)
        assert (loss[rows] == 0).all() and (dz[rows] == 0).all()
        dz.fill_(7.0)
        tron.tron_distill_grad(z.cuda(), lse, i.cuda(), v.cuda(), dz, weight=w)
        assert (dz[rows] == 0).all()
        u = torch.full_like(dz, math.nan)
        tron.tron_distill_hv(z.cuda(), lse, u, dz, ids=i.cuda(), t=v.cuda(), weight=w)
        assert (dz[rows] == 0).all()
    # a row of some masks of the lowest value beside ordinary logits: they have probability 0
    z = torch.randn(m, V).to(dt)
    z[:, V // 2:] = low
    tron.tron_distill(z.cuda(), ids.cuda(), t.cuda(), loss, lse, temperature=0.5, dz=dz)
    assert torch.isfinite(loss).all() and (dz[:, V // 2:] == 0).all()
    _within(lse, torch.logsumexp(z[:, :V // 2].double() / 0.5, 1), 1e-4 * torch.ones(m), "lse")


def test_distill_against_differences():
    torch = torch_mod()
    g = _gen(9)
    m, V, K, T, h = 2, 40, 5, 1.5, 2.0 ** -6
    z, ids, t = _randn(g, m, V).float().cuda(), torch.randint(0, V, (m, K), generator=g).cuda(), _randn(g, m, K).float().cuda()
    w = torch.tensor([0.7, 1.3], device="cuda")
    loss, lse, dz, u, hu = torch.empty(m, device="cuda"), torch.empty(m, device="cuda"), torch.empty_like(z), torch.zeros_like(z), torch.empty_like(z)

    def at(z):
        tron.tron_distill(z, ids, t, loss, lse, temperature=T, weight=w, dz=dz)
        return float(loss.double().sum()), dz.double()

    _, g0 = at(z)
    lse0 = lse.clone()
    for j in (0, 17, int(ids[1, 0])):
        e = torch.zeros_like(z)
        e[1, j] = h
        up, gu = at(z + e)
        down, gd = at(z - e)
        # third derivatives of w T^2 log sum exp(z / T) are at most w / T / 4; values are rounded to 2^-22 or so
        assert abs((up - down) / (2 * h) - float(g0[1, j])) < h * h + 2.0 ** -21 / h
        tron.tron_distill_hv(z, lse0, e / h, hu, ids=ids, t=t, temperature=T, weight=w)
        assert float(((gu - gd) / (2 * h) - hu.double()).abs().max()) < h * h + 2.0 ** -22 / h


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
def test_distill_masks_of_rows_in_parts(kind):
    test_distill_masks(4, 40000, kind)


# --------------------------------------------------------------------------- streams, graphs, refusals
def test_other_streams_and_graphs():
    torch = torch_mod()
    x, w = torch.randn(3, 6000, device="cuda").bfloat16(), (torch.randn(90, 6000, device="cuda") / 80).bfloat16()
    ids, t = torch.randint(0, 90, (3, 4), device="cuda"), torch.randn(3, 4, device="cuda")

    def step(stream=None):
        a, z, dz, u = torch.empty_like(x), torch.empty(3, 90, device="cuda"), torch.empty(3, 90, device="cuda"), torch.randn(3, 90, device="cuda")
        loss, lse, dx = torch.empty(3, device="cuda"), torch.empty(3, device="cuda"), torch.empty_like(x)
        b16 = torch.empty(3, 90, device="cuda", dtype=torch.bfloat16)

        def go():
            tron.tron_rms_norm(x, a, stream=stream)
            tron.tron_linear(a, w, z, stream=stream)
            tron.tron_distill(z, ids, t, loss, lse, dz=dz, stream=stream)
            tron.tron_linear(a, w, b16, stream=stream)
            tron.tron_linear_grad(None, w, b16, dx=dx, stream=stream)
        return go, (z, loss, lse, dz, dx)

    go, want = step()
    go()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for s in (side, side.cuda_stream):
        go, got = step(s)
        side.wait_stream(torch.cuda.current_stream())
        go()
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, got))
    go, got = step()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        go()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        go()
    for _ in range(3):
        for b in got:
            b.fill_(-1.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, got))


def test_refusals():
    torch = torch_mod()
    f, b = torch.zeros(4, 8, device="cuda"), torch.zeros(4, 8, device="cuda").bfloat16()
    q = b.to(torch.float8_e4m3fn)
    v4, v8 = torch.zeros(4, device="cuda"), torch.zeros(8, device="cuda")
    ids, t = torch.zeros(4, 2, dtype=torch.int64, device="cuda"), torch.zeros(4, 2, device="cuda")
    z = torch.zeros(4, 8, device="cuda")

    def refused(call, *args, **kw):
        with pytest.raises(tron.TronError) as e:
            call(*args, **kw)
        assert e.value.code == -1, e.value

    refused(tron.tron_rms_norm, f.cpu(), f)
    refused(tron.tron_rms_norm, f, f.cpu())
    refused(tron.tron_rms_norm, f, torch.zeros(4, 7, device="cuda"))
    refused(tron.tron_rms_norm, f, b)                                  # y of another type
    refused(tron.tron_rms_norm, b, q)                                  # no scale
    refused(tron.tron_rms_norm, q, q, scale=v4)                        # input in 8 bits
    refused(tron.tron_rms_norm, f, torch.empty_like(f), eps=-1.0)
    refused(tron.tron_rms_norm, f, torch.empty_like(f), eps=math.nan)
    refused(tron.tron_rms_norm, f, torch.empty_like(f), gain=v4)
    refused(tron.tron_rms_norm, f, torch.empty_like(f), gain=v8.double())
    refused(tron.tron_rms_norm, f.t(), torch.empty(8, 4, device="cuda"))
    refused(tron.tron_rms_norm, f, v8.expand(4, 8))                    # rows that are written overlap
    refused(tron.tron_rms_norm, f[None], f[None])
    refused(tron.tron_rms_norm, f.double(), f.double())
    refused(tron.tron_rms_norm_grad, f, None, f, torch.empty_like(f))
    refused(tron.tron_rms_norm_grad, f, v4, b, torch.empty_like(f))
    refused(tron.tron_rms_norm_grad, f, v4, f, torch.empty_like(f), dgain=v8, work=torch.empty(16, dtype=torch.uint8, device="cuda"))
    refused(tron.tron_linear, f, f, f)                                 # operands in 32 bits
    refused(tron.tron_linear, b, q, torch.zeros(4, 4, device="cuda"))
    refused(tron.tron_linear, q, q, torch.zeros(4, 4, device="cuda"))  # no scales
    refused(tron.tron_linear, b, b, torch.zeros(4, 4, device="cuda"), x_scale=v4, w_scale=v4)
    refused(tron.tron_linear, b, b, torch.zeros(4, 5, device="cuda"))
    refused(tron.tron_linear, b, b, torch.zeros(4, 4, device="cuda"), residual=torch.zeros(4, 4, device="cuda").bfloat16())
    refused(tron.tron_linear, b, b, torch.zeros(4, 4, device="cuda"), act=4)
    refused(tron.tron_linear, b, b, torch.zeros(1, 4, device="cuda").expand(4, 4))
    refused(tron.tron_linear, b, b[0], torch.zeros(4, 1, device="cuda"))
    refused(tron.tron_linear_grad, b, b, f, dx=torch.empty_like(b))
    refused(tron.tron_linear_grad, b, None, torch.zeros(4, 4, device="cuda").bfloat16(), dx=torch.empty_like(b))
    refused(tron.tron_linear_grad, None, b, torch.zeros(4, 4, device="cuda").bfloat16(), dw=torch.empty_like(b))
    refused(tron.tron_linear_grad, b, b, torch.zeros(4, 4, device="cuda").bfloat16(), dx=torch.empty_like(b), act=tron.ACT_GELU)
    refused(tron.tron_distill, z, ids, t, None)
    refused(tron.tron_distill, z, ids.float(), t, v4)
    refused(tron.tron_distill, z, ids, t.double(), v4)
    refused(tron.tron_distill, z, ids, t[:, :1], v4)
    refused(tron.tron_distill, z, ids, t, v4, temperature=0.0)
    refused(tron.tron_distill, z, ids, t, v4, temperature=math.inf)
    refused(tron.tron_distill, z, ids, t, v4, weight=v8)
    refused(tron.tron_distill, z, ids, t, v4, dz=b)
    refused(tron.tron_distill, z, torch.zeros(4, 1025, dtype=torch.int64, device="cuda"), torch.zeros(4, 1025, device="cuda"), v4)
    refused(tron.tron_distill_grad, z, None, ids, t, torch.empty_like(z))
    refused(tron.tron_distill_hv, z, v4, z, None)
    refused(tron.tron_distill_hv, z, v4, z, torch.empty_like(z), ids=ids)


# --------------------------------------------------------------------------- together
def test_softmax_head_function_gradient_and_hessian_vector_product():
    torch = torch_mod()
    g = _gen(11)
    m, d, V, K, C, T = 90, 70, 33, 4, 2.0, 1.5
    hidden, residual = _randn(g, m, d).bfloat16(), _randn(g, m, d).bfloat16()
    gain = (1 + 0.1 * _randn(g, d)).float()
    ids, t, weight = torch.randint(0, V, (m, K), generator=g), _randn(g, m, K).float(), torch.rand(m, generator=g) + 0.5
    W, D = (_randn(g, V, d) / 8).bfloat16().float(), (_randn(g, V, d) / 8).bfloat16().float()   # exact in the products' type
    head = tron.SoftmaxHead(hidden.cuda(), ids.cuda(), t.cuda(), gain=gain.cuda(), residual=residual.cuda(), temperature=T, weight=weight.cuda())
    with pytest.raises(tron.TronError):
        head.hv(C, D.cuda(), torch.empty(V, d, device="cuda"))
    G, HD = torch.empty(V, d, device="cuda"), torch.empty(V, d, device="cuda")
    f = head.fun_grad(C, W.cuda(), G)
    X = head.X.double().cpu()
    _, _, y = _norm_plain(hidden, residual, gain, 1e-6)
    _within(X, y, (U["bf16"] + 130 * E) * y.abs() + 1e-30, "features")
    # the logits are rounded to bf16: from there on the values that are kept
    z = head.z.cpu()
    _within(z, X @ W.double().T, U["bf16"] * (X @ W.double().T).abs() * 1.01 + (d + 8) * 2 * E * (X.abs() @ W.double().abs().T), "logits")
    loss, _, dz, p, _, w = _distill_plain(z, ids, t, T, weight)
    want = 0.5 * float((W.double() ** 2).sum()) + C * float(loss.sum())
    assert abs(f - want) <= 1e-5 * abs(want)
    # dz is rounded to bf16 (and computed to 2^-16 of p)
    _within(G, W.double() + C * dz.T @ X, C * ((U["bf16"] + 2.0 ** -10) * dz.abs() + 2.0 ** -15 * w * T * p).T @ X.abs() + 1e-6, "gradient")
    assert head.fun_grad(C, W.cuda()) == f
    head.hv(C, D.cuda(), HD)
    u = X @ D.double().T
    h = w * (p * u - p * (p * u).sum(1, keepdim=True))
    # u is rounded to bf16 before, H u after
    off = w * p * (u.abs() + (p * u.abs()).sum(1, keepdim=True)) * (U["bf16"] + 2.0 ** -10) + h.abs() * U["bf16"]
    _within(HD, D.double() + C * h.T @ X, C * off.T @ X.abs() + 1e-6, "Hessian-vector product")


def test_the_example_trains_and_answers():
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "distilled_head.py")
    spec = importlib.util.spec_from_file_location("distilled_head", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    history, agree = module.main(["--rows", "2000", "--features", "128", "--classes", "200", "--top", "8", "--steps", "4"])
    assert len(history) >= 3 and all(b < a for a, b in zip(history, history[1:]))
    assert history[-1] < 0.6 * history[0] and agree >= 48
