"""Operators of a multi-class head at the edges of their inputs' ranges, against plain implementations in 64 bits.  Bounds as in
test_gpu_heads.py."""
import math

import pytest

import paper_2008_03433_amd as tron
import test_gpu_heads as heads
from test_gpu_heads import E, TINY, U, _check_linear, _distill_bounds, _distill_plain, _dt, _gen, _randn, _within
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


# --------------------------------------------------------------------------- rows whose lse a float does not hold
def _far_rows(kind, V, T, seed):
    """Rows whose logits lie so far from 0 that a float's lse says little about them, and ordinary ones between them."""
    torch = torch_mod()
    g, dt = _gen(seed), _dt(kind)
    top = torch.finfo(dt).max
    z = (3 * T * _randn(g, 7, V)).to(dt)
    z[0] = -top
    z[2] = top
    z[3] = (0.875 * top * torch.sign(_randn(g, V))).to(dt)   # half of them masked as deep as they can be
    z[4] = (1e4 + 8 * _randn(g, V)).to(dt)
    z[5] = -math.inf
    return z


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("T", [1.0, 0.5, 1.5])
@pytest.mark.parametrize("V", [70, 6000, 40_000, 70_003])
def test_distill_gradient_and_hessian_vector_product_of_rows_far_from_zero(V, T, kind):
    """tron_distill_grad and tron_distill_hv agree with the definition where lse has no digits left, in place too."""
    torch = torch_mod()
    z, dt, K = _far_rows(kind, V, T, V), _dt(kind), 3
    m = z.shape[0]
    ids, t, weight = torch.arange(K).repeat(m, 1), torch.zeros(m, K), torch.linspace(0.5, 2.0, m)
    # from differences to the row's maximum: 64 bits do not hold such an lse either
    p = torch.softmax(z.double() / T, 1).nan_to_num(nan=0.0)
    q, w = torch.zeros_like(p), weight.double()[:, None]
    q[:, :K] = 1 / K
    dz = w * T * (p - q)
    got_loss, lse = torch.empty(m, device="cuda"), torch.empty(m, device="cuda")
    fused, got = torch.empty(m, V, dtype=dt, device="cuda"), torch.empty(m, V, dtype=dt, device="cuda")
    args = (ids.cuda(), t.cuda())
    tron.tron_distill(z.cuda(), *args, got_loss, lse, temperature=T, weight=weight.cuda(), dz=fused)
    # exponents are differences to the row's maximum, up to 64 where p counts; below 2^-120 p may be 0.  Ordinary rows: from lse, up to some 20
    off = (V / 512 + 160) * E + 4 * 20 * E
    p_off = p * (off + 8 * E)
    bound = U[kind] * dz.abs() + (w * T * (p_off + q * 8 * E)) * (1 + U[kind]) + 4 * E * dz.abs() + TINY[kind] + 2.0 ** -120
    _within(fused, dz, bound, "dz")
    tron.tron_distill_grad(z.cuda(), lse, *args, got, temperature=T, weight=weight.cuda())
    _within(got, dz, bound, "dz from lse")
    mine = z.cuda()
    tron.tron_distill_grad(mine, lse, *args, mine, temperature=T, weight=weight.cuda())
    assert torch.equal(mine, got)

    u = _randn(_gen(V + 1), m, V).to(dt)
    u64 = u.double()
    want = w * (p * u64 - p * (p * u64).sum(1, keepdim=True))
    size = p * (u64.abs() + (p * u64.abs()).sum(1, keepdim=True))
    tron.tron_distill_hv(z.cuda(), lse, u.cuda(), got, ids=args[0], t=args[1], temperature=T, weight=weight.cuda())
    _within(got, want, U[kind] * want.abs() + w * size * (2 * off + (V / 512 + 40) * 2 * E) * (1 + U[kind]) + TINY[kind] + 2.0 ** -120, "hu")
    mine = u.cuda()
    tron.tron_distill_hv(z.cuda(), lse, mine, mine, ids=args[0], t=args[1], temperature=T, weight=weight.cuda())
    assert torch.equal(mine, got)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("V", [500, 40_000])
def test_distill_gradient_of_rows_far_from_zero_that_are_not_finite(V, kind):
    torch = torch_mod()
    dt, T = _dt(kind), 0.5
    z = torch.full((3, V), torch.finfo(dt).min).to(dt)
    z[0, 7], z[1, 8] = math.nan, math.inf
    ids, t = torch.zeros(3, 1, dtype=torch.int64, device="cuda"), torch.zeros(3, 1, device="cuda")
    loss, lse = torch.empty(3, device="cuda"), torch.empty(3, device="cuda")
    dz = torch.empty(3, V, dtype=dt, device="cuda")
    tron.tron_distill(z.cuda(), ids, t, loss, lse, temperature=T)
    tron.tron_distill_grad(z.cuda(), lse, ids, t, dz, temperature=T)
    assert torch.isnan(dz[:2].float()).all() and torch.isfinite(dz[2].float()).all()
    # rows that do not count are 0 whatever they hold
    weight = torch.tensor([0.0, 1.0, 0.0], device="cuda")
    ids[1] = -1
    tron.tron_distill_grad(z.cuda(), lse, ids, t, dz, temperature=T, weight=weight)
    assert (dz == 0).all()


# --------------------------------------------------------------------------- gradients of the matrix product
def _grad_inputs(g, m, n, k, kind, act):
    """x, w, dy, pre of a type; dpre = dy act'(pre), X and W in 64 bits."""
    torch = torch_mod()
    dt = _dt(kind)
    x, w, dy, pre = (a.to(dt) for a in (_randn(g, m, k), _randn(g, n, k) * k ** -0.5, _randn(g, m, n), _randn(g, m, n)))
    return x, w, dy, pre, _dpre(dy, pre, act)


def _dpre(dy, pre, act):
    torch = torch_mod()
    a = pre.double().requires_grad_()
    y = [lambda v: v * 1.0, torch.relu, torch.nn.functional.gelu, torch.nn.functional.silu][act](a)
    return torch.autograd.grad(y, a, dy.double())[0]


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("act", [tron.ACT_GELU, tron.ACT_SILU])
@pytest.mark.parametrize("m,n,k", [(1, 700, 600), (8, 300, 530), (5, 63, 64)])
def test_linear_gradient_of_few_rows_takes_dpre_unrounded(m, n, k, act, kind):
    torch = torch_mod()
    x, w, dy, pre, d = _grad_inputs(_gen(m + n + k), m, n, k, kind, act)
    dx = torch.empty(m, k, dtype=_dt(kind), device="cuda")
    tron.tron_linear_grad(None, w.cuda(), dy.cuda(), dx=dx, act=act, pre=pre.cuda())
    want, W = d @ w.double(), w.double().abs()
    # the factors' roundings of 32 bits, the sum, and the rounding of the result alone
    _within(dx, want, U[kind] * want.abs() + ((32 * E * dy.double().abs() + (n + 8) * 2 * E * d.abs()) @ W) * (1 + U[kind]) + TINY[kind], "dx")


@pytest.mark.parametrize("act", [tron.ACT_GELU, tron.ACT_SILU, tron.ACT_RELU])
@pytest.mark.parametrize("size", [65504.0, 2.0 ** -16])
@pytest.mark.parametrize("m,n,k", [(70, 40, 130), (200, 264, 96), (12, 50, 64)])
def test_linear_gradients_in_f16_whose_dpre_lies_beyond_its_range(m, n, k, size, act):
    """Gradients next to f16's largest value times slopes above 1, and small ones times small slopes: the products have results that f16
    holds.  (12 rows: dx by the kernel that reads w as it lies.)"""
    torch = torch_mod()
    g, u = _gen(m + n + k), U["f16"]
    dy = (size * torch.sign(_randn(g, m, n)) * (1.0 - 0.25 * torch.rand(m, n, generator=g, dtype=torch.float64))).half()
    dy[0, :2] = size
    pre = (1.5 + 0.3 * _randn(g, m, n) if size > 1 else -3.0 + 0.5 * _randn(g, m, n)).half()
    scale = 2.0 ** -14 if size > 1 else 2.0 ** 13
    x, w = (_randn(g, m, k) * scale).half(), (_randn(g, n, k) * scale).half()
    d = _dpre(dy, pre, act)
    dx, dw, db = torch.empty(m, k, dtype=torch.float16, device="cuda"), torch.empty(n, k, dtype=torch.float16, device="cuda"), torch.empty(n, device="cuda")
    tron.tron_linear_grad(x.cuda(), w.cuda(), dy.cuda(), dx=dx, dw=dw, dbias=db, act=act, pre=pre.cuda())
    # dpre rounded to f16 times a power of two by which the largest |dy| is 2^14 at least: below f16's normal numbers half of 2^-24 over that power
    off = u * d.abs() + 32 * E * dy.double().abs() + 2.0 ** -25 * float(dy.double().abs().max()) / 2.0 ** 14
    X, W = x.double(), w.double()
    for got, want, bound in ((dx, d @ W, (off + (n + 8) * 2 * E * d.abs()) @ W.abs()), (dw, d.T @ X, (off + (m + 8) * 2 * E * d.abs()).T @ X.abs())):
        assert float(want.abs().max()) < 65504.0
        _within(got, want, u * want.abs() * (1 + u) + bound * (1 + u) + TINY["f16"], "dx" if got is dx else "dw")
    _within(db, d.sum(0), ((m + 8) * 2 * E * d.abs() + 32 * E * dy.double().abs()).sum(0), "dbias")
    # all of it infinite or NaN where dy is, and nothing else
    dy[3, 5], dy[m - 1, 7] = math.inf, math.nan
    tron.tron_linear_grad(x.cuda(), w.cuda(), dy.cuda(), dx=dx, dw=dw, act=act, pre=pre.abs().cuda())
    assert torch.equal(~torch.isfinite(dx).all(1).cpu(), torch.isin(torch.arange(m), torch.tensor([3, m - 1])))
    assert torch.equal(~torch.isfinite(dw).all(1).cpu(), torch.isin(torch.arange(n), torch.tensor([5, 7])))


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("act", [tron.ACT_GELU, tron.ACT_SILU, tron.ACT_RELU])
@pytest.mark.parametrize("narrow", [False, True])
@pytest.mark.parametrize("m,n,k", [(3, 40, 70), (20, 33, 64), (130, 70, 257), (700, 24, 16), (300, 520, 264), (9000, 100, 130)])
def test_linear_gradients_have_the_rounding_of_their_type_alone(m, n, k, narrow, act, kind):
    """dpre keeps its bits in the products, unless the caller asks for fewer.  Shapes with dx and dw in one launch, in one part and in several;
    rows that lie apart."""
    torch = torch_mod()
    u = U[kind]
    x, w, dy, pre, d = _grad_inputs(_gen(m + n + k + act), m, n, k, kind, act)
    X, W, args = x.double(), w.double(), (x.cuda(), w.cuda(), dy.cuda())
    # dpre in two parts, each rounded: u of u, or of one; f16's smallest step is 2^-24 where the largest |dy| is 2^14 at least.  Sums of 2 m or 2 n terms
    rounded = 0.0 if act == tron.ACT_RELU else u if narrow else u * u
    off = rounded * d.abs() + 32 * E * dy.double().abs() + 2.0 ** -25 * float(dy.double().abs().max()) / 2.0 ** 14
    for wide in (True, False):
        dw = torch.full((n, k + 3), math.nan, dtype=torch.float32 if wide else _dt(kind), device="cuda")[:, :k]
        dx, db = torch.full((m, k + 5), math.nan, dtype=_dt(kind), device="cuda")[:, :k], torch.empty(n, device="cuda")
        tron.tron_linear_grad(*args, dx=dx, dw=dw, dbias=db, act=act, pre=pre.cuda(), narrow=narrow)
        want, bound = d @ W, (off + (2 * n + 8) * 2 * E * d.abs()) @ W.abs()
        _within(dx, want, u * want.abs() + bound * (1 + u) + TINY[kind] * (1 + W.abs().sum(0)), "dx")
        want, bound = d.T @ X, (off + (2 * m + 8) * 2 * E * d.abs()).T @ X.abs()
        ud = E if wide else u
        _within(dw, want, ud * want.abs() + bound * (1 + ud) + (0.0 if wide else TINY[kind]), "dw")
        _within(db, d.sum(0), ((m + 8) * 2 * E * d.abs() + 32 * E * dy.double().abs()).sum(0), "dbias")
        # one at a time: the same bits; with a work space of its own size
        work = torch.empty(tron.tron_linear_grad_work(m, n, k, act, False, True, False, narrow=narrow), dtype=torch.uint8, device="cuda")
        only = torch.empty(n, k, dtype=dw.dtype, device="cuda")
        tron.tron_linear_grad(args[0], None, args[2], dw=only, act=act, pre=pre.cuda(), work=work, narrow=narrow)
        assert torch.equal(only, dw)
        only = torch.empty(m, k, dtype=dx.dtype, device="cuda")
        tron.tron_linear_grad(None, *args[1:], dx=only, act=act, pre=pre.cuda(), narrow=narrow)
        assert torch.equal(only, dx)


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("act", [tron.ACT_GELU, tron.ACT_SILU])
@pytest.mark.parametrize("m,n,k", [(40, 33, 64), (300, 130, 72)])
def test_linear_gradients_keep_infinities(m, n, k, act, kind):
    """One infinite term makes a result that infinity, of its sign: what the rounding of dpre left has no part in it."""
    torch = torch_mod()
    x, w, dy, pre, d = _grad_inputs(_gen(m + n + k), m, n, k, kind, act)
    x[1, 5], w[2, 7] = math.inf, -math.inf
    for narrow in (False, True):
        dx, dw = torch.empty(m, k, dtype=_dt(kind), device="cuda"), torch.empty(n, k, device="cuda")
        tron.tron_linear_grad(x.cuda(), w.cuda(), dy.cuda(), dx=dx, dw=dw, act=act, pre=pre.cuda(), narrow=narrow)
        assert torch.equal(dw[:, 5].cpu(), torch.sign(d[1]).float() * math.inf)
        assert torch.equal(dx[:, 7].float().cpu(), torch.sign(d[:, 2]).float() * -math.inf)
        dx[:, 7], dw[:, 5] = 0.0, 0.0
        assert torch.isfinite(dx).all() and torch.isfinite(dw).all()


def test_linear_gradients_refuse_a_work_space_of_fewer_bits():
    torch = torch_mod()
    m, n, k = 100, 80, 64
    x, w, dy, pre = (torch.zeros(*s, dtype=torch.bfloat16, device="cuda") for s in ((m, k), (n, k), (m, n), (m, n)))
    dx, dw = torch.empty_like(x), torch.empty_like(w)
    sizes = [tron.tron_linear_grad_work(m, n, k, tron.ACT_SILU, True, True, False, narrow=narrow) for narrow in (False, True)]
    assert sizes[1] < sizes[0]
    work = torch.empty(sizes[1], dtype=torch.uint8, device="cuda")
    with pytest.raises(tron.TronError):
        tron.tron_linear_grad(x, w, dy, dx=dx, dw=dw, act=tron.ACT_SILU, pre=pre, work=work)
    tron.tron_linear_grad(x, w, dy, dx=dx, dw=dw, act=tron.ACT_SILU, pre=pre, work=work, narrow=True)
    for act in (tron.ACT_SILU + 256, 4, 260):   # of the gradients alone; no activation
        with pytest.raises(tron.TronError):
            tron.tron_linear(x, w, torch.empty(m, n, device="cuda"), act=act)
        if act != tron.ACT_SILU + 256:
            with pytest.raises(tron.TronError):
                tron.tron_linear_grad(x, w, dy, dx=dx, act=act, pre=pre)


# --------------------------------------------------------------------------- activations
def _phi(a):
    """Phi(a) and its density in 64 bits; erfc keeps the digits of the lower tail."""
    torch = torch_mod()
    return 0.5 * torch.special.erfc(-a * math.sqrt(0.5)), torch.exp(-0.5 * a * a) / math.sqrt(2 * math.pi)


@pytest.mark.parametrize("out", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("act", [tron.ACT_GELU, tron.ACT_SILU])
@pytest.mark.parametrize("m", [2, 40])
def test_activations_have_the_digits_of_their_output(m, act, out):
    """Values before the activation that are given exactly, by the bias: small results of the negative side too."""
    torch = torch_mod()
    n, k = 5003, 8
    a = torch.linspace(-8.0, 8.0, n) if act == tron.ACT_GELU else torch.linspace(-60.0, 60.0, n)
    a[:8] = torch.tensor([-11.0, -12.5, 0.0, 30.0, -30.0, -86.0, 86.0, 1e30])
    x, w = torch.zeros(m, k, device="cuda", dtype=torch.float16), torch.zeros(n, k, device="cuda", dtype=torch.float16)
    a64, dt = a.double(), _dt(out)
    if out == "f16":
        x, w, a64[7], a[7] = x, w, 3e4, 3e4
    y = torch.empty(m, n, dtype=dt, device="cuda")
    tron.tron_linear(x, w, y, bias=a.cuda(), act=act)
    want = a64 * (_phi(a64)[0] if act == tron.ACT_GELU else torch.sigmoid(a64))
    # a dozen roundings of 32 bits and the fit's 1.9e-7, 4 E; nothing below 2^-120
    _within(y, want.expand(m, n), (U[out] + 20 * E) * want.abs().expand(m, n) + TINY[out] + 2.0 ** -120, "y")


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("act", [tron.ACT_GELU, tron.ACT_SILU])
def test_slopes_of_activations_have_32_bits(act, kind):
    torch = torch_mod()
    n = 4001
    pre = torch.linspace(-12.0, 12.0, n).to(_dt(kind))
    dy, db = torch.ones(1, n, dtype=_dt(kind), device="cuda"), torch.empty(n, device="cuda")
    tron.tron_linear_grad(None, None, dy, dbias=db, act=act, pre=pre[None].cuda())
    a = pre.double()
    if act == tron.ACT_GELU:
        phi, density = _phi(a)
        want, size = phi + a * density, phi + a.abs() * density
    else:
        h, rest = torch.sigmoid(a), torch.sigmoid(-a)
        want, size = h * (1 + a * rest), h * (1 + a.abs() * rest)
    _within(db, want, 20 * E * size + 2.0 ** -120, "slope")


# --------------------------------------------------------------------------- scales of 8-bit operands
@pytest.mark.parametrize("m,n,k", [(3, 40, 96), (150, 140, 512), (40, 60, 20_000)])
def test_scales_whose_product_leaves_the_range_of_32_bits(m, n, k):
    """Row and column scales that lie far apart: one large and one small, two small ones and a large sum, down to numbers that are not normal."""
    torch = torch_mod()
    g = _gen(m + n)
    x, w = ((_randn(g, r, k) * 100).clamp(-440, 440).float().to(torch.float8_e4m3fn) for r in (m, n))
    xs, ws = torch.full((m,), 1.0), torch.full((n,), 1.0)
    xs[0], ws[0] = 2.0 ** -80 * 1.37, 2.0 ** -66 * 1.71       # 2^-146: three bits left of their product
    xs[1], ws[1] = 2.0 ** 120 * 1.37, 2.0 ** -120 * 1.71      # sums of 2^20 times 2^120
    xs[2], ws[2] = 2.0 ** -120 * 1.37, 2.0 ** 120 * 1.71
    ws[3], ws[4], ws[5] = 2.0 ** -140, 2.0 ** 100, 0.0
    y = torch.empty(m, n, device="cuda")
    tron.tron_linear(x.cuda(), w.cuda(), y, x_scale=xs.cuda(), w_scale=ws.cuda())
    X, W = x.float().double() * xs.double()[:, None], w.float().double() * ws.double()[:, None]
    want, size = X @ W.T, X.abs() @ W.abs().T
    inside = size < 2.0 ** 127
    assert int(inside.sum()) > m * n // 2 and bool(inside[:3, :3].diagonal().all())
    _within(torch.where(inside, y.cpu(), torch.zeros(())), torch.where(inside, want, 0.0), torch.where(inside, (k + 8) * 2 * E * size + 4 * E * want.abs(), 0.0) + TINY["f32"], "y")


# --------------------------------------------------------------------------- the head's Hessian-vector product
@pytest.mark.parametrize("kind", ["f16", "bf16"])
def test_softmax_head_hv_of_directions_of_any_size(kind):
    """The curvature term scales with its direction, from sizes that float16 does not hold to such that it rounds to 0."""
    torch = torch_mod()
    g = _gen(21)
    m, d, V, K, C = 60, 200, 37, 3, 0.5
    hidden, dt = _randn(g, m, d).to(_dt(kind)), _dt(kind)
    ids, t = torch.randint(0, V, (m, K), generator=g), _randn(g, m, K).float()
    W, D = (_randn(g, V, d) / 16).to(dt).float(), (_randn(g, V, d)).to(dt).float()
    head = tron.SoftmaxHead(hidden.cuda(), ids.cuda(), t.cuda())
    head.fun_grad(C, W.cuda())
    X, z = head.X.double().cpu(), head.z.double().cpu()
    p, u = torch.softmax(z, 1), X @ D.double().T
    h = p * u - p * (p * u).sum(1, keepdim=True)
    want = C * h.T @ X
    # u and H u are rounded to the states' type, H u down to steps of 2^-25 (f16) where |u| is below 2^12 and above 2^12 / (d 2)
    off = p * (u.abs() + (p * u.abs()).sum(1, keepdim=True)) * (U[kind] + 2.0 ** -10) + h.abs() * U[kind] + 2.0 ** -24
    bound = C * off.T @ X.abs()
    curvature = {}
    for power in (0, 20, -30, 60, -100):
        size = 2.0 ** power
        HV = torch.empty(V, d, device="cuda")
        V_ = (D * size).cuda()
        head.hv(C, V_, HV)
        assert torch.isfinite(HV).all(), power
        # the sum with V is rounded to 32 bits
        curvature[power] = (HV.double().cpu() - (D * size).double()) / size
        _within(curvature[power], want, bound + 2 * E * (want.abs() + D.double().abs()), f"direction times 2^{power}")
        again = torch.empty_like(HV)
        head.hv(C, V_, again)
        assert torch.equal(again, HV)
    # a power of two changes no bit
    assert all(torch.equal(c, curvature[0]) for c in curvature.values())
    HV.fill_(7.0)
    head.hv(C, torch.zeros(V, d, device="cuda"), HV)
    assert (HV == 0).all()


# --------------------------------------------------------------------------- every kernel of the matrix product, whatever the rule takes
@pytest.fixture
def tile():
    """Sets the tiles of products over more than 32 rows."""
    yield lambda side: tron.tron_tuning_set("linear_tile", side)
    tron.tron_tuning_set("linear_tile", 0)


# whole chunks at multiples of 16 bytes (from memory straight to LDS): one step, a step that ends inside a row of chunks, several; rows that end
# inside a chunk, and rows that lie apart (through registers); an inner index cut in many
@pytest.mark.parametrize("kind,out", [("bf16", "bf16"), ("f16", "f16"), ("e4m3", "bf16"), ("e4m3", "f32")])
@pytest.mark.parametrize("m,n,k", [(33, 40, 16), (257, 255, 1008), (300, 520, 2048), (256, 512, 64), (129, 300, 1031), (70, 60, 20_000), (300, 258, 20_001)])
def test_linear_in_tiles_of_256(tile, m, n, k, kind, out):
    tile(256)
    for act in (m % 4, 2):
        _check_linear(m, n, k, kind, out, act=act, bias=True, residual=True, pre=True)
    _check_linear(m, n, k, kind, out, act=0, bias=False, residual=False, pre=False, pads=(7, 3))


@pytest.mark.parametrize("kind", ["bf16", "f16", "e4m3"])
@pytest.mark.parametrize("m,n,k", [(4100, 4099, 272), (2300, 4099, 1040), (4000, 4099, 77)])
def test_linear_in_tiles_of_256_with_a_result_past_the_caches(tile, m, n, k, kind):
    tile(256)
    heads.test_linear_large(m, n, k, kind)


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("m,n,k", [(300, 520, 264), (300, 520, 265), (515, 262, 129), (700, 258, 300), (2000, 40, 72)])
def test_linear_gradients_in_tiles_of_256(tile, m, n, k, kind):
    """All activations, dx and dw from the padded copies, parts where the inner index is long."""
    tile(256)
    heads.test_linear_gradients(m, n, k, kind)
    tile(128)
    heads.test_linear_gradients(m, n, k, kind)


@pytest.mark.parametrize("side", [128, 256])
def test_tiles_in_a_graph(tile, side):
    """A captured product and its gradients, replayed on other inputs beside eager work."""
    torch = torch_mod()
    tile(side)
    m, n, k = 300, 264, 520
    x, w, dy = (torch.empty(*s, dtype=torch.float16, device="cuda") for s in ((m, k), (n, k), (m, n)))

    def outputs():
        return (torch.empty(m, n, device="cuda"), torch.empty(m, n, dtype=torch.float16, device="cuda"), torch.empty(m, k, dtype=torch.float16, device="cuda"),
                torch.empty(n, k, device="cuda"), torch.empty(n, device="cuda"))

    def go(y, pre, dx, dw, db):
        tron.tron_linear(x, w, pre, act=tron.ACT_NONE)
        tron.tron_linear(x, w, y, act=tron.ACT_GELU)
        tron.tron_linear_grad(x, w, dy, dx=dx, dw=dw, dbias=db, act=tron.ACT_GELU, pre=pre)

    def fill(seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        for t, std in ((x, 1.0), (w, k ** -0.5), (dy, 1.0)):
            t.copy_(torch.randn(t.shape, generator=g, device="cuda") * std)

    eager, captured = outputs(), outputs()
    fill(0)
    go(*captured)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        go(*captured)
    for seed in range(1, 4):
        fill(seed)
        for t in captured:
            t.fill_(-1.0)
        go(*eager)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(eager, captured))


# --------------------------------------------------------------------------- norms whose outputs go past the caches
@pytest.mark.parametrize("out", ["same", "e4m3"])
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("m,d", [(12_500, 1001), (2_700, 4099), (340, 33_001)])
def test_norm_with_outputs_past_the_caches(m, d, kind, out):
    """Rows of a wavefront, of a workgroup, and such that are read twice; odd strides."""
    heads.test_norm(m, d, kind, out)


@pytest.mark.parametrize("kind,m,d", [("f32", 8_100, 1001), ("bf16", 16_100, 1001), ("f16", 4_100, 4099), ("f32", 2_000, 4099), ("bf16", 1_000, 16_501)])
def test_norm_gradient_with_outputs_past_the_caches(kind, m, d):
    heads.test_norm_gradient(m, d, kind)


# --------------------------------------------------------------------------- norms of rows of any size
@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("d", [100, 3000, 20_000, 40_000])
def test_norm_and_gradient_of_rows_whose_squares_leave_the_range_of_32_bits(d, kind):
    """Rows of 1e-25 to 1e25: rstd, y (in 8 bits too) and the gradients as for rows of 1."""
    torch = torch_mod()
    g, dt, u = _gen(d), _dt(kind), U[kind]
    sizes = torch.tensor([2.0 ** -83, 2.0 ** -70, 1.0, 2.0 ** 70, 2.0 ** 83], dtype=torch.float64)[:, None]
    m = len(sizes)
    s, dy, gain = (_randn(g, m, d) * sizes).to(dt), _randn(g, m, d).to(dt), (1.0 + 0.2 * _randn(g, d)).float()
    S = s.double()
    rstd = (S * S).mean(1, keepdim=True) ** -0.5
    y = S * rstd * gain.double()
    got, q, scale, got_rstd = torch.empty(m, d, dtype=dt, device="cuda"), torch.empty(m, d, dtype=_dt("e4m3"), device="cuda"), torch.empty(m, device="cuda"), torch.empty(m, device="cuda")
    lost = 64 * E
    tron.tron_rms_norm(s.cuda(), got, gain=gain.cuda(), eps=0.0, rstd=got_rstd)
    _within(got_rstd, rstd[:, 0], lost * rstd[:, 0], "rstd")
    _within(got, y, (u + 2 * lost) * y.abs() + TINY[kind], "y")
    tron.tron_rms_norm(s.cuda(), q, gain=gain.cuda(), eps=0.0, scale=scale)
    want = y.abs().amax(1) / 448
    _within(scale, want, 2 * lost * want, "scale")
    _within(q.float().double().cpu() * scale.double().cpu()[:, None], y, (2.0 ** -4 + 4 * lost) * y.abs() + 2.0 ** -10 * (1 + lost) * want[:, None], "y in 8 bits")
    # the gradient has the size of rstd
    dx, dgain = torch.empty(m, d, dtype=dt, device="cuda"), torch.empty(d, device="cuda")
    tron.tron_rms_norm_grad(s.cuda(), got_rstd, dy.cuda(), dx, gain=gain.cuda(), dgain=dgain)
    R = got_rstd.double().cpu()[:, None]
    A, H = dy.double() * gain.double(), S * R
    want = R * (A - H * (A * H).mean(1, keepdim=True))
    size = R * (A.abs() + H.abs() * (A * H).abs().mean(1, keepdim=True))
    _within(dx, want, u * want.abs() + 80 * E * size + TINY[kind], "dx")
    terms = dy.double() * H
    _within(dgain, terms.sum(0), (m + 8) * 2 * E * terms.abs().sum(0), "dgain")
