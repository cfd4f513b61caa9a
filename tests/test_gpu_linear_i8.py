"""The matrix product of whole numbers of 8 bits against sums in 64 bits.

The sum is exact; behind it there are the roundings to a float, of the product of the scales' fractions, of the product with it, of the bias' addition and
of the residual's, E = 2^-24 each, and the output's own, U.  gelu and silu have a slope of at most 1.13 and are off by a dozen units of their own."""
import math

import pytest

import paper_2008_03433_amd as tron
from test_gpu_heads import E, TINY, U, _dt, _gen, _randn, _same, _within
from util import torch_mod

pytestmark = pytest.mark.gpu


def _whole(g, m, k, low=-128):
    return torch_mod().randint(low, 128, (m, k), generator=g, dtype=torch_mod().int8)


def _act(a, act):
    torch = torch_mod()
    return {0: lambda v: v, 1: torch.relu, 2: torch.nn.functional.gelu, 3: torch.nn.functional.silu}[act](a)


def _inside(t, pad, offset):
    """The same values on the GPU in rows `pad` bytes further apart, `offset` bytes into a buffer."""
    torch = torch_mod()
    m, k = t.shape
    buf = torch.full((offset + m * (k + pad),), 99, dtype=torch.int8, device="cuda")
    view = buf[offset:].view(m, k + pad)[:, :k]
    view.copy_(t)
    return view


SIZES = [(1, 1, 1), (1, 70, 15), (2, 64, 16), (3, 130, 4096), (8, 1000, 4099), (16, 33, 257), (17, 200, 1024), (32, 77, 8192), (33, 50, 31), (40, 129, 1000),
         (130, 140, 2048), (200, 333, 2051), (300, 260, 640), (257, 513, 128), (64, 64, 65536), (5, 40, 100001)]


@pytest.mark.parametrize("tile", [0, 128, 256])
@pytest.mark.parametrize("m,n,k", SIZES)
def test_product_of_whole_numbers(m, n, k, tile):
    torch = torch_mod()
    if tile and m <= 32:
        pytest.skip("few rows have no tiles")
    g = _gen(m * 1000 + n + k)
    x, w = _whole(g, m, k), _whole(g, n, k)
    xs, ws = torch.rand(m, generator=g) + 0.01, 0.01 * torch.rand(n, generator=g) + 1e-4
    bias = _randn(g, n).float() if n % 2 else None
    act, out = (m + n + k) % 4, ("f32", "bf16", "f16")[(n + k) % 3]
    residual = _randn(g, m, n).to(_dt(out)) if k % 2 else None
    total = (x.double() @ w.double().T)   # exact: below 2^53
    pre = total * xs.double()[:, None] * ws.double()
    off = 4 * E * pre.abs()
    if bias is not None:
        pre = pre + bias.double()
        off = off + E * pre.abs()
    y = _act(pre, act)
    off_y = 1.13 * off + (16 * E * y.abs() + 2.0 ** -119 if act > 1 else 0.0)
    if residual is not None:
        y = y + residual.double()
        off_y = off_y + E * y.abs()
    if out == "f16":
        assert float(y.abs().max()) < 60000
    yv, pv = torch.empty((m, n), dtype=_dt(out), device="cuda"), torch.empty((m, n + 3), dtype=_dt(out), device="cuda")[:, :n]
    aligned = k % 16 == 0
    xv, wv = (_inside(x, 16, 0), _inside(w, 0, 16)) if aligned else (_inside(x, 3, 1), _inside(w, 0, 5))
    args = dict(bias=None if bias is None else bias.cuda(), act=act, residual=None if residual is None else residual.cuda(), x_scale=xs.cuda(), w_scale=ws.cuda())
    try:
        tron.tron_tuning_set("linear_tile", tile)
        tron.tron_linear(xv, wv, yv, pre=pv, **args)
        again = torch.empty_like(yv)
        tron.tron_linear(xv, wv, again, **args)
    finally:
        tron.tron_tuning_set("linear_tile", 0)
    _within(pv, pre, U[out] * pre.abs() + (1 + U[out]) * off + TINY[out], "pre")
    _within(yv, y, U[out] * y.abs() + (1 + U[out]) * off_y + TINY[out], "y")
    assert torch.equal(yv, again)
    # whatever kernel multiplies, the sums are the same: so are rows by themselves, and rows at other places
    few = torch.empty((min(m, 7), n), dtype=_dt(out), device="cuda")
    args["residual"] = None if residual is None else args["residual"][: few.shape[0]]
    args["x_scale"] = args["x_scale"][: few.shape[0]]
    tron.tron_linear(_inside(x[: few.shape[0]], 1, 3), wv, few, **args)
    assert torch.equal(few, yv[: few.shape[0]])


def test_the_largest_sums():
    torch = torch_mod()
    k = 2 ** 17 - 1
    for m in (1, 40):
        x = torch.full((m, k), -128, dtype=torch.int8, device="cuda")
        y, one = torch.empty((m, 20), device="cuda"), torch.ones(40, device="cuda")
        tron.tron_linear(x, x[:1].expand(20, k), y, x_scale=one[:m], w_scale=one[:20])
        assert (y == float(torch.tensor(16384.0 * k, dtype=torch.float64).float())).all()
        tron.tron_linear(x, torch.full((20, k), 127, dtype=torch.int8, device="cuda"), y, x_scale=one[:m], w_scale=one[:20])
        assert (y == float(torch.tensor(-128.0 * 127.0 * k, dtype=torch.float64).float())).all()


def test_scales_out_of_range_and_not_finite():
    """The product of the scales may lie outside the range of 32 bits where the result does not; a NaN scale is a NaN row."""
    torch = torch_mod()
    g = _gen(5)
    for m in (3, 60):
        x, w = _whole(g, m, 200).cuda(), _whole(g, 50, 200).cuda()
        y = torch.empty((m, 50), device="cuda")
        tron.tron_linear(x, w, y, x_scale=torch.full((m,), 2.0 ** -120, device="cuda"), w_scale=torch.full((50,), 2.0 ** 120, device="cuda"))
        assert torch.equal(y.double(), (x.double() @ w.double().T))
        xs = torch.ones(m, device="cuda")
        xs[1] = math.nan
        tron.tron_linear(x, w, y, x_scale=xs, w_scale=torch.ones(50, device="cuda"))
        assert torch.isnan(y[1]).all() and not torch.isnan(y[[0, 2]]).any()


def test_norm_and_product_in_whole_numbers():
    """The features of a batch in 8 bits by the norm, then the product that reads them: against the same in 64 bits from what the norm stored."""
    torch = torch_mod()
    g = _gen(8)
    m, d, n = 70, 1040, 130
    h, w = _randn(g, m, d).bfloat16(), _whole(g, n, d, -127)
    x8, scale = torch.empty((m, d), dtype=torch.int8, device="cuda"), torch.empty(m, device="cuda")
    tron.tron_layer_norm(h.cuda(), x8, scale=scale)
    ws = torch.full((n,), 1 / 127.0)
    y = torch.empty((m, n), device="cuda")
    tron.tron_linear(x8, w.cuda(), y, x_scale=scale, w_scale=ws.cuda())
    want = (x8.double().cpu() @ w.double().T) * scale.double().cpu()[:, None] * ws.double()
    _within(y, want, 6 * E * want.abs() + TINY["f32"], "y")


def test_an_output_over_its_residual():
    torch = torch_mod()
    g = _gen(9)
    for m in (4, 100):
        x, w = _whole(g, m, 96).cuda(), _whole(g, 65, 96).cuda()
        s = torch.rand(165, device="cuda")
        r = torch.randn(m, 65, device="cuda").bfloat16()
        y = torch.empty_like(r)
        tron.tron_linear(x, w, y, residual=r, x_scale=s[:m], w_scale=s[100:])
        tron.tron_linear(x, w, r, residual=r, x_scale=s[:m], w_scale=s[100:])
        assert _same(r, y)


@pytest.mark.parametrize("m,n,k", [(45, 1, 60000), (333, 9, 3001), (3368, 18, 1027), (700, 64, 2944), (34, 71, 100000)])
def test_few_columns_whose_inner_index_is_cut(m, n, k):
    """Rows of the parts that share wavefronts.  Scales are powers of two and sums stay below 2^24, so that the product is exact; the sum with the residual is rounded once."""
    torch = torch_mod()
    g = _gen(m + n + k)
    x, w = torch.randint(-8, 9, (m, k), generator=g, dtype=torch.int8), torch.randint(-8, 9, (n, k), generator=g, dtype=torch.int8)   # 64 k < 2^24
    xs, ws = 2.0 ** torch.randint(-3, 4, (m,), generator=g).float(), 2.0 ** torch.randint(-3, 4, (n,), generator=g).float()
    residual = torch.randint(-9, 10, (m, n), generator=g).float()
    assert tron.tron_linear_work(m, n, k, torch.int8) >= 2 * 4 * m * n   # it is cut
    want = ((x.double() @ w.double().T) * xs.double()[:, None] * ws.double() + residual.double()).float()
    y = torch.full((m + 1, n + 5), 7.0, device="cuda")
    tron.tron_linear(x.cuda(), w.cuda(), y[:m, :n], x_scale=xs.cuda(), w_scale=ws.cuda(), residual=residual.cuda())
    assert torch.equal(y[:m, :n].cpu(), want)
    assert bool((y[m] == 7).all()) and bool((y[:, n:] == 7).all())
