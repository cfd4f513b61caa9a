"""The step of a beam search against an enumeration in 64 bits, and the reordering of the beams' states against indexing.

Scores: an exponent d = z - max is off by E |d| from the product with log2(e), the exponential by 2 E, a sum by 64 E (see below), so the logarithm of the sum by
(40 + 66) E at most where the masses' mean |d| is below 40; the score is rounded once more.  E = 2^-24.  Two candidates whose scores are nearer than twice that may
change places, and no others: where there are such among the picks, each pick's own score is held against the one of its place."""
import math

import pytest

import paper_2008_03433_amd as tron
from test_gpu_heads import E, _dt, _gen, _strided
from util import torch_mod

pytestmark = pytest.mark.gpu

LSE = 106 * E


def _plain(z, score, ended, end, picks):
    """next_score, parent, token by sorting all candidates; and the smallest distance between picks that are not equal."""
    torch = torch_mod()
    batch, beams = score.shape
    V = z.shape[1]
    z = z.double().cpu().reshape(batch, beams, V)
    c = torch.empty_like(z)
    for i in range(batch):
        for b in range(beams):
            s, row = float(score[i, b]), z[i, b]
            if not math.isfinite(s):
                c[i, b] = -math.inf
            elif ended is not None and bool(ended[i, b]):
                c[i, b] = -math.inf
                c[i, b, end] = s
            elif torch.isnan(row).any() or float(row.max()) in (math.inf, -math.inf):
                c[i, b] = -math.inf
            else:
                c[i, b] = s + (row - torch.logsumexp(row, 0))
    # a beam's candidates by z, whose differences a score of any size keeps, then all by their scores: ties stay in the order of beams and columns
    by_z = torch.sort(torch.where(torch.isfinite(c), z, -math.inf), dim=2, descending=True, stable=True)[1] + torch.arange(beams)[:, None] * V
    by_z = by_z.reshape(batch, beams * V)
    best, at = torch.sort(c.reshape(batch, beams * V).gather(1, by_z), dim=1, descending=True, stable=True)
    at = by_z.gather(1, at)
    more = best[:, : picks + 1]
    gaps = (more[:, :-1] - more[:, 1:])
    gaps = gaps[torch.isfinite(gaps) & (gaps > 0)]
    at = at[:, :picks]
    return best[:, :picks], torch.arange(batch)[:, None] * beams + at // V, at % V, float(gaps.min()) if gaps.numel() else math.inf, c.reshape(batch * beams, V)


def _check(z, score, picks, ended=None, end=-1, zv=None):
    torch = torch_mod()
    batch, beams = score.shape
    want, parent, token, least, c = _plain(z, score, ended, end, picks)
    out = (torch.full((batch, picks), 7.0, device="cuda"), torch.full((batch, picks), -7, dtype=torch.int32, device="cuda"),
           torch.full((batch, picks), -7, dtype=torch.int32, device="cuda"), torch.empty((batch, picks), dtype=torch.bool, device="cuda"))
    tron.tron_beam_select(z.cuda() if zv is None else zv, score.cuda(), out[0], out[1], out[2], ended=None if ended is None else ended.cuda(), end=end, next_ended=out[3])
    got = out[0].double().cpu()
    if least > 2 * LSE:
        assert torch.equal(out[2].cpu().long(), token), "token"
        assert torch.equal(out[1].cpu().long(), parent), "parent"
    else:
        parent, token = out[1].cpu().long(), out[2].cpu().long()
        assert (parent // beams == torch.arange(batch)[:, None]).all() and len(set(zip(parent.flatten().tolist(), token.flatten().tolist()))) == batch * picks
        own = c[parent, token]
        assert ((own == want) | ((own - want).abs() <= 2 * LSE)).all()
    impossible = torch.isinf(want)
    assert torch.equal(got[impossible], want[impossible])
    assert float(((got - want).abs()[~impossible] - LSE - 1.01 * E * want.abs()[~impossible]).max()) <= 0 if (~impossible).any() else True
    was = torch.zeros(batch * beams, dtype=torch.bool) if ended is None else ended.reshape(-1).bool()
    assert torch.equal(out[3].cpu(), was[parent] | (token == end))
    return out


SIZES = [(1, 1, 1, 1), (1, 1, 2, 2), (2, 3, 5, 15), (1, 4, 100, 4), (3, 2, 511, 7), (2, 8, 2049, 16), (1, 4, 32000, 4), (2, 5, 50021, 10), (1, 64, 700, 64), (5, 16, 3000, 64),
         (1, 1, 200000, 64), (70, 8, 4100, 16), (600, 1, 5000, 1), (1, 2, 65536, 33), (1, 30, 17000, 60)]


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("batch,beams,V,picks", SIZES)
def test_selection(batch, beams, V, picks, kind):
    torch = torch_mod()
    g = _gen(batch * 31 + beams * 7 + V + picks)
    z = (3.0 * torch.randn(batch * beams, V, generator=g, dtype=torch.float64)).to(_dt(kind))
    score = -10.0 * torch.rand(batch, beams, generator=g)
    ended, end = None, -1
    if (batch + V) % 2:
        end = V // 3
        ended = torch.rand(batch, beams, generator=g) < 0.2
        score[:, 1:][torch.rand(batch, beams - 1, generator=g) < 0.2] = -math.inf
    pad = 3 if batch * beams > 1 else 0
    _check(z, score, picks, ended, end, zv=_strided(z, pad, 1))


def test_the_same_call_gives_the_same_bits_whatever_lies_beside_it():
    torch = torch_mod()
    g = _gen(3)
    z, score = (3.0 * torch.randn(6 * 4, 9000, generator=g)).bfloat16().cuda(), -torch.rand(6, 4, generator=g).cuda()

    def select(z, score):
        out = (torch.empty((score.shape[0], 9), device="cuda"), torch.empty((score.shape[0], 9), dtype=torch.int32, device="cuda"),
               torch.empty((score.shape[0], 9), dtype=torch.int32, device="cuda"))
        tron.tron_beam_select(z, score, *out)
        return out

    first = select(z, score)
    for _ in range(5):
        again = select(z, score)
        assert all(torch.equal(a, b) for a, b in zip(first, again))
    # beams that are alike: the lower one's come first
    _check(z[:4].repeat(2, 1).cpu(), score[:1].repeat(1, 2).cpu(), 9)


@pytest.mark.parametrize("V", [3, 64, 2000, 2049, 40000])
def test_equal_and_ordered_logits(V):
    torch = torch_mod()
    picks, beams = min(40, 3 * V), 3
    score = torch.tensor([[-1.0, -1.0, -1.0], [-2.0, -1.0, -3.0]])
    for row in (torch.zeros(V), torch.full((V,), torch.finfo(torch.float32).min), torch.full((V,), 1e30)):
        _check(row.expand(6, V).contiguous(), score, picks)
    up = torch.arange(V, dtype=torch.float32) * (1.0 / 64)
    scores = torch.tensor([[-1.0, -1.4, -1.9]])
    _check(torch.stack([up, up.flip(0), -up]), scores, picks)
    # plateaus, the highest one at the end
    steps = torch.floor(torch.arange(V, dtype=torch.float32) / 700)
    _check(torch.stack([steps, steps.flip(0), steps]), torch.tensor([[-1.0, -1.4, -2.9]]), picks)


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("V", [70, 5000, 33000])
def test_masks_and_rows_that_say_nothing(V, kind):
    torch = torch_mod()
    g = _gen(V)
    dt = _dt(kind)
    z = (2.0 * torch.randn(4 * 6, V, generator=g)).to(dt)
    z[0] = -math.inf                       # no probability anywhere
    z[1, V // 2] = math.nan
    z[2, V - 1] = math.inf
    z[3, 5:] = -math.inf                   # five columns are possible
    z[4] = torch.finfo(dt).min             # uniform
    z[5, : V // 2] = torch.finfo(dt).min
    z[6:12] = -math.inf                    # an item of which nothing is possible
    z[12:18, 3:] = -math.inf               # one of which few are
    z[18] = math.nan                       # ended: not looked at
    score = -torch.rand(4, 6, generator=g)
    score[3, 2:] = torch.tensor([math.nan, math.inf, -math.inf, -0.0])
    ended = torch.zeros(4, 6, dtype=torch.uint8)
    ended[3, 0] = 255
    for picks in (1, 5, 30, 64):
        _check(z, score, picks, ended, 1)


def test_scores_far_apart_and_rows_of_work_spaces_and_none():
    torch = torch_mod()
    z = torch.randn(2, 100, generator=_gen(1))
    _check(z, torch.tensor([[-1e30, -3.0]]), 64)
    _check(z, torch.tensor([[-1e-30], [3e38]]), 1)
    out = (torch.full((0, 4), 1.0, device="cuda"), torch.empty((0, 4), dtype=torch.int32, device="cuda"), torch.empty((0, 4), dtype=torch.int32, device="cuda"))
    tron.tron_beam_select(z[:0].cuda(), torch.empty((0, 2), device="cuda"), *out)


def test_the_next_beams_in_the_place_of_the_last_ones():
    torch = torch_mod()
    g = _gen(21)
    z, score, ended = torch.randn(90 * 6, 3000, generator=g), -torch.rand(90, 6, generator=g), torch.rand(90, 6, generator=g) < 0.4
    want = _check(z, score, 6, ended, 5)
    s, e = score.cuda(), ended.cuda()
    parent, token = torch.empty((90, 6), dtype=torch.int32, device="cuda"), torch.empty((90, 6), dtype=torch.int32, device="cuda")
    tron.tron_beam_select(z.cuda(), s, s, parent, token, ended=e, end=5, next_ended=e)
    assert all(torch.equal(a, b) for a, b in zip(want, (s, parent, token, e)))


# --------------------------------------------------------------------------- states
def _states(g, shape, dtype):
    torch = torch_mod()
    n = torch.Size(shape).numel() * torch.empty(0, dtype=dtype).element_size()
    return torch.randint(0, 256, (n,), generator=g, dtype=torch.uint8).view(dtype).view(shape)


@pytest.mark.parametrize("dtype", ["uint8", "bfloat16", "float32", "int64"])
@pytest.mark.parametrize("layers,rows,positions,tail,batch,per", [(1, 1, 1, (1,), 1, 1), (3, 6, 5, (3,), 2, 3), (2, 8, 129, (7, 11), 2, 5), (1, 4, 1, (40000,), 1, 9), (4, 12, 600, (16,), 3, 4)])
def test_reorder(layers, rows, positions, tail, batch, per, dtype):
    torch = torch_mod()
    g, dt = _gen(rows + positions), getattr(torch, dtype)
    size = torch.empty(0, dtype=dt).element_size()
    src, was = _states(g, (layers, rows, positions) + tail, dt), _states(g, (layers, batch * per, positions) + tail, dt)
    at = torch.randint(0, rows, (batch, per + 2), generator=g, dtype=torch.int32)
    if batch * per > 2:
        at[0, 1], at[-1, 0] = -1, rows
    lengths = torch.randint(-1, positions + 2, (rows,), generator=g, dtype=torch.int32)
    for n in (None, lengths):
        want = was.clone()
        for i in range(batch * per):
            r = int(at[i // per, i % per])
            if 0 <= r < rows:
                live = positions if n is None else max(0, min(positions, int(n[r])))
                want[:, i, :live] = src[:, r, :live]
        # rows one behind the other, and with room between layers and rows, at an odd place
        out = was.cuda()
        tron.tron_beam_reorder(at.cuda()[:, :per], src.cuda(), out, lengths=None if n is None else n.cuda())
        assert torch.equal(out.cpu().view(torch.uint8), want.view(torch.uint8))
        one = torch.Size(tail).numel() * positions
        room = torch.full((layers * (batch * per * (one + 3) + 5) + 1,), 77, dtype=torch.uint8, device="cuda").repeat_interleave(size)[: (layers * (batch * per * (one + 3) + 5) + 1) * size]
        room = room.view(dt)
        strided = torch.as_strided(room, (layers, batch * per, positions) + tail, (batch * per * (one + 3) + 5, one + 3) + was.stride()[2:], 1)
        strided.copy_(was)
        before = room.clone()
        tron.tron_beam_reorder(at.cuda()[:, :per], src.cuda().transpose(0, 1).contiguous().transpose(0, 1), strided, lengths=None if n is None else n.cuda())
        assert torch.equal(strided.cpu().contiguous().view(torch.uint8), want.view(torch.uint8))
        strided.copy_(was)
        assert torch.equal(room.view(torch.uint8), before.view(torch.uint8))


def test_reorder_of_nothing():
    torch = torch_mod()
    s, out = torch.ones((2, 3, 4, 5), device="cuda"), torch.zeros((2, 2, 4, 5), device="cuda")
    at = torch.tensor([2, 0], dtype=torch.int32, device="cuda")
    tron.tron_beam_reorder(at[:0], s, out[:, :0])
    tron.tron_beam_reorder(at, s[:0], out[:0])
    tron.tron_beam_reorder(at, s[:, :, :0], out[:, :, :0])
    tron.tron_beam_reorder(at, s[:, :0], out)      # no row of src
    assert (out == 0).all()
    with pytest.raises(tron.TronError):
        tron.tron_beam_reorder(at, s, s[:, 1:])    # over itself
    assert (s == 1).all()


def test_reorder_between_the_halves_of_each_layer():
    torch = torch_mod()
    both = torch.randn(3, 2, 4, 5, 6, device="cuda")
    was = both.clone()
    at = torch.tensor([[3, 0], [2, 2]], dtype=torch.int32, device="cuda")
    tron.tron_beam_reorder(at, both[:, 0], both[:, 1])
    assert torch.equal(both[:, 0], was[:, 0]) and torch.equal(both[:, 1], was[:, 0][:, at.flatten().long()])
    tron.tron_beam_reorder(at, both[:, 1], both[:, 0])
    assert torch.equal(both[:, 0], both[:, 1][:, at.flatten().long()])
    with pytest.raises(tron.TronError):
        tron.tron_beam_reorder(at, both[:, 1], both.view(3, 8, 5, 6)[:, 3:7])


@pytest.mark.parametrize("dtype,bits", [("bf16", 0x7F81), ("bf16", 0xFFFF - 0x10000), ("f16", 0x7C01), ("f32", 0x7F800001)])
def test_rows_with_one_nan_of_any_kind(dtype, bits):
    """Signalling ones too, beside the largest values and before them: the row offers nothing, the others all."""
    torch = torch_mod()
    batch, beams, V, picks = 6, 5, 9001, 8
    g = _gen(bits & 0xFFFF)
    z = (4 * torch.randn(batch * beams, V, generator=g)).to(_dt(dtype))
    words = z.view(torch.int32 if dtype == "f32" else torch.int16)
    for i, row in enumerate(range(0, batch * beams, 3)):
        words[row, (0, 1, 7, 8, 511, 2048, 4099, V - 1)[i % 8]] = bits
        z[row, (1, 0, 6, 9, 510, 2049, 4098, V - 2)[i % 8]] = 60.0
    assert int(torch.isnan(z).any(1).sum()) == 10
    _check(z, torch.randn(batch, beams, generator=g), picks)
    one = z[:beams].clone()
    words = one.view(torch.int32 if dtype == "f32" else torch.int16)
    words[:, 5] = bits
    out = _check(one, torch.zeros(1, beams), picks)   # no row is left
    assert bool(torch.isinf(out[0]).all()) and out[2].cpu().tolist() == [list(range(picks))]


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("V,picks", [(100, 8), (100, 64), (2500, 20), (40000, 33)])
def test_scores_that_take_the_differences_of_a_beams_logits(V, picks, kind):
    """Where all candidates of a beam have one score in 64 bits, they go by their z: those that are taken and their order."""
    torch = torch_mod()
    z = torch.randn(4, V, generator=_gen(V + picks)).to(_dt(kind))
    for score in (-1e30, 3e38, -3.4e38):
        _check(z[:1], torch.tensor([[score]]), picks)
        _check(z[:2], torch.tensor([[score], [-score]]), picks)
        _check(z[:2], torch.tensor([[score, score]]), picks)
        # a beam that has ended before one of them, and behind it
        _check(z[:2], torch.tensor([[-1.0, score]]), picks, torch.tensor([[True, False]]), 1)
        _check(z[:3], torch.tensor([[score, -1.0, score]]), picks, torch.tensor([[False, True, False]]), 1)
    # ordinary scores, and logits that differ by less than the last place of theirs
    tiny = (torch.randn(4, V, generator=_gen(V + 1)) * 1e-20).to(_dt(kind))
    if kind != "f16":   # which has no such numbers
        _check(tiny[:1], torch.tensor([[-3.0]]), picks)
        _check(tiny, torch.tensor([[-3.0, -3.0], [-1.0, -1e30]]), picks)
    # equal z among them: the lower column
    steps = (torch.randint(0, 5, (2, V), generator=_gen(V + 2)).float()).to(_dt(kind))
    _check(steps, torch.tensor([[1e30, 1e30]]), picks)


def test_many_offers_of_scores_that_take_the_differences():
    """More than are ranked at once: beam, z and column decide, digit by digit."""
    torch = torch_mod()
    g = _gen(5)
    for z in (torch.randn(64, 300, generator=g), torch.randint(0, 3, (64, 300), generator=g).float(), torch.randn(64, 300, generator=g).half()):
        _check(z, torch.full((1, 64), -1e30), 64)
        few = torch.full((1, 64), -1e30)
        few[0, :63] = -math.inf
        few[0, 3] = -2e30
        _check(z, few, 64)
    # 64 of several beams, the first of which have fewer than that
    z = torch.randn(64, 300, generator=g)
    z[:, 10:] = -math.inf
    _check(z, torch.full((1, 64), 1e30), 64)
    _check(z[:, :20].contiguous(), torch.full((1, 64), 1e30), 64)


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,V,picks", [(1, 3000001, 64), (2, 1200007, 32)])
def test_selection_over_millions_of_columns(rows, V, picks, kind):
    torch = torch_mod()
    z = (3.0 * torch.randn(rows, V, generator=_gen(V))).to(_dt(kind))
    _check(z, -torch.rand(1, rows, generator=_gen(1)), picks)


def test_more_rows_than_a_dimension_of_a_launch():
    torch = torch_mod()
    rows, V = 70001, 100
    z, score = torch.randn(rows, V, generator=_gen(9)).bfloat16(), -torch.rand(rows, 1, generator=_gen(10))
    out = (torch.empty((rows, 2), device="cuda"), torch.empty((rows, 2), dtype=torch.int32, device="cuda"), torch.empty((rows, 2), dtype=torch.int32, device="cuda"))
    tron.tron_beam_select(z.cuda(), score.cuda(), *out)
    best, at = torch.sort(z.double(), dim=1, descending=True, stable=True)
    assert torch.equal(out[1].cpu(), torch.arange(rows, dtype=torch.int32)[:, None].expand(rows, 2)) and torch.equal(out[2].cpu().long(), at[:, :2])
    want = score.double() + best[:, :2] - torch.logsumexp(z.double(), 1)[:, None]
    assert float(((out[0].double().cpu() - want).abs() - LSE - 1.01 * E * want.abs()).max()) <= 0


def test_the_most_offers_in_a_graph():
    """64 beams with 64 picks: the workgroups that join them have more LDS than others."""
    torch = torch_mod()
    z, score = torch.randn(2 * 64, 700, generator=_gen(11)).cuda(), -torch.rand(2, 64, generator=_gen(12)).cuda()
    new = lambda dtype: torch.zeros((2, 64), dtype=dtype, device="cuda")  # noqa: E731
    want, out = [(new(torch.float32), new(torch.int32), new(torch.int32)) for _ in range(2)]
    tron.tron_beam_select(z, score, *want)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        tron.tron_beam_select(z, score, *out)
    for _ in range(3):
        for t in out:
            t.zero_()
        tron.tron_beam_select(z, score, *want)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, out))
