"""A token's way into a softmax head and out of it again: the operators together, on other streams and in graphs, and what they refuse."""
import math

import pytest

import paper_2008_03433_amd as tron
from test_gpu_beam import LSE, _check, _plain
from test_gpu_heads import E, TINY, U, _distill_plain, _gen, _randn, _within
from test_gpu_layer_norm import _plain as _layer_plain
from test_gpu_layer_norm import _plain_grad
from util import torch_mod

pytestmark = pytest.mark.gpu


CLOSE = LSE + 5 * E * 64   # a score's error, and what the roundings of five steps' scores (below 64) add to it


class _Decoder:
    """A head without layers before it: each step's hidden state is the token's embedding plus half the state so far, which is kept for each beam."""

    def __init__(self, batch, beams, V, d, steps, stream=None):
        torch = torch_mod()
        g = _gen(V + d)
        w = _randn(g, V, d).float()
        self.scale = (w.abs().amax(1) / 127.0).cuda()
        self.W = (w.cuda() / self.scale[:, None]).round().to(torch.int8)
        self.batch, self.beams, self.V, self.d, self.stream = batch, beams, V, d, stream
        rows = batch * beams
        new = lambda *s, dtype=torch.float32: torch.zeros(s, dtype=dtype, device="cuda")  # noqa: E731
        self.score = [new(batch, beams), new(batch, beams)]
        self.ended = [new(batch, beams, dtype=torch.bool), new(batch, beams, dtype=torch.bool)]
        self.state = [new(1, rows, steps, d, dtype=torch.bfloat16), new(1, rows, steps, d, dtype=torch.bfloat16)]   # positions: the steps so far
        self.parent = [new(batch, beams, dtype=torch.int32) for _ in range(steps)]
        self.token = [new(batch, beams, dtype=torch.int32) for _ in range(steps)]
        self.length = [torch.full((rows,), i + 1, dtype=torch.int32, device="cuda") for i in range(steps)]
        self.ids = torch.randint(0, V, (rows,), generator=g).cuda().to(torch.int32)
        self.h, self.total = new(rows, d, dtype=torch.bfloat16), new(rows, d, dtype=torch.bfloat16)
        self.x8, self.x_scale = new(rows, d, dtype=torch.int8), new(rows)
        self.z = [new(rows, V) for _ in range(steps)]
        self.steps = steps

    def run(self):
        s = self.stream
        self.score[0].zero_()
        self.score[0][:, 1:].fill_(-math.inf)
        self.ended[0].zero_()
        for i in range(self.steps):
            now, then = i % 2, (i + 1) % 2
            ids = self.ids if i == 0 else self.token[i - 1].view(-1)
            tron.tron_embed(ids, self.W, self.h, scale=1.5, row_scale=self.scale, stream=s)
            before = self.state[now][0, :, i - 1] if i else None
            # the sum is the state of this step, in its place among the positions
            tron.tron_layer_norm(self.h, self.x8, residual=before, total=self.state[now][0, :, i], scale=self.x_scale, stream=s)
            tron.tron_linear(self.x8, self.W, self.z[i], x_scale=self.x_scale, w_scale=self.scale, stream=s)
            tron.tron_beam_select(self.z[i], self.score[now], self.score[then], self.parent[i], self.token[i], ended=self.ended[now], end=1, next_ended=self.ended[then], stream=s)
            tron.tron_beam_reorder(self.parent[i], self.state[now], self.state[then], lengths=self.length[i], stream=s)

    def outputs(self):
        return [self.score[self.steps % 2], self.ended[self.steps % 2], self.state[self.steps % 2]] + self.parent + self.token + self.z


def test_a_beam_search_step_by_step():
    torch = torch_mod()
    batch, beams, V, d, steps = 3, 4, 700, 96, 5
    D = _Decoder(batch, beams, V, d, steps)
    D.run()
    torch.cuda.synchronize()
    W = D.W.double().cpu() * D.scale.double().cpu()[:, None]
    score, ended = torch.zeros(batch, beams), torch.zeros(batch, beams, dtype=torch.bool)
    score[:, 1:] = -math.inf
    state = torch.zeros(batch * beams, 0, d, dtype=torch.float64)
    ids = D.ids.cpu().long()
    for i in range(steps):
        # the logits, from the formulas: embedding and state are rounded to bf16, features to 127 steps of the row's largest, the rest in 32 bits
        h = (1.5 * W[ids]).bfloat16().double()
        s = h + (state[:, i - 1] if i else 0.0)
        x = s - s.mean(1, keepdim=True)
        x = x / (x.pow(2).mean(1, keepdim=True) + 1e-5).sqrt()
        step = x.abs().amax(1, keepdim=True) / 127.0
        # half a step of each feature, and what 2^-9 of the embedding and 2^-9 of the state change of the others
        off = ((0.51 * step + 2.0 ** -7 * (x.abs() + x.abs().mean(1, keepdim=True))) @ W.abs().T)
        z = x @ W.T
        assert ((D.z[i].double().cpu() - z).abs() <= off).all()
        # the selection, from the logits that are there
        want, parent, token, least, c = _plain(D.z[i], score, ended, 1, beams)
        if least > 2 * CLOSE:
            assert torch.equal(D.parent[i].cpu().long(), parent) and torch.equal(D.token[i].cpu().long(), token)
        else:   # near ones may have changed places
            parent, token = D.parent[i].cpu().long(), D.token[i].cpu().long()
            assert len(set(zip(parent.flatten().tolist(), token.flatten().tolist()))) == batch * beams
            want, best = c[parent, token], want
            assert ((want == best) | ((want - best).abs() <= 2 * CLOSE)).all()
        state = torch.cat([state, s.bfloat16().double()[:, None]], 1)[parent.view(-1)]
        ended = ended.view(-1)[parent] | (token == 1)
        score, ids = want.float(), token.view(-1)
    assert torch.equal(D.state[steps % 2][0].cpu().double(), state)
    assert torch.equal(D.ended[steps % 2].cpu(), ended) and float((D.score[steps % 2].cpu() - score).abs().max()) <= 5 * CLOSE


def test_beam_searches_on_two_streams_and_in_a_graph():
    torch = torch_mod()
    args = (2, 3, 5000, 160, 4)
    first = _Decoder(*args)
    first.run()
    torch.cuda.synchronize()
    want = [t.clone() for t in first.outputs()]
    sides = [torch.cuda.Stream(), torch.cuda.Stream()]
    for as_address in (False, True):
        others = []
        for side in sides:
            D = _Decoder(*args, stream=side.cuda_stream if as_address else side)
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(side):   # the fills' stream, too
                D.run()
            others.append(D)
        torch.cuda.synchronize()
        for D in others:
            assert all(torch.equal(a, b) for a, b in zip(want, D.outputs()))
    D = _Decoder(*args)
    sides[0].wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(sides[0]):
        D.run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        D.run()
    for _ in range(4):
        for t in D.outputs():
            t.fill_(1)
        first.run()   # eager work of the same operators between the replays
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, D.outputs()))


class _Training:
    """Loss and gradients of a head over the embeddings of tokens, with one table for both."""

    def __init__(self, m, V, d, K=4, stream=None):
        torch = torch_mod()
        g = _gen(m + V)
        self.stream = stream
        dt = torch.float16
        self.ids = torch.randint(0, V, (m,), generator=g).cuda()
        self.ids[3] = -1
        self.W = (_randn(g, V, d) / 4).to(dt).cuda()
        self.gain, self.shift = (1 + 0.1 * _randn(g, d)).float().cuda(), (0.1 * _randn(g, d)).float().cuda()
        self.teacher, self.t = torch.randint(0, V, (m, K), generator=g).cuda(), _randn(g, m, K).float().cuda()
        new = lambda *s, dtype=torch.float32: torch.zeros(s, dtype=dtype, device="cuda")  # noqa: E731
        self.e, self.x, self.z, self.dz = new(m, d, dtype=dt), new(m, d, dtype=dt), new(m, V, dtype=dt), new(m, V, dtype=dt)
        self.mean, self.rstd, self.loss, self.lse = new(m), new(m), new(m), new(m)
        self.dx, self.de, self.dgain, self.dshift, self.dW = new(m, d, dtype=dt), new(m, d, dtype=dt), new(d), new(d), new(V, d)

    def run(self):
        s = self.stream
        tron.tron_embed(self.ids, self.W, self.e, scale=3.0, stream=s)
        tron.tron_layer_norm(self.e, self.x, gain=self.gain, shift=self.shift, mean=self.mean, rstd=self.rstd, stream=s)
        tron.tron_linear(self.x, self.W, self.z, stream=s)
        tron.tron_distill(self.z, self.teacher, self.t, self.loss, self.lse, dz=self.dz, stream=s)
        tron.tron_linear_grad(self.x, self.W, self.dz, dx=self.dx, dw=self.dW, stream=s)
        tron.tron_layer_norm_grad(self.e, self.mean, self.rstd, self.dx, self.de, gain=self.gain, dgain=self.dgain, dshift=self.dshift, stream=s)
        tron.tron_embed_grad(self.ids, self.de, self.dW, scale=3.0, add=True, stream=s)   # to the gradient that the product left there

    def outputs(self):
        return [self.loss, self.dgain, self.dshift, self.dW, self.de]


def test_a_training_step():
    """Each operator's output against the formula in 64 bits of what the one before it stored, and the table's gradient of both ways."""
    torch = torch_mod()
    m, V, d = 150, 90, 70
    T = _Training(m, V, d)
    T.run()
    u = U["f16"]
    W, ids = T.W.cpu().double(), T.ids.cpu()
    there = (ids >= 0)[:, None]
    e = torch.where(there, 3.0 * W[ids.clamp(min=0)], 0.0)
    _within(T.e, e, (u + 4 * E) * e.abs() + TINY["f16"], "embeddings")
    _, mean, rstd, y, off_mean, off_rstd, off_y = _layer_plain(T.e.cpu(), None, T.gain.cpu(), T.shift.cpu(), 1e-5)
    _within(T.x, y, u * y.abs() + 1.01 * off_y + TINY["f16"], "features")
    _within(T.mean, mean, off_mean + TINY["f32"], "mean")
    x = T.x.cpu().double()
    _within(T.z, x @ W.T, u * (x @ W.T).abs() * 1.01 + (d + 8) * 2 * E * (x.abs() @ W.abs().T), "logits")
    loss, _, dz, p, _, w = _distill_plain(T.z.cpu(), T.teacher.cpu(), T.t.cpu(), 1.0, torch.ones(m))
    _within(T.loss, loss, 1e-5 * loss.abs() + 1e-5, "loss")
    _within(T.dz, dz, (u + 2.0 ** -15) * dz.abs() + 2.0 ** -15 * p + TINY["f16"], "gradient of the logits")
    kept = T.dz.cpu().double()
    dx = kept @ W
    _within(T.dx, dx, u * dx.abs() * 1.01 + (V + 8) * 2 * E * (kept.abs() @ W.abs()) + TINY["f16"], "gradient of the features")
    de, off, dgain, off_g, dshift, off_b = _plain_grad(T.e.cpu(), T.mean.cpu(), T.rstd.cpu(), T.gain.cpu(), T.dx.cpu(), None)
    _within(T.de, de, u * de.abs() + 1.01 * off + TINY["f16"], "gradient of the embeddings")
    _within(T.dgain, dgain, off_g, "dgain")
    _within(T.dshift, dshift, off_b, "dshift")
    de = T.de.cpu().double()
    by_token, size = torch.zeros(V, d, dtype=torch.float64), torch.zeros(V, d, dtype=torch.float64)
    by_token.index_add_(0, ids[ids >= 0], 3.0 * de[ids >= 0])
    size.index_add_(0, ids[ids >= 0], 3.0 * de[ids >= 0].abs())
    by_product = kept.T @ x
    _within(T.dW, by_product + by_token, (m + 8) * 2 * E * (kept.abs().T @ x.abs()) + (m + 4) * E * size + 2 * E * (by_product + by_token).abs(), "gradient of the table")


def test_training_on_other_streams_and_in_a_graph():
    torch = torch_mod()
    args = (300, 2000, 700)
    first = _Training(*args)
    first.run()
    torch.cuda.synchronize()
    want = [t.clone() for t in first.outputs()]
    side = torch.cuda.Stream()
    for s in (side, side.cuda_stream):
        T = _Training(*args, stream=s)
        side.wait_stream(torch.cuda.current_stream())
        T.run()
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, T.outputs()))
    graphs = []
    for _ in range(2):   # two, each with a work space of its own
        T = _Training(*args)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            T.run()
        graphs.append((graph, T))
    for _ in range(3):
        for _, T in graphs:
            for t in T.outputs():
                t.fill_(math.nan)
        first.run()
        torch.cuda.synchronize()
        for graph, _ in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for _, T in graphs:
            assert all(torch.equal(a, b) for a, b in zip(want, T.outputs()))


def test_softmax_head_over_layer_norms():
    torch = torch_mod()
    g = _gen(4)
    m, d, V, K = 60, 50, 20, 3
    hidden, gain, shift = _randn(g, m, d).bfloat16(), (1 + 0.1 * _randn(g, d)).float(), (0.1 * _randn(g, d)).float()
    ids, t = torch.randint(0, V, (m, K), generator=g).cuda(), _randn(g, m, K).float().cuda()
    head = tron.SoftmaxHead(hidden.cuda(), ids, t, gain=gain.cuda(), eps=1e-5, norm="layer", shift=shift.cuda())
    _, _, _, y, _, _, off = _layer_plain(hidden, None, gain, shift, 1e-5)
    _within(head.X, y, U["bf16"] * y.abs() + 1.01 * off + TINY["bf16"], "features")
    W, G = torch.randn(V, d, device="cuda").bfloat16().float(), torch.empty(V, d, device="cuda")
    f = head.fun_grad(1.0, W, G)
    assert math.isfinite(f) and torch.isfinite(G).all()
    for kw in ({"norm": "batch"}, {"shift": shift.cuda()}):
        with pytest.raises(tron.TronError):
            tron.SoftmaxHead(hidden.cuda(), ids, t, **kw)


def test_selection_of_many_offers():
    """More offers than are ranked at once, of equal and of different scores."""
    torch = torch_mod()
    g = _gen(77)
    z = torch.randint(0, 3, (64, 300), generator=g).float()
    _check(z, torch.zeros(1, 64), 64)
    _check(z, -torch.randint(0, 3, (1, 64), generator=g).float(), 64)
    _check(torch.randn(64, 300, generator=g), -torch.rand(1, 64, generator=g), 64)
    one = torch.full((64, 300), -math.inf)
    one[:, 0] = 0.0
    _check(one, torch.zeros(1, 64), 64)
    _check(torch.full((64, 300), -math.inf), torch.zeros(1, 64), 64)


def test_refusals():
    torch = torch_mod()
    f, b = torch.zeros(4, 8, device="cuda"), torch.zeros(4, 8, device="cuda").bfloat16()
    q = torch.zeros(4, 8, dtype=torch.int8, device="cuda")
    v4, v8 = torch.zeros(4, device="cuda"), torch.zeros(8, device="cuda")

    def refused(call, *args, **kw):
        with pytest.raises(tron.TronError) as e:
            call(*args, **kw)
        assert e.value.code == -1, e.value

    small = torch.empty(16, dtype=torch.uint8, device="cuda")
    for norm in (tron.tron_layer_norm, tron.tron_rms_norm):
        refused(norm, b, q)                                          # no scale
        refused(norm, q, q, scale=v4)                                # input in 8 bits
        refused(norm, b, q, scale=v8)
    refused(tron.tron_layer_norm, f.cpu(), f)
    refused(tron.tron_layer_norm, f, torch.zeros(4, 7, device="cuda"))
    refused(tron.tron_layer_norm, f, b)
    refused(tron.tron_layer_norm, f, torch.empty_like(f), eps=-1.0)
    refused(tron.tron_layer_norm, f, torch.empty_like(f), shift=v4)
    refused(tron.tron_layer_norm, f, torch.empty_like(f), mean=v8)
    refused(tron.tron_layer_norm, f, v8.expand(4, 8))
    refused(tron.tron_layer_norm_grad, f, None, v4, f, torch.empty_like(f))
    refused(tron.tron_layer_norm_grad, f, v4, None, f, torch.empty_like(f))
    refused(tron.tron_layer_norm_grad, f, v4, v4, b, torch.empty_like(f))
    refused(tron.tron_layer_norm_grad, f, v4, v4, f, torch.empty_like(f), dshift=v8, work=small)
    y = torch.zeros(4, 4, device="cuda")
    refused(tron.tron_linear, q, q, y)                               # no scales
    refused(tron.tron_linear, q, q, y, x_scale=v4)
    refused(tron.tron_linear, q, b, y, x_scale=v4, w_scale=v4)
    long = torch.zeros(1, 1 << 17, dtype=torch.int8, device="cuda")
    refused(tron.tron_linear, long, long, torch.zeros(1, 1, device="cuda"), x_scale=v4[:1], w_scale=v4[:1])
    refused(tron.tron_linear_grad, q, q, torch.zeros(4, 4, dtype=torch.int8, device="cuda"), dx=torch.empty_like(q))
    refused(tron.tron_linear, b, b, torch.zeros(4, 4, dtype=torch.int8, device="cuda"))   # an output in 8 bits
    refused(tron.tron_distill, q, torch.zeros(4, 2, dtype=torch.int64, device="cuda"), torch.zeros(4, 2, device="cuda"), v4)

    z, score, nxt = torch.zeros(4, 8, device="cuda"), torch.zeros(2, 2, device="cuda"), torch.zeros(2, 3, device="cuda")
    p, t = torch.zeros(2, 3, dtype=torch.int32, device="cuda"), torch.zeros(2, 3, dtype=torch.int32, device="cuda")
    flags = torch.zeros(2, 2, dtype=torch.bool, device="cuda")
    refused(tron.tron_beam_select, z.cpu(), score, nxt, p, t)
    refused(tron.tron_beam_select, z[:3], score, nxt, p, t)
    refused(tron.tron_beam_select, z.to(torch.int8), score, nxt, p, t)
    refused(tron.tron_beam_select, z, score.double(), nxt, p, t)
    refused(tron.tron_beam_select, z, score, nxt, p.long(), t)
    refused(tron.tron_beam_select, z, score, nxt, p, t[:, :2])
    refused(tron.tron_beam_select, z, score, nxt, p, t, ended=flags)            # no end
    refused(tron.tron_beam_select, z, score, nxt, p, t, ended=flags, end=8)
    refused(tron.tron_beam_select, z, score, nxt, p, t, ended=flags.float(), end=1)
    refused(tron.tron_beam_select, z, score, nxt, p, t, end=-2)
    refused(tron.tron_beam_select, z, score, nxt, p, t, work=small)
    refused(tron.tron_beam_select, z, torch.zeros(4, device="cuda"), nxt, p, t)
    refused(tron.tron_beam_select, z[:, :1], score, nxt, p, t)                  # more picks than candidates
    many = torch.zeros(2, 65, device="cuda")
    refused(tron.tron_beam_select, torch.zeros(4, 100, device="cuda"), score, many, many.int(), many.int())
    refused(tron.tron_beam_select, torch.zeros(65, 100, device="cuda"), torch.zeros(1, 65, device="cuda"), nxt[:1], p[:1], t[:1])

    s, out, rows = torch.zeros(2, 4, 5, 6, device="cuda"), torch.zeros(2, 3, 5, 6, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")
    refused(tron.tron_beam_reorder, rows.long(), s, out)
    refused(tron.tron_beam_reorder, rows, s, out[:, :2])
    refused(tron.tron_beam_reorder, rows, s, out.double())
    refused(tron.tron_beam_reorder, rows, s, out.cpu())
    refused(tron.tron_beam_reorder, rows, s[0], out[0, 0])
    refused(tron.tron_beam_reorder, rows, s, out, lengths=rows)
    refused(tron.tron_beam_reorder, rows, s.transpose(2, 3), out.transpose(2, 3))
    refused(tron.tron_beam_reorder, rows, s, out[:, :1].expand(2, 3, 5, 6))
    refused(tron.tron_beam_reorder, rows, s, s[:, :3])

    ids = torch.zeros(4, dtype=torch.int64, device="cuda")
    refused(tron.tron_embed, ids.float(), f, torch.empty_like(f))
    refused(tron.tron_embed, ids.cpu(), f, torch.empty_like(f))
    refused(tron.tron_embed, ids[:3], f, torch.empty_like(f))
    refused(tron.tron_embed, ids, q, torch.empty_like(f))                       # no scales
    refused(tron.tron_embed, ids, f, torch.empty_like(f), row_scale=v4)
    refused(tron.tron_embed, ids, f, torch.empty_like(q))
    refused(tron.tron_embed, ids, f, v8.expand(4, 8))
    refused(tron.tron_embed, ids, f.t(), torch.empty(4, 4, device="cuda"))
    refused(tron.tron_embed_grad, ids, f, torch.zeros(9, 7, device="cuda"))
    refused(tron.tron_embed_grad, ids, q, torch.zeros(9, 8, device="cuda"))
    refused(tron.tron_embed_grad, ids, f, torch.zeros(9, 8, dtype=torch.int8, device="cuda"))
    refused(tron.tron_embed_grad, ids, f, v8.expand(9, 8))
    refused(tron.tron_embed_grad, ids, f, torch.zeros(9, 8, device="cuda"), work=small)


def test_softmax_head_over_layer_norms_is_the_problem_of_its_features():
    """Function, gradient and Hessian-vector product from the formulas on the features and logits that are there, as of the head over RMS norms."""
    torch = torch_mod()
    g = _gen(13)
    m, d, V, K, C, T = 90, 70, 33, 4, 2.0, 1.5
    hidden, residual = (_randn(g, m, d) + _randn(g, m, 1)).bfloat16(), _randn(g, m, d).bfloat16()
    gain, shift = (1 + 0.1 * _randn(g, d)).float(), (0.1 * _randn(g, d)).float()
    ids, t, weight = torch.randint(0, V, (m, K), generator=g), _randn(g, m, K).float(), torch.rand(m, generator=g) + 0.5
    W, D = (_randn(g, V, d) / 8).bfloat16().float(), (_randn(g, V, d) / 8).bfloat16().float()   # exact in the products' type
    head = tron.SoftmaxHead(hidden.cuda(), ids.cuda(), t.cuda(), gain=gain.cuda(), residual=residual.cuda(), temperature=T, weight=weight.cuda(), eps=1e-5, norm="layer",
                            shift=shift.cuda())
    G, HD = torch.empty(V, d, device="cuda"), torch.empty(V, d, device="cuda")
    f = head.fun_grad(C, W.cuda(), G)
    X = head.X.double().cpu()
    _, _, _, y, _, _, off = _layer_plain(hidden, residual, gain, shift, 1e-5)
    _within(X, y, U["bf16"] * y.abs() + 1.01 * off + TINY["bf16"], "features")
    z = head.z.cpu()
    _within(z, X @ W.double().T, U["bf16"] * (X @ W.double().T).abs() * 1.01 + (d + 8) * 2 * E * (X.abs() @ W.double().abs().T), "logits")
    loss, _, dz, p, _, w = _distill_plain(z, ids, t, T, weight)
    want = 0.5 * float((W.double() ** 2).sum()) + C * float(loss.sum())
    assert abs(f - want) <= 1e-5 * abs(want)
    # dz is rounded to bf16 (and computed to 2^-16 of p)
    _within(G, W.double() + C * dz.T @ X, C * ((U["bf16"] + 2.0 ** -10) * dz.abs() + 2.0 ** -15 * w * T * p).T @ X.abs() + 1e-6, "gradient")
    head.hv(C, D.cuda(), HD)
    u = X @ D.double().T
    h = w * (p * u - p * (p * u).sum(1, keepdim=True))
    # u is rounded to bf16 before, H u after
    off = w * p * (u.abs() + (p * u.abs()).sum(1, keepdim=True)) * (U["bf16"] + 2.0 ** -10) + h.abs() * U["bf16"]
    _within(HD, D.double() + C * h.T @ X, C * off.T @ X.abs() + 1e-6, "Hessian-vector product")
