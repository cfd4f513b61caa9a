"""The way of a token into a multi-class head and out of it again, as cases that can be timed: the lookup of its embedding, the layer norm that makes
its features, the matrix product of 8-bit integers that makes its logits, the step of a beam search over these (with the states of
the beams that go on), and, for training, the gradients of the norm and of the lookup.

`run` computes them with elementary torch operations in 32 bits (the beams' scores, whose order decides, in 64), or, where `own` is true,
with this library's calls on the same state.  Inputs are drawn on the GPU from the seed: hidden states with a few large features and a
mean that is not 0, weights of variance 1 / k, logits of standard deviation 3, tokens of which some are frequent and some missing."""
import math

import numpy as np
import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16, "e4m3": torch.float8_e4m3fn, "i8": torch.int8}
BYTES = {"f32": 4, "bf16": 2, "f16": 2, "e4m3": 1, "i8": 1}
ACTS = {"none": 0, "relu": 1, "gelu": 2, "silu": 3}
EPS = 1e-5
E4M3_MAX = 448.0
I8_MAX = 127.0


def listed():
    return [
        # the features of one token on their way to a product in 8 bits: the smallest call, where latency counts
        {"name": "norm_token_e4m3", "op": "norm", "m": 1, "d": 4096, "type": "bf16", "out": "e4m3", "residual": True},
        # those of a batch of prompts: the widest rows
        {"name": "norm_prompts", "op": "norm", "m": 16384, "d": 8192, "type": "bf16", "out": "bf16", "residual": True},
        # the backward pass of the norm in training
        {"name": "norm_grad", "op": "norm_grad", "m": 16384, "d": 4096, "type": "bf16", "residual": True},
        # the same of a small model, an odd width
        {"name": "norm_grad_odd", "op": "norm_grad", "m": 30011, "d": 1023, "type": "f16", "residual": False},
        # logits of the beams of one prompt: the weights are read once, nothing else counts
        {"name": "linear_beams", "op": "linear", "m": 8, "n": 32000, "k": 4096, "out": "f32", "act": "none", "bias": False, "residual": False},
        # a hidden layer of the head over a batch of prompts: the most arithmetic
        {"name": "linear_prompts", "op": "linear", "m": 8192, "n": 8192, "k": 4096, "out": "bf16", "act": "silu", "bias": True, "residual": False},
        # a thousand classes on a few hundred rows, every size odd
        {"name": "linear_odd", "op": "linear", "m": 515, "n": 1003, "k": 2051, "out": "f16", "act": "none", "bias": True, "residual": True},
        # a step of the search for one prompt, its beams' states of a few layers moved along: latency
        {"name": "beam_one", "op": "beam", "batch": 1, "beams": 4, "v": 32000, "picks": 4, "type": "f32", "layers": 4, "positions": 64, "width": 256},
        # the same for a batch of prompts over a large vocabulary; twice as many candidates as beams are kept
        {"name": "beam_batch", "op": "beam", "batch": 64, "beams": 8, "v": 128000, "picks": 16, "type": "bf16", "layers": 2, "positions": 129, "width": 128},
        # the embeddings of the beams' tokens, from the head's own weights in 8 bits
        {"name": "embed_beams", "op": "embed", "m": 8, "d": 4096, "v": 32000, "type": "i8", "out": "bf16", "ids": "i32"},
        # the gradient of the lookup of a training batch: every row of the table is written
        {"name": "embed_grad", "op": "embed_grad", "m": 32768, "d": 4096, "v": 128000, "type": "bf16", "out": "f32", "ids": "i64"},
        # the same of a small model, an odd width
        {"name": "embed_grad_odd", "op": "embed_grad", "m": 9001, "d": 511, "v": 50021, "type": "f16", "out": "f16", "ids": "i32"},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "norm", "norm_grad", "norm_grad", "linear", "linear", "linear", "beam", "beam", "beam", "embed", "embed_grad", "embed_grad"])
    kind = rng.choice(["bf16", "bf16", "f16", "f32"])
    if op in ("norm", "norm_grad"):
        d = _log(rng, 64, 16384)
        m = _log(rng, 1, min(65536, (16384 * 8192) // (d * (2 if kind == "f32" else 1))))
        case = {"op": op, "m": m, "d": d, "type": kind, "residual": rng.random() < 0.6}
        return case | ({"out": rng.choice(["e4m3", kind])} if op == "norm" else {})
    if op == "linear":
        while True:
            m, n, k = _log(rng, 1, 16384), _log(rng, 16, 32768), _log(rng, 32, 8192)
            if rng.random() < 0.5:  # what programs choose; the others are odd as often as even
                n, k = max(64, n // 128 * 128), max(64, k // 128 * 128)
            if m * n * k <= 8192 * 8192 * 4096 and m * n <= 16384 * 16384:
                break
        return {"op": op, "m": m, "n": n, "k": k, "out": rng.choice(["bf16", "f16", "f32"]), "act": rng.choice(["none", "none", "relu", "gelu", "silu"]),
                "bias": rng.random() < 0.7, "residual": rng.random() < 0.3}
    if op == "beam":
        v = _log(rng, 100, 200_000)
        beams = rng.choice([1, 2, 3, 4, 4, 5, 8, 8, 12, 16])
        batch = _log(rng, 1, max(1, min(256, 64 * 8 * 128000 // (v * beams * (2 if kind == "f32" else 1)))))
        layers, positions, width = rng.choice([1, 2, 4, 8]), _log(rng, 1, 512), rng.choice([32, 64, 100, 128, 256])
        while layers * batch * beams * positions * width > 1 << 25 and positions > 1:
            positions //= 2
        return {"op": op, "batch": batch, "beams": beams, "v": v, "picks": min(beams * rng.choice([1, 1, 2]), 32), "type": kind, "layers": layers,
                "positions": positions, "width": width}
    v, d = _log(rng, 100, 200_000), _log(rng, 64, 8192)
    while v * d > 128000 * 4096:
        d //= 2
    m = _log(rng, 1, min(65536, 32768 * 4096 // d))
    case = {"op": op, "m": m, "d": d, "v": v, "ids": rng.choice(["i64", "i32"])}
    if op == "embed":
        kind = rng.choice([kind, "e4m3", "i8"])
        return case | {"type": kind, "out": kind if kind in ("bf16", "f16", "f32") else rng.choice(["bf16", "f16"])}
    return case | {"type": kind, "out": rng.choice(["f32", kind])}


# ------------------------------------------------------------------------------------------ inputs
def _normal(g, shape, dtype, std=1.0):
    return torch.empty(shape, dtype=torch.float32, device="cuda").normal_(0.0, std, generator=g).to(dtype)


def _hidden(g, m, d, dtype):
    """Hidden states: about one feature in a hundred is ten times as large as the others, and rows have a mean of their own."""
    size = torch.where(torch.rand(d, generator=g, device="cuda") < 0.01, 10.0, 1.0)
    x = torch.empty((m, d), device="cuda").normal_(generator=g) * size
    return (x + torch.empty((m, 1), device="cuda").normal_(generator=g)).to(dtype)


def _in_8_bits(a, kind):
    largest = E4M3_MAX if kind == "e4m3" else I8_MAX
    scale = a.abs().amax(1).clamp(min=1e-30) / largest
    a = a / scale[:, None]
    return (a.to(torch.float8_e4m3fn) if kind == "e4m3" else a.round().clamp(-I8_MAX, I8_MAX).to(torch.int8)), scale


def _tokens(g, m, v, kind):
    """Low ids are frequent, as in vocabularies that are sorted by frequency; one token in sixteen is missing."""
    ids = (torch.rand(m, generator=g, device="cuda", dtype=torch.float64) ** 3 * v).long().clamp(max=v - 1)
    ids[torch.rand(m, generator=g, device="cuda") < 1 / 16] = -1
    return ids if kind == "i64" else ids.to(torch.int32)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    op = case["op"]
    new = lambda *shape, dtype=torch.float32: torch.empty(shape, dtype=dtype, device="cuda")  # noqa: E731
    s = {"case": case}
    if op == "norm":
        m, d, dt, out = case["m"], case["d"], DTYPES[case["type"]], DTYPES[case["out"]]
        s["x"] = _hidden(g, m, d, dt)
        s["residual"] = _normal(g, (m, d), dt) if case["residual"] else None
        s["gain"], s["shift"] = 1.0 + _normal(g, (d,), torch.float32, 0.1), _normal(g, (d,), torch.float32, 0.1)
        s["y"], s["mean"], s["rstd"] = new(m, d, dtype=out), new(m), new(m)
        s["total"] = new(m, d, dtype=dt) if case["residual"] else None
        s["scale"] = new(m) if case["out"] == "e4m3" else None
    elif op == "norm_grad":
        m, d, dt = case["m"], case["d"], DTYPES[case["type"]]
        s["total"] = _hidden(g, m, d, dt)
        total = s["total"].float()
        s["mean"] = total.mean(1)
        s["rstd"] = ((total - s["mean"][:, None]).square().mean(1) + EPS).rsqrt()
        s["gain"] = 1.0 + _normal(g, (d,), torch.float32, 0.1)
        s["dy"] = _normal(g, (m, d), dt)
        s["dtotal"] = _normal(g, (m, d), dt) if case["residual"] else None
        s["dx"], s["dgain"], s["dshift"] = new(m, d, dtype=dt), new(d), new(d)
    elif op == "linear":
        m, n, k, out = case["m"], case["n"], case["k"], DTYPES[case["out"]]
        s["x"], s["x_scale"] = _in_8_bits(_hidden(g, m, k, torch.float32), "i8")
        s["w"], s["w_scale"] = _in_8_bits(_normal(g, (n, k), torch.float32, k ** -0.5), "i8")
        s["bias"] = _normal(g, (n,), torch.float32, 0.1) if case["bias"] else None
        s["residual"] = _normal(g, (m, n), out) if case["residual"] else None
        s["y"] = new(m, n, dtype=out)
    elif op == "beam":
        batch, beams, v, picks, dt = case["batch"], case["beams"], case["v"], case["picks"], DTYPES[case["type"]]
        rows, shape = batch * beams, (case["positions"], case["width"])
        s["z"] = _normal(g, (rows, v), dt, 3.0)
        # sums of log-probabilities so far; one prompt in eight is at its first step, where a single beam is there
        score = -10.0 * torch.rand((batch, beams), generator=g, device="cuda")
        first = torch.rand(batch, generator=g, device="cuda") < 0.125
        score[:, 1:].masked_fill_(first[:, None], -math.inf)
        s["score"] = score
        ended = torch.rand((batch, beams), generator=g, device="cuda") < 1 / 16
        ended[first] = False
        s["ended"], s["end"] = ended, 2
        s["next_score"] = new(batch, picks)
        s["parent"], s["token"] = new(batch, picks, dtype=torch.int32), new(batch, picks, dtype=torch.int32)
        s["next_ended"] = new(batch, picks, dtype=torch.bool)
        # the states of the beams so far, and room for those that go on (as many as there were)
        s["states"] = _normal(g, (case["layers"], rows) + shape, torch.bfloat16)
        s["next_states"] = torch.zeros((case["layers"], batch * min(picks, beams)) + shape, dtype=torch.bfloat16, device="cuda")
        low = (case["positions"] + 1) // 2
        s["lengths"] = torch.randint(low, case["positions"] + 1, (batch, 1), generator=g, device="cuda").expand(batch, beams).reshape(rows).to(torch.int32)
    else:
        m, d, v = case["m"], case["d"], case["v"]
        s["ids"] = _tokens(g, m, v, case["ids"])
        if op == "embed":
            table, s["row_scale"] = _normal(g, (v, d), torch.float32, d ** -0.5), None
            if BYTES[case["type"]] == 1:
                s["table"], s["row_scale"] = _in_8_bits(table, case["type"])
            else:
                s["table"] = table.to(DTYPES[case["type"]])
            s["y"] = new(m, d, dtype=DTYPES[case["out"]])
        else:
            s["dy"] = _normal(g, (m, d), DTYPES[case["type"]])
            s["dtable"] = new(v, d, dtype=DTYPES[case["out"]])
        s["factor"] = float(d) ** 0.5
    return s


# ------------------------------------------------------------------------------------------ the plain forms
def _act(a, name):
    if name == "relu":
        return a.clamp(min=0.0)
    if name == "gelu":
        return 0.5 * a * (1.0 + torch.erf(a * math.sqrt(0.5)))
    return a / (1.0 + torch.exp(-a)) if name == "silu" else a


def _plain(s):
    case = s["case"]
    op = case["op"]
    f = lambda a: None if a is None else a.float()  # noqa: E731
    if op == "norm":
        total = f(s["x"]) if s["residual"] is None else f(s["x"]) + f(s["residual"])
        mean = total.mean(1)
        centred = total - mean[:, None]
        rstd = 1.0 / torch.sqrt((centred * centred).mean(1) + EPS)
        y = centred * rstd[:, None] * s["gain"] + s["shift"]
        out = {"mean": mean, "rstd": rstd}
        if s["total"] is not None:
            out["total"] = total.to(s["total"].dtype)
        if s["scale"] is None:
            return out | {"y": y.to(s["y"].dtype)}
        top = y.abs().amax(1)
        scale = torch.where(top > 0, top / E4M3_MAX, 1.0)
        return out | {"y": (y / scale[:, None]).to(torch.float8_e4m3fn), "scale": scale}
    if op == "norm_grad":
        dy, rstd = f(s["dy"]), s["rstd"][:, None]
        h = (f(s["total"]) - s["mean"][:, None]) * rstd
        a = dy * s["gain"]
        dx = rstd * (a - a.mean(1, keepdim=True) - h * (a * h).mean(1, keepdim=True))
        if s["dtotal"] is not None:
            dx = dx + f(s["dtotal"])
        return {"dx": dx.to(s["dx"].dtype), "dgain": (dy * h).sum(0), "dshift": dy.sum(0)}
    if op == "linear":
        y = (f(s["x"]) @ f(s["w"]).T) * s["x_scale"][:, None] * s["w_scale"]
        if s["bias"] is not None:
            y = y + s["bias"]
        y = _act(y, case["act"])
        if s["residual"] is not None:
            y = y + f(s["residual"])
        return {"y": y.to(s["y"].dtype)}
    if op == "beam":
        batch, beams, v, picks = case["batch"], case["beams"], case["v"], case["picks"]
        z = s["z"].double()
        top = z.amax(1, keepdim=True)
        z = z - (top + torch.log(torch.exp(z - top).sum(1, keepdim=True)))
        score = s["score"].double().reshape(-1, 1)
        ended = s["ended"].reshape(-1, 1)
        # an ended beam has one candidate, the end once more, at no cost
        stays = torch.where(torch.arange(v, device=z.device) == s["end"], 0.0, -math.inf)
        z = (torch.where(ended, stays, z) + score).reshape(batch, beams * v)
        best, at = torch.sort(z, dim=1, descending=True, stable=True)
        best, at = best[:, :picks], at[:, :picks]
        first = torch.arange(batch, device=z.device)[:, None] * beams
        parent, token = first + at // v, at % v
        go_on = parent[:, : min(picks, beams)].reshape(-1)
        live = torch.arange(case["positions"], device=z.device) < s["lengths"].long()[go_on][:, None]
        states = torch.where(live[None, :, :, None], s["states"][:, go_on], 0.0)
        return {"next_score": best.float(), "parent": parent.to(torch.int32), "token": token.to(torch.int32),
                "next_ended": ended[:, 0][parent] | (token == s["end"]), "states": states}
    ids = s["ids"].long()
    there = ids >= 0
    if op == "embed":
        row = torch.where(there, ids, 0)
        y = f(s["table"][row]) * s["factor"]
        if s["row_scale"] is not None:
            y = y * s["row_scale"][row][:, None]
        return {"y": torch.where(there[:, None], y, 0.0).to(s["y"].dtype)}
    sums = torch.zeros((case["v"] + 1, case["d"]), device=ids.device).index_add_(0, torch.where(there, ids, case["v"]), f(s["dy"]))
    return {"dtable": (sums[: case["v"]] * s["factor"]).to(s["dtable"].dtype)}


def _own(s):
    import paper_2008_03433_amd as tron

    case = s["case"]
    op = case["op"]
    if op == "norm":
        tron.tron_layer_norm(s["x"], s["y"], gain=s["gain"], shift=s["shift"], eps=EPS, residual=s["residual"], total=s["total"], scale=s["scale"], mean=s["mean"], rstd=s["rstd"])
        return {k: s[k] for k in ("mean", "rstd", "total", "y", "scale") if s[k] is not None}
    if op == "norm_grad":
        tron.tron_layer_norm_grad(s["total"], s["mean"], s["rstd"], s["dy"], s["dx"], gain=s["gain"], dtotal=s["dtotal"], dgain=s["dgain"], dshift=s["dshift"])
        return {"dx": s["dx"], "dgain": s["dgain"], "dshift": s["dshift"]}
    if op == "linear":
        tron.tron_linear(s["x"], s["w"], s["y"], bias=s["bias"], act=ACTS[case["act"]], residual=s["residual"], x_scale=s["x_scale"], w_scale=s["w_scale"])
        return {"y": s["y"]}
    if op == "beam":
        tron.tron_beam_select(s["z"], s["score"], s["next_score"], s["parent"], s["token"], ended=s["ended"], end=s["end"], next_ended=s["next_ended"])
        tron.tron_beam_reorder(s["parent"][:, : min(case["picks"], case["beams"])], s["states"], s["next_states"], lengths=s["lengths"])
        return {"next_score": s["next_score"], "parent": s["parent"], "token": s["token"], "next_ended": s["next_ended"], "states": s["next_states"]}
    if op == "embed":
        tron.tron_embed(s["ids"], s["table"], s["y"], scale=s["factor"], row_scale=s["row_scale"])
        return {"y": s["y"]}
    tron.tron_embed_grad(s["ids"], s["dy"], s["dtable"], scale=s["factor"])
    return {"dtable": s["dtable"]}


def run(state):
    return _own(state) if own else _plain(state)


def _distinct(case):
    """Expected number of different tokens among m: token t has probability ((t + 1) / v)^(1/3) - (t / v)^(1/3)."""
    p = np.diff(np.cbrt(np.arange(case["v"] + 1) / case["v"]))
    return float(np.sum(-np.expm1(case["m"] * (15 / 16) * np.log1p(-np.minimum(p, 1 - 1e-12)))))


def work(case):
    op = case["op"]
    if op in ("norm", "norm_grad"):
        m, d, b, extra = case["m"], case["d"], BYTES[case["type"]], 2 if case["residual"] else 0
        if op == "norm":  # x, and the residual and the sum; y, its scales, mean, rstd, gain, shift
            return {"bytes": m * d * (b * (1 + extra) + BYTES[case["out"]]) + m * (12 if case["out"] == "e4m3" else 8) + 8 * d, "flops": 8 * m * d}
        return {"bytes": m * d * b * (3 + extra // 2) + 8 * m + 12 * d, "flops": 13 * m * d}
    if op == "linear":
        m, n, k, o = case["m"], case["n"], case["k"], BYTES[case["out"]]
        return {"bytes": k * (m + n) + o * m * n * (1 + case["residual"]) + 4 * (m + n) + 4 * n * case["bias"], "flops": 2 * m * n * k}
    if op == "beam":
        rows, b = case["batch"] * case["beams"], BYTES[case["type"]]
        moved = case["layers"] * case["batch"] * min(case["picks"], case["beams"]) * case["positions"] * case["width"] * 2
        # about one beam in ten is not read: ended, or a first step's; states are on average three quarters full
        return {"bytes": int(rows * 0.9) * case["v"] * b + case["batch"] * case["picks"] * 13 + 9 * rows + int(1.5 * moved), "flops": 4 * rows * case["v"]}
    m, d, v, ids = case["m"], case["d"], case["v"], 8 if case["ids"] == "i64" else 4
    b, o = BYTES[case["type"]], BYTES[case["out"]]
    if op == "embed":
        return {"bytes": int(_distinct(case) * d * b) + m * d * o + m * ids, "flops": m * d}
    return {"bytes": int(m * 15 / 16) * d * b + v * d * o + m * ids, "flops": m * d + v * d}


# ------------------------------------------------------------------------------------------ the definitions in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    D = lambda name: s[name].double()  # noqa: E731
    if op == "norm":
        a = D("x")
        if s["residual"] is not None:
            a += D("residual")
        mean = a.sum(1) / case["d"]
        variance = a.sub(mean.unsqueeze(1)).pow_(2).sum(1) / case["d"]
        r = (variance + EPS).pow(-0.5)
        y = a.mul(r.unsqueeze(1)).sub_((mean * r).unsqueeze(1)).mul_(D("gain")).add_(D("shift"))
        out = {"mean": mean, "rstd": r, "y": y}
        if s["total"] is not None:
            out["total"] = a
        if s["scale"] is not None:
            largest = torch.linalg.vector_norm(y, math.inf, 1)
            out["scale"] = largest.div(E4M3_MAX).masked_fill(largest == 0, 1.0)
            out["y"] = y.div(out["scale"].unsqueeze(1))
        return out
    if op == "norm_grad":
        # h is the row with its mean and its own direction taken out: d h_j / d total_l = rstd (delta_jl - 1 / d - h_j h_l / d)
        h = D("total").sub_(D("mean").unsqueeze(1)).mul_(D("rstd").unsqueeze(1))
        a = D("dy").mul_(D("gain"))
        along = a.mul(h).sum(1, True).div_(case["d"])
        dx = a.sub(a.sum(1, True).div_(case["d"])).sub_(h.mul(along)).mul_(D("rstd").unsqueeze(1))
        return {"dx": dx if s["dtotal"] is None else dx.add_(D("dtotal")), "dgain": D("dy").mul_(h).sum(0), "dshift": D("dy").sum(0)}
    if op == "linear":
        y = torch.mm(D("x").mul_(D("x_scale").unsqueeze(1)), D("w").mul_(D("w_scale").unsqueeze(1)).t())
        if s["bias"] is not None:
            y.add_(D("bias"))
        y = {"none": lambda v: v, "relu": torch.relu, "gelu": torch.nn.functional.gelu, "silu": torch.nn.functional.silu}[case["act"]](y)
        return {"y": y if s["residual"] is None else y.add_(D("residual"))}
    if op == "beam":
        batch, beams, v, picks = case["batch"], case["beams"], case["v"], case["picks"]
        rows = torch.log_softmax(D("z"), 1).add_(D("score").reshape(-1, 1))
        ended = s["ended"].reshape(-1)
        rows[ended] = -math.inf
        rows[ended, s["end"]] = D("score").reshape(-1)[ended]
        # pick after pick, each the lowest index of what is largest; what is impossible ranks above what is taken
        left = rows.reshape(batch, beams * v).clamp_(min=-1e300)
        item, place = torch.arange(batch, device=left.device), torch.arange(beams * v, device=left.device)
        score, at = [], []
        for _ in range(picks):
            most = left.amax(1, keepdim=True)
            i = torch.where(left == most, place, beams * v).amin(1)
            score.append(most[:, 0])
            at.append(i)
            left[item, i] = -math.inf
        score, at = torch.stack(score, 1), torch.stack(at, 1)
        beam = torch.div(at, v, rounding_mode="floor")
        parent, token = beam + item[:, None] * beams, at - beam * v
        go_on = parent[:, : min(picks, beams)].reshape(-1)
        states = D("states").index_select(1, go_on)
        for i, n in enumerate(s["lengths"].index_select(0, go_on).tolist()):
            states[:, i, n:] = 0.0
        return {"next_score": score.masked_fill(score <= -1e300, -math.inf), "parent": parent.to(torch.int32), "token": token.to(torch.int32),
                "next_ended": (token == s["end"]).logical_or_(ended[parent]), "states": states}
    if op == "embed":
        table = s["table"].index_select(0, s["ids"].long().clamp(min=0)).double()
        if s["row_scale"] is not None:
            table.mul_(s["row_scale"].index_select(0, s["ids"].long().clamp(min=0)).double().unsqueeze(1))
        return {"y": table.mul_(s["factor"]).mul_(s["ids"].ge(0).double().unsqueeze(1))}
    # by sorted tokens: differences of running sums would lose digits, so the rows of each are added where they lie
    order = torch.argsort(s["ids"].long(), stable=True)
    order = order[s["ids"].long()[order] >= 0]
    out = torch.zeros((case["v"], case["d"]), dtype=torch.float64, device="cuda")
    out.index_put_((s["ids"].long()[order],), D("dy")[order], accumulate=True)
    return {"dtable": out.mul_(s["factor"])}
