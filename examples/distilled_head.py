#!/usr/bin/env python3
"""Trains a softmax head against a teacher's top logits by truncated Newton, on synthetic hidden states, and answers single tokens with
the trained head in 8 bits.

    python examples/distilled_head.py [--rows M] [--features D] [--classes V] [--top K] [--steps N]

One evaluation is SoftmaxHead.fun_grad (norm once; logits, loss and gradient), one product of the inner conjugate-gradient solve is
SoftmaxHead.hv; serving takes the norm with an output in 8 bits and the matrix product of 8-bit operands."""
import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch  # noqa: E402

import paper_2008_03433_amd as tron  # noqa: E402


def newton_step(head, C, W, G, most_products=20, xi=0.1):
    """The conjugate-gradient solution of H s = -G to |r| <= xi |G|."""
    s, r = torch.zeros_like(W), -G
    p, Hp = r.clone(), torch.empty_like(W)
    rr, target = float((r * r).sum()), xi * xi * float((G * G).sum())
    products = 0
    while products < most_products and rr > target:
        head.hv(C, p, Hp)
        products += 1
        alpha = rr / float((p * Hp).sum())
        s += alpha * p
        r -= alpha * Hp
        rr, before = float((r * r).sum()), rr
        p = r + (rr / before) * p
    return s, products


def train(head, classes, C, steps, say=print):
    W = torch.zeros((classes, head.d), device=head.X.device)
    G = torch.empty_like(W)
    f = head.fun_grad(C, W, G)
    history = [f]
    for step in range(steps):
        s, products = newton_step(head, C, W, G)
        scale = 1.0
        while True:   # halve the step until f falls
            trial = W + scale * s
            f_trial = head.fun_grad(C, trial)
            if f_trial < f or scale < 1e-3:
                break
            scale *= 0.5
        if f_trial >= f:
            break
        W = trial
        f = head.fun_grad(C, W, G)
        history.append(f)
        say(f"step {step + 1}: f = {f:.6g}, |g| = {float(G.norm()):.4g}, {products} products")
    return W, history


def answer(hidden, residual, gain, W8, w_scale):
    """Logits of some tokens from weights in 8 bits, which were laid out once."""
    m, d = hidden.shape
    x, scale = torch.empty((m, d), dtype=torch.float8_e4m3fn, device=hidden.device), torch.empty(m, device=hidden.device)
    tron.tron_rms_norm(hidden, x, gain=gain, residual=residual, scale=scale)
    z = torch.empty((m, W8.shape[0]), device=hidden.device)
    tron.tron_linear(x, W8, z, x_scale=scale, w_scale=w_scale)
    return z


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--rows", type=int, default=4000)
    ap.add_argument("--features", type=int, default=256)
    ap.add_argument("--classes", type=int, default=1000)
    ap.add_argument("--top", type=int, default=16)
    ap.add_argument("--steps", type=int, default=5)
    a = ap.parse_args(argv)
    g = torch.Generator(device="cuda").manual_seed(1)
    hidden = torch.randn((a.rows, a.features), generator=g, device="cuda").bfloat16()
    residual = torch.randn((a.rows, a.features), generator=g, device="cuda").bfloat16()
    gain = 1.0 + 0.1 * torch.randn(a.features, generator=g, device="cuda")
    planted = torch.randn((a.classes, a.features), generator=g, device="cuda") * (3.0 * a.features ** -0.5)
    # a teacher's logits, of which it gives the largest
    s = hidden.float() + residual.float()
    features = s * (s.square().mean(1, keepdim=True) + 1e-6).rsqrt() * gain
    t, ids = (features @ planted.T).topk(a.top, 1)

    head = tron.SoftmaxHead(hidden, ids, t, gain=gain, residual=residual)
    W, history = train(head, a.classes, C=1.0, steps=a.steps)
    w_scale = W.abs().amax(1).clamp(min=1e-30) / 448.0
    W8 = (W / w_scale[:, None]).to(torch.float8_e4m3fn)
    agree = sum(int(answer(hidden[i:i + 1], residual[i:i + 1], gain, W8, w_scale).argmax(1)) == int(ids[i, 0]) for i in range(64))
    print(f"f: {history[0]:.6g} -> {history[-1]:.6g} in {len(history) - 1} steps; {agree} of 64 tokens have the teacher's first class")
    return history, agree


if __name__ == "__main__":
    main()
