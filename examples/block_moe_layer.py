"""A mixture-of-experts layer whose weights are E4M3 codes with a scale for each 128 x 128 block and
whose router scores by sigmoid, with a balance bias and groups of experts.

    python examples/block_moe_layer.py [--tokens 32] [--experts 64] [--budget 24] [--steps 20]

It quantizes random weights once (block_quantize), then runs the layer three ways: with the
router's own choice (router_logits, gate, block_experts), with the batch-level set selection in
its place (route, block_experts), which reads fewer experts' weights, and its shared expert
as plain products (block_linear) beside the one-expert form of block_experts.  Last it trains a
router to a teacher's weights with gate_backward.  It prints times, how many experts were read and
how far the results are from the layer in 32-bit torch operations.
"""
import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2602_07265_amd import xshare as X  # noqa: E402

GATE = dict(score="sigmoid", n_groups=8, top_groups=4, group_score="top2", scale=2.5)


def quantized(n, rows, cols, gen):
    """n random matrices as (codes [n, rows, cols], scales of their 128 x 128 blocks)."""
    q, s = [], []
    for _ in range(n):
        w = torch.randn((rows, cols), generator=gen, device="cuda") * 0.02
        c, f = X.block_quantize(w.to(torch.bfloat16), 128)
        q.append(c)
        s.append(f)
    return torch.stack(q), torch.stack(s)


def plain_weight(q, s):
    s = s.repeat_interleave(128, 0)[:q.shape[0]].repeat_interleave(128, 1)[:, :q.shape[1]]
    return q.view(torch.float8_e4m3fn).float() * s


def plain_experts(x, ids, w, mats):
    """The routed experts without quantized activations, one expert after the other."""
    y = torch.zeros_like(x, dtype=torch.float32)
    for e in ids.unique().tolist():
        t, r = (ids == e).nonzero(as_tuple=True)
        w1, w3, w2 = (plain_weight(q[e], s[e]) for q, s in mats)
        v = x[t].float()
        h = torch.nn.functional.silu(v @ w1.t()) * (v @ w3.t())
        y.index_add_(0, t, w[t, r, None] * (h @ w2.t()))
    return y


def timed(steps, call):
    out = call()
    torch.cuda.synchronize()
    t = time.perf_counter()
    for _ in range(steps):
        out = call()
    torch.cuda.synchronize()
    return out, (time.perf_counter() - t) / steps * 1e6


def off(y, ref):
    return float((y.float() - ref).norm() / ref.norm())


def experts(x, ids, w, mats):
    return X.block_experts(x, ids, w, *(q for q, _ in mats), *(s for _, s in mats))


def train_router(x, k, gen, steps=60):
    """A router learns the weights that a teacher gives the experts of its choice."""
    T, d = x.shape
    teacher = torch.randn((d, 64), generator=gen, device="cuda") / d ** 0.5
    wg = 0.1 * torch.randn((d, 64), generator=gen, device="cuda") / d ** 0.5
    want = torch.sigmoid(x.float() @ teacher)
    first = last = 0.0
    for step in range(steps):
        h = x.float() @ wg
        g = X.gate(h, k, score="sigmoid", renormalize=False)
        miss = g["w"] - want.gather(1, g["ids"].long())
        dh = X.gate_backward(h, g["ids"], 2 * miss / T, score="sigmoid", renormalize=False)
        wg -= 0.5 * (x.float().t() @ dh)
        last = float(miss.square().mean())
        first = first or last
    return first, last


def main():
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--tokens", type=int, default=32)
    p.add_argument("--experts", type=int, default=64)
    p.add_argument("--top-k", type=int, default=8)
    p.add_argument("--budget", type=int, default=24, help="experts of the batch-level selection")
    p.add_argument("--hidden", type=int, default=2048)
    p.add_argument("--ffn", type=int, default=768)
    p.add_argument("--steps", type=int, default=20)
    a = p.parse_args()
    gen = torch.Generator(device="cuda")
    gen.manual_seed(0)
    N, d, f, k = a.experts, a.hidden, a.ffn, a.top_k
    mats = [quantized(N, f, d, gen), quantized(N, f, d, gen), quantized(N, d, f, gen)]
    shared = [quantized(1, f, d, gen), quantized(1, f, d, gen), quantized(1, d, f, gen)]
    wg = (torch.randn((N, d), generator=gen, device="cuda") * 1.5 / d ** 0.5).to(torch.bfloat16)
    bias = 0.05 * torch.randn(N, generator=gen, device="cuda")
    x = torch.randn((a.tokens, d), generator=gen, device="cuda").to(torch.bfloat16)

    def routed():
        g = X.gate(X.router_logits(x, wg), k, bias=bias, **GATE)
        return experts(x, g["ids"], g["w"], mats), g["ids"], g["w"]

    def selected():
        r = X.route(X.router_logits(x, wg), k, 1, a.budget)
        return experts(x, r["ids"], r["w"], mats), r["ids"], r["w"]

    for name, call in (("router's choice", routed), ("batch-level selection", selected)):
        (y, ids, w), us = timed(a.steps, call)
        print(f"{name}: {us:.1f} us, {ids.unique().numel()} of {N} experts read, off by "
              f"{off(y, plain_experts(x, ids, w, mats)):.2e}", flush=True)

    one, ones = torch.zeros((a.tokens, 1), dtype=torch.int32, device="cuda"), \
        torch.ones((a.tokens, 1), device="cuda")

    def products():
        up = X.block_linear(x, *(t[0] for t in shared[0])).float()
        h = torch.nn.functional.silu(up) * X.block_linear(x, *(t[0] for t in shared[1])).float()
        return X.block_linear(h.to(torch.bfloat16), *(t[0] for t in shared[2]))

    ref = plain_experts(x, one, ones, shared)
    for name, call in (("shared expert as products", products),
                       ("shared expert as one expert", lambda: experts(x, one, ones, shared))):
        y, us = timed(a.steps, call)
        print(f"{name}: {us:.1f} us, off by {off(y, ref):.2e}", flush=True)

    first, last = train_router(x, k, gen)
    print(f"router training: miss {first:.4f} -> {last:.4f}", flush=True)


if __name__ == "__main__":
    main()
