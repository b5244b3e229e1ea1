"""The calls on groups of rows as a program uses them together: a training step of a MoE layer from the
router's logits to every gradient, adapters beside a block-scaled projection, both captured in
graphs and on streams of their own."""
import pytest
import torch

from helpers import DEV, say
from test_gpu_blocks import _weight

pytestmark = pytest.mark.gpu
T, E, K, D, F = 300, 12, 3, 264, 136


def _inputs(seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    rn = lambda *s: torch.randn(*s, generator=g, device=DEV)  # noqa: E731
    return dict(x=rn(T, D).to(torch.bfloat16), logits=rn(T, E), dy=rn(T, D).to(torch.bfloat16))


def _weights():
    g = torch.Generator(device=DEV).manual_seed(99)
    rn = lambda *s: (0.1 * torch.randn(*s, generator=g, device=DEV)).to(torch.bfloat16)  # noqa: E731
    return rn(E, 2 * F, D), rn(E, D, F)


def step(x, logits, dy, w13, w2):
    """y and the gradients of x, the logits and the weights; SwiGLU in torch, in fp32, rounded once."""
    from paper_2602_07265_amd import xshare as X
    r = X.gate(logits, K)
    o = X.expert_order(r["ids"], E)
    rows = X.dispatch(x, o)
    gu = X.grouped_linear(rows, w13, o["offsets"])
    a, b = gu.float().split(F, 1)
    s = torch.sigmoid(a)
    h = (a * s * b).to(torch.bfloat16)
    z = X.grouped_linear(h, w2, o["offsets"])
    y = X.combine(z, r["w"], o)
    back = X.combine_backward(dy, z, r["w"], o)
    dh = X.grouped_linear_backward_x(back["drows"], w2, o["offsets"])
    dw2 = X.grouped_linear_backward_w(back["drows"], h, o["offsets"])
    g = dh.float()
    dgu = torch.cat([g * b * (s + a * s * (1 - s)), g * a * s], 1).to(torch.bfloat16)
    drows = X.grouped_linear_backward_x(dgu, w13, o["offsets"])
    dw13 = X.grouped_linear_backward_w(dgu, rows, o["offsets"])
    dx = X.dispatch_backward(drows, o)
    dlogits = X.gate_backward(logits, r["ids"], back["dw"])
    return dict(y=y, dx=dx, dlogits=dlogits, dw13=dw13, dw2=dw2, ids=r["ids"], dw=back["dw"])


def _reference(x, logits, dy, w13, w2, ids):
    """float64 autograd of the layer with these ids; and, for each output, its terms' magnitudes: the
    same products of absolute values (silu(a) and its slope are at most |a| and 1.1)."""
    x, logits, w13, w2 = (t.double().requires_grad_(True) for t in (x, logits, w13, w2))
    dy = dy.double()
    w = torch.softmax(logits, 1).gather(1, ids.long())
    w = w / w.sum(1, keepdim=True)
    y = torch.zeros_like(dy)
    mag = {n: torch.zeros(s, dtype=torch.float64, device=DEV)
           for n, s in (("y", dy.shape), ("dx", dy.shape), ("dw13", w13.shape), ("dw2", w2.shape))}
    mag["dw"] = torch.zeros(ids.shape, dtype=torch.float64, device=DEV)
    for e in range(E):
        t, r = (ids == e).nonzero(as_tuple=True)
        if not t.numel():
            continue
        gu = x[t] @ w13[e].t()
        a, b = gu.split(F, 1)
        z = (torch.nn.functional.silu(a) * b) @ w2[e].t()
        y = y.index_add(0, t, w[t, r, None] * z)
        with torch.no_grad():
            A = x[t].abs() @ w13[e].abs().t()
            ga, gb = A.split(F, 1)
            Z = (ga * gb) @ w2[e].abs().t()
            mag["y"].index_add_(0, t, w[t, r, None] * Z)
            mag["dw"][t, r] = (dy[t].abs() * Z).sum(1)
            R = w[t, r, None] * dy[t].abs()
            H = R @ w2[e].abs()
            G = torch.cat([1.1 * H * gb, H * ga], 1)
            mag["dw2"][e] = R.t().contiguous() @ (ga * gb)
            mag["dw13"][e] = G.t().contiguous() @ x[t].abs()
            mag["dx"].index_add_(0, t, G @ w13[e].abs())
    grads = torch.autograd.grad((y * dy).sum(), (x, logits, w13, w2))
    return dict(zip(("y", "dx", "dlogits", "dw13", "dw2"), (y.detach(), *grads))), mag


def test_a_training_step():
    say("run case: a training step of a MoE layer")
    c, w = _inputs(0), _weights()
    got = step(**c, w13=w[0], w2=w[1])
    torch.cuda.synchronize()
    ref, mag = _reference(**c, w13=w[0], w2=w[1], ids=got["ids"])
    # Roundings to bf16 on the way, each at most 2^-8 of what the next step takes: y: gate, up (1.1 by
    # silu's slope), hidden, rows, y; dx: w dy, dh, then gate, up and dh again in dgate, dup (silu's
    # second derivative is below 0.5, so 1.1 and 0.5 for the gate), d(gate, up), rows, dx; the
    # weights': those of their factors.  Sums in fp32 add less than a hundredth of a rounding.
    steps = dict(y=5.2, dx=8.0, dw13=7.0, dw2=4.2)
    for name, n in steps.items():
        err = (got[name].double() - ref[name]).abs()
        assert (err <= n * 2.0 ** -8 * mag[name] + 1e-30).all(), \
            (name, float((err / mag[name].clamp(min=1e-30)).max()) * 2 ** 8)
        # and by far nearer on the whole: no part is missing
        assert float(err.norm() / ref[name].norm()) <= 0.02, name
    # the logits' gradient from dw's: off by at most the weights' Jacobian of dw's errors
    ids = got["ids"].long()
    p = torch.softmax(c["logits"].double(), 1).gather(1, ids)
    p = p / p.sum(1, keepdim=True)
    tol = 4.2 * 2.0 ** -8 * mag["dw"]
    full = torch.zeros(T, E, dtype=torch.float64, device=DEV)
    full.scatter_(1, ids, p * (tol + (p * tol).sum(1, keepdim=True)))
    assert ((got["dlogits"].double() - ref["dlogits"]).abs() <= full * 1.001 + 1e-6).all()


def test_a_training_step_in_a_graph():
    w = _weights()
    inputs = [_inputs(s) for s in range(3)]
    held = {name: v.clone() for name, v in inputs[0].items()}
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(**held, w13=w[0], w2=w[1])
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    say("run case: a training step in a graph: capture")
    with torch.cuda.graph(graph):
        out = step(**held, w13=w[0], w2=w[1])
    for rep in range(3):
        for i, c in enumerate(inputs):
            say(f"run case: replay {rep} input {i}")
            for name, v in c.items():
                held[name].copy_(v)
            graph.replay()
            torch.cuda.synchronize()
            ref = step(**c, w13=w[0], w2=w[1])
            torch.cuda.synchronize()
            for name in out:
                assert torch.equal(out[name], ref[name]), (name, rep, i)


def _tuned(X, x, dy, ids, q, s, a, b, scales):
    """A frozen block-scaled projection with adapters, and the way back."""
    y = X.block_linear(x, q, s)
    y = X.adapters(x, a, b, ids, scales=scales, base=y, out=y)
    dx = X.block_linear(dy, q.t().contiguous(), s.t().contiguous())
    g = X.adapters_backward(dy, x, a, b, ids, scales=scales, base=dx, out=dict(dx=dx))
    return dict(y=y, **g)


def _tuning(rows, seed=3):
    import numpy as np
    g = torch.Generator(device=DEV).manual_seed(seed)
    n, d, r, L = 272, 400, 24, 4
    rn = lambda *s: torch.randn(*s, generator=g, device=DEV).to(torch.bfloat16)  # noqa: E731
    q, s = (t.to(DEV) for t in _weight(np.random.default_rng(seed), n, d))
    ids = torch.randint(-1, L, (rows,), generator=g, device=DEV).to(torch.int32)
    return dict(x=rn(rows, d), dy=rn(rows, n), ids=ids, q=q, s=s, a=rn(L, r, d), b=rn(L, n, r),
                scales=torch.rand(L, generator=g, device=DEV))


@pytest.mark.parametrize("rows", [7, 250])
def test_adapters_beside_a_block_projection(rows):
    from paper_2602_07265_amd import xshare as X
    say(f"run case: adapters beside block_linear, {rows} tokens")
    c = _tuning(rows)
    got = _tuned(X, **c)
    torch.cuda.synchronize()
    base = X.block_linear(c["x"], c["q"], c["s"])
    dbase = X.block_linear(c["dy"], c["q"].t().contiguous(), c["s"].t().contiguous())
    want = X.adapters(c["x"], c["a"], c["b"], c["ids"], scales=c["scales"], base=base)
    g = X.adapters_backward(c["dy"], c["x"], c["a"], c["b"], c["ids"], scales=c["scales"], base=dbase)
    torch.cuda.synchronize()
    assert torch.equal(got["y"], want) and not torch.equal(want, base)
    for name in ("dx", "da", "db"):
        assert torch.equal(got[name], g[name]), name
    off = c["ids"] < 0
    assert torch.equal(got["y"][off], base[off]) and torch.equal(got["dx"][off], dbase[off])


def test_adapters_in_two_graphs_of_one_workspace():
    """Decode steps and training steps captured with the same workspace, replayed in turn."""
    from paper_2602_07265_amd import xshare as X
    few, many = _tuning(9), _tuning(300, 5)
    need = X.adapters_workspace_bytes(300, 4, 24, 272, 400, True)
    ws = torch.empty(need, dtype=torch.uint8, device=DEV)

    def run(c):
        args = (c["x"], c["a"], c["b"], c["ids"])
        y = X.adapters(*args, scales=c["scales"], workspace=ws)
        return dict(y=y, **X.adapters_backward(c["dy"], *args, scales=c["scales"], workspace=ws))

    ref = [{n: v.clone() for n, v in run(c).items()} for c in (few, many)]
    torch.cuda.synchronize()
    graphs, outs = [], []
    for c in (few, many):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            outs.append(run(c))
    for rep in range(3):
        say(f"run case: two graphs of one workspace, replay {rep}")
        for i in (0, 1):
            for v in outs[i].values():
                v.zero_()
            graphs[i].replay()
            torch.cuda.synchronize()
            for name, v in outs[i].items():
                assert torch.equal(v, ref[i][name]), (name, rep, i)


def _stream_of_memory(t):
    for seg in torch.cuda.memory_snapshot():
        if seg["address"] <= t.data_ptr() < seg["address"] + seg["total_size"]:
            return seg["stream"]
    raise AssertionError("not the caching allocator's memory")


def test_calls_on_a_stream_that_is_not_current():
    from paper_2602_07265_amd import xshare as X
    c, (w13, w2), t = _inputs(0), _weights(), _tuning(250)
    r = X.gate(c["logits"], K)
    ids = r["ids"].repeat(20, 1)                       # enough pairs for two launches
    o = X.expert_order(r["ids"], E)
    rows = X.dispatch(c["x"], o)
    gu = X.grouped_linear(rows, w13, o["offsets"])
    ad = (t["x"], t["a"], t["b"], t["ids"])
    calls = {
        "order": lambda **kw: X.expert_order(ids, E, **kw)["rows"],
        "dispatch": lambda **kw: X.dispatch(c["x"], o, **kw),
        "dispatch_backward": lambda **kw: X.dispatch_backward(rows, o, **kw),
        "combine": lambda **kw: X.combine(rows, r["w"], o, **kw),
        "combine_backward": lambda **kw: X.combine_backward(c["dy"], rows, r["w"], o, **kw)["drows"],
        "linear": lambda **kw: X.grouped_linear(rows, w13, o["offsets"], **kw),
        "backward_x": lambda **kw: X.grouped_linear_backward_x(gu, w13, o["offsets"], **kw),
        "backward_w": lambda **kw: X.grouped_linear_backward_w(gu, rows, o["offsets"], **kw),
        "adapters": lambda **kw: X.adapters(*ad, **kw),
        "adapters_backward": lambda **kw: X.adapters_backward(t["dy"], *ad, **kw)["da"],
    }
    ref = {name: call().clone() for name, call in calls.items()}
    torch.cuda.synchronize()
    side = [torch.cuda.Stream(), torch.cuda.Stream()]
    for name, call in calls.items():
        say(f"run case: {name} on another stream")
        got = []
        for rep in range(6):
            got.append(call(stream=side[rep % 2]))
            assert _stream_of_memory(got[-1]) == side[rep % 2].cuda_stream, name
            for size in (1 << 12, 1 << 16, 1 << 19, 1 << 21, 1 << 26):   # what the call has dropped
                torch.full((size,), 0xFF, dtype=torch.uint8, device=DEV)
        torch.cuda.synchronize()
        for v in got:
            assert torch.equal(v, ref[name]), name


def test_rows_side_by_side_in_one_buffer():
    """Inputs and outputs that are columns of one buffer, their rows as far apart."""
    from paper_2602_07265_amd import xshare as X
    v = _inputs(3)
    w13, _ = _weights()
    o = X.expert_order(X.gate(v["logits"], K)["ids"], E)
    want = X.grouped_linear(X.dispatch(v["x"], o), w13, o["offsets"])
    buf = torch.zeros(T * K, D + 2 * F, device=DEV, dtype=torch.bfloat16)
    X.dispatch(v["x"], o, out=buf[:, :D])
    y = X.grouped_linear(buf[:, :D], w13, o["offsets"], y=buf[:, D:])
    assert torch.equal(y, want) and torch.equal(buf[:, D:], want)


def test_a_residual_as_base_is_not_the_output():
    from paper_2602_07265_amd import xshare as X
    x = _inputs(4)["x"]
    g = torch.Generator(device=DEV).manual_seed(5)
    a = torch.randn(4, 16, D, generator=g, device=DEV).to(torch.bfloat16)
    b = torch.randn(4, D, 16, generator=g, device=DEV).to(torch.bfloat16)
    ids = torch.randint(-1, 4, (T,), generator=g, device=DEV, dtype=torch.int32)
    want = X.adapters(x, a, b, ids, base=x.clone())
    assert torch.equal(X.adapters(x, a, b, ids, base=x), want)
    for n in (T, 5):
        with pytest.raises(X.XShareError):
            X.adapters(x[:n], a, b, ids[:n], base=x[:n], out=x[:n])
        with pytest.raises(X.XShareError):
            X.adapters_backward(x[:n], want[:n], a, b, ids[:n], base=x[:n], out=dict(dx=x[:n]))
