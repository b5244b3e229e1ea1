"""Tokens in expert order, the products of groups of rows, and low-rank adapters, as cases that
can be timed and compared.

The operators, each a public entry point of ``paper_2602_07265_amd.xshare``:

* order: the (token, rank) pairs of a routing sorted by expert, ties by pair: each expert's first
  row, each pair's row and each row's pair.  A pair whose id is no expert's has no row;
* move: tokens copied to their pairs' rows (dispatch) and the rows back, weighted and summed per
  token (combine); in its training form also both gradients: of the tokens, rows and weights;
* products: y_p = W_e x_p for the rows p of each group e; in its training form also the gradients
  of x and of W;
* adapters: y_t = base_t + s_e B_e A_e x_t for each token t's adapter e (base_t alone for a token
  without one); in its training form also the gradients of x, of A and of B.

Shapes are those of this repository's benchmark (Mixtral-, Qwen-MoE- and DeepSeek-R1-shaped
layers) and sizes of no particular model.  Where ``own`` is false, ``run`` computes the same in
elementary torch operations in 32 bits.  Rows past the last group's keep what they held.
"""
import math

import torch

own = False


# ---------------------------------------------------------------------------- cases

def _order(T, E, k, share=1):
    """share: GPUs that the experts are spread over; the pairs whose expert lives elsewhere have
    id -1."""
    return dict(op="order", T=T, E=E, k=k, share=share)


def _move(T, E, k, d, dtype="bf16", grad=False, share=1):
    return dict(op="move", T=T, E=E, k=k, d=d, dtype=dtype, grad=grad, share=share)


def _products(T, E, k, N, K, grad=False, share=1):
    """The rows of T tokens' k pairs each, products with one [N, K] matrix an expert."""
    return dict(op="products", T=T, E=E, k=k, N=N, K=K, grad=grad, share=share)


def _adapters(T, L, r, n, d, grad=False, none=0.0):
    """none: the share of requests that have no adapter."""
    return dict(op="adapters", T=T, L=L, r=r, n=n, d=d, grad=grad, none=none)


def listed():
    return [
        # one token's pairs: a decode step's latency
        dict(_order(1, 256, 8), name="order_t1"),
        # a long prefill's, or a training step's
        dict(_order(16384, 128, 8), name="order_t16384"),
        # a decode batch to its experts' rows and back
        dict(_move(32, 256, 8, 7168), name="move_t32"),
        # a training step's, on one of two GPUs that share the experts
        dict(_move(4099, 128, 8, 2048, grad=True, share=2), name="move_train_t4099"),
        # a training step in fp32 whose rows end inside every vector and tile
        dict(_move(1023, 37, 3, 1367, "fp32", grad=True), name="move_train_fp32_t1023"),
        # one token's gate and up projections (held as one matrix): latency
        dict(_products(1, 128, 8, 1536, 2048), name="products_t1"),
        # a prefill chunk's down projection over few, large experts
        dict(_products(2048, 8, 2, 4096, 14336), name="products_t2048"),
        # a training step of many small experts' gate and up projections: the largest call
        dict(_products(4096, 128, 8, 1536, 2048, grad=True), name="products_train_t4096"),
        # a small training step whose sizes end inside their tiles, half of it on another GPU
        dict(_products(1000, 34, 2, 1368, 1000, grad=True, share=2),
             name="products_train_t1000_ragged"),
        # one user's decode step: latency
        dict(_adapters(1, 8, 16, 4096, 4096), name="adapters_t1"),
        # a decode batch of many users' adapters, some without one
        dict(_adapters(45, 20, 32, 2048, 7168, none=0.2), name="adapters_t45"),
        # a training step over a few adapters
        dict(_adapters(4000, 5, 16, 4096, 4096, grad=True), name="adapters_train_t4000"),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _cost(c):
    w = work(c)
    return max(w["bytes"], w["flops"] / 250)


def _draw_once(rng):
    op = rng.choice(["order"] + ["move"] * 3 + ["products"] * 4 + ["adapters"] * 4)
    T = _log_uniform(rng, 1, 16384)
    if op == "adapters":
        return _adapters(min(T, 8192), _log_uniform(rng, 1, 64), 8 * rng.randint(1, 16),
                         8 * _log_uniform(rng, 8, 1024), 8 * _log_uniform(rng, 8, 1024),
                         rng.random() < 0.5, rng.choice([0.0, 0.0, 0.3]))
    share = rng.choice([1, 1, 2, 4])
    E = share * max(1, _log_uniform(rng, 1, 384) // share)
    k = rng.randint(1, min(8, E))
    if op == "order":
        return _order(T, E, k, share)
    if op == "move":
        return _move(T, E, k, _log_uniform(rng, 64, 8192), rng.choice(["bf16", "bf16", "fp32"]),
                     rng.random() < 0.5, share)
    return _products(T, E, k, 8 * _log_uniform(rng, 8, 1792), 8 * _log_uniform(rng, 8, 1792),
                     rng.random() < 0.5, share)


def draw(rng):
    """One more case of the ranges that the listed ones stand for."""
    known = [{a: b for a, b in c.items() if a != "name"} for c in listed()]
    most = max(_cost(c) for c in listed())
    most_bytes = max(work(c)["bytes"] for c in listed())
    while True:
        c = _draw_once(rng)
        if c not in known and _cost(c) <= most and work(c)["bytes"] <= most_bytes:
            return c


def work(case):
    """Bytes and operations that one pass cannot do without."""
    c, T = case, case["T"]
    if c["op"] == "adapters":
        L, r, n, d = c["L"], c["r"], c["n"], c["d"]
        lora = (n + d) * r
        held = min(L, T)
        b = 2 * T * (d + 2 * n) + 2 * held * lora
        f = 2 * T * lora
        if c["grad"]:               # dy, the shared part of dx, dx; the factors' gradients
            b += 2 * T * (n + 2 * d) + 4 * L * lora
            f += 4 * T * lora
        return {"bytes": b + 4 * T, "flops": f}
    E, k = c["E"], c["k"]
    P = T * k / c["share"]
    if c["op"] == "order":
        return {"bytes": 12 * T * k + 4 * E // c["share"], "flops": 4 * T * k}
    if c["op"] == "move":
        size = 4 if c["dtype"] == "fp32" else 2
        d = c["d"]
        b = size * (2 * T * d + 2 * P * d) + 8 * T * k
        if c["grad"]:               # of the rows and weights from dy, of the tokens from rows'
            b += size * (2 * T * d + 3 * P * d) + 8 * T * k
        return {"bytes": b, "flops": 2 * P * d * (4 if c["grad"] else 1)}
    N, K = c["N"], c["K"]
    held = E // c["share"]
    active = held * (1 - (1 - k / E) ** T)
    b = 2 * (active * N * K + P * (N + K))
    f = 2 * P * N * K
    if c["grad"]:
        b += 2 * (active * N * K + P * (N + K)) + 4 * held * N * K
        f *= 3
    return {"bytes": b, "flops": f}


# ---------------------------------------------------------------------------- inputs

def _gen(seed, what):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 1000003 + what)
    return g


def _randn(g, *shape, dtype=torch.float32):
    return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32).to(dtype)


def _routing(g, c):
    """Each token's k experts, of a router that likes some more than others; -1: elsewhere."""
    h = 0.5 * _randn(g, 1, c["E"]) + _randn(g, c["T"], c["E"])
    ids = h.topk(c["k"], dim=1).indices
    held = c["E"] // c["share"]
    return torch.where(ids < held, ids, torch.full_like(ids, -1)).to(torch.int32), held


def _matrices(g, n, rows, cols, std):
    """[n, rows, cols] bf16 of N(0, std)."""
    w = torch.empty((n, rows, cols), dtype=torch.bfloat16, device="cuda")
    step = max(1, (1 << 28) // (rows * cols))
    for e in range(0, n, step):
        w[e:e + step] = std * _randn(g, min(step, n - e), rows, cols)
    return w


def _prepare_adapters(c, seed):
    g = _gen(seed, 14)
    T, L, r, n, d = (c[a] for a in ("T", "L", "r", "n", "d"))
    if c["grad"]:                                  # sequences of a few hundred tokens
        of = torch.arange(T, device="cuda") // 250
        ids = torch.randint(0, L, (int(of[-1]) + 1,), generator=g, device="cuda")
        off = torch.rand(ids.shape, generator=g, device="cuda") < c["none"]
        ids = ids.masked_fill(off, -1)[of]
    else:
        ids = torch.randint(0, L, (T,), generator=g, device="cuda")
        ids = ids.masked_fill(torch.rand((T,), generator=g, device="cuda") < c["none"], -1)
    bf = torch.bfloat16
    s = dict(case=c, ids=ids.to(torch.int32), x=_randn(g, T, d, dtype=bf),
             a=_matrices(g, L, r, d, d ** -0.5), b=_matrices(g, L, n, r, 0.05),
             scales=0.5 + torch.rand((L,), generator=g, device="cuda"),
             base=_randn(g, T, n, dtype=bf))
    if c["grad"]:
        s["dy"] = _randn(g, T, n, dtype=bf)
        s["base_dx"] = _randn(g, T, d, dtype=bf)
    return s


def prepare(case, seed):
    """A program's activations, routing, weights and the buffers that it keeps."""
    c = case
    if c["op"] == "adapters":
        return _prepare_adapters(c, seed)
    g = _gen(seed, 11)
    ids, held = _routing(g, c)
    s = dict(case=c, ids=ids, held=held)
    P = c["T"] * c["k"]
    if c["op"] == "order":
        return s
    if c["op"] == "move":
        dtype = torch.float32 if c["dtype"] == "fp32" else torch.bfloat16
        T, d = c["T"], c["d"]
        s["order"] = _plain_order(ids, held)
        s["w"] = torch.softmax(_randn(g, T, c["k"]), 1)
        s["x"] = _randn(g, T, d, dtype=dtype)
        s["moved"] = torch.zeros((P, d), dtype=dtype, device="cuda")
        s["results"] = _randn(g, P, d, dtype=dtype)            # the experts' outputs
        if c["grad"]:
            s["dy"] = _randn(g, T, d, dtype=dtype)
            s["dmoved"] = _randn(g, P, d, dtype=dtype)         # the gradient of their inputs
            s["dresults"] = torch.zeros((P, d), dtype=dtype, device="cuda")
        return s
    N, K, bf = c["N"], c["K"], torch.bfloat16
    s["offsets"] = _plain_order(ids, held)["offsets"]
    s["x"] = _randn(g, P, K, dtype=bf)
    s["w"] = _matrices(g, held, N, K, 0.02)
    s["y"] = torch.zeros((P, N), dtype=bf, device="cuda")
    if c["grad"]:
        s["dy"] = _randn(g, P, N, dtype=bf)
        s["dx"] = torch.zeros((P, K), dtype=bf, device="cuda")
    return s


# ---------------------------------------------------------------------------- plain forms

def _plain_order(ids, n):
    flat = ids.reshape(-1).long()
    key = torch.where((flat >= 0) & (flat < n), flat, torch.full_like(flat, n))
    pairs = key.sort(stable=True).indices
    at = torch.empty_like(pairs)
    at[pairs] = torch.arange(pairs.numel(), device=ids.device)
    upto = (key[None, :] < torch.arange(n + 1, device=ids.device)[:, None]).sum(1)
    dead = key == n
    return dict(offsets=upto.to(torch.int32),
                rows=at.masked_fill(dead, -1).view(ids.shape).to(torch.int32),
                pairs=pairs.masked_fill(dead[pairs], -1).to(torch.int32))


def _back(rows, at, w=None):
    """Each token's rows, times w, summed."""
    v = rows.float()[at.clamp(min=0).long()]
    if w is not None:
        v = v * w[:, :, None]
    return v.masked_fill(at[:, :, None] < 0, 0.0).sum(1)


def _plain_move(s):
    c, o = s["case"], s["order"]
    at, k = o["rows"], c["k"]
    live = (o["pairs"] >= 0).nonzero()[:, 0]
    pair = o["pairs"][live].long()
    s["moved"][live] = s["x"][pair // k]
    out = dict(moved=s["moved"], y=_back(s["results"], at, s["w"]).to(s["x"].dtype))
    if c["grad"]:
        dy = s["dy"].float()
        grad = dy[pair // k]
        s["dresults"][live] = (grad * s["w"].reshape(-1)[pair][:, None]).to(s["x"].dtype)
        dw = torch.zeros(c["T"] * k, device=dy.device)
        dw[pair] = (grad * s["results"].float()[live]).sum(1)
        out.update(dresults=s["dresults"], dw=dw.view(c["T"], k),
                   dx=_back(s["dmoved"], at).to(s["x"].dtype))
    return out


def _places(offsets, P):
    """For the rows up to the last group's end: which, their groups, their places in them; and
    the most rows of a group."""
    o = offsets.long()
    p = torch.arange(P, device=o.device)
    p = p[p < o[-1]]
    e = (o[None, 1:] <= p[:, None]).sum(1)
    return p, e, p - o[e], max(1, int((o[1:] - o[:-1]).max()))


def _padded(v, place, n):
    """Rows of v as [n, the most rows of a group, columns] in 32 bits, zeros past each group."""
    p, e, at, most = place
    out = torch.zeros((n, most, v.shape[1]), device=v.device)
    out[e, at] = v[p].float()
    return out


def _plain_products(s):
    c = s["case"]
    n = s["held"]
    place = _places(s["offsets"], s["x"].shape[0])
    p, e, at, _ = place
    x = _padded(s["x"], place, n)
    w = s["w"].float()
    s["y"][p] = (x @ w.transpose(1, 2))[e, at].to(torch.bfloat16)
    if not c["grad"]:
        return dict(y=s["y"])
    dy = _padded(s["dy"], place, n)
    s["dx"][p] = (dy @ w)[e, at].to(torch.bfloat16)
    return dict(y=s["y"], dx=s["dx"], dw=dy.transpose(1, 2) @ x)


def _plain_adapters(s):
    c, L = s["case"], s["case"]["L"]
    order = _plain_order(s["ids"][:, None], L)
    token = order["pairs"].clamp(min=0).long()
    place = _places(order["offsets"], c["T"])
    p, e, at, _ = place
    t = token[p]
    x = _padded(s["x"][token], place, L)
    a, b, scale = s["a"].float(), s["b"].float(), s["scales"][:, None, None]
    h = x @ a.transpose(1, 2)
    y = s["base"].float()
    y[t] += (scale * (h @ b.transpose(1, 2)))[e, at]
    out = dict(y=y.to(torch.bfloat16))
    if c["grad"]:
        dy = scale * _padded(s["dy"][token], place, L)
        dh = dy @ b
        dx = s["base_dx"].float()
        dx[t] += (dh @ a)[e, at]
        out.update(dx=dx.to(torch.bfloat16), da=dh.transpose(1, 2) @ x,
                   db=dy.transpose(1, 2) @ h)
    return out


# ---------------------------------------------------------------------------- one pass

def _run_own(s):
    from paper_2602_07265_amd import xshare as X
    c = s["case"]
    if c["op"] == "order":
        return X.expert_order(s["ids"], s["held"])
    if c["op"] == "move":
        o = s["order"]
        out = dict(moved=X.dispatch(s["x"], o, out=s["moved"]),
                   y=X.combine(s["results"], s["w"], o))
        if c["grad"]:
            g = X.combine_backward(s["dy"], s["results"], s["w"], o,
                                   out=dict(drows=s["dresults"]))
            out.update(dresults=g["drows"], dw=g["dw"], dx=X.dispatch_backward(s["dmoved"], o))
        return out
    if c["op"] == "products":
        out = dict(y=X.grouped_linear(s["x"], s["w"], s["offsets"], y=s["y"]))
        if c["grad"]:
            out["dx"] = X.grouped_linear_backward_x(s["dy"], s["w"], s["offsets"], out=s["dx"])
            out["dw"] = X.grouped_linear_backward_w(s["dy"], s["x"], s["offsets"])
        return out
    out = dict(y=X.adapters(s["x"], s["a"], s["b"], s["ids"], scales=s["scales"],
                            base=s["base"]))
    if c["grad"]:
        out.update(X.adapters_backward(s["dy"], s["x"], s["a"], s["b"], s["ids"],
                                       scales=s["scales"], base=s["base_dx"]))
    return out


def run(state):
    """One pass through an operator."""
    if own:
        return _run_own(state)
    op = state["case"]["op"]
    if op == "order":
        return _plain_order(state["ids"], state["held"])
    if op == "move":
        return _plain_move(state)
    return _plain_products(state) if op == "products" else _plain_adapters(state)


# ---------------------------------------------------------------------------- 64 bits

def _exact_move(s):
    x, w, res = s["x"].double(), s["w"].double(), s["results"].double()
    at, out = s["order"]["rows"].long(), {}
    moved, y = torch.zeros_like(res), torch.zeros_like(x)
    if s["case"]["grad"]:
        dy, dmoved = s["dy"].double(), s["dmoved"].double()
        dres, dx, dw = torch.zeros_like(res), torch.zeros_like(x), torch.zeros_like(w)
    for r in range(at.shape[1]):
        t = (at[:, r] >= 0).nonzero()[:, 0]
        p = at[t, r]
        moved[p] = x[t]
        y[t] += w[t, r, None] * res[p]
        if s["case"]["grad"]:
            dres[p] = w[t, r, None] * dy[t]
            dw[t, r] = (dy[t] * res[p]).sum(1)
            dx[t] += dmoved[p]
    out = dict(moved=moved, y=y)
    if s["case"]["grad"]:
        out.update(dresults=dres, dw=dw, dx=dx)
    return out


def _exact_products(s):
    x, grad = s["x"].double(), s["case"]["grad"]
    edge = s["offsets"].tolist()
    y = torch.zeros(s["y"].shape, dtype=torch.float64, device=x.device)
    if grad:
        dy = s["dy"].double()
        dx = torch.zeros_like(x)
        dw = torch.zeros(s["w"].shape, dtype=torch.float64, device=x.device)
    for e in range(len(edge) - 1):
        lo, hi = edge[e], edge[e + 1]
        if lo == hi:
            continue
        w = s["w"][e].double()
        y[lo:hi] = x[lo:hi] @ w.t()
        if grad:
            dx[lo:hi] = dy[lo:hi] @ w
            dw[e] = dy[lo:hi].t() @ x[lo:hi]
    return dict(y=y, dx=dx, dw=dw) if grad else dict(y=y)


def _exact_adapters(s):
    grad = s["case"]["grad"]
    y, x = s["base"].double(), s["x"].double()
    if grad:
        dx, dy = s["base_dx"].double(), s["dy"].double()
        da = torch.zeros(s["a"].shape, dtype=torch.float64, device=x.device)
        db = torch.zeros(s["b"].shape, dtype=torch.float64, device=x.device)
    for e in range(s["case"]["L"]):
        t = (s["ids"] == e).nonzero()[:, 0]
        if not t.numel():
            continue
        a, b, scale = s["a"][e].double(), s["b"][e].double(), s["scales"][e].double()
        h = x[t] @ a.t()
        y[t] += scale * (h @ b.t())
        if grad:
            dh = scale * (dy[t] @ b)
            dx[t] += dh @ a
            da[e] = dh.t() @ x[t]
            db[e] = scale * (dy[t].t() @ h)
    return dict(y=y, dx=dx, da=da, db=db) if grad else dict(y=y)


def _exact_order(s):
    ids = s["ids"].reshape(-1).tolist()
    by = [[] for _ in range(s["held"])]
    for i, e in enumerate(ids):
        if e >= 0:
            by[e].append(i)
    pairs = [i for one in by for i in one]
    rows = [-1] * len(ids)
    for p, i in enumerate(pairs):
        rows[i] = p
    edge = [0]
    for one in by:
        edge.append(edge[-1] + len(one))
    make = lambda v: torch.tensor(v, dtype=torch.int32, device=s["ids"].device)  # noqa: E731
    return dict(offsets=make(edge), rows=make(rows).view(s["ids"].shape),
                pairs=make(pairs + [-1] * (len(ids) - len(pairs))))


def exact(case, seed):
    """The outputs from the definition in 64 bits."""
    s = prepare(case, seed)
    if case["op"] == "order":
        return _exact_order(s)
    if case["op"] == "move":
        return _exact_move(s)
    return _exact_products(s) if case["op"] == "products" else _exact_adapters(s)
