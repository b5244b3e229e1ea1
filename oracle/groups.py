"""Tokens in expert order and back, products of groups of rows, low-rank adapters, and their
gradients, from their definitions in 64 bits (torch, on the device of the arguments).  Each product
also comes with the sum of its terms' magnitudes, from which the tests derive what a sum in 32 bits
may be off by."""
import torch


def expert_order(ids, n):
    """(offsets [n + 1], rows [T, k], pairs [T k]) of ids [T, k] as lists of Python integers."""
    flat = [int(i) for row in ids.tolist() for i in row]
    by = [[p for p, e in enumerate(flat) if e == want] for want in range(n)]
    pairs = [p for one in by for p in one]
    offsets = [0]
    for one in by:
        offsets.append(offsets[-1] + len(one))
    rows = [-1] * len(flat)
    for row, p in enumerate(pairs):
        rows[p] = row
    return offsets, rows, pairs + [-1] * (len(flat) - len(pairs))


def dispatch(x, rows, out):
    """out (float64 [T k, d]) with out[rows[t, r]] = x[t]."""
    for t in range(rows.shape[0]):
        for row in rows[t].tolist():
            if row >= 0:
                out[row] = x[t].double()
    return out


def combine(src, w, rows):
    """(y, magnitudes), [T, d]; w None: every weight 1."""
    y = torch.zeros(rows.shape[0], src.shape[1], dtype=torch.float64, device=src.device)
    m = torch.zeros_like(y)
    for t in range(rows.shape[0]):
        for r, row in enumerate(rows[t].tolist()):
            if row >= 0:
                v = src[row].double() * (1.0 if w is None else w[t, r].double())
                y[t] += v
                m[t] += v.abs()
    return y, m


def combine_backward(dy, src, w, rows, dsrc):
    """(dsrc, dw, dw's magnitudes); dsrc (float64 [T k, d]) is written where a pair has a row."""
    dw = torch.zeros(w.shape, dtype=torch.float64, device=dy.device)
    m = torch.zeros_like(dw)
    for t in range(rows.shape[0]):
        for r, row in enumerate(rows[t].tolist()):
            if row >= 0:
                dsrc[row] = w[t, r].double() * dy[t].double()
                v = dy[t].double() * src[row].double()
                dw[t, r] = v.sum()
                m[t, r] = v.abs().sum()
    return dsrc, dw, m


def groups(offsets):
    edge = [int(i) for i in offsets]
    return [(e, edge[e], edge[e + 1]) for e in range(len(edge) - 1) if edge[e + 1] > edge[e]]


def grouped_linear(x, w, offsets, y):
    """y (float64 [P, n]) with the groups' rows written, and their magnitudes."""
    m = torch.zeros_like(y)
    for e, lo, hi in groups(offsets):
        a, b = x[lo:hi].double(), w[e].double().t().contiguous()
        y[lo:hi] = a @ b
        m[lo:hi] = a.abs() @ b.abs()
    return y, m


def grouped_linear_backward_x(dy, w, offsets, dx):
    m = torch.zeros_like(dx)
    for e, lo, hi in groups(offsets):
        a, b = dy[lo:hi].double(), w[e].double()
        dx[lo:hi] = a @ b
        m[lo:hi] = a.abs() @ b.abs()
    return dx, m


def grouped_linear_backward_w(dy, x, offsets):
    n = len(offsets) - 1
    dw = torch.zeros(n, dy.shape[1], x.shape[1], dtype=torch.float64, device=x.device)
    m = torch.zeros_like(dw)
    for e, lo, hi in groups(offsets):
        a, b = dy[lo:hi].double().t().contiguous(), x[lo:hi].double()
        dw[e] = a @ b
        m[e] = a.abs() @ b.abs()
    return dw, m


def adapters(x, a, b, ids, scales, base):
    """(y, magnitudes of base + the products' terms)."""
    n = b.shape[1]
    y = torch.zeros(x.shape[0], n, dtype=torch.float64, device=x.device) if base is None \
        else base.double().clone()
    m = y.abs()
    for e in range(a.shape[0]):
        t = (ids == e).nonzero()[:, 0]
        if t.numel():
            s = 1.0 if scales is None else scales[e].double()
            at, bt = a[e].double().t().contiguous(), b[e].double().t().contiguous()
            y[t] += s * (x[t].double() @ at @ bt)
            m[t] += abs(s) * (x[t].double().abs() @ at.abs() @ bt.abs())
    return y, m


def adapters_backward(dy, x, a, b, ids, scales, base):
    """dict(dx, da, db) and dict of their magnitudes."""
    out = dict(dx=torch.zeros(x.shape, dtype=torch.float64, device=x.device) if base is None
               else base.double().clone(),
               da=torch.zeros(a.shape, dtype=torch.float64, device=x.device),
               db=torch.zeros(b.shape, dtype=torch.float64, device=x.device))
    mag = {name: v.abs() for name, v in out.items()}
    for e in range(a.shape[0]):
        t = (ids == e).nonzero()[:, 0]
        if not t.numel():
            continue
        s = 1.0 if scales is None else scales[e].double()
        for to, f in ((out, lambda v: v), (mag, torch.abs)):
            xe, g, ae, be = f(x[t].double()), f(dy[t].double()), f(a[e].double()), f(b[e].double())
            k = s if to is out else abs(s)
            dh = k * (g @ be)
            to["dx"][t] += dh @ ae
            to["da"][e] = dh.t().contiguous() @ xe
            to["db"][e] = k * (g.t().contiguous() @ (xe @ ae.t().contiguous()))
    return out, mag
