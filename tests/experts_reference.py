"""Plain 64-bit implementations of the experts' operators, and how far an evaluation in 32 bits may be from them.

U = 2^-24.  A sum of c products in 32 bits is off by at most (c + 16) 2 U times the sum of their absolute values: c roundings of U each, twice that because
the matrix cores may cut what they add up instead of rounding it, 16 for the joining of parts.  s(g) = 1/(1 + exp(-g)) is off by (|g| + 8) U of itself (the
exponent's product with log2 e, the exponential, the addition, the division); what follows is bounded step by step.  A result in 16 bits has half a
unit of its own on top; results below the smallest normal number may come back as 0.
"""
import numpy as np
import torch

from rows_reference import HALF_UNIT, U, close, rounded  # noqa: F401  (used by the tests beside what is here)

TINY = 1e-36


def choices(n, k, experts, gen, dropped=0.1):
    """(n, k) int32 on the CPU: experts of uneven popularity, some without any, some choices none."""
    popularity = torch.rand(experts, generator=gen) ** 3
    if experts > 2:
        popularity[gen.initial_seed() % experts] = 0.0
    popularity += 1e-9
    idx = torch.multinomial(popularity.expand(n, experts), k, replacement=True, generator=gen).to(torch.int32) if n else torch.empty(0, k, dtype=torch.int32)
    idx[torch.rand(n, k, generator=gen) < dropped] = -1
    return idx


def order(idx, experts):
    """(start, order, place) by plain loops."""
    n, k = idx.shape
    flat = idx.reshape(-1).tolist()
    rows = [[] for _ in range(experts)]
    for s, e in enumerate(flat):
        if 0 <= e < experts:
            rows[e].append(s)
    start = np.concatenate([[0], np.cumsum([len(r) for r in rows])]).astype(np.int64)
    listed = [s for r in rows for s in r]
    order = np.full(n * k, -1, np.int32)
    order[:len(listed)] = listed
    place = np.full(n * k, -1, np.int32)
    place[listed] = np.arange(len(listed))
    return torch.from_numpy(start), torch.from_numpy(order), torch.from_numpy(place.reshape(n, k))


def source(X, order, k):
    """The rows of X that a product takes, for the rows that have one."""
    return X if order is None else X[(order.long().clamp(min=0) // k)]


def experts_of(start, rows):
    """The expert of each row, -1 for those of none."""
    e = torch.full((rows,), -1, dtype=torch.long)
    for i in range(len(start) - 1):
        e[start[i]:start[i + 1]] = i
    return e


def sums(rows, W, start):
    """z and the bound of its 32-bit evaluation, all CPU float64; rows of no expert NaN."""
    z = torch.full((rows.shape[0], W.shape[1]), np.nan, dtype=torch.float64)
    tol = torch.zeros_like(z)
    for e in range(W.shape[0]):
        a, b = int(start[e]), int(start[e + 1])
        z[a:b] = rows[a:b] @ W[e].t()
        tol[a:b] = (rows[a:b].abs() @ W[e].abs().t()) * 2 * U * (W.shape[2] + 16) + TINY
    return z, tol


def gate(z, tol):
    """(h, its bound)"""
    m = z.shape[1] // 2
    g, u, tg, tu = z[:, :m], z[:, m:], tol[:, :m], tol[:, m:]
    silu = g * torch.sigmoid(g)
    h = silu * u
    return h, 1.1 * tg * (u.abs() + tu) + (silu.abs() + 1.1 * tg) * tu + (g.abs() + 12) * U * h.abs() + TINY * (1 + u.abs())


def gate_grad(D, tol, saved):
    """(the gradient to (g, u), its bound)"""
    m = D.shape[1]
    g, u = saved[:, :m], saved[:, m:]
    p = torch.sigmoid(g)
    f = p * (1 + g * (1 - p))
    tf = U * (p * (g ** 2 + 9 * g.abs() + 4) + f.abs() * (g.abs() + 8)) + TINY
    dg, du = D * u * f, D * g * p
    t_g = u.abs() * (tol * f.abs() + (D.abs() + tol) * tf) + 4 * U * dg.abs()
    t_u = (g * p).abs() * (tol + (D.abs() + tol) * (g.abs() + 10) * U) + TINY * (1 + D.abs() * (1 + g.abs()))
    return torch.cat([dg, du], 1), torch.cat([t_g, t_u], 1)


def weight_grad(dY, rows, start):
    """(dW, its bound)"""
    E = len(start) - 1
    dW = torch.zeros(E, dY.shape[1], rows.shape[1], dtype=torch.float64)
    tol = torch.zeros_like(dW)
    for e in range(E):
        a, b = int(start[e]), int(start[e + 1])
        dW[e] = dY[a:b].t() @ rows[a:b]
        tol[e] = (dY[a:b].abs().t() @ rows[a:b].abs()) * 2 * U * (b - a + 16) + (TINY if b > a else 0.0)
    return dW, tol


def combine(Y, place, weight):
    n, k = place.shape
    out = torch.zeros(n, Y.shape[1], dtype=torch.float64)
    size = torch.zeros_like(out)
    for l in range(k):
        live = ((place[:, l] >= 0) & (place[:, l] < Y.shape[0]))
        rows = Y[place[live, l].long()] * (1.0 if weight is None else weight[live, l, None])
        out[live] += rows
        size[live] += rows.abs()
    return out, size * U * (k + 2) + TINY


def combine_grad(g_out, Y, place, weight, rows):
    """(dY with NaN where no choice has the row, its bound, g_weight, its bound)"""
    n, k = place.shape
    dY = torch.full((rows, g_out.shape[1]), np.nan, dtype=torch.float64)
    gw, tol = torch.zeros(n, k, dtype=torch.float64), torch.zeros(n, k, dtype=torch.float64)
    for l in range(k):
        live = (place[:, l] >= 0) & (place[:, l] < rows)
        p = place[live, l].long()
        dY[p] = g_out[live] * (1.0 if weight is None else weight[live, l, None])
        if Y is not None:
            gw[live, l] = (g_out[live] * Y[p]).sum(1)
            tol[live, l] = (g_out[live] * Y[p]).abs().sum(1) * U * (Y.shape[1] + 16) + TINY
    return dY, dY.abs().nan_to_num() * 2 * U + TINY, gw, tol
