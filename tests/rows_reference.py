"""Plain 64-bit implementations of the row operators, and how far a 32-bit evaluation may be from them.

U = 2^-24 is the relative error of one 32-bit operation.  The bounds are sums of the errors an evaluation in 32 bits makes
where it rounds each step once: with z = x/eta, d = |z - max z|, T = sum p d (the mean distance from the maximum) and
  chain(m)   additions one after the other in a sum over m columns by at least 64 lanes: m/64 + 64
  exponent   forming (x - max) * const: 3 U d;  the exponential itself 2 U;  so p's numerator is off by (3 d + 2) U
  log-sum    (chain + 16 + 3 T + 2 |L|) U
  log p      log-sum + 4 U (d + |log p|)
  entropy    log-sum + U ((2 chain + 32)(T + 1) + 6 sum p d^2 + 4 (|L| + T))
  p          p * (the bound of log p + 8 U)
A result in 16 bits has half a unit of its own on top, and results below the smallest normal number may come back as 0.
"""
import numpy as np
import torch

U = 2.0 ** -24
HALF_UNIT = {torch.float32: (U, 2.0 ** -126), torch.bfloat16: (2.0 ** -8, 2.0 ** -126), torch.float16: (2.0 ** -11, 2.0 ** -24)}
TYPES = [torch.float32, torch.bfloat16, torch.float16]
TYPE_IDS = ["f32", "bf16", "f16"]


def chain(m):
    return m / 64 + 64


def sums(S, bias):
    """x = S + bias as the operators define it: one 32-bit addition.  float64 CPU."""
    x = S.detach().cpu().float()
    if bias is not None:
        x = x + bias.cpu()
    return x.double()


class Rows:
    """Distribution of each row and the bounds of its numbers; rows: `none` (no distribution) and `bad` (NaN or +inf)."""

    def __init__(self, S, bias, eta):
        self.eta = eta
        self.x = x = sums(S, bias)
        n, m = x.shape
        self.n, self.m = n, m
        self.bad = (x.isnan() | (x == np.inf)).any(1)
        self.max = x.amax(1) if m else torch.full((n,), -np.inf, dtype=torch.float64)
        self.none = (self.max == -np.inf) & ~self.bad
        mx = torch.where(self.none | self.bad, 0.0, self.max)
        self.z = (x - mx[:, None]) / eta
        e = torch.exp(self.z)
        total = e.sum(1)
        self.L = torch.log(total)
        self.p = torch.where(self.none[:, None], 0.0, e / total[:, None])
        self.d = torch.where(e > 0, -self.z, 0.0)
        self.logp = self.z - self.L[:, None]
        self.T = (self.p * self.d).sum(1)
        self.H = torch.where(self.none, 0.0, self.L + self.T)
        self.tol_L = U * (chain(m) + 16 + 3 * self.T + 2 * self.L.abs())
        self.tol_H = self.tol_L + U * ((2 * chain(m) + 32) * (self.T + 1) + 6 * (self.p * self.d ** 2).sum(1) + 4 * (self.L.abs() + self.T))
        # (a column whose p vanishes counts with the distance at which 32 bits lose it)
        near = self.d.clamp(max=110.0)
        self.tol_logp = self.tol_L[:, None] + 4 * U * (self.d + self.logp.abs())
        self.tol_p = self.p * (self.tol_L[:, None] + 8 * U * (near + self.L.abs()[:, None] + 2)) + 2.0 ** -126


def best(x, k):
    """(columns, values) of the k largest of each row of x, ties to the lower column, -1 and -inf beyond those above -inf."""
    n, m = x.shape
    order = np.argsort(-x.numpy(), axis=1, kind="stable")[:, :k]
    val = np.take_along_axis(x.numpy(), order, 1)
    idx = np.where(val > -np.inf, order, -1)
    if m < k:
        idx = np.concatenate([idx, np.full((n, k - m), -1)], 1)
        val = np.concatenate([val, np.full((n, k - m), -np.inf)], 1)
    return torch.from_numpy(idx), torch.from_numpy(val)


def close(got, want, tol, what):
    """NaN where NaN, infinities alike (a value beyond 32 bits is one), the rest within tol."""
    got = got.detach().cpu().double()
    want, tol = torch.as_tensor(want).double(), torch.as_tensor(tol).double().expand_as(want)
    want = torch.where(want.abs() > torch.finfo(torch.float32).max, want.sign() * np.inf, want)
    assert got.shape == want.shape, (what, got.shape, want.shape)
    assert torch.equal(got.isnan(), want.isnan()), f"{what}: NaN at other places"
    fin = torch.isfinite(want)
    inf = ~fin & ~want.isnan()
    assert torch.equal(got[inf], want[inf]), f"{what}: infinities at other places"
    err = (got - want).abs()[fin]
    over = err > tol[fin]
    assert not over.any(), f"{what}: {int(over.sum())} of {over.numel()} off, worst {float((err / tol[fin].clamp(min=1e-300)).max()):.3g} times the bound"


def logprob_grad(R, target, g_logprob, g_entropy):
    """(dS, bound) in 64 bits."""
    n, m = R.x.shape
    dead = R.none
    d = torch.zeros(n, m, dtype=torch.float64)
    tol = torch.zeros(n, m, dtype=torch.float64)
    if target is not None:
        t = target.cpu().long().reshape(n, -1)
        ok = (t >= 0) & (t < m)
        g = torch.where(ok, g_logprob.cpu().double().reshape(n, -1), 0.0)
        total, size, count = g.sum(1, keepdim=True), g.abs().sum(1, keepdim=True), t.shape[1]
        d -= R.p * total
        tol += size * R.tol_p + R.p * size * U * (count + 4)
        if m:
            d.scatter_add_(1, t.clamp(0, m - 1), g)
            at = torch.zeros_like(d).scatter_add_(1, t.clamp(0, m - 1), g.abs())
            tol += at * U * (count + 4)
    if g_entropy is not None:
        h = g_entropy.cpu().double()[:, None]
        logp = torch.where(R.p > 0, R.logp, 0.0)
        d -= h * R.p * (logp + R.H[:, None])
        far = (logp.abs() + R.H[:, None])
        tol += h.abs() * (R.tol_p * (far + 1) + R.p * (torch.where(R.p > 0, R.tol_logp, 0.0) + R.tol_H[:, None] + 8 * U * far))
    d, tol = d / R.eta, tol / R.eta
    d[dead], tol[dead] = 0.0, 0.0
    d[R.bad] = np.nan
    return d, tol


def rounded(want, tol, dtype):
    rel, least = HALF_UNIT[dtype]
    return tol + rel * (want.abs() + tol) + least


def distill(S, t_idx, t_score, eta, row_weight):
    """(loss, its bound, dS, its bound)."""
    R = Rows(S, None, eta)
    n, m = R.x.shape
    t = t_idx.cpu().long()
    k = t.shape[1]
    ok = (t >= 0) & (t < m)
    raw = t_score.cpu().double()
    s = torch.where(ok, raw / eta, -np.inf)
    bad_t = (ok & (raw.isnan() | (raw == np.inf))).any(1)
    pad = (s.amax(1) == -np.inf) & ~bad_t
    s = s - torch.where(pad | bad_t, 0.0, s.amax(1))[:, None]
    q = torch.exp(s)
    q_total = q.sum(1, keepdim=True)
    q = torch.where(pad[:, None], 0.0, q / q_total)
    log_q = s - torch.log(q_total)
    live = q > 2.0 ** -140
    at = t.clamp(0, max(m - 1, 0))
    logp = (torch.where(R.none[:, None], -np.inf, R.logp).gather(1, at) if m else torch.full((n, k), -np.inf, dtype=torch.float64))
    terms = torch.where(live, q * (torch.where(live, log_q, 0.0) - torch.where(live, logp, 0.0)), 0.0)
    loss = terms.sum(1)
    tol_q = U * (k + 16 + 4 * torch.where(live, s.abs(), 0.0) + 2 * torch.where(live, log_q.abs(), 0.0))  # of log q; relative of q
    tol_lp = torch.where(torch.isfinite(logp), R.tol_logp.gather(1, at), 0.0) if m else torch.zeros(n, k, dtype=torch.float64)
    fine = torch.where(live & torch.isfinite(logp), logp.abs(), 0.0)
    size = torch.where(live, log_q.abs(), 0.0) + fine
    tol_loss = (q * (tol_q * (size + 1) + tol_lp + U * (k + 8) * size)).sum(1) + 1e-30
    w = (row_weight.cpu().double() if row_weight is not None else torch.ones(n, dtype=torch.float64))[:, None] / eta
    listed, tol_listed = torch.zeros(n, m, dtype=torch.float64), torch.zeros(n, m, dtype=torch.float64)
    if m:
        listed.scatter_add_(1, at, q)
        tol_listed.scatter_add_(1, at, q * (tol_q + (k + 4) * U))
    d = w * (R.p - listed)
    tol = w.abs() * (R.tol_p + tol_listed + 8 * U * (R.p + listed))
    d[R.none], tol[R.none] = 0.0, 0.0
    for v, where in ((np.nan, R.bad | bad_t), (0.0, pad)):
        loss[where], d[where] = v, v
        if v == 0.0:
            tol[where] = 0.0
    return loss, tol_loss, d, tol


def route_scores(S, score):
    x = S.detach().cpu().double()
    if score == "sigmoid":
        return torch.sigmoid(x)
    if x.shape[1] == 0:
        return x
    mx = x.amax(1, keepdim=True)
    e = torch.exp(x - torch.where(mx == -np.inf, 0.0, mx))
    return torch.where(mx == -np.inf, 0.0, e / e.sum(1, keepdim=True))


def route_keys(S, bias, bias_on, score, groups, kept, group_by):
    """(keys after the groups, in 64 bits; least distance between group values at the cut), by plain loops over groups."""
    x, s = S.detach().cpu().double(), route_scores(S, score)
    n, m = x.shape
    key = x.clone() if bias is None else (s if bias_on == "score" else x) + bias.cpu().double()
    key[x == -np.inf] = -np.inf
    if groups == 1:
        return key, np.inf
    by = torch.where(key == -np.inf, -np.inf, s if bias is None else key).reshape(n, groups, -1)
    two = by.sort(dim=2, descending=True).values
    value = two[:, :, 0].clone()
    if group_by == "top2" and two.shape[2] > 1:
        value = torch.where(two[:, :, 1] > -np.inf, value + two[:, :, 1], value)
    order = np.argsort(-value.numpy(), axis=1, kind="stable")
    shut = torch.ones(n, groups, dtype=torch.bool).scatter_(1, torch.from_numpy(order[:, :kept].copy()), False)
    least = np.inf
    if kept < groups:
        v = np.take_along_axis(value.numpy(), order, 1)
        with np.errstate(invalid="ignore"):
            gap = v[:, kept - 1] - v[:, kept]
        gap = gap[np.isfinite(gap) & (gap > 0)]
        least = gap.min() if gap.size else np.inf
    return key.masked_fill(shut.repeat_interleave(m // groups, dim=1), -np.inf), least
