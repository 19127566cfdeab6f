"""The row operators as cases that can be timed and compared: log probabilities of given columns with the entropy and the
top alternatives of a row (and the gradient), distillation from a teacher's top entries (loss and gradient), routing of
rows to columns (forward, and with its gradient).

A case is one call, or one forward and backward pair, on seeded scores S of n rows against m columns in the types that
models hold.  `own` chooses what runs: the plain form (elementary torch operations in 32 bits) or the framework's kernels.
"""
import math

import torch

own = False

_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_MOST_BYTES = 4096 * 131072 * 2  # scores of the largest case


def listed():
    return [
        # one token of a served model: its log probability, the entropy and the 20 best alternatives
        dict(name="answer_one", kind="logprob", n=1, m=131072, type="bf16", k=20, targets=1, eta=1.0, bias=False, masked=0.0),
        # a batch of answers at a temperature, a third of the columns closed by a grammar; 50000 columns
        dict(name="answer_batch", kind="logprob", n=64, m=50000, type="f16", k=8, targets=1, eta=0.7, bias=False, masked=0.3),
        # balanced targets: the best columns of each row under the column duals of a solve, an odd number of them, fp32 scores
        dict(name="targets_balanced", kind="logprob", n=1500, m=10007, type="f32", k=32, targets=2, eta=0.1, bias=True, masked=0.0),
        # prompts scored whole: the largest
        dict(name="score_prompts", kind="logprob", n=4096, m=131072, type="bf16", k=20, targets=1, eta=1.0, bias=False, masked=0.0),
        # a policy's step: gradients of log probabilities and entropy to the scores
        dict(name="policy_grad", kind="logprob_grad", n=2048, m=40000, type="bf16", k=0, targets=1, eta=1.0, bias=False, masked=0.0),
        # the same on fp32 scores of ragged length with the bias and several given columns
        dict(name="policy_grad_ragged", kind="logprob_grad", n=700, m=4999, type="f32", k=0, targets=3, eta=0.5, bias=True, masked=0.1),
        # a student's step against balanced targets over 10000 columns, fp32
        dict(name="distill_small", kind="distill", n=256, m=10000, type="f32", k=32, eta=0.1, padded=0.0),
        # a student's step on a ragged batch, a tenth of the rows padding; rows start at odd multiples of 2 bytes
        dict(name="distill_ragged", kind="distill", n=999, m=33333, type="bf16", k=50, eta=2.0, padded=0.1),
        # a student's step over the largest vocabulary
        dict(name="distill_large", kind="distill", n=4096, m=131072, type="bf16", k=64, eta=1.0, padded=0.0),
        # one token of a served model to its experts: sigmoid scores, bias, groups
        dict(name="route_one", kind="route", n=1, m=256, type="f32", k=8, score="sigmoid", bias="score", groups=8, kept=4, group_by="top2", renorm=True),
        # a prompt's tokens to few experts, softmax without groups, balanced by duals on the scores themselves
        dict(name="route_prompt", kind="route", n=8192, m=60, type="bf16", k=4, score="softmax", bias="logit", groups=1, kept=1, group_by="max", renorm=False),
        # a training batch's tokens to many experts, with the gradient
        dict(name="route_train", kind="route_train", n=65536, m=256, type="f32", k=8, score="sigmoid", bias="score", groups=8, kept=4, group_by="top2", renorm=True),
    ]


def _log_between(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["logprob", "logprob", "logprob_grad", "distill", "distill", "route", "route_train"])
    kind_of = rng.choice(["bf16", "bf16", "f16", "f32"])
    b = _TYPES[kind_of].itemsize
    if kind in ("route", "route_train"):
        groups = rng.choice([1, 1, 2, 4, 8])
        m = groups * _log_between(rng, max(2, 16 // groups), 512 // groups)
        kept = rng.randint((groups + 1) // 2, groups)
        return dict(kind=kind, n=_log_between(rng, 1 if kind == "route" else 64, 65536), m=m, type=kind_of,
                    k=rng.randint(1, min(10, kept * (m // groups))), score=rng.choice(["softmax", "sigmoid"]),
                    bias=rng.choice(["none", "score", "logit"]), groups=groups, kept=kept,
                    group_by=rng.choice(["max", "top2"]), renorm=rng.random() < 0.6)
    m = _log_between(rng, 300, 131072)
    n = _log_between(rng, 1 if kind == "logprob" else 16, min(16384, _MOST_BYTES // (m * b)))
    if kind == "distill":
        return dict(kind=kind, n=n, m=m, type=kind_of, k=rng.randint(1, 100), eta=rng.choice([0.1, 1.0, 1.0, 2.0]),
                    padded=rng.choice([0.0, 0.2]))
    return dict(kind=kind, n=n, m=m, type=kind_of, k=rng.randint(0, 64) if kind == "logprob" else 0, targets=rng.randint(1, 4),
                eta=rng.choice([0.2, 0.7, 1.0, 1.0]), bias=rng.random() < 0.3, masked=rng.choice([0.0, 0.0, 0.2]))


def work(case):
    n, m, b = case["n"], case["m"], _TYPES[case["type"]].itemsize
    kind, k = case["kind"], case["k"]
    if kind == "logprob":
        t = case["targets"]
        return dict(bytes=n * m * b + n * (8 * t + 12 + 8 * k) + 4 * m * case["bias"], flops=6 * n * m)
    if kind == "logprob_grad":
        t = case["targets"]
        return dict(bytes=2 * n * m * b + n * (8 * t + 16) + 4 * m * case["bias"], flops=8 * n * m)
    if kind == "distill":
        return dict(bytes=2 * n * m * b + n * (8 * k + 8), flops=8 * n * m)
    once = n * m * b + 8 * n * k + 4 * m * (case["bias"] != "none")
    return dict(bytes=once + (n * m * b + 4 * n * k) * (kind == "route_train"), flops=(6 if kind == "route" else 12) * n * m)


# ---- inputs ----------------------------------------------------------------------------------------------------------

def _scores(case, gen):
    """Rows as a model gives them: a broad body, a few columns far above it."""
    n, m = case["n"], case["m"]
    S = torch.randn(n, m, generator=gen, device="cuda").mul_(2.0)
    peaks = min(24, m)
    at = torch.randint(0, m, (n, peaks), generator=gen, device="cuda")
    S.scatter_add_(1, at, torch.rand(n, peaks, generator=gen, device="cuda").clamp_(min=1e-6).log_().mul_(-3.0))
    if case["eta"] < 0.5:
        S.mul_(case["eta"])  # scores of the size of the regularisation
    if case.get("masked"):
        closed = torch.rand(m, generator=gen, device="cuda") < case["masked"]
        closed[0] = False
        S.masked_fill_(closed, -math.inf)
    return S.to(_TYPES[case["type"]])


def _loss_scale(case):
    """What a program multiplies its loss by so that 16-bit gradients of five exponent bits do not vanish."""
    return 65536.0 if case["type"] == "f16" else 1.0


def _selection(case, S, bias, wide):
    """(keys that experts are chosen by, keys that groups are valued by, scores), in `wide` bits."""
    x = S.to(wide)
    if case["score"] == "softmax":
        e = torch.exp(x - x.max(1, keepdim=True).values)
        s = e / e.sum(1, keepdim=True)
    else:
        s = 1.0 / (1.0 + torch.exp(-x))
    if bias is None:
        return x, s, s
    key = (s if case["bias"] == "score" else x) + bias.to(wide)
    return key, key, s


def _group_values(case, key):
    parts = key.view(case["n"], case["groups"], -1)
    if case["group_by"] == "max" or parts.shape[2] == 1:
        return parts.max(2).values
    return parts.topk(2, dim=2).values.sum(2)


def _close_calls(case, S, bias):
    """Rows whose choice hangs on the last bits of 32: two keys, or two groups, within 1e-5 of each other but not equal."""
    key, by, _ = _selection(case, S, bias, torch.float64)
    close = torch.zeros(case["n"], dtype=torch.bool, device=S.device)
    if case["groups"] > 1:
        v = _group_values(case, by).sort(1, descending=True).values
        gap = v[:, :-1] - v[:, 1:]
        close |= ((gap > 0) & (gap < 1e-5 * v.abs().max(1, keepdim=True).values)).any(1)
    if bias is not None:
        v = key.sort(1, descending=True).values
        gap = (v[:, :-1] - v[:, 1:])[:, :4 * case["k"] + 8]
        close |= ((gap > 0) & (gap < 1e-5 * v.abs().max(1, keepdim=True).values)).any(1)
    return close


def _router_scores(case, gen):
    n, m = case["n"], case["m"]
    lean = torch.randn(m, generator=gen, device="cuda").mul_(0.5)
    fresh = lambda: (torch.randn(n, m, generator=gen, device="cuda") + lean).to(_TYPES[case["type"]])  # noqa: E731
    size = {"none": None, "score": 0.05 if case["score"] == "sigmoid" else 0.3 / m, "logit": 0.5}[case["bias"]]
    bias = None if size is None else torch.randn(m, generator=gen, device="cuda").mul_(size)
    S = fresh()
    for _ in range(12):  # whole numbers are compared: no choice is left to the last bit of a sum
        S = torch.where(_close_calls(case, S, bias)[:, None], fresh(), S)
    return S, bias


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    n, m, kind, k = case["n"], case["m"], case["kind"], case["k"]
    st = dict(case=case)
    if kind in ("route", "route_train"):
        st["S"], st["bias"] = _router_scores(case, gen)
        st["g_weight"] = torch.randn(n, k, generator=gen, device="cuda") if kind == "route_train" else None
        return st
    S = st["S"] = _scores(case, gen)
    if kind == "distill":
        k = min(k, m)
        t = S.float()
        t += torch.randn(n, m, generator=gen, device="cuda").mul_(0.5 * min(1.0, case["eta"]))
        score, idx = t.topk(k, dim=1)
        st["t_score"], st["t_idx"] = score.contiguous(), idx.to(torch.int32).contiguous()
        live = torch.rand(n, generator=gen, device="cuda") >= case["padded"]
        st["t_idx"][~live] = -1
        st["row_weight"] = live.float() / live.sum().clamp(min=1) * _loss_scale(case)
        return st
    st["bias"] = torch.randn(m, generator=gen, device="cuda").mul_(0.3 * case["eta"]) if case["bias"] else None
    x = S.float() if st["bias"] is None else S.float() + st["bias"]
    likely = torch.rand(n, m, generator=gen, device="cuda").clamp_(min=1e-20).log_().neg_().log_().neg_().mul_(case["eta"]).add_(x)
    st["target"] = likely.topk(case["targets"], dim=1).indices.to(torch.int32).contiguous()  # drawn from the rows' own distributions
    if kind == "logprob_grad":
        z = x.double() / case["eta"]
        mx = z.max(1, keepdim=True).values
        e = torch.exp(z - mx)
        total = e.sum(1, keepdim=True)
        st["stats"] = torch.cat([x.max(1, keepdim=True).values, total.log().float()], 1).contiguous()
        st["entropy"] = (total.log() - torch.where(e > 0, e * (z - mx), 0.0).sum(1, keepdim=True) / total)[:, 0].float().contiguous()
        st["g_logprob"] = torch.randn(n, case["targets"], generator=gen, device="cuda") * (_loss_scale(case) / n)
        st["g_entropy"] = torch.full((n,), 0.01 * _loss_scale(case) / n, device="cuda")
    return st


# ---- the plain form --------------------------------------------------------------------------------------------------

def _best(x, k):
    """Columns of the k largest of each row, largest first, ties to the lower column."""
    b = (x + 0.0).view(torch.int32)
    order = torch.where(b < 0, b ^ 0x7FFFFFFF, b).long()
    column = torch.arange(x.shape[1], device=x.device)
    return ((order << 32) | (0xFFFFFFFF - column)).topk(k, dim=1).indices


def _plain_logprob(st):
    c = st["case"]
    x = st["S"].float()
    if st["bias"] is not None:
        x = x + st["bias"]
    top = x.max(1, keepdim=True).values
    z = (x - top) / c["eta"]
    e = torch.exp(z)
    total = e.sum(1, keepdim=True)
    log_total = torch.log(total)
    out = dict(logprob=z.gather(1, st["target"].long()) - log_total,
               entropy=(log_total - torch.where(e > 0, e * z, 0.0).sum(1, keepdim=True) / total)[:, 0],
               stats=torch.cat([top, log_total], 1))
    if c["k"]:
        idx = _best(x, c["k"])
        out["top_idx"], out["top_logprob"] = idx.to(torch.int32), z.gather(1, idx) - log_total
    return out


def _plain_logprob_grad(st):
    c = st["case"]
    x = st["S"].float()
    if st["bias"] is not None:
        x = x + st["bias"]
    logp = (x - st["stats"][:, :1]) / c["eta"] - st["stats"][:, 1:]
    p = torch.exp(logp)
    d = -p * st["g_logprob"].sum(1, keepdim=True)
    d = d - torch.where(p > 0, st["g_entropy"][:, None] * p * (logp + st["entropy"][:, None]), 0.0)
    d.scatter_add_(1, st["target"].long(), st["g_logprob"])
    return (d / c["eta"]).to(st["S"].dtype)


def _plain_distill(st):
    c = st["case"]
    x = st["S"].float()
    z = (x - x.max(1, keepdim=True).values) / c["eta"]
    e = torch.exp(z)
    total = e.sum(1, keepdim=True)
    there = st["t_idx"] >= 0
    at = st["t_idx"].clamp(min=0).long()
    t = st["t_score"] / c["eta"]
    t = t - t.max(1, keepdim=True).values
    q = torch.exp(t)
    q_total = q.sum(1, keepdim=True)
    q = torch.where(there, q / q_total, 0.0)
    loss = (q * (t - torch.log(q_total) - z.gather(1, at) + torch.log(total))).sum(1)
    d = (e / total) * q.sum(1, keepdim=True)
    d.scatter_add_(1, at, -q)
    return dict(loss=loss, grad=(d * (st["row_weight"][:, None] / c["eta"])).to(st["S"].dtype))


def _plain_route(st):
    c = st["case"]
    key, by, s = _selection(c, st["S"], st["bias"], torch.float32)
    if c["groups"] > 1:
        v = _group_values(c, by)
        g = torch.arange(c["groups"], device=v.device)
        better = (v[:, None, :] > v[:, :, None]) | ((v[:, None, :] == v[:, :, None]) & (g[None, :] < g[:, None]))
        kept = better.sum(2) < c["kept"]
        key = torch.where(kept.repeat_interleave(c["m"] // c["groups"], dim=1), key, -math.inf)
    idx = _best(key, c["k"])
    chosen = s.gather(1, idx)
    weight = chosen / chosen.sum(1, keepdim=True) if c["renorm"] else chosen
    out = dict(idx=idx.to(torch.int32), weight=weight * 2.5)
    if c["kind"] == "route_train":
        g = st["g_weight"] * 2.5
        if c["renorm"]:
            g = (g - (g * weight).sum(1, keepdim=True)) / chosen.sum(1, keepdim=True)
        ds = torch.zeros_like(s).scatter_(1, idx, g)
        d = s * (ds - (ds * s).sum(1, keepdim=True)) if c["score"] == "softmax" else ds * s * (1.0 - s)
        out["grad"] = d.to(st["S"].dtype)
    return out


# ---- the framework's calls -------------------------------------------------------------------------------------------

def _own_handle(st):
    """The buffers that a program keeps for calls of one size; made at the first call."""
    from paper_2605_08793_amd.rows import RowDistill, RowLogprob, RowRoute
    c, dtype = st["case"], st["S"].dtype
    if c["kind"] == "distill":
        st["op"] = RowDistill(c["n"], c["m"], st["t_idx"].shape[1], dtype=dtype)
    elif c["kind"] in ("logprob", "logprob_grad"):
        st["op"] = RowLogprob(c["n"], c["m"], k=c["k"], targets=c["targets"], dtype=dtype)
    else:
        st["op"] = RowRoute(c["n"], c["m"], c["k"], score=c["score"], bias_on=None if c["bias"] == "none" else c["bias"],
                            groups=c["groups"], groups_kept=c["kept"], group_by=c["group_by"], renormalise=c["renorm"],
                            scale=2.5, dtype=dtype)
    return st["op"]


def _own_run(st):
    c = st["case"]
    op = st.get("op") or _own_handle(st)
    if c["kind"] == "logprob":
        op.logprob(st["S"], st["target"], eta=c["eta"], bias=st["bias"])
        out = dict(logprob=op.logprob_out, entropy=op.entropy, stats=op.stats)
        if c["k"]:
            out["top_idx"], out["top_logprob"] = op.top_idx, op.top_logprob
        return out
    if c["kind"] == "logprob_grad":
        return op.grad(st["S"], st["target"], st["g_logprob"], st["g_entropy"], eta=c["eta"], bias=st["bias"],
                       stats=st["stats"], entropy=st["entropy"])
    if c["kind"] == "distill":
        op.distill(st["S"], st["t_idx"], st["t_score"], eta=c["eta"], row_weight=st["row_weight"])
        return dict(loss=op.loss, grad=op.grad)
    op.route(st["S"], bias=st["bias"])
    out = dict(idx=op.idx, weight=op.weight)
    if c["kind"] == "route_train":
        out["grad"] = op.grad(st["S"], st["g_weight"])
    return out


def run(state):
    if own:
        return _own_run(state)
    return {"logprob": _plain_logprob, "logprob_grad": _plain_logprob_grad, "distill": _plain_distill,
            "route": _plain_route, "route_train": _plain_route}[state["case"]["kind"]](state)


# ---- the definitions in 64 bits --------------------------------------------------------------------------------------

def _exact_rows(c, st, i, j):
    """(log p, p) of rows i to j."""
    x = st["S"][i:j].double()
    if st.get("bias") is not None:
        x = x + st["bias"].double()
    lp = torch.log_softmax(x / c["eta"], dim=1)
    return x, lp, lp.exp()


def _exact_logprob(c, st, i, j):
    x, lp, p = _exact_rows(c, st, i, j)
    out = dict(logprob=lp.gather(1, st["target"][i:j].long()), entropy=torch.special.entr(p).sum(1),
               stats=torch.stack([x.amax(1), torch.logsumexp(x / c["eta"], 1) - x.amax(1) / c["eta"]], 1))
    if c["k"]:
        out["top_logprob"] = lp.topk(c["k"], dim=1).values
    return out


def _exact_logprob_grad(c, st, i, j):
    x, lp, p = _exact_rows(c, st, i, j)
    entropy = torch.special.entr(p).sum(1, keepdim=True)
    d = torch.special.entr(p) - p * entropy  # dH/dz
    d *= st["g_entropy"][i:j, None].double()
    for t in range(c["targets"]):
        g = st["g_logprob"][i:j, t].double()
        d -= g[:, None] * p
        d[torch.arange(j - i, device=d.device), st["target"][i:j, t].long()] += g
    return dict(grad=d / c["eta"])


def _exact_distill(c, st, i, j):
    x, lp, p = _exact_rows(c, st, i, j)
    there = st["t_idx"][i:j] >= 0
    q = torch.softmax(st["t_score"][i:j].double() / c["eta"], dim=1) * there
    at = st["t_idx"][i:j].long() * there
    loss = (torch.xlogy(q, q) - q * lp.gather(1, at)).sum(1)
    target = torch.zeros_like(p).scatter_add_(1, at, q)
    return dict(loss=loss, grad=st["row_weight"][i:j, None].double() * (p * target.sum(1, keepdim=True) - target) / c["eta"])


def _exact_route(c, st, i, j):
    x = st["S"][i:j].double().requires_grad_(True)
    s = torch.softmax(x, 1) if c["score"] == "softmax" else torch.sigmoid(x)
    key = s if c["bias"] == "score" else x
    by = s if c["bias"] == "none" else key
    if st["bias"] is not None:
        key, by = key + st["bias"].double(), by + st["bias"].double()
    groups = by.detach().reshape(j - i, c["groups"], -1)
    value = groups.topk(1 if c["group_by"] == "max" else min(2, groups.shape[2]), dim=2).values.sum(2)
    best = value.sort(dim=1, descending=True, stable=True).indices[:, :c["kept"]]
    shut = torch.ones_like(value, dtype=torch.bool).scatter_(1, best, False)
    key = key.detach().masked_fill(shut.repeat_interleave(c["m"] // c["groups"], dim=1), -math.inf)
    idx = key.sort(dim=1, descending=True, stable=True).indices[:, :c["k"]]
    w = s.gather(1, idx)
    w = 2.5 * (w / w.sum(1, keepdim=True) if c["renorm"] else w)
    out = dict(weight=w.detach())
    if c["kind"] == "route_train":
        out["grad"] = torch.autograd.grad((w * st["g_weight"][i:j].double()).sum(), x)[0]
    return out


def exact(case, seed):
    st = prepare(case, seed)
    of = {"logprob": _exact_logprob, "logprob_grad": _exact_logprob_grad, "distill": _exact_distill,
          "route": _exact_route, "route_train": _exact_route}[case["kind"]]
    rows = max(1, (1 << 27) // case["m"])
    parts = [of(case, st, i, min(i + rows, case["n"])) for i in range(0, case["n"], rows)]
    whole = {key: torch.cat([p[key] for p in parts]) for key in parts[0]}
    return whole["grad"] if case["kind"] == "logprob_grad" else whole
