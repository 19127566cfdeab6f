"""The experts' operators as cases that can be timed and compared: the order of a router's choices, products grouped by expert
with their gradients, the weighted sum of the experts' rows with its gradient, and the norm over many gradients with clipping.

A case is one call, or the calls of one backward step, on seeded data in the types that models hold: n tokens, each with k choices
among `experts`, whose loads differ as those of a balanced router do.  `own` chooses what runs: the plain form (elementary torch operations
in 32 bits) or the framework's kernels.
"""
import math

import torch

own = False

_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_MOST_FLOPS = 4 * 131072 * 2048 * 1024   # of the largest case
_MOST_WEIGHTS = 256 * 2048 * 2048        # numbers that a case's experts have
_MOST_ROWS = 65536 * 8 * 2048            # numbers that a case's rows have
_LEAN = 0.2                              # how far apart the experts' loads are (standard deviation of their logarithms)


def listed():
    return [
        # a prompt's choices put into the order of the experts before their products
        dict(name="order_prompt", kind="order", n=8192, k=4, experts=60, dropped=0.0),
        # a training batch's choices, some of them dropped where an expert was full
        dict(name="order_train", kind="order", n=65536, k=8, experts=256, dropped=0.02),
        # one token of a served model: a row each for eight of 256 experts, the gated product of their weights
        dict(name="serve_one", kind="product", n=1, k=8, experts=256, d=2048, m=1024, type="bf16", gated=True, keep=False),
        # a step of a batch of served sequences: few rows for each expert, the product behind the gate
        dict(name="serve_batch", kind="product", n=64, k=4, experts=60, d=1400, m=2048, type="f16", gated=False, keep=False),
        # a prompt, or the forward pass of training, which keeps what the gradient needs
        dict(name="prompt", kind="product", n=8192, k=4, experts=60, d=2048, m=1024, type="bf16", gated=True, keep=True),
        # a backward step: gradients to the rows and to the weights (held in 32 bits); the largest
        dict(name="grad_train", kind="product_grad", n=16384, k=8, experts=64, d=2048, m=1024, type="bf16", behind_gate=False, dw="f32"),
        # a backward step of the product behind the gate, few experts
        dict(name="grad_gate", kind="product_grad", n=4096, k=2, experts=8, d=1408, m=2048, type="bf16", behind_gate=True, dw="bf16"),
        # a backward step of a small model in 32 bits: odd sizes, so rows start at odd multiples of 4 bytes
        dict(name="grad_ragged", kind="product_grad", n=999, k=3, experts=12, d=777, m=555, type="f32", behind_gate=False, dw="f32"),
        # the experts' answers of a batch of served sequences brought together
        dict(name="combine_batch", kind="combine", n=64, k=4, m=2048, type="f16", dropped=0.0),
        # the same in training, with the gradients to the experts' rows and to the router's weights
        dict(name="combine_train", kind="combine_grad", n=65536, k=8, m=2048, type="bf16", dropped=0.02),
        # the gradients of a small model, whose norm is below the limit
        dict(name="clip_small", kind="clip", tensors=24, total=3_000_000, type="f32", limit=2.0, kept=False),
        # the gradients of a larger one, over the limit; the clipped ones go to other memory
        dict(name="clip_large", kind="clip", tensors=300, total=600_000_000, type="bf16", limit=0.3, kept=True),
    ]


def _log_between(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def _width(rng, lo, hi):
    """Rows' lengths: mostly whole multiples of 64 or 8, some of them anything."""
    v = _log_between(rng, lo, hi)
    step = rng.choice([64, 64, 8, 8, 1])
    return max(lo, v // step * step)


def draw(rng):
    kind = rng.choice(["order", "product", "product", "product", "product_grad", "product_grad", "combine", "combine_grad", "clip"])
    type_ = rng.choice(["bf16", "bf16", "f16", "f32"])
    if kind == "clip":
        limit = rng.choice([0.3, 0.9, 2.0])  # (where it is passed, the gradients stay: a pass in place would leave the next one nothing to clip)
        return dict(kind=kind, tensors=_log_between(rng, 1, 400), total=_log_between(rng, 1000, 600_000_000 // (2 if type_ == "f32" else 1)),
                    type=type_, limit=limit, kept=limit < 1.0 or rng.random() < 0.3)
    k = rng.randint(1, 8)
    if kind == "order":
        return dict(kind=kind, n=_log_between(rng, 1, 65536), k=k, experts=_log_between(rng, max(4, k), 512), dropped=rng.choice([0.0, 0.05]))
    if kind in ("combine", "combine_grad"):
        m = _width(rng, 64, 4096)
        most = _MOST_ROWS // (k * m * (2 if type_ == "f32" else 1))
        return dict(kind=kind, n=_log_between(rng, 1, min(65536, most)), k=k, m=m, type=type_, dropped=rng.choice([0.0, 0.05]))
    d, m = _width(rng, 64, 4096), _width(rng, 64, 4096)
    gated = rng.random() < 0.5
    experts = _log_between(rng, max(4, k), min(256, _MOST_WEIGHTS // (d * m * (2 if gated else 1))))
    times = 2 if kind == "product" and gated else 1
    # (32-bit products cost several times what those of 16 bits do)
    most = _MOST_FLOPS // (2 * d * m * k * (2 if kind == "product_grad" else times) * (8 if type_ == "f32" else 1))
    n = _log_between(rng, 1, max(1, min(16384, most)))
    if kind == "product":
        return dict(kind=kind, n=n, k=k, experts=experts, d=d, m=m, type=type_, gated=gated, keep=gated and rng.random() < 0.5)
    return dict(kind=kind, n=n, k=k, experts=experts, d=d, m=m, type=type_, behind_gate=gated, dw=rng.choice([type_, "f32"]))


def work(case):
    kind = case["kind"]
    if kind == "order":
        return dict(bytes=12 * case["n"] * case["k"] + 8 * case["experts"], flops=0)
    b = _TYPES[case["type"]].itemsize
    if kind == "clip":
        return dict(bytes=case["total"] * b * (2 if case["kept"] else 1), flops=3 * case["total"])
    n, k, m = case["n"], case["k"], case["m"]
    rows = n * k
    if kind == "combine":
        return dict(bytes=(rows + n) * m * b + 8 * rows, flops=2 * rows * m)
    if kind == "combine_grad":
        return dict(bytes=(2 * rows + 2 * n) * m * b + 12 * rows, flops=5 * rows * m)
    d, used = case["d"], min(case["experts"], rows)
    if kind == "product":
        wide = 2 * m if case["gated"] else m
        return dict(bytes=(n * d + used * wide * d + rows * m + case["keep"] * rows * wide) * b + 4 * rows, flops=2 * rows * wide * d)
    moved = (rows * m + used * m * d + (5 * rows if case["behind_gate"] else rows + n) * d) * b
    return dict(bytes=moved + case["experts"] * m * d * _TYPES[case["dw"]].itemsize, flops=4 * rows * m * d)


# ---- inputs ----------------------------------------------------------------------------------------------------------

def _choices(case, gen):
    """(n, k) different experts for each token, some dropped: -1."""
    n, k, experts = case["n"], case["k"], case.get("experts", 64)
    lean = torch.randn(experts, generator=gen, device="cuda") * _LEAN
    key = torch.rand(n, experts, generator=gen, device="cuda").clamp_(min=1e-20).log_().neg_().log_().neg_().add_(lean)
    idx = key.topk(k, dim=1).indices.to(torch.int32)
    if case.get("dropped"):
        idx[torch.rand(n, k, generator=gen, device="cuda") < case["dropped"]] = -1
    return idx


def _order(idx, experts):
    """(start, order, place) of choices, as a program has them from the call before."""
    flat = idx.reshape(-1).long()
    key = torch.where(flat < 0, experts, flat)
    sorted_key, order = key.sort(stable=True)
    start = torch.searchsorted(sorted_key, torch.arange(experts + 1, device=flat.device))
    rows = torch.arange(flat.numel(), device=flat.device)
    live = sorted_key < experts
    place = torch.empty_like(flat).scatter_(0, order, torch.where(live, rows, -1))
    return start, torch.where(live, order, -1).to(torch.int32), place.to(torch.int32).reshape(idx.shape)


def _random(gen, *shape, dtype, scale=1.0):
    return torch.empty(*shape, dtype=dtype, device="cuda").normal_(0.0, scale, generator=gen)


def _prepare_clip(case, gen):
    """Tensors of all sizes, a few of them most of the whole, in one memory."""
    dtype, tensors = _TYPES[case["type"]], case["tensors"]
    cpu = torch.Generator().manual_seed(tensors)  # (a model's tensors have the same sizes each time)
    share = torch.rand(tensors, generator=cpu).mul_(6.0).exp_().double()
    sizes = (share / share.sum() * case["total"]).long().clamp_(min=1)
    starts = torch.cat([torch.zeros(1, dtype=torch.long), ((sizes + 63) // 64 * 64).cumsum(0)])
    flat = torch.zeros(int(starts[-1]), dtype=dtype, device="cuda")
    flat.normal_(0.0, 1e-3, generator=gen)
    cut = lambda whole: [whole[a:a + s] for a, s in zip(starts.tolist(), sizes.tolist())]  # noqa: E731
    st = dict(case=case, flat=flat, tensors=cut(flat), limit=case["limit"] * 1e-3 * math.sqrt(int(sizes.sum())), out=None)
    if case["kept"]:
        st["out"] = torch.zeros_like(flat)
        st["out_tensors"] = cut(st["out"])
    return st


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    if case["kind"] == "clip":
        return _prepare_clip(case, gen)
    st = dict(case=case, idx=_choices(case, gen))
    if case["kind"] == "order":
        return st
    st["start"], st["order"], st["place"] = _order(st["idx"], case.get("experts", 64))
    n, k, m, dtype = case["n"], case["k"], case["m"], _TYPES[case["type"]]
    rows = n * k
    if case["kind"] in ("combine", "combine_grad"):
        st["Y"] = _random(gen, rows, m, dtype=dtype)
        w = torch.rand(n, k, generator=gen, device="cuda") + 0.1
        st["weight"] = w / w.sum(1, keepdim=True)
        if case["kind"] == "combine_grad":
            st["g_out"] = _random(gen, n, m, dtype=dtype)
        return st
    d, experts = case["d"], case["experts"]
    st["most"] = int((st["start"][1:] - st["start"][:-1]).max())  # the rows of the fullest expert, which a program that pads knows
    wide = 2 * m if case["kind"] == "product" and case["gated"] else m
    st["W"] = _random(gen, experts, wide, d, dtype=dtype, scale=d ** -0.5)
    if case["kind"] == "product":
        st["X"] = _random(gen, n, d, dtype=dtype)
        return st
    st["g_Y"] = _random(gen, rows, m, dtype=dtype)
    if case["behind_gate"]:
        st["saved"] = _random(gen, rows, 2 * d, dtype=dtype)
        g, u = st["saved"][:, :d].float(), st["saved"][:, d:].float()
        st["X"] = (g / (1.0 + torch.exp(-g)) * u).to(dtype)
    else:
        st["X"] = _random(gen, n, d, dtype=dtype)
    return st


# ---- the plain form --------------------------------------------------------------------------------------------------

def _plain_order(st):
    start, order, place = _order(st["idx"], st["case"]["experts"])
    return dict(start=start, order=order, place=place)


def _slots(st):
    """Where each row is among padded ones: expert times the most rows of one, plus its number there."""
    rows = torch.arange(st["order"].numel(), device="cuda")
    expert = torch.searchsorted(st["start"][1:], rows, right=True)
    return expert, expert * st["most"] + rows - st["start"][expert]


def _padded(st, rows, at):
    """Rows of each expert below each other, zeros behind: (experts, most, length)."""
    out = torch.zeros(st["case"]["experts"] * st["most"], rows.shape[1], device="cuda")
    out[at] = rows.float()
    return out.view(st["case"]["experts"], st["most"], -1)


def _grouped(st, rows, turned):
    """rows W^T, or rows W where `turned`, with each row's own expert; few rows take a copy of their expert's weights each."""
    expert, at = _slots(st)
    few = st["case"]["n"] * st["case"]["k"] < st["case"]["experts"]
    W = (st["W"][expert] if few else st["W"]).float()
    if not turned:
        W = W.transpose(1, 2)
    if few:
        return torch.bmm(rows.float()[:, None, :], W)[:, 0]
    return torch.bmm(_padded(st, rows, at), W).reshape(-1, W.shape[2])[at]


def _plain_product(st):
    c = st["case"]
    Z = _grouped(st, st["X"][st["order"].long() // c["k"]], False)
    if not c["gated"]:
        return dict(Y=Z.to(st["X"].dtype))
    g, u = Z[:, :c["m"]], Z[:, c["m"]:]
    out = dict(Y=(g / (1.0 + torch.exp(-g)) * u).to(st["X"].dtype))
    if c["keep"]:
        out["saved"] = Z.to(st["X"].dtype)
    return out


def _plain_product_grad(st):
    c = st["case"]
    D = _grouped(st, st["g_Y"], True)
    if c["behind_gate"]:
        X = st["X"]
        g, u = st["saved"][:, :c["d"]].float(), st["saved"][:, c["d"]:].float()
        s = 1.0 / (1.0 + torch.exp(-g))
        D = torch.cat([D * u * s * (1.0 + g * (1.0 - s)), D * g * s], 1)
    else:
        X = st["X"][st["order"].long() // c["k"]]
    _, at = _slots(st)
    dW = torch.bmm(_padded(st, st["g_Y"], at).transpose(1, 2), _padded(st, X, at))
    return dict(dX=D.to(X.dtype), dW=dW.to(_TYPES[c["dw"]]))


def _plain_combine(st):
    c = st["case"]
    live = st["place"] >= 0
    rows = st["Y"][st["place"].clamp(min=0).long()].float()
    w = torch.where(live, st["weight"], 0.0)
    out = dict(out=(rows * w[:, :, None]).sum(1).to(st["Y"].dtype))
    if c["kind"] == "combine_grad":
        g = st["g_out"].float()
        out["g_weight"] = torch.where(live, (rows * g[:, None, :]).sum(2), 0.0)
        spare = st["Y"].shape[0]  # (where the rows of dropped choices go)
        dY = torch.zeros(spare + 1, c["m"], dtype=st["Y"].dtype, device="cuda")
        dY[torch.where(live, st["place"], spare).long()] = (g[:, None, :] * w[:, :, None]).to(dY.dtype)
        out["dY"] = dY[:spare]
    return out


def _plain_clip(st):
    norm = torch.stack([t.float().square().sum() for t in st["tensors"]]).sum().sqrt()
    factor = (st["limit"] / norm).clamp(max=1.0)
    to = st["tensors"] if st["out"] is None else st["out_tensors"]
    [o.copy_(t.float() * factor) for o, t in zip(to, st["tensors"])]
    return dict(norm=norm.reshape(1), factor=factor.reshape(1), tensors=st["flat"] if st["out"] is None else st["out"])


# ---- the framework's calls -------------------------------------------------------------------------------------------

def _own_handle(st):
    """The buffers that a program keeps for calls of one size; made at the first call."""
    from paper_2605_08793_amd.experts import ExpertCombine, ExpertOrder, ExpertProduct, GradClip
    c, kind = st["case"], st["case"]["kind"]
    if kind == "order":
        st["op"] = ExpertOrder(c["n"], c["k"], c["experts"])
    elif kind == "clip":
        st["op"] = GradClip(st["tensors"], out=st.get("out_tensors"))
    elif kind in ("combine", "combine_grad"):
        st["op"] = ExpertCombine(c["n"], c["k"], c["m"], dtype=st["Y"].dtype)
        if kind == "combine_grad":
            st["op"].dY = torch.zeros_like(st["Y"])  # (rows that nobody chose stay as they are)
    elif kind == "product":
        st["op"] = ExpertProduct(c["n"] * c["k"], c["m"], c["d"], c["experts"], gated=c["gated"], keep=c["keep"], dtype=st["X"].dtype)
    else:
        st["op"] = ExpertProduct(c["n"] * c["k"], c["m"], c["d"], c["experts"], dtype=st["X"].dtype, grad_dtype=_TYPES[c["dw"]])
    return st["op"]


def _own_run(st):
    c, kind = st["case"], st["case"]["kind"]
    op = st.get("op") or _own_handle(st)
    if kind == "order":
        op.sort(st["idx"])
        return dict(start=op.start, order=op.order, place=op.place)
    if kind == "clip":
        op.clip(st["limit"])
        return dict(norm=op.norm_out, factor=op.factor, tensors=st["flat"] if st["out"] is None else st["out"])
    if kind in ("combine", "combine_grad"):
        op.combine(st["Y"], st["place"], st["weight"])
        out = dict(out=op.out)
        if kind == "combine_grad":
            op.grad(st["g_out"], st["Y"], st["place"], st["weight"])
            out["g_weight"], out["dY"] = op.g_weight, op.dY
        return out
    if kind == "product":
        op.product(st["X"], st["W"], st["start"], order=st["order"], k=c["k"])
        return dict(Y=op.Y, saved=op.saved) if c["keep"] else dict(Y=op.Y)
    if c["behind_gate"]:
        op.input_grad(st["g_Y"], st["W"], st["start"], saved=st["saved"])
        op.weight_grad(st["g_Y"], st["X"], st["start"])
    else:
        op.input_grad(st["g_Y"], st["W"], st["start"])
        op.weight_grad(st["g_Y"], st["X"], st["start"], order=st["order"], k=c["k"])
    return dict(dX=op.dX, dW=op.dW)


def run(state):
    if own:
        return _own_run(state)
    return {"order": _plain_order, "product": _plain_product, "product_grad": _plain_product_grad, "combine": _plain_combine,
            "combine_grad": _plain_combine, "clip": _plain_clip}[state["case"]["kind"]](state)


# ---- the definitions in 64 bits --------------------------------------------------------------------------------------

def _exact_product(c, st):
    out = dict(Y=torch.empty(c["n"] * c["k"], c["m"], dtype=torch.float64, device="cuda"))
    if c["keep"]:
        out["saved"] = torch.empty(c["n"] * c["k"], 2 * c["m"], dtype=torch.float64, device="cuda")
    at = st["start"].tolist()
    for e in range(c["experts"]):
        mine = slice(at[e], at[e + 1])
        token = torch.div(st["order"][mine].long(), c["k"], rounding_mode="floor")
        Z = st["X"].index_select(0, token).double() @ st["W"][e].double().t()
        if c["gated"]:
            out["Y"][mine] = torch.nn.functional.silu(Z[:, :c["m"]]) * Z[:, c["m"]:]
            if c["keep"]:
                out["saved"][mine] = Z
        else:
            out["Y"][mine] = Z
    return out


def _exact_product_grad(c, st):
    rows = c["n"] * c["k"]
    dX = torch.empty(rows, 2 * c["d"] if c["behind_gate"] else c["d"], dtype=torch.float64, device="cuda")
    dW = torch.empty(c["experts"], c["m"], c["d"], dtype=torch.float64, device="cuda")
    at = st["start"].tolist()
    for e in range(c["experts"]):
        mine = slice(at[e], at[e + 1])
        G = st["g_Y"][mine].double()
        D = G @ st["W"][e].double()
        if c["behind_gate"]:
            s = st["saved"][mine].double().requires_grad_(True)
            h = torch.nn.functional.silu(s[:, :c["d"]]) * s[:, c["d"]:]
            D = torch.autograd.grad(h, s, D)[0]
            X = st["X"][mine].double()
        else:
            X = st["X"].index_select(0, torch.div(st["order"][mine].long(), c["k"], rounding_mode="floor")).double()
        dX[mine] = D
        dW[e] = G.t() @ X
    return dict(dX=dX, dW=dW)


def _exact_combine(c, st):
    out = torch.zeros(c["n"], c["m"], dtype=torch.float64, device="cuda")
    g_weight = torch.zeros(c["n"], c["k"], dtype=torch.float64, device="cuda")
    dY = torch.zeros(c["n"] * c["k"], c["m"], dtype=torch.float64, device="cuda") if c["kind"] == "combine_grad" else None
    for l in range(c["k"]):
        for i in range(0, c["n"], 8192):
            p = st["place"][i:i + 8192, l].long()
            live = torch.nonzero(p >= 0)[:, 0]
            w = st["weight"][i + live, l, None].double()
            rows = st["Y"][p[live]].double()
            out[i + live] += w * rows
            if dY is not None:
                g = st["g_out"][i + live].double()
                g_weight[i + live, l] = torch.linalg.vecdot(rows, g)
                dY[p[live]] = w * g
    return dict(out=out) if dY is None else dict(out=out, g_weight=g_weight, dY=dY)


def _exact_clip(c, st):
    norm = math.sqrt(math.fsum(float(torch.linalg.vector_norm(t, dtype=torch.float64)) ** 2 for t in st["tensors"]))
    factor = st["limit"] / norm if norm > st["limit"] else 1.0
    whole = torch.zeros_like(st["flat"], dtype=torch.float64) if c["kept"] else st["flat"].double()
    at = 0
    for t in st["tensors"]:
        whole[at:at + t.numel()] = t.double() * factor
        at += (t.numel() + 63) // 64 * 64
    number = lambda v: torch.tensor([v], dtype=torch.float64, device="cuda")  # noqa: E731
    return dict(norm=number(norm), factor=number(factor), tensors=whole)


def exact(case, seed):
    if case["kind"] == "order":
        return None
    st = prepare(case, seed)
    return {"product": _exact_product, "product_grad": _exact_product_grad, "combine": _exact_combine, "combine_grad": _exact_combine,
            "clip": _exact_clip}[case["kind"]](case, st)
