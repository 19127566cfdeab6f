"""Balanced targets and balanced routing: the solver's column duals beside a model's scores.

    python -m paper_2605_08793_amd.balanced

Three uses of one idea.  Scores of n rows against m columns are the negative costs of a transport problem with uniform
marginals; its column duals beta, added to the scores, spread the rows evenly over the columns.

`train_student`: a teacher's scores of samples against prototypes are balanced by a few Sinkhorn sweeps; the best columns of
each row under those duals (RowLogprob with bias) are the targets that a linear student learns (RowDistill: loss and
gradient in one call), and its answers are looked at with RowLogprob.

`route_tokens`: a router's scores of tokens against experts are balanced in the same way; RowRoute takes the duals as its
bias, and regot_pattern_transpose puts the choices into the order of the experts.

`train_experts`: a layer of gated experts behind such a router learns a map.  ExpertOrder puts the choices into the order of the experts,
ExpertProduct multiplies each expert's tokens by its weights, ExpertCombine adds a token's answers up under the router's weights; their
gradients lead back to the weights and, through RowRoute, to the router, and GradClip bounds the norm of a step.
"""
import torch

from . import binding as B
from .driver import DualPass
from .experts import ExpertCombine, ExpertOrder, ExpertProduct, GradClip
from .rows import RowDistill, RowLogprob, RowRoute


def column_duals(scores, eta: float, sweeps: int):
    """Duals beta (m, fp32) of the columns: rows and columns with uniform marginals, costs = -scores."""
    n, m = scores.shape
    M = (-scores).double().contiguous()
    a = torch.full((n,), 1.0 / n, dtype=torch.float64, device=M.device)
    b = torch.full((m,), 1.0 / m, dtype=torch.float64, device=M.device)
    _, beta = DualPass(n, m, device=M.device).sinkhorn_sweeps(M, a, b, eta, sweeps)
    return beta.float()


def train_student(n=2048, m=1500, features=96, k=16, eta=0.1, sweeps=10, steps=60, rate=300.0, dtype=torch.bfloat16, seed=0):
    """Returns the mean loss of each step, the share of the most used column with and without the duals, and the student's
    mean entropy and log probability of the teacher's best column at the end."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    X = torch.nn.functional.normalize(torch.randn(n, features, generator=gen, device="cuda"), dim=1)
    prototypes = torch.nn.functional.normalize(torch.randn(m, features, generator=gen, device="cuda"), dim=1)
    prototypes *= 0.5 + 2.5 * torch.rand(m, 1, generator=gen, device="cuda") ** 8  # (long ones take most rows)
    teacher = (X @ prototypes.t()).to(dtype)

    beta = column_duals(teacher, eta, sweeps)
    targets, plain = (RowLogprob(n, m, k=k, targets=0, dtype=dtype) for _ in range(2))
    targets.logprob(teacher, eta=eta, bias=beta)
    plain.logprob(teacher, eta=eta)
    most = [float(torch.bincount(t.top_idx[:, 0].long(), minlength=m).max()) / n for t in (targets, plain)]

    W = torch.zeros(features, m, device="cuda")
    step, answer = RowDistill(n, m, k, dtype=dtype), RowLogprob(n, m, targets=1, dtype=dtype)
    weight = torch.full((n,), 1.0 / n, device="cuda")
    losses = []
    best = targets.top_idx[:, :1].contiguous()
    for _ in range(steps):
        scores = (X @ W).to(dtype)
        # (log probabilities are scores at temperature 1, which is the student's)
        step.distill(scores, targets.top_idx, targets.top_logprob, row_weight=weight)
        W -= rate * (X.t() @ step.grad.float())
        losses.append(step.loss.mean())
    answer.logprob((X @ W).to(dtype), best)
    return dict(loss=torch.stack(losses).tolist(), most_balanced=most[0], most_plain=most[1],
                entropy=float(answer.entropy.mean()), logprob=float(answer.logprob_out.mean()))


def route_tokens(n=4096, experts=64, k=2, sweeps=8, dtype=torch.float32, seed=0):
    """Returns the tokens of the most used expert over the mean, with the duals as bias and without, the tokens in the order of their
    experts, where each expert's begin, and the weights' gradient to the scores."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    scores = (torch.randn(n, experts, generator=gen, device="cuda") + torch.randn(experts, generator=gen, device="cuda")).to(dtype)
    beta = column_duals(scores, 1.0, sweeps)
    balanced, plain = RowRoute(n, experts, k, bias_on="logit", dtype=dtype), RowRoute(n, experts, k, dtype=dtype)
    balanced.route(scores, bias=beta)
    plain.route(scores)
    load = [float(torch.bincount(r.idx.reshape(-1).long(), minlength=experts).max()) * experts / (n * k) for r in (balanced, plain)]

    row_ptr = torch.arange(0, n * k + 1, k, dtype=torch.int64, device="cuda")
    col_idx = balanced.idx.sort(dim=1).values.reshape(-1)  # (a pattern's columns ascend in its rows)
    start = torch.empty(experts + 1, dtype=torch.int64, device="cuda")
    tokens = torch.empty(n * k, dtype=torch.int32, device="cuda")
    place = torch.empty(n * k, dtype=torch.int64, device="cuda")
    ws = torch.empty(max(B.regot_pattern_transpose_workspace_bytes(n, experts, n * k), 256), dtype=torch.uint8, device="cuda")
    B.regot_pattern_transpose(n, experts, n * k, row_ptr, col_idx, start, tokens, place, workspace=ws)
    grad = balanced.grad(scores, torch.ones_like(balanced.weight))
    return dict(load_balanced=load[0], load_plain=load[1], start=start, tokens=tokens, idx=balanced.idx, weight=balanced.weight, grad=grad)


class ExpertLayer:
    """A gated layer of n tokens: k of `experts` experts each, features -> 2 x hidden -> features.

    `forward` leaves the answers in .out, `backward` the gradients in .grads: of W_up (experts, 2 hidden, features), of W_down (experts, features, hidden), of
    the router's scores, and of the tokens as the experts take them."""

    def __init__(self, n, features, hidden, experts, k, dtype=torch.bfloat16):
        self.k = k
        self.route = RowRoute(n, experts, k, bias_on="logit", dtype=torch.float32)
        self.order = ExpertOrder(n, k, experts)
        self.up = ExpertProduct(n * k, hidden, features, experts, gated=True, keep=True, dtype=dtype, grad_dtype=torch.float32)
        self.down = ExpertProduct(n * k, features, hidden, experts, dtype=dtype, grad_dtype=torch.float32)
        self.total, self.tokens = (ExpertCombine(n, k, features, dtype=dtype) for _ in range(2))
        self.up.dW = torch.empty(experts, 2 * hidden, features, device="cuda")
        self.down.dW = torch.empty(experts, features, hidden, device="cuda")
        self.out = self.total.out

    def forward(self, X, scores, bias, W_up, W_down):
        self.route.route(scores, bias=bias)
        self.order.sort(self.route.idx)
        self.up.product(X, W_up, self.order.start, self.order.order, self.k)
        self.down.product(self.up.Y, W_down, self.order.start)
        self.total.combine(self.down.Y, self.order.place, self.route.weight)

    def backward(self, X, scores, W_up, W_down, g_out):
        start = self.order.start
        self.total.grad(g_out, self.down.Y, self.order.place, self.route.weight)
        self.down.weight_grad(self.total.dY, self.up.Y, start)
        self.down.input_grad(self.total.dY, W_down, start, saved=self.up.saved)
        self.up.weight_grad(self.down.dX, X, start, self.order.order, self.k)
        self.up.input_grad(self.down.dX, W_up, start)
        self.tokens.combine(self.up.dX, self.order.place)
        self.grads = self.up.dW, self.down.dW, self.route.grad(scores, self.total.g_weight), self.tokens.out


def train_experts(n=2048, features=64, hidden=48, experts=16, k=2, sweeps=6, steps=40, rate=4.0, max_norm=0.5, dtype=torch.bfloat16, seed=0):
    """Returns the loss of each step, the gradients' norms before they were clipped, and the tokens of the most used expert over the mean at the end."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    X = torch.randn(n, features, generator=gen, device="cuda")
    wanted = torch.tanh(X @ torch.randn(features, features, generator=gen, device="cuda") * features ** -0.5)
    X = X.to(dtype)
    W_up = torch.randn(experts, 2 * hidden, features, generator=gen, device="cuda") * features ** -0.5
    W_down = torch.randn(experts, features, hidden, generator=gen, device="cuda") * hidden ** -0.5
    R = torch.randn(features, experts, generator=gen, device="cuda") * features ** -0.5

    layer = ExpertLayer(n, features, hidden, experts, k, dtype)
    dR = torch.empty_like(R)
    clip = GradClip([layer.up.dW, layer.down.dW, dR])
    losses, norms = [], []
    for _ in range(steps):
        scores, up, down = X.float() @ R, W_up.to(dtype), W_down.to(dtype)
        layer.forward(X, scores, column_duals(scores, 1.0, sweeps), up, down)
        off = layer.out.float() - wanted
        layer.backward(X, scores, up, down, (off / n).to(dtype))
        torch.mm(X.float().t(), layer.grads[2], out=dR)
        clip.clip(max_norm)
        for W, g in ((W_up, layer.up.dW), (W_down, layer.down.dW), (R, dR)):
            W -= rate * g
        losses.append(0.5 * off.square().sum(1).mean())
        norms.append(clip.norm_out.clone())
    load = (layer.order.start[1:] - layer.order.start[:-1]).max() * experts / (n * k)
    return dict(loss=torch.stack(losses).tolist(), norm=torch.cat(norms).tolist(), load=float(load))


if __name__ == "__main__":
    s = train_student()
    print(f"student: loss {s['loss'][0]:.4f} -> {s['loss'][-1]:.4f}, entropy {s['entropy']:.3f}, log probability of the target {s['logprob']:.3f}; "
          f"most used column {100 * s['most_plain']:.2f} % of the rows, balanced {100 * s['most_balanced']:.2f} %")
    r = route_tokens()
    print(f"router: most used expert {r['load_plain']:.2f} times the mean, balanced {r['load_balanced']:.2f}")
    e = train_experts()
    print(f"experts: loss {e['loss'][0]:.3f} -> {e['loss'][-1]:.3f}, norm of the gradients {e['norm'][0]:.3f} -> {e['norm'][-1]:.3f}, most used expert {e['load']:.2f} times the mean")
