"""What the row calls refuse, before anything is enqueued (no GPU needed)."""
import ctypes

import pytest
import torch

from paper_2605_08793_amd import binding as B

P = ctypes.c_void_p(0x10000)     # never dereferenced
ODD = ctypes.c_void_p(0x10001)
HALF = ctypes.c_void_p(0x10002)
WS = ctypes.c_void_p(0x20000)
BIG = 1 << 40
NULL, DIM, ETA, LD, ALIGN, WORKSPACE, ARG = -1, -2, -3, -4, -5, -6, -7

LOGPROB = dict(n=4, m=8, S=P, type=0, ldS=8, bias=P, eta=1.0, target=P, targets=1, k=2, logprob=P, entropy=P, stats=P, top_idx=P,
               top_logprob=P, ws=WS, ws_bytes=BIG, stream=None)
LOGPROB_GRAD = dict(n=4, m=8, S=P, type=0, ldS=8, bias=P, eta=1.0, target=P, targets=1, stats=P, entropy=P, g_logprob=P, g_entropy=P, dS=P,
                    ldD=8, stream=None)
DISTILL = dict(n=4, m=8, S=P, type=0, ldS=8, eta=1.0, t_idx=P, t_score=P, k=2, row_weight=P, loss=P, dS=P, ldD=8, ws=WS, ws_bytes=BIG,
               stream=None)
ROUTE = dict(n=4, m=8, S=P, type=0, ldS=8, bias=P, bias_on=0, score=0, groups=2, groups_kept=1, group_by=0, k=2, renormalise=1, scale=1.0,
             idx=P, weight=P, stream=None)
ROUTE_GRAD = dict(n=4, m=8, S=P, type=0, ldS=8, score=0, idx=P, k=2, renormalise=1, scale=1.0, g_weight=P, dS=P, ldD=8, stream=None)
CALLS = {"regot_row_logprob": LOGPROB, "regot_row_logprob_grad": LOGPROB_GRAD, "regot_row_distill": DISTILL, "regot_row_route": ROUTE,
         "regot_row_route_grad": ROUTE_GRAD}

REFUSED = [("regot_row_logprob", a, s) for a, s in [
    (dict(targets=-1), ARG), (dict(targets=1025), ARG), (dict(k=-1), ARG), (dict(k=129), ARG), (dict(target=None), NULL), (dict(logprob=None), NULL),
    (dict(top_idx=None), NULL), (dict(top_logprob=None), NULL), (dict(ws=None), NULL), (dict(ws=P, ws_bytes=0), WORKSPACE),
    (dict(ws=ctypes.c_void_p(0x20010)), ALIGN), (dict(target=HALF), ALIGN), (dict(bias=HALF), ALIGN), (dict(stats=HALF), ALIGN)]] + [
    ("regot_row_logprob_grad", a, s) for a, s in [
        (dict(targets=1025), ARG), (dict(stats=None), NULL), (dict(target=None), NULL), (dict(g_logprob=None), NULL), (dict(entropy=None), NULL),
        (dict(dS=None), NULL), (dict(ldD=7), LD), (dict(dS=HALF), ALIGN), (dict(dS=ODD, type=1), ALIGN), (dict(g_entropy=HALF), ALIGN)]] + [
    ("regot_row_distill", a, s) for a, s in [
        (dict(k=0), ARG), (dict(k=1025), ARG), (dict(t_idx=None), NULL), (dict(t_score=None), NULL), (dict(loss=None), NULL), (dict(ldD=7), LD),
        (dict(ws=None), NULL), (dict(ws_bytes=0), WORKSPACE), (dict(loss=HALF), ALIGN), (dict(row_weight=HALF), ALIGN)]] + [
    ("regot_row_route", a, s) for a, s in [
        (dict(m=1025, ldS=1025), DIM), (dict(k=0), ARG), (dict(k=33), ARG), (dict(score=2), ARG), (dict(bias_on=2), ARG), (dict(groups=0), ARG),
        (dict(groups=65), ARG), (dict(groups=3), ARG), (dict(groups_kept=0), ARG), (dict(groups_kept=3), ARG), (dict(group_by=2), ARG),
        (dict(renormalise=2), ARG), (dict(scale=float("nan")), ARG), (dict(scale=1e300), ARG), (dict(idx=None), NULL), (dict(weight=None), NULL),
        (dict(idx=HALF), ALIGN)]] + [
    ("regot_row_route_grad", a, s) for a, s in [
        (dict(m=1025, ldS=1025, ldD=1025), DIM), (dict(k=0), ARG), (dict(k=33), ARG), (dict(score=-1), ARG), (dict(idx=None), NULL),
        (dict(g_weight=None), NULL), (dict(dS=None), NULL), (dict(ldD=7), LD), (dict(scale=float("inf")), ARG)]]


def call(name, **changed):
    args = {**CALLS[name], **changed}
    assert set(args) == set(CALLS[name])
    return getattr(B.load(), name)(*args.values())


@pytest.mark.parametrize("name", sorted(CALLS))
def test_scores_and_eta(name):
    for changed, status in ((dict(n=-1), DIM), (dict(m=-1), DIM), (dict(n=1 << 31), DIM), (dict(type=3), ARG), (dict(type=-1), ARG), (dict(S=None), NULL),
                            (dict(ldS=7), LD), (dict(S=HALF), ALIGN), (dict(S=ODD, type=1), ALIGN)):
        assert call(name, **changed) == status, changed
    if "eta" in CALLS[name]:
        for eta in (0.0, -1.0, float("nan"), float("inf"), 1e-60, 1e60):
            assert call(name, eta=eta) == ETA, eta


@pytest.mark.parametrize("name,changed,status", REFUSED)
def test_refused(name, changed, status):
    assert call(name, **changed) == status


@pytest.mark.parametrize("name", sorted(CALLS))
def test_nothing_to_do_is_fine(name):
    for m in (0, 8, 1000, 1 << 20, (1 << 31) - 1):
        if m > 1024 and "route" in name:
            continue
        changed = dict(n=0, m=m, ldS=m)
        if "ldD" in CALLS[name]:
            changed["ldD"] = m
        assert call(name, **changed) == 0


def test_workspaces_of_all_sizes():
    """Asked for on the host for any size; for k alternatives no smaller than for none, and a small part of the scores."""
    for n in (0, 1, 2, 63, 96, 97, 192, 193, 10 ** 6):
        for m in (0, 1, 4097, 53248, 131072, 10 ** 6, (1 << 31) - 1):
            none, some = B.regot_row_logprob_workspace_bytes(n, m, 0), B.regot_row_logprob_workspace_bytes(n, m, 20)
            assert 256 <= none <= some <= 256 + n * (64 * 12 + 32 * 1024) + 512
            assert 256 <= B.regot_row_distill_workspace_bytes(n, m, 20) <= 256 + n * 64 * 12 + 512


def test_workspaces():
    assert B.regot_row_logprob_workspace_bytes(0, 0, 0) >= 0
    for f, least in ((B.load().regot_row_logprob_workspace_bytes, 0), (B.load().regot_row_distill_workspace_bytes, 1)):
        out = ctypes.c_size_t()
        assert f(4, 8, 5, ctypes.byref(out)) == 0 and out.value % 256 == 0
        assert f(4, 8, 5, None) == NULL
        assert f(-1, 8, 5, ctypes.byref(out)) == DIM and f(4, 1 << 31, 5, ctypes.byref(out)) == DIM
        assert f(4, 8, least - 1, ctypes.byref(out)) == ARG and f(4, 8, 5000, ctypes.byref(out)) == ARG


class FakeCuda(torch.Tensor):
    """A CPU tensor that says it is on the GPU: the checks of shape, type and layout look at nothing else."""
    @property
    def is_cuda(self):
        return True


def fake(*shape, dtype=torch.float32):
    return torch.zeros(*shape, dtype=dtype).as_subclass(FakeCuda)


def test_the_binding_checks_tensors():
    with pytest.raises(TypeError):
        B._scores(torch.zeros(3, 4))
    with pytest.raises(TypeError):
        B._scores(fake(3, 4, dtype=torch.float64))
    with pytest.raises(TypeError):
        B._scores(fake(3, 4).t())
    with pytest.raises(TypeError):
        B._scores(fake(1, 4).expand(3, 4))
    with pytest.raises(TypeError):
        B._scores(fake(12))
    assert B._scores(fake(3, 9)[:, 2:6])[:4] == (3, 4, 0, 9)
    assert B._scores(fake(1, 9)[:, 2:6])[:4] == (1, 4, 0, 4)
    for bad in (fake(3, 2), fake(3, 4, dtype=torch.int64), fake(4, 3).t(), torch.zeros(3, 4), None):
        with pytest.raises(TypeError):
            B._list(bad, 3, 4, "list")
    assert B._list(None, 3, 4, "list", optional=True) == 0
    with pytest.raises(TypeError):
        B._width(fake(4, 2), 3, "list")
    with pytest.raises(TypeError):
        B._same_scores(fake(3, 4, dtype=torch.bfloat16), fake(3, 4))
