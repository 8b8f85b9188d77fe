"""The balance loss and its gradient at logits and factors far from 1, against plain forms in 64 bits.

Tolerances as derived in tests/test_gpu_router.py (K of the parts' magnitudes, the types' roundings).  A score that counts as 0
is below 2^-126 of its row's largest; its gradient is that times the row's factors, which are not below 1 here: `factor`."""
import numpy as np
import pytest
import torch

from paper_2004_13336_b200 import binding as B
from tests import _regularizer_ref as R
from tests.test_gpu_router import BF16, DEV, F32, K, TINY, f64, make, np_lists, np_valid
from tests._util import to_np

pytestmark = pytest.mark.gpu


def call(picks, logits, dlogits, valid, experts, score="softmax", coef=1e-2, z=0.0, upstream=None, loss=True):
    routers = B.RouterSet(experts, picks, valid, logits, dlogits, score)
    counts = torch.empty(len(logits), experts + 1, dtype=torch.int64, device=DEV)
    B.ws_router_counts(routers, counts)
    got = torch.full((len(logits), 2), float("nan"), device=DEV) if loss else None
    ws = torch.full((routers.workspace_bytes(),), 255, dtype=torch.uint8, device=DEV)
    B.ws_balance_loss(routers, counts, got, coef, z, upstream, False, ws)
    return got, counts


def expect_gradient(t, want, size, factor):
    bound = K * size
    bound = bound + torch.finfo(t.dtype).eps / 2 * (np.abs(want) + bound) + TINY * factor
    assert (np.abs(f64(t) - want) <= bound).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("top", [1e3, -1e4, 1.04e6, -1.06e6, 3e8, -3e8, 6e9, -6e9, 1e10, -1e10, 1e15, -1e15, -1e30, 9e36, -9e36, 2e38])
def test_rows_whose_largest_logit_is_far_from_zero(top, dtype):
    """Experts masked with a large finite number, rows of nothing else among them: they are a softmax like any other.  The z loss
    where the logits' squares and their sum are fp32 numbers."""
    picks, logits, dlogits, _, _ = make(1, [40], 32, 2, dtype)
    x = logits[0][0]
    x[0] = top
    x[1, ::2] = top
    x[2, 3:] = top
    x[3] = top
    x[3, 7] = -float("inf")
    x[4] = -abs(top)
    x[4, 9] = abs(top)
    # distinct logits next to the largest one, some units of the type's last place apart
    x[5:8] = (top + abs(top) * torch.finfo(dtype).eps * torch.arange(-48, 48, device=DEV).view(3, 32)).to(dtype)
    z = 1e-3 if abs(top) <= 1e15 else 0.0
    got, counts = call(picks, logits, dlogits, None, 32, z=z)
    ref, grads, sizes = R.balance(np_lists(logits), None, to_np(counts), 2, "softmax", 1e-2, z)
    # the row's factors 2 z / N |lse| + coef E / N (N = 40), and 2^(2^-4) where all exponents of a row are off by 2^-4
    expect_gradient(dlogits[0][0], grads[0][0], sizes[0][0], 2 ** 0.0625 * (2 * z / 40 * (abs(top) * 1.01 + 4) + 0.008))
    _, lse, _, far = R.scores(f64(x), "softmax")
    bound = K * np.array([ref[0, 0], 2 * z / 40 * (np.abs(lse) * (np.abs(lse) + far + 1)).sum()]) + 2.0 ** -24 * ref[0]
    assert (np.abs(f64(got)[0] - ref[0]) <= bound).all()
    assert bool(torch.isfinite(got).all()) and bool(torch.isfinite(dlogits[0][0]).all())


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("up", [float("inf"), -float("inf"), float("nan")])
def test_factors_that_are_no_numbers_leave_rows_without_scores_at_0(up, dtype, score):
    """An overflowed loss scale shows in the valid rows; masked tokens and rows that leave no expert have gradient 0, and a layer
    without tokens has nothing else."""
    for experts, tokens in ((24, [90, 33]), (33, [90, 33]), (64, [3000, 10])):
        picks, logits, dlogits, valid, _ = make(2, tokens, experts, 2, dtype, valid=0.8)
        empty = torch.zeros(tokens[0], dtype=torch.bool, device=DEV)
        empty[::7] = True
        for layer in logits:
            layer[0][empty] = -float("inf")
        z = 1e-3 if score == "softmax" else 0.0
        call(picks, logits, dlogits, valid, experts, score, z=z, upstream=torch.tensor([up], device=DEV))
        for layer in dlogits:
            gone = empty | ~valid[0]
            assert bool((layer[0][gone] == 0).all()) and not bool(torch.isfinite(layer[0][~gone]).all(1).any())
            assert not bool(torch.isfinite(layer[1]).all(1).any())
        none = [torch.zeros(n, dtype=torch.uint8, device=DEV) for n in tokens]
        call(picks, logits, dlogits, none, experts, score, z=z, upstream=torch.tensor([up], device=DEV))
        assert not any(bool(t.any()) for layer in dlogits for t in layer)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_coefficients_past_fp32_with_a_small_factor(score):
    """coef and z_coef are 64-bit numbers: only their products with the factor have to be fp32 numbers."""
    for scale in (1e40, 1e-50):
        picks, logits, dlogits, valid, _ = make(1, [90, 33], 24, 2, valid=0.8)
        z = scale * 0.1 if score == "softmax" else 0.0
        up = torch.tensor([1e-10 if scale > 1 else 1e30], device=DEV)
        _, counts = call(picks, logits, dlogits, valid, 24, score, scale, z, up, loss=False)
        _, grads, sizes = R.balance(np_lists(logits), np_valid(valid), to_np(counts), 2, score, scale, z, float(up))
        for k in range(2):
            expect_gradient(dlogits[0][k], grads[0][k], sizes[0][k], max(1.0, float(up) * scale * 100))


@pytest.mark.parametrize("experts", [2, 7, 64, 256])
def test_z_loss_where_one_expert_has_nearly_everything(experts):
    """Rows 0, -t, -infinity ...: lse = log(1 + exp(-t)), read off the z loss's gradient 2 / N lse p.  1 + exp(-t) is rounded by 2^-24 at
    most; exp(-t) <= 0.0068 is off by 2^-19 of itself, the logarithm and the products by 2^-21 of lse <= 0.0068: 2^-25 together."""
    n = 4096
    t = torch.linspace(5, 12, n, device=DEV)
    x = torch.full((n, experts), -float("inf"), device=DEV)
    x[:, 0], x[:, -1] = 0, -t
    d = torch.empty_like(x)
    counts = torch.full((1, experts + 1), n, dtype=torch.int64, device=DEV)
    routers = B.RouterSet(experts, logits=[[x]], dlogits=[[d]], topk=1)
    B.ws_balance_loss(routers, counts, None, 0.0, 1.0, workspace=torch.empty(routers.workspace_bytes(), dtype=torch.uint8, device=DEV))
    two = torch.stack([torch.zeros_like(t), -t], 1).double()
    lse = d[:, 0].double() * (n / 2) / torch.softmax(two, 1)[:, 0]
    assert float((lse - torch.logsumexp(two, 1)).abs().max()) <= 2.0 ** -24 + 2.0 ** -25


def test_balance_loss_finds_its_own_scratch():
    """Without a workspace, eager and captured: the same bits as with one."""
    picks, logits, dlogits, valid, _ = make(3, [5000, 17], 64, 2, valid=0.8)
    want, counts = call(picks, logits, dlogits, valid, 64, z=1e-3)
    first = [t.clone() for layer in dlogits for t in layer]
    routers = B.RouterSet(64, picks, valid, logits, dlogits)
    loss = torch.empty_like(want)
    B.ws_balance_loss(routers, counts, loss, 1e-2, 1e-3)
    assert torch.equal(loss, want)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.ws_balance_loss(routers, counts, loss, 1e-2, 1e-3)
    for _ in range(2):
        loss.fill_(9)
        for layer in dlogits:
            for t in layer:
                t.fill_(9)
        graph.replay()
        assert torch.equal(loss, want) and all(torch.equal(a, b) for a, b in zip(first, (t for layer in dlogits for t in layer)))
    with pytest.raises(B.WsError):
        B.ws_balance_loss(B.RouterSet(64, picks), counts, loss, 1e-2)          # no logits
