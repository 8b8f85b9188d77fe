"""Counts of the experts' picks and the balance loss with its gradient on the GPU against plain forms in 64 bits.

Tolerance of a gradient: its fp32 parts are scores exp(x - top), off by 2^-24 (|x - top| + 2), |x - top| <= 104 where the score
is not 0, sums over at most 1024 experts of at most 32 + 5 additions, and a few products; 200 x 2^-24 of the parts' magnitudes
covers them (half of that for each of the two sums), then the rounding to the type.  The losses are the rows' parts summed in
64 bits, so the same share of their magnitudes, and one rounding.  Below fp32's normal range a relative tolerance says nothing:
a score under 2^-126 of the row's largest counts as 0, which a gradient of parts below 1 shows as at most 2^-126, and the types'
own smallest steps (bf16 2^-133, fp32 2^-149) are smaller than that."""
import numpy as np
import pytest
import torch

from paper_2004_13336_b200 import binding as B
from tests import _regularizer_ref as R
from tests._util import bf16_to_f64, to_np

pytestmark = pytest.mark.gpu
DEV = "cuda"
F32, BF16 = torch.float32, torch.bfloat16
K = 200 * 2.0 ** -24
TINY = 2.0 ** -126


def f64(t):
    return bf16_to_f64(to_np(t)) if t.dtype == BF16 else to_np(t).astype(np.float64)


def make(layers, tokens, experts, topk, dtype=F32, index=torch.int64, valid=None, seed=0, std=2.0, pad=0, shift=0, refused=0.1):
    """Nested lists of picks, logits, dlogits (filled with 55, in buffers with guards), and the valid bytes."""
    gen = torch.Generator(device=DEV).manual_seed(seed)
    picks, logits, dlogits, bufs = [], [], [], []
    for _ in range(layers):
        for lst in (picks, logits, dlogits):
            lst.append([])
        for n in tokens:
            q = torch.stack([torch.randperm(experts, generator=gen, device=DEV)[:topk] for _ in range(min(n, 16))] or [torch.zeros(topk, dtype=torch.int64, device=DEV)])
            q = q[torch.arange(n, device=DEV) % len(q)]
            q = torch.where(torch.rand(q.shape, generator=gen, device=DEV) < refused, -1, q)
            picks[-1].append(q.to(index).contiguous())
            x = torch.empty(n, experts, device=DEV).normal_(0, std, generator=gen).to(dtype)
            buf = torch.full((n * (experts + pad) + shift + 16,), 9.0, dtype=dtype, device=DEV)
            view = buf[shift:shift + n * (experts + pad)].view(n, experts + pad)[:, :experts]
            view.copy_(x)
            logits[-1].append(view)
            buf = torch.full((n * (experts + pad) + shift + 16,), 55.0, dtype=dtype, device=DEV)
            bufs.append(buf)
            dlogits[-1].append(buf[shift:shift + n * (experts + pad)].view(n, experts + pad)[:, :experts])
    if valid is not None:
        valid = [torch.rand(n, generator=gen, device=DEV) < valid if i != 1 else None for i, n in enumerate(tokens)]
    return picks, logits, dlogits, valid, bufs


def np_lists(x):
    return [[f64(t) if t.is_floating_point() else to_np(t) for t in layer] for layer in x]


def np_valid(v):
    return None if v is None else [None if t is None else to_np(t) for t in v]


def check(picks, logits, dlogits, valid, experts, topk, score="softmax", coef=1e-2, z=0.0, upstream=None, before=None, loss=True):
    routers = B.RouterSet(experts, picks, valid, logits, dlogits, score)
    counts = torch.full((len(logits), experts + 1), -3, dtype=torch.int64, device=DEV)
    B.ws_router_counts(routers, counts)
    want = R.counts(np_lists(picks), np_valid(valid), experts)
    assert (to_np(counts) == want).all()
    x = np_lists(logits)
    got = torch.full((len(logits), 2), float("nan"), device=DEV) if loss else None
    ws = torch.full((routers.workspace_bytes(),), 255, dtype=torch.uint8, device=DEV)
    B.ws_balance_loss(routers, counts, got, coef, z, upstream, before is not None, ws)
    ref, grads, sizes = R.balance(x, np_valid(valid), want, topk, score, coef, z, 1.0 if upstream is None else float(upstream))
    if loss:
        lse = [sum(np.sum(np.where(np.isfinite(s := R.scores(t[live_of(np_valid(valid), k, t)], "softmax")[1]), np.abs(s) * (np.abs(s) + R.scores(t[live_of(np_valid(valid), k, t)], "softmax")[3] + 1), 0))
                   for k, t in enumerate(layer)) for layer in x] if z else [0.0] * len(x)
        inv = np.array([1.0 / max(1, n) for n in want[:, -1]])
        bound = K * np.stack([np.abs(ref[:, 0]), 2 * z * inv * np.array(lse)], 1) + 2.0 ** -24 * np.abs(ref)
        assert (np.abs(f64(got) - ref) <= bound).all(), (f64(got), ref)
    if dlogits is not None:
        for l, layer in enumerate(dlogits):
            for k, t in enumerate(layer):
                old = 0.0 if before is None else f64(before[l][k])
                w = grads[l][k] + old
                bound = K * sizes[l][k] + 2.0 ** -24 * np.abs(old)
                bound = bound + torch.finfo(t.dtype).eps / 2 * (np.abs(w) + bound) + TINY
                assert (np.abs(f64(t) - w) <= bound).all(), (l, k)
    return got, counts, routers


def live_of(valid, k, t):
    return np.ones(len(t), dtype=bool) if valid is None or valid[k] is None else valid[k].astype(bool)


EXPERTS = [(1, 1), (2, 1), (4, 2), (7, 3), (8, 2), (12, 12), (16, 4), (33, 2), (60, 4), (64, 8), (100, 6), (128, 8), (256, 8), (257, 1), (384, 6), (515, 5), (1000, 8), (1024, 32)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("experts,topk", EXPERTS)
def test_numbers_of_experts(experts, topk, dtype):
    picks, logits, dlogits, valid, bufs = make(2, [37, 5, 0, 70], experts, topk, dtype, valid=0.8, seed=experts)
    check(picks, logits, dlogits, valid, experts, topk, z=1e-3 if experts % 2 else 0.0)
    check(picks, logits, dlogits, valid, experts, topk, score="sigmoid")


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("pad,shift", [(0, 0), (8, 0), (3, 0), (0, 1), (8, 8)])
def test_strides_and_alignment(pad, shift, dtype, score):
    picks, logits, dlogits, valid, bufs = make(1, [50, 3], 64, 2, dtype, torch.int32, pad=pad, shift=shift)
    check(picks, logits, dlogits, valid, 64, 2, score)
    for t in dlogits[0]:
        t.fill_(55.0)
    assert all(bool((b == 55.0).all()) for b in bufs)          # nothing between and behind the rows was touched


@pytest.mark.parametrize("tokens", [[0], [1], [1, 0, 2], [0, 0], [4097], [3000, 1, 9000, 255, 257], [1] * 20, [5] * 512])
@pytest.mark.parametrize("index", [torch.int32, torch.int64])
def test_lengths(tokens, index):
    picks, logits, dlogits, valid, _ = make(2 if len(tokens) < 100 else 1, tokens, 16, 2, F32, index, valid=0.7, seed=len(tokens))
    check(picks, logits, dlogits, valid, 16, 2, z=1e-2)


def test_more_layers_than_one_launch_takes():
    picks, logits, dlogits, valid, _ = make(150, [3, 0, 2, 9], 8, 2, BF16, valid=0.7)
    check(picks, logits, dlogits, valid, 8, 2, z=1e-2)


def test_picks_that_are_none_and_picks_twice():
    q = torch.tensor([[0, 0], [3, -1], [-1, -1], [7, 8], [1 << 40, -(1 << 40)], [2, 2]], device=DEV)
    counts = torch.empty(1, 9, dtype=torch.int64, device=DEV)
    B.ws_router_counts(B.RouterSet(8, [[q]]), counts)
    assert counts.tolist() == [[2, 0, 2, 1, 0, 0, 0, 1, 6]]
    B.ws_router_counts(B.RouterSet(8, [[q]]), counts, accumulate=True)
    assert counts.tolist() == [[4, 0, 4, 2, 0, 0, 0, 2, 12]]


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("tokens", [[100], [70000], [9000, 0, 33000]])
def test_counts_with_everything_on_one_expert(tokens, accumulate):
    picks = [[torch.full((n, 2), 5, dtype=torch.int32, device=DEV) for n in tokens] for _ in range(2)]
    counts = torch.full((2, 9), 7, dtype=torch.int64, device=DEV)
    B.ws_router_counts(B.RouterSet(8, picks), counts, accumulate)
    n, c = sum(tokens), 7 if accumulate else 0
    assert counts.tolist() == [[c] * 5 + [c + 2 * n] + [c] * 2 + [c + n]] * 2


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rows_with_masked_experts(dtype, score):
    """-infinity, the type's lowest value, and rows that leave no expert; masked tokens may hold anything."""
    picks, logits, dlogits, _, _ = make(1, [64], 32, 2, dtype)
    x, low = logits[0][0], torch.finfo(dtype).min
    x[0] = -float("inf")
    x[1, 1:] = -float("inf")
    x[2] = low
    x[3, :31] = low
    x[4, ::2] = -float("inf")
    x[5] -= 200
    x[6] = -88.0
    x[7] += 300
    x[8] = 0
    x[9] = float("nan")
    x[10] = float("inf")
    valid = [torch.ones(64, dtype=torch.uint8, device=DEV)]
    valid[0][9:11] = 0
    got, _, _ = check(picks, logits, dlogits, valid, 32, 2, score, z=0.0)
    d = dlogits[0][0]
    assert bool((d[0] == 0).all()) and bool((d[9:11] == 0).all()) and bool((d[4, ::2] == 0).all())
    if score == "softmax":        # the z loss of such rows: without those whose square leaves fp32's range
        x[2], x[3, :31] = 0, -1000
        check(picks, logits, dlogits, valid, 32, 2, score, z=1e-3)


def test_no_tokens_at_all():
    picks, logits, dlogits, _, _ = make(2, [40, 6], 8, 2)
    valid = [torch.zeros(40, dtype=torch.bool, device=DEV), torch.zeros(6, dtype=torch.bool, device=DEV)]
    got, counts, _ = check(picks, logits, dlogits, valid, 8, 2, z=1e-3)
    assert not got.any() and not counts.any() and not any(t.any() for layer in dlogits for t in layer)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_nan_shows(score):
    picks, logits, dlogits, _, _ = make(1, [40], 8, 2)
    logits[0][0][3, 2] = float("nan")
    routers = B.RouterSet(8, picks, None, logits, dlogits, score)
    counts, loss = torch.empty(1, 9, dtype=torch.int64, device=DEV), torch.empty(1, 2, device=DEV)
    ws = torch.empty(routers.workspace_bytes(), dtype=torch.uint8, device=DEV)
    B.ws_router_counts(routers, counts)
    B.ws_balance_loss(routers, counts, loss, 1e-2, workspace=ws)
    assert bool(loss[0, 0].isnan()) and bool(dlogits[0][0][3].isnan().all()) and not dlogits[0][0].isnan()[4:].any()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_gradient_is_added_and_scaled_on_request(dtype):
    picks, logits, dlogits, valid, _ = make(2, [90, 33], 24, 2, dtype, valid=0.8)
    up = torch.tensor([1024.0], device=DEV)
    before = [[t.normal_().clone() for t in layer] for layer in dlogits]
    check(picks, logits, dlogits, valid, 24, 2, z=1e-3, upstream=up, before=before)
    for layer, old in zip(dlogits, before):
        gone = ~valid[0]
        assert torch.equal(layer[0][gone], old[0][gone])          # masked tokens: as it was
    check(picks, logits, dlogits, valid, 24, 2, z=1e-3, upstream=-up, loss=False)
    check(picks, logits, None, valid, 24, 2, z=1e-3, upstream=up)


def test_gradient_in_place_of_the_logits():
    picks, logits, dlogits, valid, _ = make(1, [90, 33], 24, 2)
    _, counts, routers = check(picks, logits, dlogits, valid, 24, 2, z=1e-3)
    same = B.RouterSet(24, picks, valid, logits, logits)
    ws = torch.empty(same.workspace_bytes(), dtype=torch.uint8, device=DEV)
    B.ws_balance_loss(same, counts, None, 1e-2, 1e-3, workspace=ws)
    assert all(torch.equal(a, b) for a, b in zip(logits[0], dlogits[0]))


def test_replicas_one_by_one_add_up():
    """As real replicas run it: each counts its own tokens, the counts are summed, each takes the loss of its own logits."""
    picks, logits, dlogits, valid, _ = make(3, [200, 17, 0, 64], 40, 4, BF16, valid=0.8)
    loss, counts, _ = check(picks, logits, dlogits, valid, 40, 4, z=1e-3)
    total, parts = torch.zeros_like(counts), torch.zeros(3, 2, dtype=torch.float64, device=DEV)
    one = [[[t[k]] for t in picks] for k in range(4)]
    for k in range(4):
        B.ws_router_counts(B.RouterSet(40, one[k], [valid[k]]), total, accumulate=True)
    assert torch.equal(total, counts)
    for k in range(4):
        d = [[torch.empty_like(t[k])] for t in dlogits]
        s = B.RouterSet(40, one[k], [valid[k]], [[t[k]] for t in logits], d)
        part = torch.empty(3, 2, device=DEV)
        B.ws_balance_loss(s, total, part, 1e-2, 1e-3, workspace=torch.empty(s.workspace_bytes(), dtype=torch.uint8, device=DEV))
        parts += part
        assert all(torch.equal(a[0], b[k]) for a, b in zip(d, dlogits))
    np.testing.assert_allclose(parts.cpu().numpy(), f64(loss), rtol=5 * 2.0 ** -24)


def test_same_call_same_bits_and_captured():
    picks, logits, dlogits, valid, _ = make(4, [5000, 3000], 64, 2, valid=0.9)
    loss, counts, routers = check(picks, logits, dlogits, valid, 64, 2, z=1e-3)
    first = [t.clone() for layer in dlogits for t in layer]
    ws = torch.empty(routers.workspace_bytes(), dtype=torch.uint8, device=DEV)
    got, again = torch.empty_like(loss), torch.empty_like(counts)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.ws_router_counts(routers, again)
        B.ws_balance_loss(routers, again, got, 1e-2, 1e-3, workspace=ws)
    for _ in range(3):
        got.fill_(9)
        again.fill_(9)
        ws.fill_(255)
        for t in (t for layer in dlogits for t in layer):
            t.fill_(9)
        graph.replay()
        assert torch.equal(got, loss) and torch.equal(again, counts)
        assert all(torch.equal(a, b) for a, b in zip(first, (t for layer in dlogits for t in layer)))


def test_two_streams_at_once():
    """Two sets, each with its own counts and workspace, against the same calls one after the other."""
    sets = []
    for seed in (1, 2):
        picks, logits, dlogits, valid, _ = make(6, [9000, 5000], 64, 2, seed=seed, valid=0.9)
        routers = B.RouterSet(64, picks, valid, logits, dlogits)
        sets.append((routers, torch.empty(6, 65, dtype=torch.int64, device=DEV), torch.empty(6, 2, device=DEV),
                     torch.empty(routers.workspace_bytes(), dtype=torch.uint8, device=DEV), dlogits))

    def call(routers, counts, loss, ws, dlogits):
        B.ws_router_counts(routers, counts)
        B.ws_balance_loss(routers, counts, loss, 1e-2, 1e-3, workspace=ws)

    want = []
    for s in sets:
        call(*s)
        want.append([s[1].clone(), s[2].clone()] + [t.clone() for layer in s[4] for t in layer])
    for s in sets:
        for t in (s[1], s[2], *(t for layer in s[4] for t in layer)):
            t.zero_()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    for _ in range(5):
        for s, stream in zip(sets, streams):
            with torch.cuda.stream(stream):
                call(*s)
    torch.cuda.synchronize()
    for s, w in zip(sets, want):
        assert all(torch.equal(a, b) for a, b in zip([s[1], s[2]] + [t for layer in s[4] for t in layer], w))


def test_many_small_replicas_and_layers_of_one_call():
    """More (layer, replica) pairs than a launch takes, replicas that share a CTA, one that has nothing."""
    tokens = [3, 0, 1, 7, 2, 11, 0, 5, 4, 1, 1, 6, 9, 2, 8, 3, 2]
    for dtype, score in ((F32, "softmax"), (BF16, "sigmoid")):
        picks, logits, dlogits, valid, _ = make(40, tokens, 24, 3, dtype, torch.int32, valid=0.8)
        check(picks, logits, dlogits, valid, 24, 3, score, z=1e-2 if score == "softmax" else 0.0)


def test_gradient_follows_differences_of_the_loss():
    """Steps of 2^-6 along single logits: (L(x + h) - L(x - h)) / 2h against the gradient.  L is a float32 (2^-24 of it), its
    third derivative at most 6 L per logit, so the difference is off by h^2 L + 2^-24 L / h < 2^-11 L at most."""
    picks, logits, dlogits, valid, _ = make(1, [9], 6, 2, std=1.0)
    _, counts, routers = check(picks, logits, dlogits, valid, 6, 2, coef=1.0)
    x, d = logits[0][0], dlogits[0][0].clone()
    ws, loss, h = torch.empty(routers.workspace_bytes(), dtype=torch.uint8, device=DEV), torch.empty(1, 2, device=DEV), 2.0 ** -6
    for i in (0, 4, 8):
        for e in range(6):
            vals = []
            for sign in (1, -1):
                old = x[i, e].clone()
                x[i, e] = old + sign * h
                step = float(x[i, e] - old)
                B.ws_balance_loss(routers, counts, loss, 1.0, workspace=ws)
                vals.append((float(loss[0, 0]), step))
                x[i, e] = old
            diff = (vals[0][0] - vals[1][0]) / (vals[0][1] - vals[1][1])
            assert abs(diff - float(d[i, e])) < 2.0 ** -11 * vals[0][0]


def test_offsets_past_32_bits():
    """2^31 elements and more in one replica's logits: the last rows against those rows alone."""
    n, experts = (1 << 23) + 77, 256
    gen = torch.Generator(device=DEV).manual_seed(1)
    x = torch.empty(n, experts, dtype=BF16, device=DEV)
    x.normal_(0, 2, generator=gen)
    d = torch.empty_like(x)
    q = torch.topk(x, 2, dim=-1).indices
    routers = B.RouterSet(experts, [[q]], None, [[x]], [[d]])
    counts, loss = torch.empty(1, experts + 1, dtype=torch.int64, device=DEV), torch.empty(1, 2, device=DEV)
    B.ws_router_counts(routers, counts)
    want = torch.bincount(q.view(-1), minlength=experts)
    assert torch.equal(counts[0, :-1], want) and int(counts[0, -1]) == n
    ws = torch.empty(routers.workspace_bytes(), dtype=torch.uint8, device=DEV)
    B.ws_balance_loss(routers, counts, loss, 1e-2, workspace=ws)
    tail = torch.empty(300, experts, dtype=BF16, device=DEV)
    part = B.RouterSet(experts, None, None, [[x[-300:]]], [[tail]], topk=2)
    B.ws_balance_loss(part, counts, None, 1e-2, workspace=ws)
    assert torch.equal(tail, d[-300:])
    f = want.double() / (2 * n)
    s = sum(float((torch.softmax(c.double(), 1) @ f).sum()) for c in x.split(1 << 19))
    assert abs(float(loss[0, 0]) - 1e-2 * experts * s / n) <= (K + 2.0 ** -24) * 1e-2 * experts * s / n


def test_router_of_a_dropped_out_layer_trains():
    """The set together: the router's weight is handed out under dropout, its logits balanced over the replicas, the gradient
    summed under the same masks and applied by the sharded update; against autograd in float64."""
    d_model, experts, topk, replicas, p, coef, z = 32, 16, 2, 3, 0.25, 0.5, 1e-2
    gen = torch.Generator(device=DEV).manual_seed(5)
    plan = B.Plan([(d_model, experts)], 4)
    w0 = torch.empty(d_model * experts, device=DEV).normal_(0, 0.3, generator=gen)
    w, m = torch.empty(plan.G, device=DEV), torch.zeros(plan.G, device=DEV)
    B.ws_pack(plan, [w0], w)
    x = [torch.empty(40 + 9 * k, d_model, device=DEV).normal_(generator=gen) for k in range(replicas)]
    valid = [torch.rand(len(t), generator=gen, device=DEV) < 0.8 for t in x]
    copies, grads = ([torch.empty(d_model * experts, device=DEV) for _ in range(replicas)] for _ in range(2))
    drop = B.make_dropout(p, 6, 1)
    B.ws_unpack_dropout(plan, -1, w, B.TensorTable(plan, [[c] for c in copies]), drop)
    logits = [(t.double() @ c.double().view(d_model, experts)).float() for t, c in zip(x, copies)]
    picks = [torch.topk(t, topk, dim=1).indices for t in logits]
    dlogits = [torch.empty_like(t) for t in logits]
    routers = B.RouterSet(experts, [picks], valid, [logits], [dlogits])
    counts, loss = torch.empty(1, experts + 1, dtype=torch.int64, device=DEV), torch.empty(1, 2, device=DEV)
    B.ws_router_counts(routers, counts)
    B.ws_balance_loss(routers, counts, loss, coef, z, workspace=torch.empty(routers.workspace_bytes(), dtype=torch.uint8, device=DEV))
    for g, t, dl in zip(grads, x, dlogits):
        g.copy_((t.double().t() @ dl.double()).reshape(-1))
    total = torch.empty(plan.G, device=DEV)
    B.ws_reduce_dropout(plan, -1, B.TensorTable(plan, [[g] for g in grads]), drop, total)
    hyper = dict(lr=1.0, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.0, momentum=0.0, grad_scale=1.0, step=1)
    B.ws_shard_update(plan, -1, [total], w, m, None, B.make_hyper("sgdm", hyper))
    out = torch.empty(d_model * experts, device=DEV)
    B.ws_unpack(plan, w, [out])
    leaf = w0.double().requires_grad_()
    f = counts[0, :-1].double() / (topk * counts[0, -1])
    live = torch.cat([(t.double() @ (leaf * torch.from_numpy(R.keep(p, 6, 1, k, 0, leaf.numel())).to(DEV) * R.scale(p)).view(d_model, experts))[valid[k]]
                      for k, t in enumerate(x)])
    want = coef * experts * (f * torch.softmax(live, 1).mean(0)).sum() + z * torch.logsumexp(live, 1).square().mean()
    want.backward()
    step = (out.double() - w0.double())
    # the gradient's errors (K of its parts, summed over the tokens) and the weight's rounding
    bound = 4 * K * leaf.grad.abs().max() * 10 + 2.0 ** -23 * w0.abs().max()
    assert float((step + leaf.grad).abs().max()) < float(bound)
    want = float(want.detach())
    assert abs(float(loss.sum()) - want) < 4 * K * want
