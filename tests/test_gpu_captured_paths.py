"""The framework's own paths captured in CUDA graphs and replayed, on a one-rank NCCL group."""
import socket

import numpy as np
import pytest
import torch
import torch.distributed as dist

from tests import _regularizer_ref as R

pytestmark = pytest.mark.gpu
DEV = "cuda"
SHAPES = [(1,), (7,), (3, 3, 16, 32), (64, 128), (1031,), (0, 3), (300, 301)]


@pytest.fixture(scope="module")
def world_of_one():
    with socket.socket() as s:
        s.bind(("127.0.0.1", 0))
        port = s.getsockname()[1]
    torch.cuda.set_device(0)
    dist.init_process_group("nccl", init_method=f"tcp://127.0.0.1:{port}", rank=0, world_size=1)
    yield
    dist.destroy_process_group()


def test_replayed_step_with_dropout_draws_new_masks(world_of_one):
    """Eager steps and replays in turn follow the plain run, whose masks move on by one with every step."""
    from paper_2004_13336_b200 import binding as B
    from paper_2004_13336_b200.collective import ShardedUpdate
    p, seed = 0.2, 31
    n = [int(np.prod(s)) for s in SHAPES]
    gen = torch.Generator(device=DEV).manual_seed(2)
    w0 = [torch.empty(k, device=DEV).normal_(generator=gen) for k in n]
    zero = [torch.zeros(k, device=DEV) for k in n]
    hyper = dict(lr=0.1, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.0, momentum=0.9, grad_scale=1.0, step=1)
    su = ShardedUpdate(SHAPES, "sgdm", hyper, device=DEV, dropout=(p, seed))
    su.load_state(w0, zero, zero)
    weights, grads = ([torch.zeros(k, device=DEV) for k in n] for _ in range(2))
    wt, gt = B.TensorTable(su.plan, [weights]), B.TensorTable(su.plan, [grads])
    w, m = [t.double().cpu().numpy() for t in w0], [np.zeros(k) for k in n]
    su.hand_out(wt)
    graph = torch.cuda.CUDAGraph()
    try:
        for step in range(7):
            for t in range(len(n)):
                want = R.hand_out(w[t], p, seed, step, 0, t)
                got = weights[t].double().cpu().numpy()
                # a few fp32 roundings a step (2^-22 of values below 8), the scale and its product two more
                assert (np.abs(got - want) <= 2.0 ** -17).all() and ((got == 0) == (want == 0)).all(), (step, t)
            assert su.drawn == step
            for t in range(len(n)):
                grads[t].normal_(generator=gen)
                g, _ = R.masked_sum([grads[t].cpu().numpy()], p, seed, step, 0, t)
                m[t] = 0.9 * m[t] + g
                w[t] = w[t] - 0.1 * m[t]
            if step == 1:
                torch.cuda.synchronize()
                with torch.cuda.graph(graph, capture_error_mode="thread_local"):
                    su.step(gt, wt)
            if step in (0, 4):
                su.step(gt, wt)
            else:
                graph.replay()
        torch.cuda.synchronize()
    finally:
        graph.reset()           # it holds the group's collectives


def test_tables_are_not_made_in_a_capture(world_of_one):
    """The upload of a table in a capture would read freed host memory at replay: refused, by itself and where a step is given
    plain lists; the capture goes on, and a step with tables made before it replays."""
    from paper_2004_13336_b200 import binding as B
    from paper_2004_13336_b200.collective import ShardedUpdate
    n = [int(np.prod(s)) for s in SHAPES]
    hyper = dict(lr=0.5, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.0, momentum=0.0, grad_scale=1.0, step=1)
    su = ShardedUpdate(SHAPES, "sgdm", hyper, device=DEV, dropout=(0.0, 3))
    w0, zero = [torch.randn(k, device=DEV) for k in n], [torch.zeros(k, device=DEV) for k in n]
    su.load_state(w0, zero, zero)
    weights, grads = [torch.zeros(k, device=DEV) for k in n], [torch.randn(k, device=DEV) for k in n]
    wt, gt = B.TensorTable(su.plan, [weights]), B.TensorTable(su.plan, [grads])
    su.step(gt, wt)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    try:
        with torch.cuda.graph(graph, capture_error_mode="thread_local"):
            for call in (lambda: B.TensorTable(su.plan, [weights]), lambda: su.step(grads, wt),
                         lambda: B.TensorTable.from_pointers(su.plan, [[t.data_ptr() for t in weights]], torch.float32, DEV)):
                with pytest.raises(B.WsError) as e:
                    call()
                assert e.value.status == 1
            su.step(gt, wt)
        for k in range(2, 5):
            graph.replay()
            for a, b, g in zip(weights, w0, grads):      # values below 16: three roundings of 2^-21 a step
                assert bool(((a.double() - b.double() + 0.5 * k * g.double()).abs() <= k * 3 * 2.0 ** -21).all())
    finally:
        graph.reset()


def _routers(B, tokens, experts, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    logits = [[torch.empty(tokens, experts, device=DEV).normal_(generator=gen)] for _ in range(2)]
    picks = [[torch.topk(t[0], 2, dim=1).indices] for t in logits]
    return B.RouterSet(experts, picks, None, logits, [[torch.empty_like(t[0])] for t in logits])


def test_replayed_balance_keeps_to_its_own_memory(world_of_one):
    """A captured step, then one that needs more scratch, then replays: they give the loss, and write to nobody else's memory."""
    from paper_2004_13336_b200 import binding as B
    from paper_2004_13336_b200.collective import ExpertBalance
    balance = ExpertBalance(2, 64, 0.01, 1e-3)
    small, large = _routers(B, 3000, 64, 1), _routers(B, 60000, 64, 2)
    assert small.workspace_bytes() < large.workspace_bytes()
    want = balance.step(small).clone()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    try:
        with torch.cuda.graph(graph, capture_error_mode="thread_local"):
            loss = balance.step(small)
        balance.step(large)
        others = [torch.full((small.workspace_bytes(),), 0x5A, dtype=torch.uint8, device=DEV) for _ in range(3000)]
        for _ in range(3):
            loss.fill_(9)
            graph.replay()
            assert torch.equal(loss, want)
        assert all(bool((t == 0x5A).all()) for t in others)
    finally:
        graph.reset()


def test_steps_captured_apart_share_nothing(world_of_one):
    """Two steps of one object, captured apart: each replay leaves the other's counts and losses alone."""
    from paper_2004_13336_b200 import binding as B
    from paper_2004_13336_b200.collective import ExpertBalance
    balance = ExpertBalance(2, 64, 0.01, 1e-3)
    sets = [_routers(B, n, 64, seed) for n, seed in ((3000, 3), (2500, 4))]
    want = [(balance.step(s).clone(), balance.counts.clone()) for s in sets]
    torch.cuda.synchronize()
    graphs, got = [torch.cuda.CUDAGraph() for _ in sets], []
    try:
        for g, s in zip(graphs, sets):
            with torch.cuda.graph(g, capture_error_mode="thread_local"):
                loss = balance.step(s)
            got.append((loss, balance.counts))
        for order in ((0, 1), (1, 0)):
            for x in got:
                x[0].fill_(9)
                x[1].fill_(9)
            for i in order:
                graphs[i].replay()
            assert all(torch.equal(a, b) for x, y in zip(got, want) for a, b in zip(x, y))
    finally:
        for g in graphs:
            g.reset()
