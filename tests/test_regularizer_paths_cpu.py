"""The sharded update with weight dropout and the experts' balance as objects that live over many steps, on a one-rank gloo
group with the plain forms behind the binding's call names."""
import socket

import numpy as np
import pytest
import torch
import torch.distributed as dist

from paper_2004_13336_b200.collective import ExpertBalance, ShardedUpdate
from tests import _regularizer_ops as ops
from tests import _regularizer_ref as R


@pytest.fixture(scope="module")
def world_of_one():
    with socket.socket() as s:
        s.bind(("127.0.0.1", 0))
        port = s.getsockname()[1]
    dist.init_process_group("gloo", init_method=f"tcp://127.0.0.1:{port}", rank=0, world_size=1)
    yield
    dist.destroy_process_group()


def test_a_loss_that_was_returned_stays(world_of_one):
    """The losses of two microbatches, both kept."""
    balance, seen = ExpertBalance(2, 5, 0.3, 0.01, device="cpu", ops=ops), []
    for seed in (1, 2):
        g = torch.Generator().manual_seed(seed)
        picks = [[torch.randint(0, 5, (9, 2), generator=g)] for _ in range(2)]
        logits = [[torch.randn(9, 5, generator=g)] for _ in range(2)]
        routers = ops.RouterSet(5, picks, None, logits, [[torch.empty(9, 5)] for _ in range(2)])
        want = R.balance(routers.arrays(logits), None, R.counts(routers.arrays(picks), None, 5), 2, "softmax", 0.3, 0.01)[0]
        seen.append((balance.step(routers), want))
        assert balance.loss is seen[-1][0]
    for got, want in seen:
        np.testing.assert_allclose(got.numpy(), want, rtol=1e-6)


SHAPES = [(13, 7), (31,), (5, 3, 2)]


def _run(su, weights, steps):
    """Steps with gradients that the step's number gives; the parts handed out."""
    seen = []
    for step in steps:
        g = torch.Generator().manual_seed(step)
        su.step([torch.randn(int(np.prod(s)), generator=g) for s in SHAPES], weights, step=step + 1)
        seen.append([t.clone() for t in weights])
    return seen


def test_a_resumed_run_goes_on_with_its_masks(world_of_one):
    """Four steps, against two, a checkpoint and two more in a new object: the same parts to the bit."""
    hyper = dict(lr=0.1, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.0, momentum=0.9, grad_scale=1.0, step=1)
    new = lambda: ShardedUpdate(SHAPES, "sgdm", hyper, device="cpu", ops=ops, dropout=(0.4, 9))  # noqa: E731
    empty = lambda: [torch.zeros(int(np.prod(s))) for s in SHAPES]  # noqa: E731
    w0 = [torch.randn(int(np.prod(s)), generator=torch.Generator().manual_seed(50)) for s in SHAPES]
    su, weights = new(), empty()
    su.load_state(w0, empty(), empty())
    su.hand_out(weights)
    first = _run(su, weights, [0, 1])
    saved = [empty() for _ in range(3)]
    for shard, out in zip((su.w, su.m, su.v), saved):
        su.gather_slot(shard, out)
    drawn = su.drawn
    want = _run(su, weights, [2, 3])
    again, weights = new(), empty()
    again.load_state(*saved, drawn=drawn)
    again.hand_out(weights)
    assert drawn == 2 and all(torch.equal(a, b) for a, b in zip(weights, first[-1]))
    got = _run(again, weights, [2, 3])
    assert again.drawn == su.drawn == 4
    assert all(torch.equal(a, b) for x, y in zip(got, want) for a, b in zip(x, y))
    for n in (0, 7, (1 << 31) - 1, 1 << 31, (1 << 32) - 1):
        again.drawn = n
        assert again.drawn == n
