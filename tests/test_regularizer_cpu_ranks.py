"""Weight dropout in the sharded update and the experts' balance across replicas, on gloo ranks: real collectives around the
plain forms, against the same step computed in one place."""
import os
import socket

import numpy as np
import pytest
import torch
import torch.distributed as dist
import torch.multiprocessing as mp

from tests import _regularizer_ref as R

SHAPES = [(13, 7), (31,), (5, 3, 2)]
P, SEED = 0.3, 77


def _data(rank, step):
    g = torch.Generator().manual_seed(100 * rank + step)
    return [torch.randn(int(np.prod(s)), generator=g) for s in SHAPES]


def _routers(rank):
    g = torch.Generator().manual_seed(7 + rank)
    n = 11 + 6 * rank
    picks = [[torch.randint(-1, 6, (n, 2), generator=g)] for _ in range(3)]
    logits = [[torch.randn(n, 6, generator=g)] for _ in range(3)]
    return picks, [torch.rand(n, generator=g) < 0.8], logits


def _worker(rank, world, port, out):
    os.environ.update(MASTER_ADDR="127.0.0.1", MASTER_PORT=str(port))
    dist.init_process_group("gloo", rank=rank, world_size=world)
    from paper_2004_13336_b200.collective import ExpertBalance, ShardedUpdate
    from tests import _regularizer_ops as ops
    hyper = dict(lr=0.1, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.0, momentum=0.9, grad_scale=1.0, step=1)
    su = ShardedUpdate(SHAPES, "sgdm", hyper, device="cpu", ops=ops, dropout=(P, SEED))
    w = _data(99, 0)
    zero = [torch.zeros_like(t) for t in w]
    su.load_state(w, zero, zero)
    weights = [torch.empty_like(t) for t in w]
    seen = []
    su.hand_out(weights)
    seen.append([t.numpy().copy() for t in weights])
    for step in range(2):
        su.step(_data(rank, step), weights, step=step + 1)
        seen.append([t.numpy().copy() for t in weights])
    full = [torch.empty_like(t) for t in w]
    su.gather_slot(su.w, full)
    picks, valid, logits = _routers(rank)
    d = [[torch.empty_like(t[0])] for t in logits]
    loss = ExpertBalance(3, 6, 0.2, 0.01, device="cpu", ops=ops).step(ops.RouterSet(6, picks, valid, logits, d))
    torch.save({"seen": seen, "full": [t.numpy() for t in full], "loss": loss.numpy(), "d": [t[0].numpy() for t in d]}, out % rank)
    dist.destroy_process_group()


@pytest.mark.parametrize("world", [2, 3])
def test_every_rank_trains_on_its_own_part_and_balances_the_whole_batch(world, tmp_path):
    with socket.socket() as s:
        s.bind(("127.0.0.1", 0))
        port = s.getsockname()[1]
    out = str(tmp_path / "rank%d.pt")
    mp.spawn(_worker, args=(world, port, out), nprocs=world)
    got = [torch.load(out % r, weights_only=False) for r in range(world)]
    # the same run in one place, in float64
    w = [t.double().numpy() for t in _data(99, 0)]
    m = [np.zeros_like(t) for t in w]
    for step in range(3):
        for r in range(world):
            for t in range(len(w)):
                want = R.hand_out(w[t], P, SEED, step, r, t)
                np.testing.assert_allclose(got[r]["seen"][step][t], want, rtol=1e-5, atol=1e-6)
                assert ((got[r]["seen"][step][t] == 0) == (want == 0)).all()
        if step == 2:
            break
        for t in range(len(w)):
            g, _ = R.masked_sum([_data(r, step)[t].numpy() for r in range(world)], P, SEED, step, 0, t)
            m[t] = 0.9 * m[t] + g
            w[t] = w[t] - 0.1 * m[t]
    for r in range(world):
        for t in range(len(w)):
            np.testing.assert_allclose(got[r]["full"][t], w[t], rtol=1e-5, atol=1e-6)
    # the balance of all ranks' tokens
    parts = [_routers(r) for r in range(world)]
    picks = [[p[0][l][0].numpy() for p in parts] for l in range(3)]
    logits = [[p[2][l][0].numpy() for p in parts] for l in range(3)]
    valid = [p[1][0].numpy() for p in parts]
    loss, grads, _ = R.balance(logits, valid, R.counts(picks, valid, 6), 2, "softmax", 0.2, 0.01)
    for r in range(world):
        np.testing.assert_allclose(got[r]["loss"], loss, rtol=1e-6)
        for l in range(3):
            np.testing.assert_allclose(got[r]["d"][l], grads[l][r], rtol=1e-6, atol=1e-9)
