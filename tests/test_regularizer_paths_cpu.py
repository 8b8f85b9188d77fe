"""The sharded update with weight dropout and the experts' balance as objects that live over many steps, on a one-rank gloo
group with the plain forms behind the binding's call names."""
import socket

import numpy as np
import pytest
import torch
import torch.distributed as dist

from paper_2004_13336_b200.collective import ExpertBalance
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
