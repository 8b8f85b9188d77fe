"""Stand-in for the CUDA binding on CPU ranks with weight dropout and the experts' balance: tests/_oracle_ops.py and the plain
numpy forms behind the binding's call names."""
import numpy as np
import torch

from tests import _regularizer_ref as R
from tests._oracle_ops import *  # noqa: F401,F403
from tests._oracle_ops import _np, ws_pack, ws_unpack
from oracle import ws_oracle as O


class TensorTable:
    def __init__(self, plan, sets):
        self.sets = [list(s) for s in sets]


class _Drop:
    def __init__(self, p, seed, step, replica):
        self.p, self.seed, self.step, self.replica = p, seed, step, replica


def make_dropout(p, seed, step=0, replica=0):
    return _Drop(p, seed, step, replica)


def _f64(t):
    return t.double().numpy().ravel()


def ws_unpack_dropout(plan, r, flat, lists, drop):
    assert r == -1
    full = [torch.empty(n, dtype=flat.dtype) for n in plan.numels]
    ws_unpack(plan, flat, full)
    for k, tensors in enumerate(lists.sets):
        for t, (src, dst) in enumerate(zip(full, tensors)):
            dst.copy_(torch.from_numpy(R.hand_out(_f64(src), drop.p, drop.seed, drop.step, drop.replica + k, t)).view_as(dst))


def ws_reduce_dropout(plan, r, grads, drop, flat):
    assert r == -1
    sums = [torch.from_numpy(R.masked_sum([_f64(s[t]) for s in grads.sets], drop.p, drop.seed, drop.step, drop.replica, t)[0]).to(flat.dtype)
            for t in range(plan.T)]
    ws_pack(plan, sums, flat)


class RouterSet:
    def __init__(self, experts, picks=None, valid=None, logits=None, dlogits=None, score="softmax"):
        self.experts, self.picks, self.valid, self.logits, self.dlogits, self.score = experts, picks, valid, logits, dlogits, score

    def workspace_bytes(self):
        return 16

    def arrays(self, lists):
        return [[t.numpy() for t in layer] for layer in lists]

    def masks(self):
        return None if self.valid is None else [None if t is None else t.numpy() for t in self.valid]


def ws_router_counts(routers, counts, accumulate=False):
    c = torch.from_numpy(R.counts(routers.arrays(routers.picks), routers.masks(), routers.experts))
    counts.copy_(counts + c if accumulate else c)


def ws_balance_loss(routers, counts, loss, coef, z_coef=0.0, upstream=None, accumulate=False, workspace=None):
    value, grads, _ = R.balance(routers.arrays(routers.logits), routers.masks(), counts.numpy(), routers.picks[0][0].shape[1], routers.score, coef, z_coef,
                                1.0 if upstream is None else float(upstream))
    loss.copy_(torch.from_numpy(value))
    for layer, g in zip(routers.dlogits, grads):
        for dst, src in zip(layer, g):
            dst.copy_(torch.from_numpy(src) + (dst if accumulate else 0))
