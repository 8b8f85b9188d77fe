"""Weight dropout in every form its dispatch knows (a CTA or a warp per tile, one vector of a tile in flight or four, one copy to
more than 8), in all types, against plain forms in 64 bits; and the sums without dropout.

Tolerance of a sum of n copies, U = 2^-24, S the sum of their magnitudes under the masks: up to 8 copies take 7 roundings at most,
7 U S.  More are summed in blocks of 4, or of 8 bf16 copies: at most 7 additions in a block (the first, to 0, is exact), 7 U of its
magnitudes; the blocks are added with compensation, 2 U of the sum and terms of n U^2 S, which 2^-19 of the first term covers
(n <= 40).  The scale and the product with it: 2 U.  Then the type's rounding."""
import numpy as np
import pytest
import torch

from paper_2004_13336_b200 import binding as B
from tests import _regularizer_ref as R
from tests.test_gpu_dropout import BF16, DEV, F32, U, _half_ulp, arenas, expect_hand_out, f64, numels, to_flat

pytestmark = pytest.mark.gpu


def expect_sum(out, grads, drop, t):
    ref, size = R.masked_sum([f64(g) for g in grads], drop.p, drop.seed, drop.step, drop.replica, t)
    bound = 7 * U * (1 + 2.0 ** -19) * size + 4 * U * np.abs(ref)
    bound = bound + _half_ulp(out.dtype) * (np.abs(ref) + bound)
    assert (np.abs(f64(out).ravel() - ref) <= bound).all(), t


# Tensors, shards, alignment, tile length: short tiles in numbers (a warp each); tiles of the usual length and shorter, of which
# bf16 lists from 4 on take one vector at a time; long ones, of which they take four.
PLANS = {
    "short": ([(8 * (i % 37) + i % 5 + 1,) for i in range(700)], 64, 8, 0),
    "short concat": ([(8 * (i % 37) + i % 5 + 1,) for i in range(9000)], 3, 8, 0),
    "usual": ([(7,), (700, 601), (4099, 3)], 2, 32, 0),
    "long": ([(7,), (300, 301), (4099, 3), (64, 128)], 1, 32, 8192),
    "middle": ([(1031 + i,) for i in range(40)], 1, 8, 0),
}


@pytest.mark.parametrize("flat_dtype", [F32, BF16])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("sets", [1, 2, 4, 7, 9, 19])
@pytest.mark.parametrize("name", PLANS)
def test_hand_out_and_sum(name, sets, dtype, flat_dtype):
    shapes, shards, align, tile = PLANS[name]
    layout = "concat" if "concat" in name else "per_tensor"
    n = numels(shapes)
    plan = B.Plan(shapes, shards, align, tile, layout=layout, one_launch=False)
    tiles = plan.ntiles if layout == "concat" else plan.ntiles * shards
    average = (plan.G if layout == "concat" else plan.S) / plan.ntiles
    if name.startswith("short"):
        assert tiles > 32 * 148 and average <= 256
    else:
        assert tiles < 32 * 148 and (average >= 1536) == (name == "long")
    drop = B.make_dropout(0.3, 77 + sets, 5, sets)
    some = [t for t in range(0, len(n), max(1, len(n) // 23)) if n[t]]
    _, (w,) = arenas(plan, n, 1, flat_dtype, seed=1)
    bufs, lists = arenas(plan, n, sets, dtype, fill=777.0)
    B.ws_unpack_dropout(plan, -1, to_flat(plan, w, flat_dtype), B.TensorTable(plan, lists), drop)
    for k in range(sets):
        for t in some:
            expect_hand_out(f64(w[t]), drop, k, t, lists[k][t])
        for x in lists[k]:
            x.fill_(777.0)
        assert bool((bufs[k] == 777.0).all())                 # nothing around the tensors was touched
    _, grads = arenas(plan, n, sets, dtype, seed=2)
    total = torch.full((plan.G,), float("nan"), dtype=flat_dtype, device=DEV)
    B.ws_reduce_dropout(plan, -1, B.TensorTable(plan, grads), drop, total)
    out = [torch.zeros(k, dtype=flat_dtype, device=DEV) for k in n]
    B.ws_unpack(plan, total, out)
    for t in some:
        expect_sum(out[t], [g[t] for g in grads], drop, t)
    again = torch.empty_like(total)
    B.ws_pack(plan, out, again)
    assert torch.equal(total.view(torch.uint8), again.view(torch.uint8))          # pads are +0


@pytest.mark.parametrize("sets", [1, 3, 8, 12, 40])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_without_dropout_it_is_a_plain_sum(sets, dtype):
    shapes = [(1,), (7,), (3, 3, 16, 32), (1031,), (300, 301)]
    n = numels(shapes)
    plan = B.Plan(shapes, 4)
    _, grads = arenas(plan, n, sets, dtype, seed=sets)
    total = torch.empty(plan.G, device=DEV)
    B.ws_reduce_dropout(plan, -1, B.TensorTable(plan, grads), B.make_dropout(0.0, 1), total)
    out = [torch.empty(k, device=DEV) for k in n]
    B.ws_unpack(plan, total, out)
    for t in range(len(n)):
        each = torch.stack([g[t].double() for g in grads])
        want, size = each.sum(0), each.abs().sum(0)
        assert bool(((out[t].double() - want).abs() <= 7 * U * (1 + 2.0 ** -19) * size + 5 * U * want.abs()).all())
        if sets == 1:
            assert torch.equal(out[t], grads[0][t].float())
