"""Weight dropout on the GPU (ws_unpack_dropout, ws_reduce_dropout) against plain forms in 64 bits.

Tolerances, from the roundings: a handed-out value is w times an fp32 scale (off by 2^-24) rounded to fp32 (2^-24) and to its
type (eps / 2).  A sum of n <= 8 copies takes at most 7 additions (7 x 2^-24 of the sum of magnitudes), more copies blocks of
4 (3 x 2^-24) with compensation (2 x 2^-24 and terms of 2^-48); then the scale, its product and the type's rounding."""
import numpy as np
import pytest
import torch

from paper_2004_13336_b200 import binding as B
from paper_2004_13336_b200 import workloads as W
from tests import _regularizer_ref as R
from tests._util import bf16_to_f64, to_np

pytestmark = pytest.mark.gpu
DEV = "cuda"
SHAPES = [(1,), (7,), (0, 4), (8,), (9, 5), (3, 3, 16, 32), (64, 128), (1031,), (), (4099, 3), (300, 301), (0,)]
F32, BF16 = torch.float32, torch.bfloat16
U = 2.0 ** -24


def _half_ulp(dtype):
    return torch.finfo(dtype).eps / 2


def f64(t):
    return bf16_to_f64(to_np(t)) if t.dtype == BF16 else to_np(t).astype(np.float64)


def numels(shapes):
    return [int(np.prod(s)) for s in shapes]


def arenas(plan, n, sets, dtype, seed=0, shift=0, fill=None):
    """`sets` tensor lists as views into one buffer each, with 8 guard elements and more around every tensor; `shift`: elements
    that every tensor starts past a 32-byte boundary."""
    gen = torch.Generator(device=DEV).manual_seed(seed)
    bufs, lists = [], []
    for _ in range(sets):
        offs, at = [], 0
        for k in n:
            at = (at + 15) // 16 * 16 + 16 + shift
            offs.append(at)
            at += k
        buf = torch.empty(at + 32, device=DEV).normal_(generator=gen).to(dtype) if fill is None else torch.full((at + 32,), fill, dtype=dtype, device=DEV)
        bufs.append(buf)
        lists.append([buf[o:o + k] for o, k in zip(offs, n)])
    return bufs, lists


def to_flat(plan, tensors, dtype):
    """Random pads, the tensors packed between them."""
    flat = torch.empty(plan.G, dtype=dtype, device=DEV)
    B.ws_pack(plan, tensors, flat)
    return flat


def expect_hand_out(w, drop, k, t, out):
    ref = R.hand_out(w, drop.p, drop.seed, drop.step, drop.replica + k, t)
    bound = (2 * U + _half_ulp(out.dtype) * (1 + 2 * U)) * np.abs(ref)
    assert (np.abs(f64(out).ravel() - ref) <= bound).all(), (k, t)


def expect_sum(flat_tensors, grads, drop, t):
    ref, size = R.masked_sum([f64(g) for g in grads], drop.p, drop.seed, drop.step, drop.replica, t)
    got = f64(flat_tensors[t]).ravel()
    bound = 7 * U * size + 2 * U * np.abs(ref)
    bound = bound + _half_ulp(flat_tensors[t].dtype) * (np.abs(ref) + bound) * 1.01
    assert (np.abs(got - ref) <= bound).all(), t


CASES = [(1, "per_tensor", 32, 1, F32, F32, 0.1), (3, "per_tensor", 32, 3, F32, BF16, 0.5), (8, "per_tensor", 8, 2, BF16, BF16, 0.25),
         (3, "concat", 32, 4, BF16, F32, 0.1), (8, "concat", 8, 5, F32, F32, 0.0), (5, "concat", 16, 9, F32, BF16, 0.9999999),
         (40, "per_tensor", 8, 33, BF16, BF16, 0.1), (1, "concat", 32, 12, F32, F32, 0.3)]


@pytest.mark.parametrize("shift", [0, 4])       # 4 fp32 elements: 16-byte alignment only
@pytest.mark.parametrize("shards,layout,align,sets,flat_dtype,dtype,p", CASES)
def test_hand_out_and_sum_match_the_definition(shards, layout, align, sets, flat_dtype, dtype, p, shift):
    if shift and dtype == BF16:
        shift = 8
    n = numels(SHAPES)
    plan = B.Plan(SHAPES, shards, align, layout=layout)
    drop = B.make_dropout(p, 0x1234567890ABCDEF + shards, step=77, replica=65536 - sets if shards == 5 else 3 * shards)
    _, (w,) = arenas(plan, n, 1, flat_dtype, seed=1)
    flat = to_flat(plan, w, flat_dtype)
    bufs, lists = arenas(plan, n, sets, dtype, shift=shift, fill=777.0)
    B.ws_unpack_dropout(plan, -1, flat, B.TensorTable(plan, lists), drop)
    for k in range(sets):
        for t in range(plan.T):
            if n[t]:
                expect_hand_out(f64(w[t]), drop, k, t, lists[k][t])
                lists[k][t].fill_(777.0)
        assert bool((bufs[k] == 777.0).all())                     # nothing around the tensors was touched
    # the sum of gradients, whose pads come out as +0 whatever was there
    gbufs, grads = arenas(plan, n, sets, dtype, seed=2, shift=shift)
    before = [b.clone() for b in gbufs]
    total = torch.full((plan.G,), float("nan"), dtype=flat_dtype, device=DEV)
    B.ws_reduce_dropout(plan, -1, B.TensorTable(plan, grads), drop, total)
    out = [torch.zeros(k, dtype=flat_dtype, device=DEV) for k in n]
    B.ws_unpack(plan, total, out)
    for t in range(plan.T):
        if n[t]:
            expect_sum(out, [g[t] for g in grads], drop, t)
    again = torch.empty_like(total)
    B.ws_pack(plan, out, again)
    assert torch.equal(total.view(torch.uint8), again.view(torch.uint8))
    assert all(torch.equal(a, b) for a, b in zip(before, gbufs))


@pytest.mark.parametrize("layout", ["per_tensor", "concat"])
@pytest.mark.parametrize("tile", [0, 1024, 16384])
def test_shards_one_by_one_are_the_whole(layout, tile):
    n, shards, sets = numels(SHAPES), 4, 3
    plan = B.Plan(SHAPES, shards, 32, tile, layout=layout)
    drop = B.make_dropout(0.2, 5, 1, 0)
    flat = torch.randn(plan.G, device=DEV)
    _, whole = arenas(plan, n, sets, BF16, fill=1.0)
    _, parts = arenas(plan, n, sets, BF16, fill=1.0)
    B.ws_unpack_dropout(plan, -1, flat, B.TensorTable(plan, whole), drop)
    table = B.TensorTable(plan, parts)
    for r in range(shards):
        B.ws_unpack_dropout(plan, r, flat[r * plan.S:(r + 1) * plan.S].clone(), table, drop)
    for a, b in zip(whole, parts):
        assert all(torch.equal(x, y) for x, y in zip(a, b))
    total = torch.empty(plan.G, device=DEV)
    B.ws_reduce_dropout(plan, -1, table, drop, total)
    for r in range(shards):
        part = torch.empty(plan.S, device=DEV)
        B.ws_reduce_dropout(plan, r, table, drop, part)
        assert torch.equal(part, total[r * plan.S:(r + 1) * plan.S])


def test_masks_do_not_depend_on_the_plan():
    n = numels(SHAPES)
    w = [torch.randn(k, device=DEV) for k in n]
    first = None
    for shards, layout, align, tile in ((1, "per_tensor", 32, 0), (7, "per_tensor", 8, 1024), (64, "per_tensor", 32, 0), (5, "concat", 8, 2048)):
        plan = B.Plan(SHAPES, shards, align, tile, layout=layout)
        outs = [torch.empty(k, device=DEV) for k in n]
        B.ws_unpack_dropout(plan, -1, to_flat(plan, w, F32), B.TensorTable(plan, [outs]), B.make_dropout(0.4, 21, 2, 9))
        first = first or outs
        assert all(torch.equal(a, b) for a, b in zip(first, outs))


def test_no_dropout_is_unpack_and_a_plain_sum():
    n = numels(SHAPES)
    plan = B.Plan(SHAPES, 4)
    flat = torch.randn(plan.G, device=DEV)
    a, b = [torch.empty(k, device=DEV) for k in n], [torch.empty(k, device=DEV) for k in n]
    B.ws_unpack(plan, flat, a)
    B.ws_unpack_dropout(plan, -1, flat, B.TensorTable(plan, [b]), B.make_dropout(0.0, 1))
    assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_dropped_elements_leave_no_trace():
    """Infinities and NaN where the mask drops; kept, they come through with their kind."""
    plan = B.Plan([(4096,)], 2)
    for sets in (1, 4, 12):
        drop = B.make_dropout(0.5, 99, 3)
        g = [torch.ones(4096, device=DEV) for _ in range(sets)]
        for k in range(sets):
            gone = torch.from_numpy(~R.keep(0.5, 99, 3, k, 0, 4096)).to(DEV)
            g[k][gone] = float("nan") if k % 2 else float("inf")
        total = torch.empty(plan.G, device=DEV)
        B.ws_reduce_dropout(plan, -1, B.TensorTable(plan, [[x] for x in g]), drop, total)
        assert bool(torch.isfinite(total).all())
        for special in (float("inf"), float("-inf"), float("nan")):
            at = int(np.flatnonzero(R.keep(0.5, 99, 3, 0, 0, 4096))[5])
            h = [x.clone() for x in g]
            h[0][at] = special
            B.ws_reduce_dropout(plan, -1, B.TensorTable(plan, [[x] for x in h]), drop, total)
            out = torch.empty(4096, device=DEV)
            B.ws_unpack(plan, total, [out])
            assert torch.equal(out[at:at + 1], torch.full((1,), special, device=DEV)) or (np.isnan(special) and bool(out[at].isnan()))
            assert int((~torch.isfinite(out)).sum()) == 1
    # an infinite copy in any place of many
    drop = B.make_dropout(0.0, 1)
    for k in range(0, 40, 3):
        g = [torch.ones(4096, device=DEV) for _ in range(40)]
        g[k][17] = float("inf")
        B.ws_reduce_dropout(plan, -1, B.TensorTable(plan, [[x] for x in g]), drop, total)
        assert float(total.max()) == float("inf") and int(torch.isfinite(total).sum()) == plan.G - 1


def test_step_word_advances_a_captured_step():
    n = numels(SHAPES)
    plan = B.Plan(SHAPES, 2)
    flat = torch.randn(plan.G, device=DEV)
    _, lists = arenas(plan, n, 2, F32, fill=0.0)
    table, total = B.TensorTable(plan, lists), torch.empty(plan.G, device=DEV)
    word = torch.zeros(1, dtype=torch.int32, device=DEV)
    drop = B.make_dropout(0.3, 8, step=0xFFFFFFFE, replica=1, step_dev=word)      # the sum runs past 2^32

    def step():
        B.ws_unpack_dropout(plan, -1, flat, table, drop)
        B.ws_reduce_dropout(plan, -1, table, drop, total)
        word.add_(1)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    word.zero_()
    for i in range(4):
        graph.replay()
        plain = B.make_dropout(0.3, 8, step=0xFFFFFFFE + i, replica=1)
        _, want = arenas(plan, n, 2, F32, fill=0.0)
        sums = torch.empty(plan.G, device=DEV)
        wt = B.TensorTable(plan, want)
        B.ws_unpack_dropout(plan, -1, flat, wt, plain)
        B.ws_reduce_dropout(plan, -1, wt, plain, sums)
        assert all(torch.equal(x, y) for a, b in zip(lists, want) for x, y in zip(a, b))
        assert torch.equal(sums, total)


def test_two_streams_at_once():
    plan = B.Plan([(1 << 20,), (1000, 777)], 4)
    flat, drops = torch.randn(plan.G, device=DEV), [B.make_dropout(0.1, s) for s in (1, 2)]
    outs = [[torch.empty(1 << 20, device=DEV), torch.empty(777000, device=DEV)] for _ in range(4)]
    tables = [B.TensorTable(plan, [o]) for o in outs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for i, s in enumerate(streams):
        with torch.cuda.stream(s):
            B.ws_unpack_dropout(plan, -1, flat, tables[i], drops[i])
    torch.cuda.synchronize()
    for i in range(2):
        B.ws_unpack_dropout(plan, -1, flat, tables[2 + i], drops[i])
        assert all(torch.equal(a, b) for a, b in zip(outs[i], outs[2 + i]))


def test_many_short_tiles():
    """Many small tensors in many shards: a warp per tile."""
    shapes = [(8 * (i % 37) + i % 5 + 1,) for i in range(700)]
    n, shards = numels(shapes), 64
    plan = B.Plan(shapes, shards, 8)
    assert plan.ntiles * shards > 32 * 148
    drop = B.make_dropout(0.2, 4, 4, 4)
    w = [torch.randn(k, device=DEV) for k in n]
    lists = [[torch.empty(k, dtype=BF16, device=DEV) for k in n] for _ in range(3)]
    table = B.TensorTable(plan, lists)
    B.ws_unpack_dropout(plan, -1, to_flat(plan, w, F32), table, drop)
    total, out = torch.empty(plan.G, device=DEV), [torch.empty(k, device=DEV) for k in n]
    B.ws_reduce_dropout(plan, -1, table, drop, total)
    B.ws_unpack(plan, total, out)
    for t in range(0, 700, 7):
        for k in range(3):
            expect_hand_out(f64(w[t]), drop, k, t, lists[k][t])
        expect_sum(out, [x[t] for x in lists], drop, t)


@pytest.mark.parametrize("p", [1e-5, 0.1, 0.75])
def test_share_kept_of_a_model(p):
    """Within 5 standard deviations of 1 - T / 65536 over a model's tensors; the mean copy is the weight."""
    wl = W.scaled_down(W.transformer(), 512)
    plan = B.Plan(wl.shapes, 8)
    ones = torch.ones(plan.G, device=DEV)
    arena = torch.empty(plan.arena_elems, device=DEV)
    views = plan.arena_views(arena, wl.numels)
    B.ws_unpack_dropout(plan, -1, ones, B.TensorTable(plan, [views]), B.make_dropout(p, 17))
    q = 1 - R.threshold(p) / 65536
    kept = sum(int((v != 0).sum()) for v in views) / wl.N
    assert abs(kept - q) <= 5 * np.sqrt(q * (1 - q) / wl.N)
    assert all(bool(((v == 0) | (v == np.float32(R.scale(p)))).all()) for v in views)


def test_offsets_past_32_bits():
    """A tensor of more than 2^31 elements (2^32 bytes and more): its first and last elements."""
    n = (1 << 31) + 1031
    plan = B.Plan([(5,), (n,)], 2, one_launch=False)
    drop = B.make_dropout(0.5, 3, 2, 1)
    flat = torch.empty(plan.G, dtype=BF16, device=DEV)
    flat.fill_(0.5)
    out = [torch.zeros(5, dtype=BF16, device=DEV), torch.zeros(n, dtype=BF16, device=DEV)]
    table = B.TensorTable(plan, [out])
    B.ws_unpack_dropout(plan, -1, flat, table, drop)
    for lo, hi in ((0, 4096), (n - 4099 - (n - 4099) % 8, n), ((1 << 30) - 4096, (1 << 30) + 4096)):
        kept = torch.from_numpy(R.keep(0.5, 3, 2, 1, 1, hi - lo, start=lo)).to(DEV)
        assert torch.equal(out[1][lo:hi] != 0, kept) and bool((out[1][lo:hi][kept] == 1.0).all())
    B.ws_reduce_dropout(plan, -1, table, drop, flat)
    back = [torch.zeros(5, dtype=BF16, device=DEV), torch.zeros(n, dtype=BF16, device=DEV)]
    B.ws_unpack(plan, flat, back)
    assert torch.equal(back[1], out[1] * 2) and torch.equal(back[0], out[0] * 2)


def test_a_training_run_with_dropout_follows_its_plain_form():
    """Hand-out, gradients of every replica's copy, their masked sum, the sharded update; three steps against float64."""
    shapes, replicas, p = [(24, 40), (40,), (40, 7)], 3, 0.25
    n = numels(shapes)
    plan = B.Plan(shapes, 4)
    gen = torch.Generator(device=DEV).manual_seed(3)
    w0 = [torch.empty(k, device=DEV).normal_(0, 0.2, generator=gen) for k in n]
    w, m = to_flat(plan, w0, F32), torch.zeros(plan.G, device=DEV)
    x = [torch.empty(16, 24, device=DEV, dtype=torch.float64).normal_(generator=gen) for _ in range(replicas)]

    def loss(params, xk):
        a, b, c = (q.view(s) for q, s in zip(params, shapes))
        return torch.tanh(xk.to(a.dtype) @ a + b).matmul(c).square().mean()

    copies = [[torch.empty(k, device=DEV) for k in n] for _ in range(replicas)]
    grads = [[torch.empty(k, device=DEV) for k in n] for _ in range(replicas)]
    ct, gt = B.TensorTable(plan, copies), B.TensorTable(plan, grads)
    total = torch.empty(plan.G, device=DEV)
    hyper = dict(lr=0.05, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.0, momentum=0.9, grad_scale=1 / replicas, step=1)
    ref, refm = [t.double() for t in w0], [torch.zeros(k, dtype=torch.float64, device=DEV) for k in n]
    for step in range(3):
        drop = B.make_dropout(p, 42, step)
        B.ws_unpack_dropout(plan, -1, w, ct, drop)
        for k in range(replicas):
            leaves = [c.double().requires_grad_() for c in copies[k]]
            for g, d in zip(grads[k], torch.autograd.grad(loss(leaves, x[k]), leaves)):
                g.copy_(d)
        B.ws_reduce_dropout(plan, -1, gt, drop, total)
        B.ws_shard_update(plan, -1, [total], w, m, None, B.make_hyper("sgdm", hyper))
        leaves = [t.clone().requires_grad_() for t in ref]
        masks = [[torch.from_numpy(R.keep(p, 42, step, k, t, n[t])).to(DEV) * R.scale(p) for t in range(3)] for k in range(replicas)]
        sum(loss([q * z for q, z in zip(leaves, masks[k])], x[k]) for k in range(replicas)).div(replicas).backward()
        for t in range(3):
            refm[t] = 0.9 * refm[t] + leaves[t].grad
            ref[t] = ref[t] - 0.05 * refm[t]
    out = [torch.empty(k, device=DEV) for k in n]
    B.ws_unpack(plan, w, out)
    # each of three steps adds a few roundings (under 2^-20 together) of values below 1 to the weights it hands on
    for a, b in zip(out, ref):
        assert float((a.double() - b).abs().max()) < 3 * 2.0 ** -20


def test_tables_of_another_plan_are_refused():
    plan, other = B.Plan([(8,), (9,)], 1), B.Plan([(8,)], 1)
    table = B.TensorTable(other, [[torch.zeros(8, device=DEV)]])
    for call in (lambda: B.ws_unpack_dropout(plan, -1, torch.zeros(plan.G, device=DEV), table, B.make_dropout(0.1, 1)),
                 lambda: B.ws_reduce_dropout(plan, -1, table, B.make_dropout(0.1, 1), torch.zeros(plan.G, device=DEV))):
        with pytest.raises(B.WsError) as e:
            call()
        assert e.value.status == 1
