"""Weight dropout and the experts' balance through the framework's own paths on the GPU: the sharded update of a replica
(a one-rank NCCL group), and the bounds-checking build."""
import json
import os
import socket
import subprocess
import sys

import numpy as np
import pytest
import torch
import torch.distributed as dist

from tests import _regularizer_ref as R

pytestmark = pytest.mark.gpu
DEV = "cuda"
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
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


@pytest.mark.parametrize("tables", [False, True])
def test_sharded_update_with_dropout(world_of_one, tables):
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
    wt, gt = (B.TensorTable(su.plan, [weights]), B.TensorTable(su.plan, [grads])) if tables else (weights, grads)
    w, m = [t.double().cpu().numpy() for t in w0], [np.zeros(k) for k in n]
    su.hand_out(wt)
    for step in range(3):
        for t in range(len(n)):
            want = R.hand_out(w[t], p, seed, step, 0, t)
            # the weights are a few fp32 roundings (2^-22 of values below 8) off, and the scale and its product two more
            assert (np.abs(weights[t].double().cpu().numpy() - want) <= 2.0 ** -18).all(), (step, t)
            assert ((weights[t].cpu().numpy() == 0) == (want == 0)).all()
        for t in range(len(n)):
            grads[t].normal_(generator=gen)
            g, _ = R.masked_sum([grads[t].cpu().numpy()], p, seed, step, 0, t)
            m[t] = 0.9 * m[t] + g
            w[t] = w[t] - 0.1 * m[t]
        su.step(gt, wt, step=step + 1)
    assert su.drawn == 3


def test_balance_of_one_rank(world_of_one):
    from paper_2004_13336_b200 import binding as B
    from paper_2004_13336_b200.collective import ExpertBalance
    gen = torch.Generator(device=DEV).manual_seed(4)
    logits = [[torch.empty(700, 24, device=DEV).normal_(generator=gen)] for _ in range(2)]
    picks = [[torch.topk(t[0], 3, dim=1).indices] for t in logits]
    d = [[torch.empty_like(t[0])] for t in logits]
    balance = ExpertBalance(2, 24, 0.01, 1e-3)
    loss = balance.step(B.RouterSet(24, picks, None, logits, d))
    lists = lambda x: [[t[0].cpu().numpy()] for t in x]  # noqa: E731
    counts = R.counts(lists(picks), None, 24)
    want, grads, sizes = R.balance(lists(logits), None, counts, 3, "softmax", 0.01, 1e-3)
    assert (balance.counts.cpu().numpy() == counts).all()
    k = 200 * 2.0 ** -24                     # as in tests/test_gpu_router.py
    assert (np.abs(loss.cpu().numpy() - want) <= 2 * k * want).all()
    for l in range(2):
        assert (np.abs(d[l][0].cpu().numpy() - grads[l][0]) <= (k + 2.0 ** -23) * sizes[l][0]).all()


CHILD = r'''
import hashlib, json, torch
from paper_2004_13336_b200 import binding as B, build as ws_build
ws_build.build(debug=B.DEBUG_BOUNDS)
L = B.lib()
out = {"enabled": int(L.ws_debug_bounds_enabled())}
if out["enabled"]:
    B.debug_bounds_read()
digest = hashlib.sha256()
shapes = [(1,), (7,), (3, 3, 16, 32), (64, 128), (1031,), (4099, 3), (0,), (20011,)]
gen = torch.Generator(device="cuda").manual_seed(1)
for shards, layout, ft, tt in ((3, "per_tensor", torch.float32, torch.bfloat16), (8, "concat", torch.bfloat16, torch.float32)):
    plan = B.Plan(shapes, shards, 8, layout=layout)
    flat = torch.empty(plan.G, device="cuda").normal_(generator=gen).to(ft)
    lists = [[torch.zeros(torch.Size(s).numel(), dtype=tt, device="cuda") for s in shapes] for _ in range(3)]
    table, drop = B.TensorTable(plan, lists), B.make_dropout(0.3, 9, 4, 2)
    for r in (-1, 1):
        lo, hi = (0, plan.G) if r < 0 else (r * plan.S, (r + 1) * plan.S)
        B.ws_unpack_dropout(plan, r, flat[lo:hi], table, drop)
        back = torch.empty(hi - lo, dtype=ft, device="cuda")
        B.ws_reduce_dropout(plan, r, table, drop, back)
        for t in [back] + [t for s in lists for t in s]:
            digest.update(t.cpu().view(torch.uint8).numpy().tobytes() if t.numel() else b"")
if out["enabled"]:
    out["bits"] = B.debug_bounds_read()
out["digest"] = digest.hexdigest()
print("RESULT " + json.dumps(out))
'''


def test_bounds_checking_build_finds_nothing_and_changes_nothing():
    got = {}
    for debug in (False, True):
        env = dict(os.environ, PYTHONPATH=ROOT)
        env.pop("WS_DEBUG_BOUNDS", None)
        if debug:
            env["WS_DEBUG_BOUNDS"] = "1"
        r = subprocess.run([sys.executable, "-c", CHILD], env=env, capture_output=True, text=True, timeout=900)
        assert r.returncode == 0, r.stderr[-2000:]
        got[debug] = json.loads(r.stdout.split("RESULT ")[1])
    assert got[True]["enabled"] == 1 and got[True]["bits"] == 0
    assert got[False]["digest"] == got[True]["digest"]
