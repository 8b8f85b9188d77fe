"""Weight dropout and the experts' balance without a GPU: the generator against its published answers, the plain forms the
GPU tests rest on against independent ones, and the arguments that the entry points refuse before any launch."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2004_13336_b200 import binding as B
from paper_2004_13336_b200 import build as ws_build
from tests import _regularizer_ref as R

INVALID, ALIGNMENT, DTYPE, WORKSPACE, NOT_UPLOADED = 1, 2, 3, 4, 5


@pytest.fixture(scope="module", autouse=True)
def _built():
    ws_build.build()


# Known answers published with the generator (key, counter all zero, all ones, digits of pi).
@pytest.mark.parametrize("rounds,key,counter,want", [
    (7, (0, 0), (0, 0, 0, 0), (0x5F6FB709, 0x0D893F64, 0x4F121F81, 0x4F730A48)),
    (7, (0xFFFFFFFF,) * 2, (0xFFFFFFFF,) * 4, (0x5207DDC2, 0x45165E59, 0x4D8EE751, 0x8C52F662)),
    (10, (0, 0), (0, 0, 0, 0), (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
    (10, (0xFFFFFFFF,) * 2, (0xFFFFFFFF,) * 4, (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
])
def test_generator_gives_the_published_words(rounds, key, counter, want):
    assert tuple(int(x) for x in R.philox(key, counter, rounds)) == want


def test_masks_keep_their_share_and_do_not_repeat():
    """The share kept of 2^20 elements is within 5 standard deviations of 1 - T / 65536, and two masks of other replicas,
    steps, tensors or seeds agree as often as independent ones do."""
    n, p = 1 << 20, 0.3
    q = 1 - R.threshold(p) / 65536
    base = R.keep(p, 11, 5, 2, 3, n)
    assert abs(base.mean() - q) < 5 * np.sqrt(q * (1 - q) / n)
    agree = q * q + (1 - q) * (1 - q)
    for other in (R.keep(p, 12, 5, 2, 3, n), R.keep(p, 11, 6, 2, 3, n), R.keep(p, 11, 5, 3, 3, n), R.keep(p, 11, 5, 2, 4, n),
                  R.keep(p, 11 + (1 << 32), 5, 2, 3, n), np.roll(base, 1), np.roll(base, 8)):
        assert abs((base == other).mean() - agree) < 5 * np.sqrt(agree * (1 - agree) / n)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_plain_balance_gradient_is_that_of_the_formula_and_of_differences(score):
    rng = np.random.default_rng(4)
    experts, topk, coef, z = 5, 2, 0.3, 0.02 if score == "softmax" else 0.0
    logits = [[rng.normal(size=(4, experts)), rng.normal(size=(3, experts)) * 3]]
    valid = [np.array([1, 1, 0, 1]), None]
    picks = [[rng.integers(0, experts, (4, topk)), rng.integers(-1, experts, (3, topk))]]
    cnt = R.counts(picks, valid, experts)
    loss, d, _ = R.balance(logits, valid, cnt, topk, score, coef, z)
    # the formula, by autograd
    x = [torch.tensor(t, requires_grad=True) for t in logits[0]]
    live = torch.cat([x[0][[0, 1, 3]], x[1]])
    s = torch.softmax(live, 1) if score == "softmax" else torch.sigmoid(live) / torch.sigmoid(live).sum(1, keepdim=True)
    f = torch.tensor(cnt[0, :-1]).double() / (topk * 6)
    want = torch.stack([coef * experts * (f * s.mean(0)).sum(), z * torch.logsumexp(live, 1).square().mean()])
    want.sum().backward()
    np.testing.assert_allclose(loss[0], want.detach().numpy(), rtol=1e-12)
    for a, b in zip(d[0], x):
        np.testing.assert_allclose(a, b.grad.numpy(), rtol=1e-10, atol=1e-15)
    # differences: (L(x + h) - L(x - h)) / 2h is off by h^2/6 L''' and 2^-53 L / h
    h = 1e-5
    for k in (0, 1):
        for i in range(logits[0][k].shape[0]):
            for e in range(experts):
                up, down = ([[t.copy() for t in logits[0]]] for _ in range(2))
                up[0][k][i, e] += h
                down[0][k][i, e] -= h
                diff = (R.balance(up, valid, cnt, topk, score, coef, z)[0] - R.balance(down, valid, cnt, topk, score, coef, z)[0]).sum() / (2 * h)
                assert abs(diff - d[0][k][i, e]) < 1e-8


def test_sum_is_the_adjoint_of_the_hand_out():
    rng = np.random.default_rng(1)
    w, g = rng.normal(size=100), [rng.normal(size=100) for _ in range(3)]
    copies = [R.hand_out(w, 0.4, 9, 1, k, 6) for k in range(3)]
    total, _ = R.masked_sum(g, 0.4, 9, 1, 0, 6)
    np.testing.assert_allclose(sum((c * x).sum() for c, x in zip(copies, g)), (w * total).sum(), rtol=1e-12)


# ------------------------------------------------------------------ refusals
def _table(T, nsets=2, dtype=0, align=32, dev=256):
    return B.ws_tensor_table(dev, nsets, T, dtype, align)


@pytest.fixture()
def uploaded(monkeypatch):
    """A plan, and a library call on it that can never launch: its plan has no tables on a device."""
    return B.Plan([(64, 8), (5,)], 4, upload=False)


@pytest.mark.parametrize("name", ["ws_unpack_dropout", "ws_reduce_dropout"])
def test_dropout_refuses_bad_arguments(uploaded, name):
    plan, L = uploaded, B.lib()

    def call(handle=None, r=-1, flat=256, flat_dtype=0, table=None, drop=None, null=()):
        t, d = table or _table(2), drop or B.make_dropout(0.1, 3)
        h = plan.handle if "plan" not in null else None
        t, d = (None if "table" in null else C.byref(t)), (None if "drop" in null else C.byref(d))
        if name == "ws_unpack_dropout":
            return L.ws_unpack_dropout(h, r, flat, flat_dtype, t, d, None)
        return L.ws_reduce_dropout(h, r, t, d, flat, flat_dtype, None)

    for null in ("plan", "table", "drop"):
        assert call(null=(null,)) == INVALID
    assert call(flat=None) == INVALID
    for r in (-2, 4, 1 << 30):
        assert call(r=r) == INVALID
    for bad in (_table(3), _table(2, 0), _table(2, 1025), _table(2, dev=None)):
        assert call(table=bad) == INVALID
    for p in (-0.1, 1.0, 1.5, float("nan"), float("inf")):
        assert call(drop=B.make_dropout(p, 3)) == INVALID
    for replica in (-1, 65535, 65536):
        assert call(drop=B.make_dropout(0.1, 3, 0, replica)) == INVALID
    assert call(flat_dtype=2) == DTYPE and call(table=_table(2, dtype=7)) == DTYPE
    # everything else in order: only the tables on the device are missing
    for ok in (dict(), dict(r=3), dict(flat_dtype=1), dict(drop=B.make_dropout(0.0, -1, -1, 65534)), dict(drop=B.make_dropout(0.9999999, 1 << 80))):
        assert call(**ok) == NOT_UPLOADED


def test_make_dropout_takes_numbers_of_any_kind():
    d = B.make_dropout(np.float32(0.5), np.int64(3), np.int32(4), np.int64(5))
    assert (d.p, d.seed, d.step, d.replica, d.step_dev) == (0.5, 3, 4, 5, None)
    d = B.make_dropout(0, -1, -1)
    assert (d.p, d.seed, d.step, d.replica) == (0.0, 2 ** 64 - 1, 2 ** 32 - 1, 0)


def test_dropout_binding_refuses_what_is_no_buffer_of_its_size(uploaded, monkeypatch):
    monkeypatch.setattr(B, "_on_current_device", lambda t: None)
    lists = type("T", (), {"c": _table(2)})()
    d = B.make_dropout(0.1, 3)
    for r, n in ((-1, uploaded.S), (-1, uploaded.G - 8), (2, uploaded.G)):
        with pytest.raises(ValueError):
            B.ws_unpack_dropout(uploaded, r, torch.zeros(n), lists, d)
        with pytest.raises(ValueError):
            B.ws_reduce_dropout(uploaded, r, lists, d, torch.zeros(n))
    with pytest.raises(ValueError):
        B.ws_unpack_dropout(uploaded, -1, torch.zeros(2 * uploaded.G)[::2], lists, d)
    with pytest.raises(TypeError):
        B.ws_unpack_dropout(uploaded, -1, torch.zeros(uploaded.G, dtype=torch.float16), lists, d)
    for bad in (None, {"p": 0.1}, B.ws_hyper()):
        with pytest.raises((TypeError, C.ArgumentError)):
            B.ws_unpack_dropout(uploaded, -1, torch.zeros(uploaded.G), lists, bad)


def test_dropout_and_routers_refuse_tensors_off_the_current_device(uploaded):
    lists, d = type("T", (), {"c": _table(2)})(), B.make_dropout(0.1, 3)
    with pytest.raises(ValueError):
        B.ws_unpack_dropout(uploaded, -1, torch.zeros(uploaded.G), lists, d)
    routers = B.RouterSet(4, [[torch.zeros(3, 2, dtype=torch.int64)]])
    with pytest.raises(ValueError):
        B.ws_router_counts(routers, torch.zeros(1, 5, dtype=torch.int64))
    with pytest.raises(TypeError):
        B.make_dropout(0.1, 3, step_dev=torch.zeros(1, dtype=torch.int32))
    with pytest.raises(TypeError):
        B.make_dropout(0.1, 3, step_dev=torch.zeros(1, dtype=torch.int64))


def _set(**kw):
    """A set of one layer and two replicas with made-up device addresses."""
    keep = {"tokens": (C.c_int64 * 2)(3, 0), "picks": (C.c_void_p * 2)(256, None), "logits": (C.c_void_p * 2)(256, None),
            "dlogits": (C.c_void_p * 2)(512, None)}
    keep.update({k: v for k, v in kw.items() if k in keep})
    s = B.ws_router_set(layers=1, replicas=2, experts=8, topk=2, logits_ld=8, dlogits_ld=8, index_bytes=8)
    for k, v in kw.items():
        if k not in keep:
            setattr(s, k, v)
    for k, v in keep.items():
        if v is not None:
            setattr(s, k, C.cast(v, C.POINTER(C.c_int64 if k == "tokens" else C.c_void_p)))
    s._keep = keep
    return s


BAD_SETS = [dict(layers=0), dict(layers=65536), dict(replicas=0), dict(replicas=513), dict(experts=0), dict(experts=1025, logits_ld=2000, dlogits_ld=2000),
            dict(topk=0), dict(topk=9), dict(tokens=(C.c_int64 * 2)(-1, 0)), dict(tokens=(C.c_int64 * 2)(1 << 31, 0)), dict(tokens=None)]


@pytest.mark.parametrize("bad", BAD_SETS, ids=lambda b: next(iter(b)))
def test_router_calls_refuse_bad_sets(bad):
    L, s = B.lib(), _set(**bad)
    assert L.ws_router_counts(C.byref(s), 256, 0, None) == INVALID
    assert L.ws_balance_workspace_bytes(C.byref(s)) == 0
    assert L.ws_balance_loss(C.byref(s), 256, 256, 1.0, 0.0, None, 0, 256, 1 << 20, None) == INVALID


def test_router_counts_refuses_bad_arguments():
    L = B.lib()
    call = lambda s, counts=256: L.ws_router_counts(C.byref(s) if s else None, counts, 0, None)  # noqa: E731
    assert call(None) == INVALID and call(_set(), None) == INVALID
    assert call(_set(picks=None)) == INVALID and call(_set(picks=(C.c_void_p * 2)(None, 256))) == INVALID
    for b in (0, 2, 16):
        assert call(_set(index_bytes=b)) == INVALID
    assert call(_set(), 260) == ALIGNMENT and call(_set(picks=(C.c_void_p * 2)(260, None))) == ALIGNMENT


def test_balance_loss_refuses_bad_arguments():
    L = B.lib()

    def call(s, counts=256, loss=256, coef=1.0, z=0.0, upstream=None, workspace=256, nbytes=1 << 20):
        return L.ws_balance_loss(C.byref(s) if s else None, counts, loss, coef, z, upstream, 0, workspace, nbytes, None)

    assert call(None) == INVALID and call(_set(), counts=None) == INVALID
    assert call(_set(dlogits=None), loss=None) == INVALID
    for x in (float("nan"), float("inf")):
        assert call(_set(), coef=x) == INVALID and call(_set(), z=x) == INVALID
    assert call(_set(score=1), z=1e-3) == INVALID and call(_set(score=2)) == INVALID
    assert call(_set(dtype=2)) == DTYPE
    for bad in (dict(logits=None), dict(logits_ld=7), dict(dlogits_ld=7), dict(logits=(C.c_void_p * 2)(None, 256)), dict(dlogits=(C.c_void_p * 2)(None, 256)),
                dict(logits_ld=1 << 40)):
        assert call(_set(**bad)) == INVALID
    assert call(_set(logits=(C.c_void_p * 2)(258, None))) == ALIGNMENT and call(_set(dtype=1, dlogits=(C.c_void_p * 2)(257, None))) == ALIGNMENT
    for x in (dict(counts=260), dict(loss=257), dict(upstream=258), dict(workspace=264)):
        assert call(_set(), **x) == ALIGNMENT
    need = L.ws_balance_workspace_bytes(C.byref(_set()))
    assert need > 0
    assert call(_set(), workspace=None) == WORKSPACE and call(_set(), nbytes=need - 1) == WORKSPACE


def test_router_set_refuses_tensors_that_do_not_belong_together():
    i = lambda n, k=2: torch.zeros(n, k, dtype=torch.int64)  # noqa: E731
    x = lambda n, e=8: torch.zeros(n, e)  # noqa: E731
    B.RouterSet(8, [[i(3), i(0)], [i(3), i(0)]], [torch.ones(3, dtype=torch.bool), None], [[x(3), x(0)], [x(3), x(0)]])
    B.RouterSet(8, logits=[[torch.zeros(3, 16)[:, :8]]], dlogits=[[x(3)]], topk=2)
    assert B.RouterSet(8, [[i(3)]], topk=2).c.topk == B.RouterSet(8, logits=[[x(3)]], topk=2).c.topk == 2
    for bad in (lambda: B.RouterSet(8), lambda: B.RouterSet(8, [[torch.zeros(3, dtype=torch.int64)]]), lambda: B.RouterSet(8, []), lambda: B.RouterSet(8, [[]]),
                lambda: B.RouterSet(8, [[i(3), i(4)], [i(3)]]), lambda: B.RouterSet(8, [[i(3), i(4)], [i(3), i(5)]]),
                lambda: B.RouterSet(8, [[i(3)]], logits=[[x(4)]]), lambda: B.RouterSet(8, logits=[[x(3, 7)]], topk=2),
                lambda: B.RouterSet(8, logits=[[x(3)]]), lambda: B.RouterSet(8, [[i(3)]], topk=3),
                lambda: B.RouterSet(8, [[i(3)]], dlogits=[[x(3)]]), lambda: B.RouterSet(8, [[i(3)]], valid=[torch.ones(4, dtype=torch.bool)]),
                lambda: B.RouterSet(8, [[i(3)]], valid=[torch.ones(3)]), lambda: B.RouterSet(8, [[i(3)]], valid=[]),
                lambda: B.RouterSet(8, logits=[[torch.zeros(8, 3).t()]], topk=2), lambda: B.RouterSet(8, logits=[[x(3), torch.zeros(3, 16)[:, :8]]], topk=2),
                lambda: B.RouterSet(8, logits=[[x(3), x(3).bfloat16()]], topk=2)):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: B.RouterSet(8, [[i(3).to(torch.int16)]]), lambda: B.RouterSet(8, [[torch.zeros(3, 4, dtype=torch.int64)[:, :2]]]),
                lambda: B.RouterSet(8, logits=[[x(3).half()]], topk=2), lambda: B.RouterSet(8, logits=[[x(3)]], dlogits=[[x(3).bfloat16()]], topk=2)):
        with pytest.raises(TypeError):
            bad()
    routers = B.RouterSet(8, [[i(3)]])
    for bad in (torch.zeros(1, 8, dtype=torch.int64), torch.zeros(1, 9, dtype=torch.int32), torch.zeros(2, 9, dtype=torch.int64)):
        with pytest.raises(ValueError):
            B.ws_router_counts(routers, bad)
    with pytest.raises(TypeError):
        B.ws_router_counts([[i(3)]], torch.zeros(1, 9, dtype=torch.int64))
