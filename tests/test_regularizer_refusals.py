"""What the weight dropout's and the routers' calls refuse in the binding, without a GPU."""
import pytest
import torch

from paper_2004_13336_b200 import binding as B
from paper_2004_13336_b200 import build as ws_build


@pytest.fixture(scope="module", autouse=True)
def _built():
    ws_build.build()


class _On:
    """A buffer on a device that is not there."""

    def __init__(self, index):
        self.index, self.device = index, f"cuda:{index}"

    def get_device(self):
        return self.index


class _Flat(_On):
    dtype = torch.float32

    def __init__(self, index, n):
        super().__init__(index)
        self.n, self.shape = n, (n,)

    def numel(self):
        return self.n

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 256


@pytest.fixture()
def calls(monkeypatch):
    """Both calls on made-up buffers of given devices, device 0 the current one; the library itself is not reached."""
    monkeypatch.setattr(B, "_current_device", lambda: 0)
    monkeypatch.setattr(B, "_raw_stream", lambda device: 0)
    reached = []
    step = type("S", (), {n: staticmethod(lambda *a: reached.append(a) or 0) for n in ("ws_unpack_dropout", "ws_reduce_dropout")})
    monkeypatch.setattr(B, "_step", lambda: step)
    plan = B.Plan([(64, 8), (5,)], 4, upload=False)

    def run(r=-1, flat=0, plan_on=0, table=0, word=None):
        plan.dev_buf = _On(plan_on)
        lists = type("T", (), {"c": B.ws_tensor_table(256, 2, 2, 0, 32), "dev_buf": _On(table)})()
        drop = B.ws_dropout(0.1, 3, 0, 0)
        drop._keep = None if word is None else _On(word)
        buf = _Flat(flat, plan.G if r < 0 else plan.S)
        B.ws_unpack_dropout(plan, r, buf, lists, drop)
        B.ws_reduce_dropout(plan, r, lists, drop, buf)
        return len(reached)

    return run


def test_buffers_of_another_device(calls):
    assert calls() == 2 and calls(r=3, word=0) == 4
    for bad in (dict(flat=1), dict(plan_on=1), dict(table=1), dict(word=1), dict(flat=1, plan_on=1, table=1), dict(r=2, table=1)):
        with pytest.raises(ValueError):
            calls(**bad)
    assert calls() == 6


def test_numbers_that_32_bits_do_not_hold(calls):
    """Each would pass for a small one by its low 32 bits."""
    big = 1 << 32
    for replica in (big, big + 5, 1 << 31, -(1 << 31) - 1, 1 << 40):
        with pytest.raises(ValueError):
            B.make_dropout(0.1, 3, 0, replica)
    for r in (-2, 4, big, big + 1, big - 1, -big):
        with pytest.raises(ValueError):
            calls(r=r)
    q, x = [[torch.zeros(3, 2, dtype=torch.int64)]], [[torch.zeros(3, 8)]]
    for bad in (lambda: B.RouterSet(big + 8, q), lambda: B.RouterSet(8, logits=x, topk=big + 2), lambda: B.RouterSet(-big + 8, q)):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: B.RouterSet(8.0, q), lambda: B.RouterSet(8, logits=x, topk=2.0)):
        with pytest.raises(TypeError):
            bad()
    assert B.make_dropout(0.1, 3, 0, 65535).replica == 65535 and B.RouterSet(8, logits=x, topk=2).c.topk == 2
