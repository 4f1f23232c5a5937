"""The Python calls of the candidate generator's operators on the host, with a library that only looks on: whose device
is current when a call reaches it, and what it is given.  (CPU tensors say that they are on device -1: that plays another
device than the current one.)"""
import contextlib

import pytest

torch = pytest.importorskip("torch")

from paper_2603_02565_gb300 import generation as G  # noqa: E402

HERE, OTHER = 0, -1  # the current device, and the tensors'


class OnDevice(torch.Tensor):
    is_cuda = True


class Library:
    def __init__(self):
        self.current, self.calls = HERE, []

    def __getattr__(self, name):
        def call(*args):
            self.calls.append((name, self.current, args))
            return 256 if name.endswith("workspace") else 0
        return call


@pytest.fixture
def lib(monkeypatch):
    lib = Library()

    @contextlib.contextmanager
    def device(index):
        before, lib.current = lib.current, index
        try:
            yield
        finally:
            lib.current = before

    def capturing():
        lib.calls.append(("capturing", lib.current, ()))
        return False
    monkeypatch.setattr(G, "_LIB", lib)
    monkeypatch.setattr(G, "_current", lambda index: 7)
    monkeypatch.setattr(G, "_current_device", lambda: lib.current, raising=False)
    monkeypatch.setattr(G, "_capturing", capturing)
    monkeypatch.setattr(torch.cuda, "device", device)
    return lib


def cache(index=OTHER):
    x = torch.zeros(4, 2, 16, 32, dtype=torch.bfloat16)
    kv = G.PagedKV.__new__(G.PagedKV)
    kv.__dict__.update(k=x, v=x.clone(), device=x.device, dtype=x.dtype, n_pages=4, kv_heads=2, page_rows=16, head_dim=32,
                       _index=index, _fields=(0, 4, 16, 2, 32, 128, 128), _scale=1.0, _kept=G._Kept())
    return kv


def ints(*v):
    return torch.tensor(v, dtype=torch.int32)


def rows(heads, grad=False):
    return torch.zeros(3, heads, 32, dtype=torch.bfloat16, requires_grad=grad)


def append(kv, **kw):
    a = dict(k=rows(2), v=rows(2), row_start=ints(0, 1, 3), first=ints(0, 0), pages=ints(0, 1).view(2, 1), q=rows(4))
    return kv.append(**dict(a, **kw))


def attend(kv, **kw):
    a = dict(q=rows(4), row_start=ints(0, 1, 3), lengths=ints(1, 2), pages=ints(0, 1).view(2, 1), group_start=ints(0, 2),
             prefix_lengths=ints(0), prefix_pages=ints(2).view(1, 1))
    return kv.attend(**dict(a, **kw))


def loss(T=3, V=40, **kw):
    x = torch.zeros(T, V).as_subclass(OnDevice)
    return x, ints(*[0] * T), G.policy_loss(x, ints(*[0] * T), torch.zeros(T), **kw)


def test_calls_are_made_with_the_tensors_device_current(lib):
    append(cache())
    attend(cache())
    cache().workspace_bytes(1, 2, 3, 4)
    x, y, r = loss()
    G.policy_loss_backward(x, y, r)
    names = [n for n, *_ in lib.calls]
    assert {"fe_kv_append", "fe_prefix_attention_workspace", "capturing", "fe_prefix_attention", "fe_policy_loss",
            "fe_policy_loss_backward"} <= set(names)
    assert all(current == OTHER for _, current, _ in lib.calls)
    assert lib.current == HERE


def test_results_and_errors_come_through(lib):
    out, lse = attend(cache(), with_lse=True)
    assert out.shape == (3, 4, 32) and lse.shape == (3, 4)
    assert append(cache()).shape == (3, 4, 32) and append(cache(), q=None) is None
    with pytest.raises(ValueError):
        attend(cache(), lengths=ints(1, 2, 3))
    with pytest.raises(ValueError):
        append(cache(), pairs="even")
    assert lib.current == HERE


def test_nothing_is_switched_when_the_device_is_current(lib, monkeypatch):
    lib.current = OTHER

    def no(index):
        raise AssertionError("switched")
    monkeypatch.setattr(torch.cuda, "device", no)
    append(cache())
    attend(cache())
    loss()
    assert all(current == OTHER for _, current, _ in lib.calls)


class Elsewhere:
    cuda_stream, device_index = 9, 3


def test_a_stream_of_another_device_is_refused(lib, monkeypatch):
    monkeypatch.setattr(torch.cuda, "Stream", Elsewhere)
    for call in (lambda: append(cache(), stream=Elsewhere()), lambda: attend(cache(), stream=Elsewhere()),
                 lambda: loss(stream=Elsewhere())):
        with pytest.raises(ValueError):
            call()
    assert not any(n in ("fe_kv_append", "fe_prefix_attention", "fe_policy_loss") for n, *_ in lib.calls)
