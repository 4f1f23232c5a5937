"""How much memory attend's kept workspaces take: the layers of a model share one, those of threads that have ended go,
and calls of ever new sizes leave nothing behind."""
import gc
import threading

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from tests.test_prefix_attention import BF, Batch  # noqa: E402


def model(layers, seed=1, own=4):
    from paper_2603_02565_gb300 import PagedKV
    b = Batch(seed, [3, 2], [700, 90], [own] * 5, [1] * 5, 8, 2, 128, 16, BF)
    return b, b.args(), [PagedKV(b.kc.clone(), b.vc.clone()) for _ in range(layers)]


def held():
    gc.collect()
    torch.cuda.synchronize()
    return torch.cuda.memory_allocated()


def test_layers_share_a_workspace():
    b, a, caches = model(12)
    out = torch.empty_like(b.q)
    before = held()
    need = caches[0].workspace_bytes(2, 5, 5, 8)
    want = None
    for _ in range(2):
        for kv in caches:
            kv.attend(b.q, *a, out=out)
            want = out.clone() if want is None else want
            assert torch.equal(out, want)
    assert held() - before <= need + (1 << 21)
    del caches, kv
    assert held() - before <= 1 << 21


def test_they_grow_together():
    small, sa, caches = model(6)
    big = Batch(2, [600], [50], [3] * 600, [1] * 600, 8, 2, 128, 16, BF)
    ba = big.args()
    from paper_2603_02565_gb300 import PagedKV
    caches += [PagedKV(big.kc, big.vc)]
    outs = torch.empty_like(small.q), torch.empty_like(big.q)
    before = held()
    need = caches[0].workspace_bytes(1, 600, 600, 8)
    want = None
    for turn in range(3):
        for kv in caches[:-1]:
            kv.attend(small.q, *sa, out=outs[0])
            want = outs[0].clone() if want is None else want
            assert torch.equal(outs[0], want)
        caches[-1].attend(big.q, *ba, out=outs[1])
    for kv in caches[:-1]:  # (and as large a call of each)
        kv._spaces.clear()
        kv.attend(small.q, *sa, out=outs[0])
    assert held() - before <= need + (1 << 21)


def test_workspaces_of_ended_threads_go():
    b, a, (kv,) = model(1)
    out = torch.empty_like(b.q)
    kv.attend(b.q, *a, out=out)
    want = out.clone()
    before = held()
    wrong = []

    def work(gate, other):
        kv.attend(b.q, *a, out=other)
        torch.cuda.synchronize()
        if not torch.equal(other, want):
            wrong.append(other)
        gate.wait()
    for _ in range(3):
        gate = threading.Barrier(4)  # (threads at once, so that none takes another's name)
        threads = [threading.Thread(target=work, args=(gate, torch.empty_like(b.q))) for _ in range(4)]
        for t in threads:
            t.start()
        for t in threads:
            t.join()
    del threads, t
    assert not wrong
    assert len(kv._spaces) == 1 and held() - before <= 1 << 21


def test_ever_new_sizes_leave_nothing():
    b, a, (kv,) = model(1)
    n = {}
    for own in range(1, 40):
        c = Batch(own, [1], [5], [own], [own], 8, 2, 128, 16, BF)
        from paper_2603_02565_gb300 import PagedKV
        kv.k.zero_(), kv.v.zero_()
        m = min(c.kc.shape[0], kv.k.shape[0])
        args = c.args(pages=c.own.clip(0, m - 1), prefix_pages=c.pre.clip(0, m - 1))
        kv.attend(c.q, *args)
        n[own] = sum(len(x) for x in vars(kv).values() if isinstance(x, dict)) + len(kv._spaces)
    assert n[39] == n[1]
