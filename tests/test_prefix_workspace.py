"""The workspace that PagedKV keeps by thread and stream: calls of other sizes, on other streams and from other
threads leave each other's results alone."""
import threading

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from tests.test_prefix_attention import Batch  # noqa: E402


def batch(seed, groups, prefix, own):
    n = sum(groups)
    return Batch(seed, groups, prefix, [own] * n, [min(own, 3)] * n, 8, 2, 64, 16, torch.bfloat16)


def calls():
    """Three calls of unlike sizes over one cache each, with results of objects of their own."""
    from paper_2603_02565_gb300 import PagedKV
    out = []
    for b in (batch(1, [2], [5], 4), batch(2, [7] * 9, [900] * 9, 40), batch(3, [1, 30], [0, 4000], 3)):
        kv, a = PagedKV(b.kc, b.vc), b.args()
        out.append((kv, b.q, a, PagedKV(b.kc, b.vc).attend(b.q, *a)))
    torch.cuda.synchronize()
    return out


def test_sizes_in_any_order():
    from paper_2603_02565_gb300 import PagedKV
    big = batch(2, [7] * 9, [900] * 9, 40)
    kv = PagedKV(big.kc, big.vc)
    a = [x for x in big.args()]
    want = PagedKV(big.kc, big.vc).attend(big.q, *a)
    few = [a[0][:2].contiguous(), a[1][:1], a[2][:1], torch.tensor([0, 1], dtype=torch.int32, device="cuda"), a[4][:1], a[5][:1]]
    n = int(few[0][1])
    for _ in range(3):
        assert torch.equal(kv.attend(big.q[:n], *few), want[:n])
        assert torch.equal(kv.attend(big.q, *a), want)
    assert len(kv._spaces) == 1


def test_streams_and_threads():
    wrong = []

    def work(todo, stream):
        with torch.cuda.stream(stream):
            for _ in range(40):
                for kv, q, a, want in todo:
                    got = kv.attend(q, *a)
                    if not torch.equal(got, want):
                        wrong.append(got)
    todo = calls()
    one, two = torch.cuda.Stream(), torch.cuda.Stream()
    for streams in ((one, one), (one, two)):
        threads = [threading.Thread(target=work, args=(todo, s)) for s in streams]
        for t in threads:
            t.start()
        for t in threads:
            t.join()
    assert not wrong


def test_a_graph_has_its_own():
    (kv, q, a, want), *_ = calls()[1:]
    kv.attend(q, *a)
    kept = dict(kv._spaces)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = kv.attend(q, *a)
    assert kv._spaces == kept
    got.zero_()
    for _ in range(3):
        kv.attend(q, *a)
        g.replay()
    torch.cuda.synchronize()
    assert torch.equal(got, want)


def test_a_captured_stream_that_is_not_the_current_one():
    (kv, q, a, want), *_ = calls()[1:]
    s, other = torch.cuda.Stream(), torch.cuda.Stream()
    kv.attend(q, *a, stream=s)
    kept = dict(kv._spaces)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s), torch.cuda.stream(other):
        got = kv.attend(q, *a, stream=s)
    assert kv._spaces == kept
    for _ in range(2):
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, want)
