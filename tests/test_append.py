"""fe_kv_append on the GPU against float64, row by row: layouts, ragged sequences, strides, pairs and
types, and what it does with indices outside their range."""
import numpy as np
import pytest

from tests import generation_oracle as O

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DEV = torch.device("cuda:0")


def i32(a):
    return torch.tensor(np.asarray(a), dtype=torch.int32, device=DEV)


def make(seed, S, lo, hi, held, hq, hkv, d, page, dtype, strided=True):
    rng = np.random.RandomState(seed)
    rows = rng.randint(lo, hi + 1, S)
    first = rng.randint(0, held + 1, S)
    start = np.concatenate([[0], np.cumsum(rows)])
    n = -(-(first + rows) // page)
    n_pages = int(n.sum()) + 2
    table = np.full((S, max(1, n.max())), -1)
    free = rng.permutation(n_pages)
    for s in range(S):
        table[s, : n[s]], free = free[: n[s]], free[n[s]:]
    g = torch.Generator().manual_seed(seed)
    T = int(start[-1])
    x = torch.randn(T, hq + 2 * hkv, d, generator=g).to(dtype).to(DEV)
    parts = x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]
    if not strided:
        parts = tuple(p.contiguous() for p in parts)
    kc, vc = (torch.randn(n_pages, hkv, page, d, generator=g).to(dtype).to(DEV) for _ in range(2))
    return rows, first, start, table, parts, kc, vc


def rope_of(n, rot, seed=0):
    a = np.random.RandomState(seed).uniform(-3, 3, (n, rot // 2))
    return torch.tensor(np.stack([np.cos(a), np.sin(a)], -1), dtype=torch.float32, device=DEV)


def close(got, want, bound, dtype):
    got = O.f64(got)
    assert np.all(np.abs(got - want) <= O.U[dtype] * np.abs(want) + 2 * bound + O.TINY[dtype])


@pytest.mark.parametrize("pairs", ["half", "interleaved"])
@pytest.mark.parametrize("S,lo,hi,held,hq,hkv,d,page,rot,dtype", [
    (1, 1, 1, 0, 1, 1, 32, 16, 32, torch.bfloat16),        # one token of one head
    (4, 1, 1, 40, 8, 8, 64, 16, 64, torch.bfloat16),       # a step of several sequences
    (37, 0, 7, 90, 12, 4, 128, 64, 128, torch.float16),    # ragged, some without rows
    (70, 1, 1, 5, 3, 1, 64, 32, 32, torch.float16),        # partly rotated, odd heads, several search steps
    (3, 100, 300, 200, 5, 5, 32, 128, 16, torch.bfloat16),  # rows over several pages
    (2, 17, 40, 3, 40, 8, 128, 16, 48, torch.bfloat16),    # rot_dim no power of two
])
def test_matches_the_definition(S, lo, hi, held, hq, hkv, d, page, rot, dtype, pairs):
    from paper_2603_02565_gb300 import PagedKV
    rows, first, start, table, (q, k, v), kc, vc = make(S + d, S, lo, hi, held, hq, hkv, d, page, dtype)
    shift = np.random.RandomState(1).randint(0, 50, S)
    rope = rope_of(int((first + rows + shift).max()) + 1, rot)
    want = O.append(k, v, q, start, first, table, rope, pairs, shift, kc, vc)
    cache, status = PagedKV(kc, vc), i32([0])
    out = cache.append(k, v, i32(start), i32(first), i32(table), q=q, rope=rope, pairs=pairs, shift=i32(shift),
                       status=status)
    assert status.item() == 0
    close(kc, want[0], want[3], dtype)
    assert np.array_equal(O.f64(vc), want[1])
    close(out, want[2], want[4], dtype)


def test_without_rotation_and_queries_rows_are_copied():
    from paper_2603_02565_gb300 import PagedKV
    rows, first, start, table, (q, k, v), kc, vc = make(3, 9, 0, 5, 30, 2, 2, 64, 16, torch.float16, strided=False)
    want = O.append(k, v, None, start, first, table, None, "half", None, kc, vc)
    assert PagedKV(kc, vc).append(k, v, i32(start), i32(first), i32(table)) is None
    assert np.array_equal(O.f64(kc), want[0]) and np.array_equal(O.f64(vc), want[1])


def test_queries_may_be_rotated_in_place():
    from paper_2603_02565_gb300 import PagedKV
    rows, first, start, table, (q, k, v), kc, vc = make(5, 6, 1, 4, 9, 4, 2, 128, 16, torch.bfloat16, strided=False)
    rope = rope_of(40, 128)
    apart = PagedKV(kc.clone(), vc.clone()).append(k, v, i32(start), i32(first), i32(table), q=q, rope=rope)
    same = PagedKV(kc, vc).append(k, v, i32(start), i32(first), i32(table), q=q, rope=rope, q_out=q)
    assert same.data_ptr() == q.data_ptr() and torch.equal(same, apart)


def test_a_bad_page_or_position_spoils_its_own_rows_only():
    from paper_2603_02565_gb300 import PagedKV, FeError, check_status
    rows, first, start, table, (q, k, v), kc, vc = make(7, 6, 2, 2, 0, 2, 2, 32, 16, torch.bfloat16)
    rope = rope_of(2, 32)
    good = PagedKV(kc.clone(), vc.clone())
    q_good = good.append(k, v, i32(start), i32(first), i32(table), q=q, rope=rope)
    bad_table, bad_first = table.copy(), first.copy()
    bad_table[1, 0] = kc.shape[0]   # a page that does not exist
    bad_table[2, 0] = -1
    bad_first[4] = 16 * table.shape[1]  # past the page table; and past the positions of rope
    k0, v0 = kc.clone(), vc.clone()
    status = i32([0])
    cache = PagedKV(kc, vc)
    q_out = cache.append(k, v, i32(start), i32(bad_first), i32(bad_table), q=q, rope=rope, status=status)
    with pytest.raises(FeError):
        check_status(status)
    for s in range(6):
        pg = int(table[s, 0])
        want_k, want_v = (k0, v0) if s in (1, 2, 4) else (good.k, good.v)
        assert torch.equal(kc[pg], want_k[pg]) and torch.equal(vc[pg], want_v[pg]), s
        assert torch.equal(q_out[2 * s:2 * s + 2], q_good[2 * s:2 * s + 2]) == (s != 4)
    assert torch.isnan(q_out[8:10]).all()


def test_runs_on_the_stream_it_is_given_and_in_a_graph():
    from paper_2603_02565_gb300 import PagedKV
    rows, first, start, table, (q, k, v), kc, vc = make(11, 20, 1, 3, 20, 4, 2, 64, 32, torch.float16)
    rope = rope_of(64, 64)
    a = (i32(start), i32(first), i32(table))
    want = PagedKV(kc.clone(), vc.clone())
    want_q = want.append(k, v, *a, q=q, rope=rope)
    cache, side, out = PagedKV(kc, vc), torch.cuda.Stream(), torch.empty(q.shape, dtype=q.dtype, device=DEV)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        cache.append(k, v, *a, q=q, rope=rope, q_out=out)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want_q) and torch.equal(kc, want.k)
    got = cache.append(k, v, *a, q=q, rope=rope, stream=side)
    side.synchronize()
    assert torch.equal(got, want_q)
