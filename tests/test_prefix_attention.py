"""fe_prefix_attention on the GPU against float64, row by row: head layouts, types, page and tile
boundaries, rows that see nothing, stale contents, splits over long prefixes, bad indices."""
import numpy as np
import pytest

from tests import generation_oracle as O

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DEV = torch.device("cuda:0")
BF, HF = torch.bfloat16, torch.float16


def i32(a):
    return torch.tensor(np.asarray(a), dtype=torch.int32, device=DEV)


class Batch:
    """Groups of sequences with given lengths; page tables over shuffled pages, NaN wherever no row is held."""

    def __init__(self, seed, groups, prefix, lens, rows, hq, hkv, d, page, dtype, spread=1.0):
        rng = np.random.RandomState(seed)
        self.groups = np.concatenate([[0], np.cumsum(groups)])
        self.prefix, self.lens = np.array(prefix), np.array(lens)
        self.start = np.concatenate([[0], np.cumsum(rows)])
        S, T = len(lens), int(self.start[-1])
        n_pre, n_own = -(-self.prefix // page), -(-self.lens // page)
        n_pages = int(n_pre.sum() + n_own.sum()) + 3
        free = list(rng.permutation(n_pages))
        self.pre = np.full((len(prefix), max(1, n_pre.max())), -1)
        self.own = np.full((S, max(1, n_own.max())), -1)
        g = torch.Generator().manual_seed(seed)
        self.kc, self.vc = (torch.full((n_pages, hkv, page, d), float("nan"), dtype=dtype) for _ in range(2))
        for table, ln in ((self.pre, self.prefix), (self.own, self.lens)):
            for i, n in enumerate(ln):
                for c in range(-(-n // page)):
                    table[i, c] = free.pop()
                    m = min(page, n - c * page)
                    for x in (self.kc, self.vc):
                        x[table[i, c], :, :m] = torch.randn(hkv, m, d, generator=g).to(dtype)
        self.q = (torch.randn(T, hq, d, generator=g) * spread).to(dtype).to(DEV)
        self.kc, self.vc = self.kc.to(DEV), self.vc.to(DEV)
        self.dtype, self.d = dtype, d

    def args(self, **kw):
        a = dict(row_start=self.start, lengths=self.lens, pages=self.own, group_start=self.groups,
                 prefix_lengths=self.prefix, prefix_pages=self.pre)
        a.update(kw)
        return [i32(a[n]) for n in ("row_start", "lengths", "pages", "group_start", "prefix_lengths", "prefix_pages")]

    def check(self, scale=None, q=None):
        from paper_2603_02565_gb300 import PagedKV
        q = self.q if q is None else q
        status = i32([0])
        out, lse = PagedKV(self.kc, self.vc).attend(q, *self.args(), scale=scale, with_lse=True, status=status)
        assert status.item() == 0
        want, wl, eo, el = O.attend(q, self.kc, self.vc, self.start, self.lens, self.own, self.groups, self.prefix,
                                    self.pre, self.d ** -0.5 if scale is None else scale)
        got, gl, u = O.f64(out), O.f64(lse), O.U[self.dtype]
        empty = np.isneginf(wl)
        assert np.array_equal(np.isneginf(gl), empty) and np.all(got[empty] == 0)
        assert np.all(np.abs(gl[~empty] - wl[~empty]) <= el[~empty])
        # each weight is rounded to the type once (u), twice its relative error from the scores, then the result (u)
        bound = (u + 2 * el[..., None]) * eo + u * np.abs(want) + O.TINY[self.dtype] * 2 + 2.0 ** -24 * eo
        assert np.all(np.abs(got - want) <= bound), np.max(np.abs(got - want) / np.maximum(bound, 1e-30))
        return out, lse


LAYOUTS = [(1, 1, 32), (4, 4, 32), (8, 8, 64), (8, 2, 64), (3, 1, 128), (10, 2, 128), (16, 2, 32)]


@pytest.mark.parametrize("hq,hkv,d", LAYOUTS)
@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("page", [16, 64])
def test_one_row_per_sequence(hq, hkv, d, dtype, page):
    Batch(1, [3, 1, 5], [40, 0, 129], [1, 7, 16, 17, 33, 1, 64, 2, 130], [1] * 9, hq, hkv, d, page, dtype).check()


@pytest.mark.parametrize("hq,hkv,d", LAYOUTS)
@pytest.mark.parametrize("page", [32, 128])
def test_many_rows_per_sequence(hq, hkv, d, page):
    # rows of one sequence over several query tiles, sequences that share a tile, rows fewer than the length
    Batch(2, [2, 3], [70, 15], [50, 9, 1, 20, 37], [50, 4, 1, 20, 30], hq, hkv, d, page, BF).check()


@pytest.mark.parametrize("n", [1, 15, 16, 17, 127, 128, 129, 255, 256, 257])
def test_prefix_ends_around_pages_and_tiles(n):
    Batch(n, [2], [n], [3, 20], [1, 2], 4, 2, 64, 16, BF).check()
    Batch(n, [2], [0], [n, 5], [1, 1], 4, 2, 128, 128, HF).check()


def test_rows_that_see_nothing():
    # no prefix and no own row; rows before the sequence's first key; a group without sequences
    b = Batch(4, [2, 0, 1], [0, 30, 0], [0, 2, 1], [1, 4, 3], 4, 2, 64, 16, BF)
    out, lse = b.check()
    assert torch.isneginf(lse[0]).all() and torch.isneginf(lse[1:3]).all() and not torch.isneginf(lse[3:5]).any()


def test_a_sequence_without_rows_and_one_long_query_block():
    Batch(5, [3], [20], [4, 300, 6], [0, 300, 1], 2, 1, 32, 16, HF).check()


@pytest.mark.parametrize("d,hq,hkv", [(32, 2, 2), (64, 4, 1), (128, 8, 2)])
def test_long_prefixes_are_split_and_joined(d, hq, hkv):
    Batch(6, [3, 2], [5003, 777], [30, 1, 200, 9, 64], [1, 1, 2, 1, 1], hq, hkv, d, 64, BF).check()


def test_many_short_sequences():
    rng = np.random.RandomState(0)
    groups = rng.randint(1, 40, 20)
    S = int(groups.sum())
    Batch(7, groups, rng.randint(0, 60, 20), rng.randint(1, 9, S), [1] * S, 2, 2, 32, 16, BF).check()


@pytest.mark.parametrize("spread,scale", [(30.0, None), (0.01, None), (1.0, 0.0), (1.0, 3.0)])
def test_peaked_and_flat_weights(spread, scale):
    Batch(8, [2], [300], [40, 50], [1, 3], 4, 2, 64, 32, BF, spread).check(scale)


def test_scores_that_grow_along_the_keys():
    # every key tile has a larger maximum than all before it: the accumulators are rescaled each time
    b = Batch(9, [2], [700], [200, 90], [2, 1], 2, 1, 64, 16, HF)
    q = torch.ones_like(b.q)
    for table, ln in ((b.pre, b.prefix), (b.own, b.lens)):
        for i, n in enumerate(ln):
            for c in range(n):
                b.kc[table[i, c // 16], :, c % 16] = c * 0.02 - 3
    b.check(q=q)


def test_strided_queries():
    b = Batch(10, [3], [90], [5, 20, 33], [1, 4, 2], 6, 2, 64, 16, BF)
    wide = torch.randn(b.q.shape[0], 10, 64, device=DEV).to(BF)
    wide[:, 2:8] = b.q
    out, _ = b.check()
    from paper_2603_02565_gb300 import PagedKV
    assert torch.equal(PagedKV(b.kc, b.vc).attend(wide[:, 2:8], *b.args()), out)
    heads_first = b.q.transpose(0, 1).contiguous().transpose(0, 1)
    assert torch.equal(PagedKV(b.kc, b.vc).attend(heads_first, *b.args()), out)


def test_infinite_and_nan_keys_touch_only_the_rows_that_see_them():
    from paper_2603_02565_gb300 import PagedKV
    b = Batch(11, [2, 2], [100, 60], [20, 30, 10, 40], [1, 1, 1, 1], 2, 2, 64, 16, BF)
    clean = PagedKV(b.kc, b.vc).attend(b.q, *b.args()).clone()
    b.vc[b.own[1, 0], :, 3] = float("nan")    # a value of sequence 1
    b.kc[b.pre[1, 2], :, 5] = float("nan")    # a key of group 1's prefix
    out = PagedKV(b.kc, b.vc).attend(b.q, *b.args())
    assert torch.equal(out[0], clean[0])
    assert torch.isnan(out[1:]).all()


@pytest.mark.parametrize("what", ["page", "page_of_prefix", "length", "negative", "prefix_length"])
def test_bad_indices_spoil_their_own_rows_only(what):
    from paper_2603_02565_gb300 import PagedKV, FeError, check_status
    b = Batch(12, [2, 2], [100, 60], [20, 30, 10, 40], [1, 2, 1, 1], 4, 2, 32, 16, HF)
    clean = PagedKV(b.kc, b.vc).attend(b.q, *b.args()).clone()
    own, pre, lens, prefix = b.own.copy(), b.pre.copy(), b.lens.copy(), b.prefix.copy()
    if what == "page":
        own[1, 1] = b.kc.shape[0]
        bad = [1, 2]
    elif what == "page_of_prefix":
        pre[1, 0] = -1
        bad = [3, 4]
    elif what == "length":
        lens[3] = own.shape[1] * 16 + 1
        bad = [4]
    elif what == "negative":
        lens[0] = -1
        bad = [0]
    else:
        prefix[0] = pre.shape[1] * 16 + 1
        bad = [0, 1, 2]
    status = i32([0])
    out = PagedKV(b.kc, b.vc).attend(b.q, *b.args(pages=own, prefix_pages=pre, lengths=lens, prefix_lengths=prefix),
                                     status=status)
    with pytest.raises(FeError):
        check_status(status)
    good = [t for t in range(5) if t not in bad]
    assert torch.isnan(out[bad]).all() and torch.equal(out[good], clean[good])


def test_same_result_every_time_on_any_stream_and_in_a_graph():
    from paper_2603_02565_gb300 import PagedKV
    b = Batch(13, [4, 3], [3000, 500], [30] * 7, [1] * 7, 4, 2, 64, 16, BF)
    cache, a = PagedKV(b.kc, b.vc), b.args()
    want = cache.attend(b.q, *a).clone()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(5):
        assert torch.equal(cache.attend(b.q, *a), want)
        got = cache.attend(b.q, *a, stream=side)
        side.synchronize()
        assert torch.equal(got, want)
    n = cache.workspace_bytes(2, 7, 7, 4)
    ws = torch.full((n,), 255, dtype=torch.uint8, device=DEV)  # what a workspace holds before does not matter
    out = torch.empty_like(b.q)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        cache.attend(b.q, *a, out=out, workspace=ws)
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


def test_no_rows():
    from paper_2603_02565_gb300 import PagedKV
    b = Batch(14, [1], [5], [3], [0], 2, 2, 64, 16, BF)
    assert PagedKV(b.kc, b.vc).attend(b.q, *b.args()).shape == (0, 2, 64)


def test_pages_past_two_to_the_31_elements():
    # page numbers whose byte and element offsets need more than 32 bits
    from paper_2603_02565_gb300 import PagedKV
    n_pages, page, hkv, d = 2 ** 31 // (128 * 128) + 40, 128, 1, 128
    kc, vc = (torch.zeros(n_pages, hkv, page, d, dtype=BF, device=DEV) for _ in range(2))
    b = Batch(15, [2], [200], [30, 140], [1, 2], 2, 1, d, page, BF)
    far = n_pages - b.kc.shape[0]
    kc[far:], vc[far:] = b.kc, b.vc
    want = PagedKV(b.kc, b.vc).attend(b.q, *b.args())
    own, pre = np.where(b.own >= 0, b.own + far, -1), np.where(b.pre >= 0, b.pre + far, -1)
    assert torch.equal(PagedKV(kc, vc).attend(b.q, *b.args(pages=own, prefix_pages=pre)), want)
