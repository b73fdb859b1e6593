"""Page bookkeeping and page copies through the C ABI vs the sequential oracle:
every count, table entry, length, pair and result word has to be equal."""
import numpy as np
import pytest
import torch

from gpu_util import say, to_dev, to_host
from oracle.pages import BOUNDS, OK, Pages

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tk():
    from paper_2607_28633_amd import topkv
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return topkv


class Device:
    """An oracle state and the same on the device."""

    def __init__(self, tk, state, max_pairs=None):
        self.tk, self.host = tk, state
        self.refs = to_dev(np.array(state.refs, dtype=np.int32))
        self.tables = to_dev(state.tables.astype(np.int32))
        self.lens = to_dev(np.array(state.lens, dtype=np.int32))
        self.owner = tk.page_owner(self.refs, self.tables, self.lens, page_size=state.P)
        self.most = max(len(state.refs) // 2, len(state.lens), 1) if max_pairs is None else max_pairs
        self.pairs = torch.full((self.most + 3, 2), -7, dtype=torch.int32, device="cuda")
        self.work = torch.randint(-2**31, 2**31 - 1, (tk.topkv_pages_workspace_bytes(self.owner) // 4,),
                                  dtype=torch.int32, device="cuda")      # scratch needs no initial values
        self.result = torch.full((4,), 99, dtype=torch.int32, device="cuda")

    def call(self, name, *args, host_args=None):
        arrays = [to_dev(np.array(a, dtype=np.int32)) if a is not None else None for a in args]
        num = 0 if not arrays else len(args[0])
        if name == "count":
            self.tk.topkv_pages_count(self.owner, self.result)
        elif name == "free":
            self.tk.topkv_pages_free(self.owner, num, arrays[0], self.result, arrays[1] if len(arrays) > 1 else None)
        elif name == "compact":
            self.tk.topkv_pages_compact(self.owner, self.pairs, self.work, self.result, max_pairs=self.most)
        else:
            getattr(self.tk, f"topkv_pages_{name}")(self.owner, num, arrays[0], arrays[1], self.pairs, self.work,
                                                    self.result, max_pairs=self.most)
        torch.cuda.synchronize()
        want = getattr(self.host, name)(*args)
        self.check(name, want)
        return want

    def check(self, name, want):
        st, pairs, pages, bad = want
        got = self.result.tolist()
        assert got[0] == st and got[3] == bad, (name, got, want)
        assert got[1] == len(pairs), (name, got, want)
        if pages is not None:
            assert got[2] == pages, (name, got, want)
        assert [tuple(p) for p in self.pairs[:len(pairs)].tolist()] == [tuple(p) for p in pairs], name
        if name != "compact":
            assert (self.pairs[self.most:] == -7).all()
        assert self.refs.tolist() == self.host.refs, name
        assert np.array_equal(to_host(self.tables).view(np.int32), self.host.tables), name
        assert self.lens.tolist() == self.host.lens, name


def make(seed, rows, stride, pages, P, empty=0.3, zipf=False):
    rng = np.random.default_rng(seed)
    lens = rng.integers(0, stride * P + 1, rows)
    lens[rng.random(rows) < empty] = 0
    tables = np.full((rows, stride), -1)
    perm = rng.permutation(pages)
    at = 0
    for r in range(rows):
        k = -(-int(lens[r]) // P)
        if at + k > pages:
            lens[r] = 0
            continue
        tables[r, :k] = perm[at:at + k]
        at += k
    s = Pages([0] * pages, tables, lens, P)
    s.count()
    return s, rng


@pytest.mark.parametrize("rows,stride,pages,P", [(1, 1, 1, 1), (3, 2, 7, 16), (16, 9, 200, 16), (64, 5, 4096, 1),
                                                 (40, 30, 4097, 64), (300, 70, 30000, 3), (700, 3, 2500, 16)])
def test_random_steps(tk, rows, stride, pages, P):
    """Free, fork, grow and compact in turn, the state compared after every call."""
    say(f"[pages] {rows} rows x {stride}, {pages} pages of {P}")
    s, rng = make(rows + pages, rows, stride, pages, P)
    d = Device(tk, s)
    cap = stride * P
    d.call("count")
    for step in range(4):
        gone = rng.choice(rows, max(1, rows // 3), replace=False)
        keep = None if step % 2 else [int(rng.integers(0, max(1, s.lens[r] + 2))) for r in gone]
        d.call("free", *([gone] if keep is None else [gone, keep]))
        empty = [r for r in range(rows) if s.lens[r] == 0]
        if empty:
            kids = rng.permutation(empty)[:max(1, len(empty) // 2)]
            d.call("fork", rng.integers(0, rows, len(kids)), kids)
        some = rng.choice(rows, max(1, rows // 2), replace=False)
        d.call("grow", some, [int(min(cap, s.lens[r] + rng.integers(0, 2 * P + 2))) for r in some])
        if step % 2:
            d.call("compact")
    d.call("free", list(range(rows)))
    assert not any(s.refs)
    d.call("compact")


def test_grow_replaces_shared_partial_pages(tk):
    """Rows cut back inside pages that others share take pages of their own before they go on, all at once too."""
    say("[pages] copy on write")
    s = Pages([0] * 20, [[3, 5, -1], [-1] * 3, [-1] * 3, [9, -1, -1]], [7, 0, 0, 4], 4)
    d = Device(tk, s)
    d.call("count")
    d.call("fork", [0, 0], [1, 2])
    d.call("free", [0, 1, 2], [3, 2, 4])
    assert s.refs[3] == 3
    assert d.call("grow", [2, 0, 3], [4, 3, 4])[1] == []          # no token is added: nothing is written
    assert len(d.call("grow", [1, 0, 2], [3, 9, 12])[1]) == 2     # row 2 starts a page of its own
    assert s.refs[3] == 1
    d.call("compact")


def test_too_few_pages_changes_nothing(tk):
    say("[pages] out of pages")
    s = Pages([0] * 4, [[0, 1, -1, -1], [2, -1, -1, -1], [-1] * 4], [6, 1, 0], 4)
    d = Device(tk, s)
    d.call("count")
    assert d.call("grow", [0, 1], [9, 5])[:3] == (BOUNDS, [], 2)
    assert d.call("fork", [0, 0], [2, 2])[0] == BOUNDS            # the same child twice
    assert d.call("fork", [0], [2])[0] == OK
    assert d.call("grow", [1], [5])[:3] == (BOUNDS, [], 1)
    assert d.call("grow", [1], [4])[0] == OK


@pytest.mark.parametrize("call", [("fork", [0, 9], [2, 3]), ("fork", [0], [-1]), ("fork", [0], [4]), ("fork", [0], [1]),
                                  ("fork", [5], [2]), ("fork", [0, 0], [2, 2]), ("grow", [0, 0], [9, 9]),
                                  ("grow", [0], [5]), ("grow", [0], [17]), ("grow", [-2], [3]), ("grow", [6], [1]),
                                  ("grow", [0], [2**31 - 1]), ("grow", [0], [-1]),
                                  ("free", [-1, 0, 99]), ("free", [0, 1], [-5, 2]), ("free", [4, 0, 0], [0, 4, 1])])
def test_bad_rows(tk, call):
    """Rows out of range, not empty, named twice, of bad length: refused on the device."""
    say(f"[pages] {call}")
    s = Pages([0] * 30, [[3, 5, -1, -1], [7, 8, 9, 10], [-1] * 4, [-1] * 4, [1, -1, -1, -1], [2, -1, -1, -1]],
              [6, 16, 0, 0, 4, 3], 4)
    s.count()
    s.lens[5] = 17                                                # a length past the row's table
    d = Device(tk, s)
    d.call(*call)


@pytest.mark.parametrize("seed", range(4))
def test_bad_rows_are_counted_alike(tk, seed):
    """Rows named many times, some of their namings bad in themselves too: which of them counts as the good one does not
    depend on the order of the GPU's stores."""
    say(f"[pages] one row many times, seed {seed}")
    rng = np.random.default_rng(seed)
    rows, P = 700, 4
    s = Pages([0] * 900, np.full((rows, 3), -1), [0] * rows, P)
    s.count()
    assert s.grow([0, 1, 2], [12, 5, 3])[0] == OK
    d = Device(tk, s)
    some = rng.choice([3, 5, 699], 640)
    assert d.call("fork", rng.choice([0, 1, 2, 700, -1], 640), some)[0] == BOUNDS
    assert d.call("fork", [0] * 639 + [99999], some)[0] == BOUNDS
    assert d.call("grow", some, rng.choice([0, 4, 12, 13, -2], 640))[0] == BOUNDS
    assert d.call("grow", [5, 3], [9, 2])[0] == OK


def test_rows_given_back_several_times_at_once(tk):
    """Rows of many more pages than a workgroup has threads, named over and over in one call with different lengths to
    keep: each ends at the smallest, and every page comes back once."""
    say("[pages] rows named many times")
    rng = np.random.default_rng(11)
    rows, stride, P, pages = 5, 1500, 4, 9000
    tables = rng.permutation(pages)[:rows * stride].reshape(rows, stride)
    s = Pages([0] * pages, tables, [6000, 5999, 1027, 0, 4500], P)
    d = Device(tk, s)
    d.call("count")
    for most in (6001, 3000, 40):
        named = rng.integers(0, rows, 200)
        d.call("free", named, rng.integers(0, most, 200))
    d.call("free", [0, 1, 2, 3, 4] * 9)
    assert not any(s.refs)


def test_bad_entries(tk):
    """Entries that are no page are carried along or skipped, counted, and never followed."""
    say("[pages] hostile entries")
    bad = [-1, 30, 2**31 - 1, -2**31]
    s = Pages([0] * 30, [[29, bad[1], 28, 27], [bad[2], bad[3], 26, bad[1]], [-1] * 4, [-1] * 4], [15, 14, 0, 0], 4)
    d = Device(tk, s)
    d.call("count")
    d.call("fork", [0, 1], [2, 3])
    d.call("grow", [3, 1], [16, 15])
    d.call("compact")
    d.call("free", [0, 1, 2, 3], [5, 0, 0, 9])
    d.call("free", [0, 1, 2, 3])


def test_compact_with_entries_of_free_pages(tk):
    """Counts that do not agree with the tables: an entry of a free page at U or above is counted and stays, one below U
    stays too, and nothing else goes wrong."""
    say("[pages] compact, entries of free pages")
    refs, tables = to_dev(np.array([1, 0, 1, 0, 0, 0], np.int32)), to_dev(np.array([[0, 2], [4, 1]], np.int32))
    lens = to_dev(np.array([8, 7], np.int32))                     # an owner holds addresses, not the tensors
    owner = tk.page_owner(refs, tables, lens, page_size=4)
    work = torch.full((tk.topkv_pages_workspace_bytes(owner),), 0, dtype=torch.uint8, device="cuda")
    pairs, result = torch.zeros((3, 2), dtype=torch.int32, device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")
    tk.topkv_pages_compact(owner, pairs, work, result)
    assert result.tolist() == [BOUNDS, 1, 2, 1] and pairs[0].tolist() == [2, 1]
    assert refs.tolist() == [1, 1, 0, 0, 0, 0] and tables.tolist() == [[0, 1], [4, 1]]


def test_empty_calls(tk):
    s, _ = make(3, 4, 3, 20, 4)
    d = Device(tk, s)
    for name in ("free", "fork", "grow"):
        d.result.fill_(55)
        if name == "free":
            tk.topkv_pages_free(d.owner, 0, None, d.result)
        else:
            getattr(tk, f"topkv_pages_{name}")(d.owner, 0, None, None, d.pairs, d.work, d.result)
        assert d.result.tolist() == [0, 0, 0, 0]


def test_large_pool_and_last_page(tk):
    """A million pages, the free ones at the far end."""
    say("[pages] 2^20 + 5 pages")
    n = (1 << 20) + 5
    refs = np.ones(n, dtype=np.int32)
    refs[[5, n - 3, n - 1]] = 0
    refs_d = to_dev(refs)
    tables, lens = to_dev(np.full((2, 4), -1, dtype=np.int32)), to_dev(np.zeros(2, dtype=np.int32))
    owner = tk.page_owner(refs_d, tables, lens, page_size=16)
    work = torch.empty(tk.topkv_pages_workspace_bytes(owner), dtype=torch.uint8, device="cuda")
    pairs, result = torch.zeros((n // 2, 2), dtype=torch.int32, device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")
    tk.topkv_pages_grow(owner, 2, to_dev(np.array([1, 0], np.int32)), to_dev(np.array([20, 16], np.int32)), pairs, work, result)
    assert result.tolist() == [0, 0, 3, 0] and tables[:, :2].tolist() == [[n - 1, -1], [5, n - 3]]
    assert int((refs_d != 1).sum()) == 0
    tk.topkv_pages_free(owner, 2, to_dev(np.array([0, 1], np.int32)), result)
    tk.topkv_pages_compact(owner, pairs, work, result)
    assert result.tolist() == [0, 1, n - 3, 0] and pairs[0].tolist() == [n - 2, 5]


@pytest.mark.parametrize("shape,elem", [((3, 20, 2, 16, 8, 128), 2), ((2, 9, 2, 5, 7, 25), 2), ((1, 6, 1, 64, 1, 576), 2),
                                        ((2, 5, 1, 1, 1, 3), 1), ((2, 7, 2, 16, 2, 20), 4), ((1, 3, 2, 300, 8, 130), 8)])
@pytest.mark.parametrize("same", [True, False])
def test_copy_pages(tk, shape, elem, same):
    """Every layer of a range, other pages untouched, bad pairs skipped, a count below, at and past the pairs."""
    say(f"[pages] copy {shape} x {elem}")
    rng = np.random.default_rng(shape[1])
    src_h = rng.integers(0, 256, shape + (elem,), dtype=np.uint8)
    dst_h = src_h if same else rng.integers(0, 256, (shape[0], shape[1] + 2) + shape[2:] + (elem,), dtype=np.uint8)
    word = {1: np.uint8, 2: np.uint16, 4: np.uint32, 8: np.uint64}[elem]
    src = to_dev(src_h.view(word)[..., 0])
    dst = src if same else to_dev(dst_h.view(word)[..., 0])
    order = rng.permutation(shape[1])
    pairs = [(int(order[0]), int(order[1])), (-1, int(order[2])), (shape[1], int(order[2])), (int(order[0]), 2**31 - 1),
             (int(order[0]), -5)]
    if not same:
        pairs += [(int(order[0]), shape[1] + 1), (int(order[2]), int(order[2]))]
    dev = to_dev(np.array(pairs, dtype=np.int32))
    for first, layers, count in ((0, shape[0], None), (shape[0] - 1, 1, 1), (0, shape[0], 0), (0, shape[0], -3),
                                 (0, shape[0], 10**6)):
        want = dst_h.copy()
        cnt = None if count is None else to_dev(np.array([count], dtype=np.int32))
        tk.topkv_copy_pages(src, dst, first, layers, dev, count=cnt)
        torch.cuda.synchronize()
        for s, t in pairs[:len(pairs) if count is None else max(0, count)]:
            if 0 <= s < shape[1] and 0 <= t < want.shape[1]:
                want[first:first + layers, t] = src_h[first:first + layers, s]
        assert np.array_equal(to_host(dst).view(np.uint8).reshape(want.shape), want), (first, layers, count)
        dst_h[...] = want


def test_copy_pages_past_32_bits(tk):
    """Pages that lie beyond 4 GiB of a layer, in the second of two layers."""
    say("[pages] copy past 4 GiB")
    pages = 70000
    pool = torch.empty((2, pages, 2, 16, 8, 128), dtype=torch.int16, device="cuda")
    pool[1, 3] = 7
    pool[1, pages - 1] = torch.arange(2 * 16 * 8 * 128, device="cuda", dtype=torch.int32).to(torch.int16).view(2, 16, 8, 128)
    tk.topkv_copy_pages(pool, pool, 1, 1, to_dev(np.array([[pages - 1, 3], [3, pages - 2]][:1], dtype=np.int32)))
    assert torch.equal(pool[1, 3], pool[1, pages - 1])
    tk.topkv_copy_pages(pool, pool, 1, 1, to_dev(np.array([[3, pages - 2]], dtype=np.int32)))
    assert torch.equal(pool[1, pages - 2], pool[1, pages - 1])


def test_captured_steps(tk):
    """A beam step in a graph, replayed over changing tables with eager work between the replays."""
    say("[pages] captured beam step")
    rows, beams, P, stride, pages = 3, 4, 4, 6, 60
    rng = np.random.default_rng(5)
    tables = np.full((rows * (1 + beams), stride), -1)
    perm, at = rng.permutation(pages), 0
    lens = [7, 12, 5] + [0] * (rows * beams)
    for r in range(rows):
        for j in range(-(-lens[r] // P)):
            tables[r, j] = perm[at]
            at += 1
    s = Pages([0] * pages, tables, lens, P)
    s.count()
    d = Device(tk, s)
    pool = torch.randint(-30000, 30000, (2, pages, 2, P, 1, 8), dtype=torch.int16, device="cuda")
    kids_h = list(range(rows, rows * (1 + beams)))
    kids = to_dev(np.array(kids_h, dtype=np.int32))
    parents = to_dev(np.zeros(len(kids_h), dtype=np.int32))

    def step():
        tk.topkv_pages_free(d.owner, len(kids_h), kids, d.result)
        tk.topkv_pages_fork(d.owner, len(kids_h), parents, kids, d.pairs, d.work, d.result)
        tk.topkv_copy_pages(pool, pool, 0, 2, d.pairs, max_pairs=len(kids_h), count=d.result[1:])

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        step()
        side.synchronize()
        s.free(kids_h), s.fork([0] * len(kids_h), kids_h)
        with torch.cuda.graph(graph, stream=side):
            step()
    torch.cuda.current_stream().wait_stream(side)
    for k in range(4):
        chosen = rng.integers(0, rows, len(kids_h))
        parents.copy_(to_dev(chosen.astype(np.int32)))
        before = pool.clone()
        graph.replay()
        torch.cuda.synchronize()
        s.free(kids_h)
        want = s.fork(list(chosen), kids_h)
        d.check("fork", want)
        for a, b in want[1]:
            before[:, b] = before[:, a]
        assert torch.equal(pool, before)
        d.call("grow", [0], [s.lens[0] + 1])           # eager work between the replays
