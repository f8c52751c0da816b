"""Page tables on the GPU against a plain mirror on the host: whole numbers, all equal."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
mcd = pytest.importorskip("paper_2607_02119_amd.mcd", reason="libmcd.so not built")

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="no GPU")]


def i32(a):
    return torch.from_numpy(np.ascontiguousarray(a, np.int32)).to("cuda")


class Mirror:
    def __init__(self, table, n_pages):
        self.table, self.n_pages = table.copy(), n_pages

    def refs(self):
        held = self.table[self.table >= 0]
        return np.bincount(held, minlength=self.n_pages)

    def release(self, slot, length):
        for s, n in zip(slot, length):
            self.table[s, -(-max(n, 0) // 64):] = -1

    def share(self, slot, source, length):
        old, bad = self.table.copy(), False
        for s, f, n in zip(slot, source, length):
            for c in range(min(max(n, 0) // 64, self.table.shape[1])):
                if old[f, c] < 0 or self.table[s, c] >= 0:
                    bad = True
                else:
                    self.table[s, c] = old[f, c]
        return bad

    def reserve(self, slot, context, tokens):
        """where, row and position of all tokens; what the status word says."""
        free = np.flatnonzero(self.refs() == 0).tolist()
        shared, status = self.refs() > 1, 0
        where, row, position = [], [], []
        for r, (s, ctx, n) in enumerate(zip(slot, context, tokens)):
            for p in range(ctx, ctx + n):
                page = self.table[s, p // 64]
                if page < 0:
                    if free:
                        page = self.table[s, p // 64] = free.pop(0)
                    else:
                        status |= mcd.MCD_DEV_NO_PAGE
                elif shared[page]:
                    page, status = -1, status | mcd.MCD_DEV_BAD_PAGE
                where.append(page * 64 + p % 64 if page >= 0 else -1)
                row.append(r)
                position.append(p)
        return np.array(where, int), np.array(row, int), np.array(position, int), status


class Both:
    """A table on the GPU and its mirror; every call is compared."""

    def __init__(self, n_slots, columns, n_pages, table=None, rows=None):
        table = np.full((n_slots, columns), -1, np.int32) if table is None else table
        self.mirror = Mirror(table, n_pages)
        self.pages = mcd.CachePages(i32(table), n_pages)
        self.ws = self.pages.workspace(rows or n_slots)
        self.ws[256:] = 255                         # (only the status word is zeroed)
        self.check(0)

    def check(self, status):
        assert mcd.mcd_read_device_status(self.ws) == status
        assert np.array_equal(self.pages.table.cpu().numpy(), self.mirror.table)
        assert np.array_equal(self.pages.refs.cpu().numpy(), self.mirror.refs())

    def release(self, slot, length=None):
        mcd.mcd_cache_release(self.pages, i32(slot), self.ws,
                              length=None if length is None else i32(length))
        self.mirror.release(slot, length if length is not None else [0] * len(slot))
        self.check(0)

    def share(self, slot, source, length):
        mcd.mcd_cache_share(self.pages, i32(slot), i32(source), i32(length), self.ws)
        bad = self.mirror.share(slot, source, length)
        self.check(mcd.MCD_DEV_BAD_PAGE if bad else 0)

    def reserve(self, slot, context, tokens, spare=0, max_tokens=None, maps=True):
        context, tokens = np.asarray(context), np.asarray(tokens)
        N, R = int(tokens.sum()), len(tokens)
        full = lambda n, dt: torch.full((n,), 77, dtype=dt, device="cuda")  # noqa: E731
        start = full(R + 1, torch.int32)
        where, row, position = (full(N + spare, dt) for dt in (torch.int64, torch.int32, torch.int32))
        print(f"case reserve R={R} N={N} pages={self.mirror.n_pages}", flush=True)
        mcd.mcd_cache_reserve(
            self.pages, i32(context), i32(tokens), start, self.ws,
            slot=None if slot is None else i32(slot), n_tokens=N + spare,
            max_tokens=int(tokens.max(initial=0)) if max_tokens is None else max_tokens,
            max_context=int((context + tokens).max(initial=0)), where=where if maps else None,
            row=row if maps else None, position=position if maps else None)
        want = self.mirror.reserve(range(R) if slot is None else slot, context, tokens)
        assert start.tolist() == np.concatenate([[0], np.cumsum(tokens)]).tolist()
        if maps:
            for got, w in zip((where, row, position), want):
                got = got.cpu().numpy()
                assert np.array_equal(got[:N], w) and (got[N:] == 77).all()
        self.check(want[3])


def random_table(rng, slots, columns, n_pages, counts):
    table, ids, at = np.full((slots, columns), -1, np.int32), rng.permutation(n_pages), 0
    for s, c in enumerate(counts):
        table[s, :c] = ids[at:at + c]
        at += c
    return table


@pytest.mark.parametrize("R,columns,n_pages", [(1, 1, 1), (3, 4, 13), (65, 9, 700), (200, 20, 5001),
                                               (513, 5, 4096), (1000, 30, 9000),
                                               (1500, 6, 9000), (700, 60, 40000)])
def test_steps(R, columns, n_pages):
    rng = np.random.default_rng(R)
    most = max(n_pages // R - 1, 0)
    counts = rng.integers(0, min(columns, most) + 1, R)
    b = Both(R, columns, n_pages, random_table(rng, R, columns, n_pages, counts))
    context = counts * 64 - np.where(counts > 0, rng.integers(0, 64, R), 0)
    room = columns * 64 - context
    for many in (2, 100):
        tokens = np.minimum(rng.integers(0, many, R), room)
        slot = rng.permutation(R)
        b.reserve(slot, context[slot], tokens[slot], spare=3)
        context, room = context + tokens, room - tokens
    keep = rng.integers(0, context + 1)
    b.release(np.arange(R), keep)
    # nothing new: a step without a token
    b.reserve(None, keep, np.zeros(R, int), spare=1, max_tokens=1)
    b.reserve(None, keep, np.minimum(65, columns * 64 - keep), maps=False)


def test_long_rows():
    """Rows of many tokens beside rows of one: more columns of a row than a wave has lanes."""
    b = Both(6, 300, 700)
    b.reserve([5, 0, 2, 1], [0, 0, 0, 0], [1500, 1, 0, 9000])
    b.reserve([1, 2, 0, 5, 3], [9000, 0, 1, 1500, 0], [4097, 70, 1, 130, 5000])
    b.release([1, 5, 3], [13, 1500, 64])
    b.reserve([3, 1], [64, 13], [12000, 63])


@pytest.mark.parametrize("groups,rows", [(1, 1), (1, 70), (7, 300)])
def test_candidates_begin_on_their_prompts_pages(groups, rows):
    rng = np.random.default_rng(rows)
    columns = 12
    b = Both(groups + rows, columns, groups * 10 + rows * 6 + 3)
    prompts, slots = np.arange(groups), groups + rng.permutation(rows)
    base = rng.integers(0, 600, groups)
    b.reserve(prompts, np.zeros(groups, int), base, spare=1)
    of = rng.integers(0, groups, rows)
    for _ in range(2):
        b.release(slots)
        b.share(slots, prompts[of], base[of])
        context = base[of] // 64 * 64
        b.reserve(slots, context, rng.integers(0, 90, rows), spare=1)
    # the prompts go first: their pages stay while a candidate holds them
    b.release(prompts)
    b.release(np.concatenate([slots, slots, prompts]))   # the same slot twice
    assert not b.mirror.refs().any()


def test_out_of_pages():
    b = Both(4, 4, 6)
    b.reserve(None, [0, 0, 0, 0], [100, 64, 200, 1])     # 2 + 1 + 4 + 1 pages wanted
    b.release([1])
    b.reserve([3], [0], [64])


def test_many_pages():
    """More pages than 1024 chunks of the smallest size, the free ones far apart."""
    n_pages = (1 << 22) + 4097
    rng = np.random.default_rng(1)
    held = rng.permutation(n_pages)[:n_pages - 60]
    table = np.full((3 + 2100, 2000), -1, np.int32)
    flat = table[3:].reshape(-1)
    flat[:len(held)] = held
    b = Both(table.shape[0], 2000, n_pages, table, rows=3)
    b.reserve([0, 2, 1], [0, 0, 0], [1000, 2000, 900])   # 16 + 32 + 15 pages, 60 there
    assert (b.mirror.table[:3] >= 0).sum() == 60


def test_shared_entries_and_taken_entries():
    b = Both(4, 6, 20)
    b.reserve([0], [0], [300])
    b.share([1, 2], [0, 0], [256, 300])                  # 4 pages each
    b.share([1], [0], [300])                             # held already
    b.share([3], [0], [500])                             # more than there is
    b.reserve([1, 3], [250, 256], [10, 3])               # positions of a shared page: no place


def test_bad_rows_are_reported():
    b = Both(3, 2, 8)
    table = b.pages.table.clone()
    ws, one = b.ws, i32([5])
    start = torch.zeros(2, dtype=torch.int32, device="cuda")
    where = torch.full((4,), 9, dtype=torch.int64, device="cuda")

    def bad(slot, context, tokens, **kw):
        a = dict(n_tokens=4, max_tokens=4, max_context=128)
        a.update(kw)
        mcd.mcd_cache_reserve(b.pages, i32([context]), i32([tokens]), start, ws, slot=i32([slot]),
                              where=where, **a)
        assert mcd.mcd_read_device_status(ws) == mcd.MCD_DEV_BAD_PAGE
        return where.tolist(), start.tolist()

    assert bad(3, 0, 2) == ([-1, -1, 9, 9], [0, 2])
    assert bad(-1, 0, 1) == ([-1, -1, 9, 9], [0, 1])
    assert torch.equal(b.pages.table, table)
    assert bad(0, -1, 2) == ([-1, 0, 9, 9], [0, 2])      # position -1 has no place, position 0 has
    assert bad(0, 126, 3)[0][:3] == [1 * 64 + 62, 1 * 64 + 63, -1]
    assert bad(1, 0, -5)[1] == [0, 0]
    assert bad(1, 0, 9)[1] == [0, 4]
    assert bad(1, 100, 3, max_context=101)[0][1:3] == [-1, -1]
    for f in (lambda: mcd.mcd_cache_release(b.pages, one, ws),
              lambda: mcd.mcd_cache_release(b.pages, i32([2]), ws, length=i32([-1])),
              lambda: mcd.mcd_cache_share(b.pages, one, i32([0]), i32([64]), ws),
              lambda: mcd.mcd_cache_share(b.pages, i32([2]), one, i32([64]), ws),
              lambda: mcd.mcd_cache_share(b.pages, i32([2]), i32([0]), i32([-64]), ws)):
        f()
        assert mcd.mcd_read_device_status(ws) == mcd.MCD_DEV_BAD_PAGE
    # an entry beyond the pages, and one that was never counted
    b.pages.table[2, 0], b.pages.table[2, 1] = 8, 7
    mcd.mcd_cache_release(b.pages, i32([2]), ws)
    assert mcd.mcd_read_device_status(ws) == mcd.MCD_DEV_BAD_PAGE
    assert b.pages.table[2].tolist() == [-1, -1] and (b.pages.refs >= 0).all()
    assert mcd.mcd_cache_count(b.pages, ws) is None
    assert torch.equal(b.pages.refs, torch.bincount(
        b.pages.table[b.pages.table >= 0], minlength=8).int())


def test_a_slot_named_twice_loses_no_page():
    b = Both(2, 4, 9)
    start = torch.zeros(3, dtype=torch.int32, device="cuda")
    mcd.mcd_cache_reserve(b.pages, i32([0, 0]), i32([100, 100]), start, b.ws, slot=i32([1, 1]),
                          n_tokens=200, max_tokens=100, max_context=100)
    mcd.mcd_read_device_status(b.ws)
    held = b.pages.table[b.pages.table >= 0]
    assert len(held) == 2 and torch.equal(
        b.pages.refs, torch.bincount(held, minlength=9).int())
    # more tokens than one launch takes, and shares into one slot and from a slot of the call
    mcd.mcd_cache_release(b.pages, i32([1]), b.ws)
    mcd.mcd_cache_reserve(b.pages, i32([0, 0]), i32([5, 8]), start, b.ws, slot=i32([1, 1]),
                          n_tokens=20, max_tokens=8, max_context=100)
    for slot, source in (([0, 0, 0], [1, 1, 1]), ([1, 0], [0, 1])):
        mcd.mcd_cache_share(b.pages, i32(slot), i32(source), i32([64] * len(slot)), b.ws)
        held = b.pages.table[b.pages.table >= 0]
        assert torch.equal(b.pages.refs, torch.bincount(held, minlength=9).int())
    mcd.mcd_read_device_status(b.ws)


def test_captured_and_replayed():
    """Release, share and reserve in a graph; replays take new lengths from the device."""
    rng = np.random.default_rng(8)
    R = 40
    b = Both(R + 1, 8, 300)
    b.reserve([R], [0], [200])
    slot, source, length = i32(np.arange(R)), i32(np.full(R, R)), i32(np.full(R, 200))
    context, tokens = i32(np.full(R, 192)), i32(np.zeros(R))
    start = torch.zeros(R + 1, dtype=torch.int32, device="cuda")
    where = torch.zeros(R * 100, dtype=torch.int64, device="cuda")

    def calls():
        mcd.mcd_cache_release(b.pages, slot, b.ws)
        mcd.mcd_cache_share(b.pages, slot, source, length, b.ws)
        mcd.mcd_cache_reserve(b.pages, context, tokens, start, b.ws, slot=slot, n_tokens=R * 100,
                              max_tokens=100, max_context=300, where=where)

    calls()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for _ in range(4):
        new = rng.integers(0, 101, R)
        tokens.copy_(i32(new))
        graph.replay()
        b.mirror.release(range(R), [0] * R)
        b.mirror.share(range(R), [R] * R, [200] * R)
        want = b.mirror.reserve(range(R), [192] * R, new)
        N = int(new.sum())
        assert np.array_equal(where.cpu().numpy()[:N], want[0])
        b.check(want[3])


def test_release_of_lengths_out_of_range_gives_nothing_back():
    """A length below 0 or beyond the table is reported and its row keeps every page; the other
    rows of the call give theirs back."""
    b = Both(4, 3, 12)
    b.reserve(None, [0, 0, 0, 0], [192, 130, 64, 192])
    for lengths in ([-1, 65, 64, 193], [-2 ** 31, 65, 0, 2 ** 31 - 1], [-64, 1, 0, 256]):
        mcd.mcd_cache_release(b.pages, i32([0, 1, 2, 3]), b.ws, length=i32(lengths))
        b.mirror.release([1, 2], lengths[1:3])
        b.check(mcd.MCD_DEV_BAD_PAGE)
        assert (b.mirror.table[[0, 3]] >= 0).all()
    b.release([0, 3], [192, 129])                    # the table's whole length, and into its last page
    assert (b.mirror.table[[0, 3]] >= 0).all()
    # named twice, once out of range: the other length holds
    mcd.mcd_cache_release(b.pages, i32([0, 0]), b.ws, length=i32([-5, 64]))
    b.mirror.release([0], [64])
    b.check(mcd.MCD_DEV_BAD_PAGE)


def test_count_of_more_entries_than_a_launch_has_threads():
    slots, columns, n_pages = (1 << 18) + 1, 1 << 14, 1000         # 2^32 + 2^14 entries
    table = torch.full((slots, columns), -1, dtype=torch.int32, device="cuda")
    flat, rng = table.view(-1), np.random.default_rng(0)
    at = np.unique(np.concatenate([rng.integers(0, slots * columns, 5000), [0, (1 << 32) - 257,
                                   (1 << 32) - 256, (1 << 32) - 1, 1 << 32, slots * columns - 1]]))
    ids = rng.integers(0, n_pages, len(at))
    flat[torch.from_numpy(at).cuda()] = i32(ids)
    pages = mcd.CachePages(table, n_pages)
    assert np.array_equal(pages.refs.cpu().numpy(), np.bincount(ids, minlength=n_pages))
    # release and share of the last slot
    ws, last = pages.workspace(1), i32([slots - 1])
    mcd.mcd_cache_share(pages, i32([slots - 2]), last, i32([columns * 64]), ws)
    mcd.mcd_read_device_status(ws)
    mcd.mcd_cache_release(pages, last, ws)
    mcd.mcd_cache_release(pages, i32([slots - 2]), ws)
    assert mcd.mcd_read_device_status(ws) == 0 and bool((table[-2:] == -1).all())
    want = np.bincount(ids[at < (slots - 2) * columns], minlength=n_pages)
    assert np.array_equal(pages.refs.cpu().numpy(), want)


def test_a_table_that_names_other_pages():
    """Refused where the pages are counted, or reported in the workspace that the count is given;
    the entries within are counted."""
    table = i32([[0, 4, -1], [4, 5, 2 ** 31 - 1], [-7, 2, 0]])
    with pytest.raises(ValueError, match="from n_pages"):
        mcd.CachePages(table, 5)
    ws = torch.zeros(256, dtype=torch.uint8, device="cuda")
    pages = mcd.CachePages(table, 5, workspace=ws)
    assert mcd.mcd_read_device_status(ws) == mcd.MCD_DEV_BAD_PAGE
    assert pages.refs.tolist() == [2, 0, 1, 0, 2]
    table[1, 1:] = -1
    assert mcd.CachePages(table, 5).refs.tolist() == [2, 0, 1, 0, 2]
    mcd.CachePages(table, 5, workspace=ws)
    assert mcd.mcd_read_device_status(ws) == 0
    # within a capture nothing waits
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = mcd.CachePages(table, 5)
    graph.replay()
    assert captured.refs.tolist() == [2, 0, 1, 0, 2]


@pytest.mark.parametrize("captured", [False, True], ids=["eager", "captured"])
@pytest.mark.parametrize("tokens", [[1, 1, 1], [40, 2, 1], [70, 100, 0]], ids=str)
def test_no_call_writes_to_a_shared_page(tokens, captured):
    """A row that was cut off within a page that others hold: its new tokens there have no place, and
    an append of the cache with refs leaves the page alone; every other token is written."""
    rng = np.random.default_rng(sum(tokens))
    H, D, n_pages = 2, 64, 30
    b = Both(4, 6, n_pages)
    pages = torch.from_numpy(rng.integers(0, 256, (n_pages, H, mcd.mcd_cache_page_bytes(D)),
                                          dtype=np.uint8)).cuda()
    cache = mcd.Cache(pages, b.pages.table, D, refs=b.pages.refs)
    plain = mcd.Cache(pages, b.pages.table, D)
    b.reserve([0], [0], [150])
    b.share([1, 2, 3], [0, 0, 0], [150] * 3)             # two pages each, by all
    b.reserve([1, 2, 3], [128] * 3, [9, 20, 9])
    b.release([1, 3], [100, 60])                         # within their second and first pages
    slot, context = [1, 2, 3], [100, 148, 60]
    N, most = sum(tokens), max(tokens)
    kv = torch.randn((N, 2, H, D), device="cuda")
    start = torch.zeros(4, dtype=torch.int32, device="cuda")
    where = torch.zeros(N, dtype=torch.int64, device="cuda")
    before, ctx, new, at = pages.clone(), i32(context), i32(tokens), i32(slot)
    rows = mcd.CacheRows(ctx, start=start, slot=at, n_tokens=N, max_tokens=most, max_context=384)
    kr, vr = (torch.full((N, H, D), 9.0, device="cuda") for _ in range(2))

    def calls():
        mcd.mcd_cache_reserve(b.pages, ctx, new, start, b.ws, slot=at, n_tokens=N, max_tokens=most,
                              max_context=384, where=where)
        mcd.mcd_cache_append(cache, rows, kv[:, 0], kv[:, 1], b.ws)

    if captured:
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            calls()
        graph.replay()
    else:
        calls()
    want = b.mirror.reserve(slot, context, tokens)
    assert np.array_equal(where.cpu().numpy(), want[0]) and (want[0] == -1).any()
    b.check(mcd.MCD_DEV_BAD_PAGE)                        # reserve's and append's
    mcd.mcd_cache_append(cache, rows, kv[:, 0], kv[:, 1], b.ws)
    assert mcd.mcd_read_device_status(b.ws) == mcd.MCD_DEV_BAD_PAGE
    # the pages of other slots, and those that nothing was appended to, as they were
    touched = np.unique(want[0][want[0] >= 0] // 64)
    others = np.setdiff1d(np.arange(n_pages), touched)
    assert torch.equal(pages[others], before[others])
    assert set(b.mirror.table[0, :3]) <= set(others)
    # what has a place was written: as an append of those tokens alone, to a copy of the pages
    mcd.mcd_cache_read(plain, rows, kr, vr, b.ws)
    assert mcd.mcd_read_device_status(b.ws) == 0
    copy = mcd.Cache(before.clone(), i32(np.arange(n_pages)[:, None]), D)
    for t in np.flatnonzero(want[0] >= 0):
        page, pos = divmod(int(want[0][t]), 64)
        one = mcd.CacheRows(i32([pos]), slot=i32([page]), n_tokens=1, max_tokens=1, max_context=64)
        mcd.mcd_cache_append(copy, one, kv[t:t + 1, 0], kv[t:t + 1, 1], b.ws)
        k1, v1 = (torch.zeros((1, H, D), device="cuda") for _ in range(2))
        mcd.mcd_cache_read(copy, one, k1, v1, b.ws)
        assert torch.equal(k1[0], kr[t]) and torch.equal(v1[0], vr[t])
    assert mcd.mcd_read_device_status(b.ws) == 0
    if most == 1:
        assert torch.equal(copy.pages, pages)


def test_no_eviction_writes_to_a_shared_page():
    rng = np.random.default_rng(5)
    H, D, n_pages = 2, 64, 12
    pages = torch.from_numpy(rng.integers(0, 256, (n_pages, H, mcd.mcd_cache_page_bytes(D)),
                                          dtype=np.uint8)).cuda()
    src = mcd.Cache(pages, i32([[0, 1, 2]]), D)
    refs = i32([1] * n_pages)
    refs[5] = 2
    to = mcd.Cache(pages, i32([[4, 5, 6]]), D, refs=refs)
    ws = torch.zeros(256, dtype=torch.uint8, device="cuda")
    kept = torch.zeros((1, H, 192), dtype=torch.int32, device="cuda")
    out, before = torch.zeros(1, dtype=torch.int32, device="cuda"), pages.clone()
    mcd.mcd_cache_evict(src, to, i32([192]), 192, 192, kept, out, ws, 192)
    assert mcd.mcd_read_device_status(ws) == mcd.MCD_DEV_BAD_PAGE
    assert torch.equal(pages[4], before[0]) and torch.equal(pages[6], before[2])
    rest = [0, 1, 2, 3, 5, 7, 8, 9, 10, 11]
    assert torch.equal(pages[rest], before[rest])
