"""The pool of pages against the oracle's, entry by entry; every byte of the pages that are moved and of those that are not."""
import numpy as np
import pytest
import torch

from oracle.keys import Pool
from paper_2606_23743_b200 import binding as B

pytestmark = pytest.mark.gpu


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _cache(rng, form, pages, H, page, d):
    shapes = {"e4m3_page": [(pages, H, page, d), (pages, H)], "e4m3": [(pages, H, page, d), (pages, H, page)],
              "fp4": [(pages, H, page, d // 2), (pages, H, page), (pages, H, page, d // 16)]}[form]
    arrays = [[torch.from_numpy(rng.integers(0, 255, s).astype(np.uint8 if i != 1 else np.float32)).cuda() for i, s in enumerate(shapes)]
              for _ in range(2)]
    return B.make_kv_cache(*arrays, format=form), arrays[0] + arrays[1]


def _moved(before, after, pairs):
    for was, now in zip(before, after):
        want = was.clone()
        if pairs:
            src, dst = (torch.tensor(x, device="cuda") for x in zip(*pairs))
            want[dst] = was[src]
        assert torch.equal(want, now)


def _books(pool, refs, table, lengths):
    assert refs.tolist() == pool.refs and table.tolist() == pool.table and lengths.tolist() == pool.lengths


@pytest.mark.parametrize("form,H,page,d,n", [("e4m3_page", 1, 16, 64, 1), ("e4m3", 3, 7, 128, 5), ("fp4", 5, 1, 64, 9), ("e4m3_page", 24, 64, 128, 3),
                                             ("fp4", 2, 48, 128, 70)])
def test_copy(form, H, page, d, n):
    rng = np.random.default_rng(n)
    pages = 2 * n + 3
    c, arrays = _cache(rng, form, pages, H, page, d)
    order = rng.permutation(pages)
    src, dst = order[:n].copy(), order[n:2 * n].copy()
    if n > 4:
        src[1], dst[2] = -1, -4
    before = [a.clone() for a in arrays]
    status = _i32([0])
    B.kv_pages_copy(c, _i32(src), _i32(dst), status)
    _moved(before, arrays, [(s, t) for s, t in zip(src, dst) if s >= 0 and t >= 0])
    assert int(status) == 0
    if n > 4:
        before = [a.clone() for a in arrays]
        src[3], dst[4] = pages, 2 ** 31 - 1
        B.kv_pages_copy(c, _i32(src), _i32(dst), status)
        _moved(before, arrays, [(s, t) for s, t in zip(src, dst) if 0 <= s < pages and 0 <= t < pages])
        assert int(status) == B.SVA_DEV_BAD_INDEX
    B.kv_pages_copy(c, _i32([]), _i32([]))


@pytest.mark.parametrize("form,rows,most,pages,page,H", [("e4m3_page", 3, 4, 15, 16, 2), ("e4m3", 20, 9, 300, 5, 1), ("fp4", 6, 3, 40, 16, 3),
                                                         ("e4m3_page", 1500, 3, 9000, 16, 1)])
def test_a_pool_lives(form, rows, most, pages, page, H):
    """Sequences come, grow, fork, shrink and go; the pool is compacted now and then."""
    rng = np.random.default_rng(pages)
    c, arrays = _cache(rng, form, pages, H, page, 64)
    refs, table, lengths, status = _i32([0] * pages), _i32([[-1] * most] * rows), _i32([0] * rows), _i32([0])
    work = torch.empty(B.kv_pages_compact_workspace_bytes(c), dtype=torch.uint8, device="cuda")
    pool = Pool([0] * pages, [[-1] * most] * rows, [0] * rows, page)
    for turn in range(24 if rows < 100 else 8):
        what = turn % 4
        pool.moved, before = [], [a.clone() for a in arrays]
        if what in (0, 3):
            counts = [int(rng.integers(0, most * page - n + 1)) if rng.random() < 0.4 else 0 for n in pool.lengths]
            while sum(r > 0 for r in pool.refs) + sum(-(-x // page) for x in counts) > pages:
                counts[int(np.argmax(counts))] = 0
            pool.take(counts)
            B.kv_pages_take(c, refs, table, lengths, _i32(counts), status)
            pool.lengths = [a + b for a, b in zip(pool.lengths, counts)]
            lengths += _i32(counts)
        elif what == 1:
            n = max(1, rows // 3)
            who = [int(i) for i in rng.permutation(rows)]
            children, parents = who[:n], [who[n + int(rng.integers(rows - n))] for _ in range(n)]
            pool.free(children, [0] * n)
            B.kv_pages_free(c, refs, table, lengths, _i32(children), status=status)
            pool.fork(parents, children)
            B.kv_pages_fork(c, refs, table, lengths, _i32(parents), _i32(children), status)
        else:
            who = [int(i) for i in rng.permutation(rows)[:rows // 2]]
            keep = [int(rng.integers(0, most * page)) for _ in who]
            pool.free(who, keep)
            B.kv_pages_free(c, refs, table, lengths, _i32(who), _i32(keep), status)
            live = _i32([0])
            assert pool.compact() == (B.kv_pages_compact(c, refs, table, work, live, status), int(live))[1]
        _books(pool, refs, table, lengths)
        _moved(before, arrays, pool.moved)
    assert int(status) == 0


def test_a_pool_runs_out():
    rng = np.random.default_rng(3)
    c, arrays = _cache(rng, "e4m3_page", 7, 2, 16, 64)
    refs, table, lengths, status = _i32([0] * 7), _i32([[-1] * 4] * 4), _i32([0] * 4), _i32([0])
    pool = Pool([0] * 7, [[-1] * 4] * 4, [0] * 4, 16)
    pool.take([40, 33, 20, 0])
    B.kv_pages_take(c, refs, table, lengths, _i32([40, 33, 20, 0]), status)
    _books(pool, refs, table, lengths)
    assert int(status) == B.SVA_DEV_NO_PAGES and pool.short
    pool.lengths = [40, 33, 16, 0]
    lengths.copy_(_i32(pool.lengths))
    status.zero_()
    pool.fork([0], [3])                                                        # two full pages are shared, none is left for the third
    B.kv_pages_fork(c, refs, table, lengths, _i32([0]), _i32([3]), status)
    _books(pool, refs, table, lengths)
    assert int(status) == B.SVA_DEV_NO_PAGES and pool.lengths[3] == 32


def test_rows_and_entries_that_are_not_there():
    rng = np.random.default_rng(4)
    c, arrays = _cache(rng, "e4m3_page", 9, 1, 16, 64)
    refs, lengths, status = _i32([1, 1, 0, 0, 0, 0, 0, 0, 0]), _i32([20, 0]), _i32([0])
    table = _i32([[0, 1], [-1, -1]])
    before = [a.clone() for a in arrays]
    for parents, children in (([0], [5]), ([-1], [1]), ([0], [0]), ([2], [1])):
        status.zero_()
        B.kv_pages_fork(c, refs, table, lengths, _i32(parents), _i32(children), status)
        assert int(status) == B.SVA_DEV_BAD_INDEX
    status.zero_()
    B.kv_pages_free(c, refs, table, lengths, _i32([7, -1]), status=status)
    assert int(status) == B.SVA_DEV_BAD_INDEX and table.tolist() == [[0, 1], [-1, -1]] and refs.tolist() == [1, 1] + [0] * 7
    _moved(before, arrays, [])
    # a row that is named twice gives its pages back once; a page without a count is reported
    status.zero_()
    B.kv_pages_free(c, refs, table, lengths, _i32([0, 0]), status=status)
    assert refs.tolist() == [0] * 9 and table.tolist() == [[-1, -1]] * 2 and lengths.tolist() == [0, 0] and int(status) == 0
    table[1, 0] = 4
    B.kv_pages_free(c, refs, table, lengths, _i32([1]), status=status)
    assert refs.tolist() == [0] * 9 and int(status) == B.SVA_DEV_BAD_INDEX
    # a table that names pages that are free, or that there are not, is reported where the pool is compacted
    status.zero_()
    refs[8], table[0, 0], table[0, 1], table[1, 0] = 1, 8, 6, 100
    work = torch.empty(B.kv_pages_compact_workspace_bytes(c), dtype=torch.uint8, device="cuda")
    B.kv_pages_compact(c, refs, table, work, status=status)
    assert table.tolist() == [[0, -1], [-1, -1]] and refs.tolist() == [1] + [0] * 8 and int(status) == B.SVA_DEV_BAD_INDEX


def test_captured():
    rng = np.random.default_rng(5)
    c, arrays = _cache(rng, "e4m3_page", 12, 2, 16, 64)
    refs, table, lengths = _i32([1, 0, 0, 1] + [0] * 8), _i32([[3, 0, -1], [-1] * 3, [-1] * 3]), _i32([20, 0, 0])
    parents, children = _i32([0]), _i32([1])
    state = [t.clone() for t in (refs, table, lengths)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        B.kv_pages_fork(c, refs, table, lengths, parents, children)
        for t, s in zip((refs, table, lengths), state):
            t.copy_(s)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            B.kv_pages_free(c, refs, table, lengths, children)
            B.kv_pages_fork(c, refs, table, lengths, parents, children)
        for child in (1, 2, 1):
            children.fill_(child)
            graph.replay()
    side.synchronize()
    # (row 1 takes page 1, row 2 page 2; row 1 gives page 1 back and takes it again)
    assert table.tolist() == [[3, 0, -1], [3, 1, -1], [3, 2, -1]] and lengths.tolist() == [20, 20, 20]
    assert refs.tolist() == [1, 1, 1, 3] + [0] * 8
    for a in arrays:
        assert torch.equal(a[1], a[0]) and torch.equal(a[2], a[0])
