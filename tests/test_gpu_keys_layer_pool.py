"""A layer whose pool or table is short, and sequences that are cut within a page that others share: what is held stays what it was.  Each is compared bit by
bit with a layer that has room, or shares nothing, and is told the outcome."""
import pytest
import torch

from paper_2606_23743_b200 import binding as B
from paper_2606_23743_b200.attention_layer import ChunkAttentionLayer

pytestmark = pytest.mark.gpu

C, D, PAGE = 64, 64, 16


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _maker():
    gen = torch.Generator("cuda").manual_seed(7)
    return lambda *s: torch.randn(*s, generator=gen, device="cuda").to(torch.bfloat16)


def _layers(n, **kw):
    bf = _maker()
    w_qkv, w_out = bf(3 * D, C) / 8, bf(C, D) / 8
    return [ChunkAttentionLayer(w_qkv, w_out, 1, page=PAGE, **{k: v[i] if isinstance(v, tuple) else v for k, v in kw.items()}) for i in range(n)]


def _books(layer):
    named = torch.bincount(layer.table[layer.table >= 0].long(), minlength=layer.refs.numel())
    assert torch.equal(named, layer.refs.long())
    assert (layer.table >= 0).sum(1).tolist() == [-(-n // PAGE) for n in layer.lengths.tolist()]
    last = [int(layer.refs[row[n // PAGE]]) for row, n in zip(layer.table, layer.lengths.tolist()) if n % PAGE]
    assert all(n == 1 for n in last)                                           # what may be appended to is a sequence's own


@pytest.mark.parametrize("causal", [False, True])
def test_a_pool_that_runs_out(causal):
    bf = _maker()
    short, wide = _layers(2, tokens=64, rows=2, pages=(4, 8), causal=causal)
    x = [bf(2, 20, C) for _ in range(4)]
    assert torch.equal(short(x[0]), wide(x[0]))
    got, want = short(x[1]), wide(x[1], _i32([12, 12]))                        # four pages: 32 tokens of each
    assert int(short.status) == B.SVA_DEV_NO_PAGES and short.lengths.tolist() == [32, 32]
    assert torch.equal(got[:, :12], want[:, :12])
    _books(short)
    short.status.zero_()
    short(x[2], _i32([1, 0]))
    assert short.lengths.tolist() == [32, 32] and int(short.status) == B.SVA_DEV_NO_PAGES
    for layer in (short, wide):
        layer.forget(_i32([1]))
    got, want = short(x[3], _i32([20, 3])), wide(x[3], _i32([20, 0]))          # two pages are free again, and row 0 comes first
    assert torch.equal(got[0], want[0]) and short.lengths.tolist() == wide.lengths.tolist() == [52, 0]
    _books(short)


@pytest.mark.parametrize("causal", [False, True])
def test_a_table_that_is_full(causal):
    bf = _maker()
    short, wide = _layers(2, tokens=(32, 64), rows=1, causal=causal)
    x = [bf(1, n, C) for n in (20, 25, 5, 9)]
    assert torch.equal(short(x[0]), wide(x[0]))
    got, want = short(x[1]), wide(x[1], _i32([12]))
    assert int(short.status) == B.SVA_DEV_BAD_INDEX and short.lengths.tolist() == [32]
    assert torch.equal(got[:, :12], want[:, :12])
    short(x[2])
    assert short.lengths.tolist() == [32]
    short.status.zero_()
    for layer in (short, wide):
        layer.forget(_i32([0]), _i32([21]))
    assert torch.equal(short(x[3]), wide(x[3])) and int(short.status) == 0 and short.lengths.tolist() == [30]
    _books(short)


def test_a_sequence_cut_within_a_page_that_others_share():
    bf = _maker()
    shared, apart = _layers(2, tokens=96, rows=3, pages=18)
    x, y, z = bf(3, 40, C), bf(3, 9, C), bf(3, 1, C)
    x[1:] = x[:1]
    shared(x, _i32([40, 0, 0]))
    shared.fork(_i32([0, 0]), _i32([1, 2]))
    apart(x)
    for layer in (shared, apart):
        layer.forget(_i32([1, 2, 1]), _i32([20, 33, 20]))                      # (row 2: within a page of its own)
    _books(shared)
    y[1] *= 100.0                                                              # the page's scale grows, its codes are re-expressed
    for t, counts in ((y, _i32([0, 9, 9])), (z, None)):
        got, want = shared(t, counts), apart(t, counts)
        for b in range(3):
            n = t.shape[1] if counts is None else int(counts[b])
            assert torch.equal(got[b, :n], want[b, :n])
    assert int(shared.status) == 0 and shared.lengths.tolist() == apart.lengths.tolist()
    _books(shared)


def test_a_cut_without_a_page_for_the_copy():
    bf = _maker()
    x = bf(2, 32, C)
    layer, = _layers(1, tokens=64, rows=2, pages=2)
    layer(x, _i32([32, 0]))
    layer.fork(_i32([0]), _i32([1]))
    layer.forget(_i32([1]), _i32([20]))                                        # no page for a copy: its full pages are left
    assert int(layer.status) == B.SVA_DEV_NO_PAGES and layer.lengths.tolist() == [32, 16] and layer.refs.tolist() == [2, 1]
    _books(layer)
    layer, = _layers(1, tokens=64, rows=2, pages=2)
    layer(x, _i32([32, 0]))
    layer.fork(_i32([0]), _i32([1]))
    layer.forget(_i32([0, 1]), _i32([20, 20]))                                 # both are cut: the page stays with one of them
    assert int(layer.status) == B.SVA_DEV_NO_PAGES and sorted(layer.lengths.tolist()) == [16, 20] and layer.refs.tolist() == [2, 1]
    _books(layer)
    layer, = _layers(1, tokens=64, rows=2, pages=3)
    layer(x, _i32([32, 0]))
    layer.fork(_i32([0]), _i32([1]))
    layer.forget(_i32([0, 1]), _i32([20, 20]))                                 # one copy is enough for two
    assert int(layer.status) == 0 and layer.lengths.tolist() == [20, 20] and layer.refs.tolist() == [2, 1, 1]
    _books(layer)


def test_a_cut_and_a_call_are_captured():
    bf = _maker()
    live, seen = _layers(2, tokens=96, rows=2, pages=12)
    x, y = bf(2, 40, C), bf(2, 3, C)
    which, keep = _i32([1]), _i32([20])
    for layer in (live, seen):
        layer(x, _i32([40, 0]))
        layer.fork(_i32([0]), _i32([1]))
        layer(y)
        layer.forget(which, _i32([41]))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        live.forget(which, keep)
        got = live(y)
    for n in (20, 17, 5):
        keep.fill_(n)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        seen.forget(which, keep)
        assert torch.equal(got, seen(y)) and torch.equal(live.table, seen.table) and torch.equal(live.refs, seen.refs)
    _books(live)
