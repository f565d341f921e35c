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
