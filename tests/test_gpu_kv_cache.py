"""The quantised K/V cache against the fp64 oracle: bytes, scales and values exactly."""
import numpy as np
import pytest
import torch

from oracle import layer as L
from paper_2606_23743_b200 import binding as B

pytestmark = pytest.mark.gpu


def _f64(t):
    return t.float().cpu().numpy().astype(np.float64)


def _arrays(form, pages, H, page, d, fill=0x11):
    codes = torch.full((pages, H, page, d if form == "e4m3" else d // 2), fill, dtype=torch.uint8, device="cuda")
    scale = torch.full((pages, H, page), 0.5, device="cuda")
    sf = torch.full((pages, H, page, d // 16), 0x38, dtype=torch.uint8, device="cuda")
    return [codes, scale] if form == "e4m3" else [codes, scale, sf]


def _rows(rng, shape, tokens_first):
    Bq, H, T, d = shape
    x = rng.standard_normal((Bq, T, H, d) if tokens_first else shape)
    x *= np.exp(2 * rng.standard_normal(x.shape[:-1]))[..., None]           # rows of different size
    x = torch.from_numpy(x).to(torch.bfloat16).cuda()
    return x.transpose(1, 2) if tokens_first else x


def _expect(x, form):
    """x [B,H,T,d] -> (codes, scale, sf or None, values) of every row."""
    x = _f64(x)
    rows = [L.cache_row(r, form) for r in x.reshape(-1, x.shape[-1])]
    lead = x.shape[:-1]
    return [None if rows[0][i] is None else np.array([r[i] for r in rows]).reshape(*lead, -1) for i in range(4)]


CASES = [
    # form, B, H, T, d, page, tokens first
    ("e4m3", 1, 1, 1, 64, 16, False),
    ("e4m3", 5, 8, 1, 128, 16, True),
    ("e4m3", 2, 3, 37, 128, 10, False),
    ("e4m3", 1, 5, 130, 64, 64, True),
    ("fp4", 1, 1, 1, 128, 16, False),
    ("fp4", 7, 6, 1, 64, 1, True),
    ("fp4", 2, 3, 37, 128, 10, True),
    ("fp4", 1, 9, 70, 64, 48, False),
]


@pytest.mark.parametrize("form,Bq,H,T,d,page,first", CASES)
def test_write_and_read_back(form, Bq, H, T, d, page, first):
    rng = np.random.default_rng(T + d + page)
    per = -(-T // page)
    pages = Bq * per + 2
    ids = rng.permutation(pages)
    table = torch.from_numpy(ids[:Bq * per].reshape(Bq, per).astype(np.int32)).cuda()
    ka, va = _arrays(form, pages, H, page, d), _arrays(form, pages, H, page, d)
    before = [t.clone() for t in ka + va]
    c = B.make_kv_cache(ka, va, form)
    k, v = _rows(rng, (Bq, H, T, d), first), _rows(rng, (Bq, H, T, d), first)
    at = np.arange(T)
    slots = ids[:Bq * per].reshape(Bq, per)[:, at // page] * page + at % page
    skip = rng.random((Bq, T)) < 0.2 if T > 1 else np.zeros((Bq, T), bool)
    slots = np.where(skip, -1 - rng.integers(0, 1000, (Bq, T)), slots)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.kv_cache_write(c, k, v, torch.from_numpy(slots.astype(np.int32)).cuda(), status)
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    want = [b.cpu().numpy() for b in before]
    values = []
    for i, x in enumerate((k, v)):
        parts = _expect(x, form)
        for b in range(Bq):
            for t in range(T):
                if slots[b, t] >= 0:
                    where = (slots[b, t] // page, slice(None), slots[b, t] % page)
                    n = len(ka)
                    want[i * n][where] = parts[0][b, :, t]
                    want[i * n + 1][where] = parts[1][b, :, t, 0]
                    if n == 3:
                        want[i * n + 2][where] = parts[2][b, :, t]
        values.append(parts[3])
    for t, w in zip(ka + va, want):                                        # what no slot names keeps its bytes
        np.testing.assert_array_equal(t.cpu().numpy(), w)

    # read back: more rows than there are, sequences of their own lengths
    N = T + 3
    lengths = np.array([rng.integers(0, T + 1) for _ in range(Bq)])
    lengths[0] = T
    ko, vo = (torch.full((Bq, N, H, d), 7.0, dtype=torch.bfloat16, device="cuda").transpose(1, 2) for _ in range(2))
    B.kv_cache_read(c, table, torch.from_numpy(lengths.astype(np.int32)).cuda(), ko, vo, status)
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    for i, (got, val) in enumerate(((ko, values[0]), (vo, values[1]))):
        got = _f64(got)
        for b in range(Bq):
            n = lengths[b]
            assert (got[b, :, n:] == 0).all()
            keep = ~skip[b, :n]
            ref = torch.from_numpy(val[b][:, :n][:, keep]).float().to(torch.bfloat16).float().numpy()
            np.testing.assert_array_equal(got[b][:, :n][:, keep], ref)


@pytest.mark.parametrize("form", ["e4m3", "fp4"])
def test_extreme_rows(form):
    """Zeros, signed zeros, tiny, denormal and huge rows, one large value among small ones."""
    x = torch.zeros(1, 1, 8, 64)
    x[0, 0, 1] = -0.0
    x[0, 0, 2] = torch.linspace(-1, 1, 64) * 1e-36
    x[0, 0, 3] = torch.linspace(-1, 1, 64) * 3e38
    x[0, 0, 4, 3] = 9.2e-41
    x[0, 0, 5] = torch.linspace(-1, 1, 64) * 1e-3
    x[0, 0, 5, 40] = 500.0
    x[0, 0, 6] = torch.arange(64) * 0.25 - 8
    x[0, 0, 7] = 448.0 * torch.linspace(-1, 1, 64)
    x = x.to(torch.bfloat16).cuda()
    ka, va = _arrays(form, 1, 1, 8, 64), _arrays(form, 1, 1, 8, 64)
    c = B.make_kv_cache(ka, va, form)
    B.kv_cache_write(c, x, x, torch.arange(8, dtype=torch.int32, device="cuda")[None])
    codes, scale, sf, values = _expect(x, form)
    np.testing.assert_array_equal(ka[1].cpu().numpy()[0, 0], scale[0, 0, :, 0])
    out = torch.empty_like(x)
    B.kv_cache_read(c, torch.zeros(1, 1, dtype=torch.int32, device="cuda"), torch.tensor([8], dtype=torch.int32, device="cuda"), out, torch.empty_like(x))
    np.testing.assert_array_equal(_f64(out), torch.from_numpy(values).float().to(torch.bfloat16).float().numpy())
    if form == "e4m3":
        np.testing.assert_array_equal(ka[0].cpu().numpy()[0, 0], codes[0, 0])


def test_bad_slots_and_pages_are_reported_and_left_out():
    H, d, page, pages = 2, 64, 4, 3
    ka, va = _arrays("e4m3", pages, H, page, d), _arrays("e4m3", pages, H, page, d)
    before = ka[0].clone()
    c = B.make_kv_cache(ka, va)
    k = torch.randn(1, H, 2, d, device="cuda").to(torch.bfloat16)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.kv_cache_write(c, k, k, torch.tensor([[pages * page, 2 ** 31 - 1]], dtype=torch.int32, device="cuda"), status)
    torch.cuda.synchronize()
    assert int(status.item()) == B.SVA_DEV_BAD_INDEX and torch.equal(ka[0], before)
    for table in ([[0, 3, 1]], [[0, -1, 1]]):
        status.zero_()
        out = torch.full((1, H, 12, d), 7.0, dtype=torch.bfloat16, device="cuda")
        B.kv_cache_read(c, torch.tensor(table, dtype=torch.int32, device="cuda"), torch.tensor([12], dtype=torch.int32, device="cuda"), out, out.clone(), status)
        torch.cuda.synchronize()
        assert int(status.item()) == B.SVA_DEV_BAD_INDEX
        assert (out[:, :, 4:8] == 0).all() and (out[:, :, :4] != 0).all() and (out[:, :, 8:] != 0).all()
    status.zero_()                                                         # a length that goes beyond the table
    out = torch.full((1, H, 12, d), 7.0, dtype=torch.bfloat16, device="cuda")
    B.kv_cache_read(c, torch.tensor([[0, 1]], dtype=torch.int32, device="cuda"), torch.tensor([100], dtype=torch.int32, device="cuda"), out, out.clone(), status)
    torch.cuda.synchronize()
    assert int(status.item()) == B.SVA_DEV_BAD_INDEX and (out[:, :, 8:] == 0).all() and (out[:, :, :8] != 0).all()


def test_offsets_beyond_32_bits():
    """A cache of 4.5 GB of K codes: rows in its last pages."""
    H, d, page = 32, 128, 64
    pages = 17500
    ka, va = ([torch.zeros(pages, H, page, d, dtype=torch.uint8, device="cuda"), torch.zeros(pages, H, page, device="cuda")] for _ in range(2))
    assert ka[0].numel() > 2 ** 32
    c = B.make_kv_cache(ka, va)
    k, v = (torch.randn(1, H, 3, d, device="cuda").to(torch.bfloat16) for _ in range(2))
    slots = [pages * page - 1, (pages - 1) * page, 5]
    B.kv_cache_write(c, k, v, torch.tensor([slots], dtype=torch.int32, device="cuda"))
    ko, vo = torch.zeros(1, H, 128, d, dtype=torch.bfloat16, device="cuda"), torch.zeros(1, H, 128, d, dtype=torch.bfloat16, device="cuda")
    B.kv_cache_read(c, torch.tensor([[0, pages - 1]], dtype=torch.int32, device="cuda"), torch.tensor([128], dtype=torch.int32, device="cuda"), ko, vo)
    for x, got in ((k, ko), (v, vo)):
        values = torch.from_numpy(_expect(x, "e4m3")[3]).float().to(torch.bfloat16)
        for t, n in ((0, 127), (1, 64), (2, 5)):
            assert torch.equal(got[0, :, n].cpu(), values[0, :, t])
    assert int((ka[0] != 0).any(-1).sum()) == 3 * H


def test_captured():
    ka, va = _arrays("fp4", 2, 2, 16, 64), _arrays("fp4", 2, 2, 16, 64)
    c = B.make_kv_cache(ka, va, "fp4")
    k = torch.randn(1, 2, 20, 64, device="cuda").to(torch.bfloat16)
    slots = torch.arange(20, dtype=torch.int32, device="cuda")[None]
    table, lengths = torch.tensor([[0, 1]], dtype=torch.int32, device="cuda"), torch.tensor([20], dtype=torch.int32, device="cuda")
    ko, vo, kg, vg = (torch.zeros(1, 2, 24, 64, dtype=torch.bfloat16, device="cuda") for _ in range(4))
    B.kv_cache_write(c, k, k, slots)
    B.kv_cache_read(c, table, lengths, ko, vo)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        B.kv_cache_write(c, k, k, slots)
        B.kv_cache_read(c, table, lengths, kg, vg)
    for t in ka + va:
        t.zero_()
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(kg, ko) and torch.equal(vg, ko) and torch.equal(vo, ko)


@pytest.mark.parametrize("form", ["e4m3", "fp4"])
@pytest.mark.parametrize("d,pad,shift", [(64, 0, 8), (128, 8, 0), (64, 24, 8)])
def test_read_into_rows_on_16_bytes(form, d, pad, shift):
    """Rows that begin on 16 bytes but not on 32: the same values as in whole tensors, and nothing beside them."""
    Bq, H, N, page = 2, 5, 21, 8
    pages = Bq * 3
    ka, va = _arrays(form, pages, H, page, d), _arrays(form, pages, H, page, d)
    for t in ka + va:
        t.copy_(torch.rand(t.shape, device="cuda") if t.dtype == torch.float32 else torch.randint(0, 100, t.shape, device="cuda"))
    c = B.make_kv_cache(ka, va, form)
    table = torch.arange(pages, dtype=torch.int32, device="cuda").view(Bq, 3)
    lengths = torch.tensor([N, 9], dtype=torch.int32, device="cuda")
    whole = [torch.empty(Bq, H, N, d, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    B.kv_cache_read(c, table, lengths, *whole)
    row = d + pad
    held = [torch.full((shift + Bq * H * N * row,), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    parts = [h[shift:].view(Bq, H, N, row) for h in held]
    B.kv_cache_read(c, table, lengths, *[p[..., :d] for p in parts])
    for w, p, h in zip(whole, parts, held):
        assert torch.equal(w, p[..., :d]) and bool((p[..., d:] == 7.0).all()) and bool((h[:shift] == 7.0).all())


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("form", ["e4m3", "fp4"])
def test_rows_with_nan_and_infinities(form, d):
    """A NaN stays alone in e4m3 and makes its row NaN in 4 bits, an infinity makes its row NaN; no other row changes."""
    rng = np.random.default_rng(d)
    x = _rows(rng, (1, 3, 9, d), False)
    clean = x.clone()
    x[0, 0, 0, 5], x[0, 0, 1, d - 1], x[0, 1, 2] = float("nan"), -float("nan"), float("nan")
    x[0, 2, 3, 20], x[0, 0, 4, 40], x[0, 1, 5, 0:2] = float("inf"), -float("inf"), torch.tensor([float("inf"), float("nan")])
    x[0, 2, 6], x[0, 2, 6, 63] = 0.0, float("nan")
    ka, va = _arrays(form, 1, 3, 9, d), _arrays(form, 1, 3, 9, d)
    c = B.make_kv_cache(ka, va, form)
    B.kv_cache_write(c, x, clean, torch.arange(9, dtype=torch.int32, device="cuda")[None])
    out, whole = torch.empty_like(x), torch.empty_like(x)
    B.kv_cache_read(c, torch.zeros(1, 1, dtype=torch.int32, device="cuda"), torch.tensor([9], dtype=torch.int32, device="cuda"), out, whole)
    for got, given, arrays in ((out, x, ka), (whole, clean, va)):
        _, scale, _, values = _expect(given, form)
        np.testing.assert_array_equal(arrays[1].cpu().numpy()[0], scale[0, :, :, 0])
        np.testing.assert_array_equal(_f64(got), torch.from_numpy(values).float().to(torch.bfloat16).float().numpy())


@pytest.mark.parametrize("d,T", [(128, 19003), (64, 37950)])
@pytest.mark.parametrize("form", ["e4m3", "fp4"])
def test_more_heads_than_a_thread_has_in_flight(form, d, T):
    """Eight heads per CTA, a thread's pass over four twice, 13 heads; against the oracle at some tokens and, everywhere, against calls of so
    few tokens that a CTA has four heads."""
    rng = np.random.default_rng(d)
    H, page = 13, 48
    pages = -(-T // page)
    g = torch.Generator(device="cuda").manual_seed(d)
    k, v = (torch.randn(1, T, H, d, generator=g, device="cuda", dtype=torch.bfloat16).transpose(1, 2) for _ in range(2))
    ids = torch.from_numpy(rng.permutation(pages).astype(np.int32)).cuda()
    at = torch.arange(T, device="cuda")
    slots = (ids[at // page] * page + at % page).to(torch.int32)[None].contiguous()
    slots[0, 77] = -1
    a, b = ((_arrays(form, pages, H, page, d), _arrays(form, pages, H, page, d)) for _ in range(2))
    ca, cb = B.make_kv_cache(*a, form), B.make_kv_cache(*b, form)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.kv_cache_write(ca, k, v, slots, status)
    assert B.debug_last_choice() == 8
    for n in range(0, T, 5000):
        B.kv_cache_write(cb, k[:, :, n:n + 5000], v[:, :, n:n + 5000], slots[:, n:n + 5000].contiguous(), status)
        assert B.debug_last_choice() == 4
    for x, y in zip(a[0] + a[1], b[0] + b[1]):
        assert torch.equal(x, y)
    some = torch.from_numpy(np.sort(rng.permutation(T)[:60])).cuda()
    values = [torch.from_numpy(_expect(x[:, :, some], form)[3]).float().to(torch.bfloat16) for x in (k, v)]
    ko, vo = (torch.full((1, H, T, d), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    B.kv_cache_read(ca, ids[None], torch.tensor([T - 2], dtype=torch.int32, device="cuda"), ko, vo, status)
    assert B.debug_last_choice() == 8
    there = (some != 77) & (some < T - 2)
    for got, want in ((ko, values[0]), (vo, values[1])):
        assert torch.equal(got[:, :, some[there]].cpu(), want[:, :, there.cpu()]) and bool((got[:, :, T - 2:] == 0).all())
    n = page * 50
    for i in range(0, T, n):
        m = min(n, T - i)
        parts = [torch.full((1, H, m, d), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        B.kv_cache_read(ca, ids[None, i // page:].contiguous(), torch.tensor([T - 2 - i], dtype=torch.int32, device="cuda"), *parts, status)
        assert B.debug_last_choice() == 4
        assert torch.equal(parts[0], ko[:, :, i:i + m]) and torch.equal(parts[1], vo[:, :, i:i + m])
    assert int(status.item()) == 0
