"""Attention over cached and over given keys, against the fp64 oracle.

Tolerances, per output:  |o - o64| <= 2^-8 |o64| + (u + 2 e) A  with A the weights' mean magnitude of v, u half a step of the probabilities' type (fp16 2^-11
for cached keys, bf16 2^-8 for given ones), and e what a logit can be off: d + 8 fp32 operations of up to a step each on sums of magnitudes up
to L = max sum |q||k| scale, 2^-20 for the exponential, and for cached keys Q's rounding where a channel lies below 2^-14 of its row's largest
(2^-25 of it: d 2^-25 L' with L' = d max|q| max|k| scale, at most 2^-12 L in these inputs, whose largest values are some 4 times the mean).
Small probabilities are rounded to multiples of the type's smallest number: fp16's 2^-24, where a row's largest weight is 2^8 or more, so that a key's
weight is off by up to 2^-33 of the largest one, and N keys by N 2^-33 max|v| (outputs that come from such keys alone are lost); bf16 has 2^-126 there.
  |lse - lse64| <= e + 2^-22 |lse64| + 2^-20.
"""
import numpy as np
import pytest
import torch

from oracle import keys as K
from paper_2606_23743_b200 import binding as B

pytestmark = pytest.mark.gpu


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _f64(t):
    return t.float().cpu().numpy().astype(np.float64)


def _heads(rng, shape, first, size=1.0):
    b, h, t, d = shape
    x = torch.from_numpy(rng.standard_normal((b, t, h, d) if first else shape) * size).to(torch.bfloat16).cuda()
    return x.transpose(1, 2) if first else x


def _compare(o, lse, want, u, d, v):
    """o [T,d], lse [T] of one head against the oracle's; v [N,d]."""
    ref, ref_lse, size, top = want
    e = (d + 8) * 2.0 ** -23 * top + 2.0 ** -20 + (2.0 ** -12 * 2.0 ** -8 * top if u < 2.0 ** -9 else 0.0)
    floor = v.shape[0] * 2.0 ** (-33 if u < 2.0 ** -9 else -126) * np.abs(v).max(initial=0.0)
    off = np.abs(o - ref) - (2.0 ** -8 * np.abs(ref) + (u + 2 * e) * size + floor)
    assert (off <= 0).all(), (off.max(), np.unravel_index(off.argmax(), off.shape))
    empty = np.isneginf(ref_lse)
    assert np.array_equal(np.isneginf(lse), empty) and not o[empty].any()
    lse, ref_lse = lse[~empty], ref_lse[~empty]
    assert (np.abs(lse - ref_lse) <= e + 2.0 ** -22 * np.abs(ref_lse) + 2.0 ** -20).all()


# ---------------------------------------------------------------------------------------------------------- cached keys
class Cached:
    def __init__(self, rng, Bq, Hq, H, M, d, page, keys, first, spread=0.5, max_pages=None):
        self.page, self.keys = page, list(keys)
        most = max_pages or max(1, max(-(-n // page) for n in keys))
        pages = Bq * most + 2
        self.ids = rng.permutation(pages)[:Bq * most].reshape(Bq, most)
        self.codes = [rng.integers(0, 256, (pages, H, page, d)).astype(np.uint8) for _ in range(2)]
        self.scales = []
        for i, codes in enumerate(self.codes):
            x = rng.standard_normal(codes.shape) * 100
            codes[:] = K.e4m3_bytes(x)
            self.scales.append(np.exp(spread * rng.standard_normal((pages, H))).astype(np.float32).astype(np.float64) / 100)
        self.q = _heads(rng, (Bq, Hq, M, d), first)
        self.o = torch.full_like(self.q, 7.0)
        self.lse = torch.full((Bq, Hq, M), 7.0, device="cuda")
        self.group, self.d = Hq // H, d

    def run(self, causal, counts, scale=0.0, spoil=True):
        arrays = []
        for codes, scales in zip(self.codes, self.scales):
            codes = codes.copy()
            if spoil:                                      # what lies behind a sequence's last token means nothing
                for b, n in enumerate(self.keys):
                    if n % self.page:
                        codes[self.ids[b][n // self.page], :, n % self.page:] = 0x7f
            arrays.append([torch.from_numpy(codes).cuda(), torch.from_numpy(scales.astype(np.float32)).cuda()])
        c = B.make_kv_cache(*arrays, format="e4m3_page")
        table = _i32(self.ids)
        p = B.make_cached_attn(c, self.q, self.o, table, causal, scale)
        ws = torch.full((max(256, B.cached_attn_workspace_bytes(p)),), 0xff, dtype=torch.uint8, device="cuda")
        self.status = _i32([0])
        B.cached_attn_fwd(p, self.q, table, _i32(self.keys), self.o, None if counts is None else _i32(counts), self.lse, self.status, ws)
        torch.cuda.synchronize()
        return c, p, table, ws

    def check(self, causal, counts, heads=None):
        Bq, Hq, M, d = self.q.shape
        q, o, lse = _f64(self.q), _f64(self.o), _f64(self.lse)
        for b in range(Bq):
            n, cnt = self.keys[b], M if counts is None else counts[b]
            k, v = (K.gathered(a, s, self.ids[b].tolist(), n, self.page) for a, s in zip(self.codes, self.scales))
            t = np.arange(cnt)
            there = np.arange(n)[None] <= n - cnt + t[:, None] if causal else np.ones((cnt, n), bool)
            for h in range(Hq) if heads is None else heads:
                want = K.attention(q[b, h, :cnt], k[h // self.group], v[h // self.group], there, d ** -0.5)
                _compare(o[b, h, :cnt], lse[b, h, :cnt], want, 2.0 ** -11, d, v[h // self.group])
            assert (o[b, :, cnt:] == 7.0).all() and (lse[b, :, cnt:] == 7.0).all()
        assert int(self.status) == 0


CACHED = [
    # Hq, H, M, d, page, keys per sequence, counts, causal, tokens first
    (1, 1, 1, 64, 16, [1], None, False, False),
    (16, 16, 1, 128, 64, [255, 0, 256], None, False, True),
    (8, 2, 1, 128, 48, [1000, 17], None, True, True),
    (7, 1, 3, 64, 16, [3, 2, 50], None, True, False),          # (two keys, three queries: the first sees none)
    (32, 8, 5, 128, 64, [700, 64, 5], [5, 1, 0], True, True),
    (4, 4, 17, 128, 32, [333, 130], [17, 11], False, False),
    (6, 3, 130, 64, 128, [259, 1], [130, 1], True, True),
    (2, 2, 300, 128, 64, [511], None, False, True),
    (3, 1, 100, 128, 16, [385, 128], [100, 99], True, False),
    (5, 5, 129, 128, 256, [640], None, True, True),
    (2, 1, 64, 64, 64, [6000], None, False, True),
    (1, 1, 1, 128, 64, [20000], None, False, False),
]


@pytest.mark.parametrize("Hq,H,M,d,page,keys,counts,causal,first", CACHED)
def test_cached(Hq, H, M, d, page, keys, counts, causal, first):
    rng = np.random.default_rng(M + d + page + sum(keys))
    x = Cached(rng, len(keys), Hq, H, M, d, page, keys, first)
    x.run(causal, counts)
    x.check(causal, counts)


@pytest.mark.parametrize("M", [1, 200])
def test_scales_of_pages_that_lie_far_apart(M):
    """Pages of zeros (scale 0), of tiny and of large values beside one another."""
    rng = np.random.default_rng(4)
    x = Cached(rng, 1, 2, 2, M, 128, 16, [300], True)
    order = x.ids[0]
    for i, s in enumerate((0.0, 1e-3, 10.0, 1e-6, 0.0, 1.0, 1e-2)):
        x.scales[1][order[i::7]] = np.float32(s)
        if s == 0.0:
            x.codes[1][order[i::7]] = 0
    x.scales[0][order[3::5]] *= np.float32(3.0)
    x.scales = [s.astype(np.float32).astype(np.float64) for s in x.scales]
    x.run(False, None)
    x.check(False, None)


@pytest.mark.parametrize("M", [1, 150])
def test_values_of_zeros_alone(M):
    x = Cached(np.random.default_rng(6), 1, 1, 1, M, 64, 16, [40], True)
    x.codes[1][:], x.scales[1][:] = 0, 0.0
    x.run(True, None)
    x.check(True, None)


@pytest.mark.parametrize("M", [1, 150])
def test_sharp_rows_and_large_queries(M):
    """Logits up to some thousands: the softmax is all but one key; queries far from 1."""
    rng = np.random.default_rng(7)
    x = Cached(rng, 1, 2, 1, M, 128, 32, [500], True)
    x.q *= 200.0
    x.q[:, 1] *= 2.0 ** -30
    x.run(False, None)
    x.check(False, None)


@pytest.mark.parametrize("M", [1, 140])
def test_bad_pages_are_left_out(M):
    rng = np.random.default_rng(8)
    x = Cached(rng, 1, 2, 2, M, 128, 16, [150], True)
    c, p, table, ws = x.run(False, None)
    good = x.ids.copy()
    bad = good.copy()
    bad[0, 2], bad[0, 5] = -1, 10 ** 6
    status = _i32([0])
    B.cached_attn_fwd(p, x.q, _i32(bad), _i32([150]), x.o, None, x.lse, status, ws)
    assert int(status) == B.SVA_DEV_BAD_INDEX
    k, v = (K.gathered(a, s, good[0].tolist(), 150, 16) for a, s in zip(x.codes, x.scales))
    there = ~np.isin(np.arange(150) // 16, (2, 5))
    for h in range(2):
        _compare(_f64(x.o)[0, h], _f64(x.lse)[0, h], K.attention(_f64(x.q)[0, h], k[h], v[h], there, 128 ** -0.5), 2.0 ** -11, 128, v[h])
@pytest.mark.parametrize("M", [1, 140])
def test_more_tokens_than_the_table_has_pages_for(M):
    x = Cached(np.random.default_rng(17), 1, 1, 1, M, 128, 16, [160], True)
    c, p, table, ws = x.run(True, None)
    o, lse = x.o.clone(), x.lse.clone()
    B.cached_attn_fwd(p, x.q, table, _i32([10 ** 6]), x.o, None, x.lse, None, ws)
    assert torch.equal(o, x.o) and torch.equal(lse, x.lse)
    B.cached_attn_fwd(p, x.q, table, _i32([-3]), x.o, None, x.lse, None, ws)
    assert not x.o.any() and torch.isneginf(x.lse).all()


@pytest.mark.parametrize("M", [1, 140])
def test_a_page_that_is_not_a_number(M):
    """A NaN scale spoils the rows that see its page, and no others."""
    x = Cached(np.random.default_rng(9), 1, 2, 2, M, 64, 16, [200], True)
    x.scales[0][x.ids[0][12], 1] = np.nan                      # K of the last page, head 1
    x.run(False, None)
    assert torch.isnan(x.o[:, 1]).all() and not torch.isnan(x.o[:, 0]).any()
    x.scales[0][x.ids[0][12], 1] = 0.01
    x.scales[1][x.ids[0][3], 0] = np.nan
    x.run(False, None)
    assert torch.isnan(x.o[:, 0]).all() and not torch.isnan(x.o[:, 1]).any()


# ---------------------------------------------------------------------------------------------------------- given keys
CROSS = [
    # B, Hq, Hk, N, S, d, lengths, mask (part of the keys), tokens first
    (1, 1, 1, 1, 1, 64, None, None, False),
    (2, 16, 16, 1, 77, 64, [77, 12], None, True),
    (3, 2, 2, 5, 130, 128, [0, 130, 1], None, True),
    (1, 4, 2, 300, 512, 128, None, None, False),
    (2, 3, 1, 129, 127, 128, [127, 64], 0.5, True),
    (2, 6, 2, 200, 640, 64, None, 0.1, False),
    (1, 2, 2, 513, 257, 128, [256], None, True),
    (1, 1, 1, 700, 1000, 128, None, 0.003, True),
    (1, 7, 1, 50, 0, 64, None, None, False),
    (1, 1, 1, 3, 9000, 64, None, 0.9, True),
]


def _cross(q, k, v, lengths, mask, scale=0.0, fill=7.0):
    o, lse = torch.full_like(q, fill), torch.full(q.shape[:3], fill, device="cuda")
    p = B.make_cross_attn(q, k, v, o, scale)
    ws = torch.full((max(256, B.cross_attn_workspace_bytes(p)),), 0xff, dtype=torch.uint8, device="cuda")
    status = _i32([0])
    B.cross_attn_fwd(p, q, k, v, o, lengths, mask, lse, status, ws)
    torch.cuda.synchronize()
    assert int(status) == 0
    return o, lse


def _cross_check(q, k, v, there, o, lse, scale=None):
    Bq, Hq, N, d = q.shape
    group = Hq // k.shape[1]
    q, k, v, o, lse = (_f64(t) for t in (q, k, v, o, lse))
    for b in range(Bq):
        for h in range(Hq):
            _compare(o[b, h], lse[b, h], K.attention(q[b, h], k[b, h // group], v[b, h // group], there[b], scale or d ** -0.5), 2.0 ** -8, d, v[b, h // group][there[b]])


@pytest.mark.parametrize("Bq,Hq,Hk,N,S,d,lengths,part,first", CROSS)
def test_cross(Bq, Hq, Hk, N, S, d, lengths, part, first):
    rng = np.random.default_rng(N + S + d)
    q, k, v = _heads(rng, (Bq, Hq, N, d), first), _heads(rng, (Bq, Hk, S, d), first), _heads(rng, (Bq, Hk, S, d), first)
    there = np.ones((Bq, S), bool)
    if lengths is not None:
        there &= np.arange(S)[None] < np.array(lengths)[:, None]
    mask = None
    if part is not None:
        on = rng.random((Bq, S)) < part
        mask = torch.from_numpy(on).cuda()
        there &= on
    # what is left out holds anything
    k2, v2 = k.clone(memory_format=torch.preserve_format), v.clone(memory_format=torch.preserve_format)
    out = torch.from_numpy(~there).cuda()[:, None, :, None].expand(k.shape)
    k2[out], v2[out] = float("nan"), float("inf")
    o, lse = _cross(q, k2, v2, None if lengths is None else _i32(lengths), mask)
    _cross_check(q, k, v, there, o, lse)


@pytest.mark.parametrize("N", [2, 300])
def test_shared_states_and_strides(N):
    """States that items or heads share (strides of 0), slices of a packed projection, a mask that items share."""
    rng = np.random.default_rng(11)
    Bq, H, S, d = 3, 2, 150, 64
    packed = _heads(rng, (Bq, 3 * H, N, d), True)
    q = packed[:, H:2 * H]
    kv = _heads(rng, (1, 2, S, d), True)
    k, v = kv[:, :1].expand(Bq, H, S, d), kv[:, 1:].expand(Bq, H, S, d)
    on = rng.random((1, S)) < 0.7
    o, lse = _cross(q, k, v, None, torch.from_numpy(on).cuda().expand(Bq, S))
    _cross_check(q, k, v, np.broadcast_to(on, (Bq, S)), o, lse)


@pytest.mark.parametrize("N", [2, 300])
def test_sharp_cross_and_scale(N):
    rng = np.random.default_rng(12)
    q, k, v = _heads(rng, (1, 2, N, 128), True, 30.0), _heads(rng, (1, 2, 400, 128), True), _heads(rng, (1, 2, 400, 128), True, 1e4)
    o, lse = _cross(q, k, v, None, None, 0.2)
    _cross_check(q, k, v, np.ones((1, 400), bool), o, lse, 0.2)


@pytest.mark.parametrize("N", [2, 300])
def test_rows_that_are_not_numbers_keep_to_themselves(N):
    rng = np.random.default_rng(13)
    q, k, v = _heads(rng, (1, 1, N, 64), True), _heads(rng, (1, 1, 200, 64), True), _heads(rng, (1, 1, 200, 64), True)
    clean, _ = _cross(q, k, v, None, None)
    q[0, 0, 1, 5] = float("nan")
    o, lse = _cross(q, k, v, None, None)
    assert torch.isnan(o[0, 0, 1]).all() and torch.isnan(lse[0, 0, 1])
    assert torch.equal(o[0, 0, 0], clean[0, 0, 0]) and torch.equal(o[0, 0, 2:], clean[0, 0, 2:])


@pytest.mark.parametrize("N,S", [(1, 4000), (300, 3000)])
def test_the_same_bits_every_time(N, S):
    rng = np.random.default_rng(14)
    q, k, v = _heads(rng, (1, 2, N, 128), True), _heads(rng, (1, 2, S, 128), True), _heads(rng, (1, 2, S, 128), True)
    first = _cross(q, k, v, None, None)
    for _ in range(3):
        again = _cross(q, k, v, None, None)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


@pytest.mark.parametrize("N,S", [(1, 2000), (200, 2000)])
def test_two_graphs_and_streams(N, S):
    """Captured calls follow what their inputs hold when they are replayed; two of them with a workspace each may overlap."""
    rng = np.random.default_rng(15)
    q, k, v = _heads(rng, (1, 2, N, 128), True), _heads(rng, (1, 2, S, 128), True), _heads(rng, (1, 2, S, 128), True)
    p = B.make_cross_attn(q, k, v, q)
    lengths = [_i32([S]), _i32([S - 7])]
    out = [torch.zeros_like(q) for _ in range(2)]
    spaces = [torch.empty(max(256, B.cross_attn_workspace_bytes(p)), dtype=torch.uint8, device="cuda") for _ in range(2)]
    streams, graphs = [torch.cuda.Stream() for _ in range(2)], []
    _cross(q, k, v, None, None)
    for i in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=streams[i]):
            B.cross_attn_fwd(p, q, k, v, out[i], lengths[i], workspace=spaces[i])
        graphs.append(g)
    want = [_cross(q, k, v, _i32([n]), None)[0] for n in (S - 100, S - 7)]
    lengths[0].fill_(S - 100)
    torch.cuda.synchronize()
    for _ in range(3):
        for s, g in zip(streams, graphs):
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1])


def test_a_long_cache():
    """Offsets beyond 32 bits: more than 2^32 bytes of codes, the sequence on the last pages."""
    H, d, page, pages = 8, 128, 128, 33000                                     # 4.3e9 bytes each
    codes = torch.zeros(pages, H, page, d, dtype=torch.uint8, device="cuda")
    scale = torch.zeros(pages, H, device="cuda")
    c = B.make_kv_cache([codes, scale], [codes, scale], format="e4m3_page")
    rng = np.random.default_rng(16)
    N, M = 300, 150
    x = _heads(rng, (1, H, N, d), True)
    table = _i32([[pages - 1, 3, pages - 2]])
    B.kv_cache_append(c, x, x, table, _i32([0]))
    q = _heads(rng, (1, H, M, d), True)
    for m in (1, M):
        qm = q[:, :, :m]
        o, lse = torch.empty_like(qm), torch.empty(1, H, m, device="cuda")
        p = B.make_cached_attn(c, qm, o, table)
        ws = torch.empty(max(256, B.cached_attn_workspace_bytes(p)), dtype=torch.uint8, device="cuda")
        B.cached_attn_fwd(p, qm, table, _i32([N]), o, None, lse, workspace=ws)
        some = [codes[i].cpu().numpy() for i in table[0].tolist()]
        kept = np.stack(some), scale[table[0].long()].cpu().numpy().astype(np.float64)
        kv = K.gathered(*kept, [0, 1, 2], N, page)
        for h in (0, H - 1):
            _compare(_f64(o)[0, h], _f64(lse)[0, h], K.attention(_f64(qm)[0, h], kv[h], kv[h], np.ones(N, bool), d ** -0.5), 2.0 ** -11, d, kv[h])
