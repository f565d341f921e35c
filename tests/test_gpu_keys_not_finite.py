"""Attention over keys of their own where numbers end: logits beyond fp32, pages whose scale is a NaN or an infinity, scales next to zero.  A row becomes NaNs
with the keys that it sees, whichever kernel and whichever place of a tile serves them, and by no others.  Tolerances as in test_gpu_keys.
"""
import numpy as np
import pytest
import torch

from oracle import keys as K
from paper_2606_23743_b200 import binding as B
from test_gpu_keys import Cached, _compare, _cross, _f64, _i32

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("how", ["infinity", "product"])
@pytest.mark.parametrize("N", [2, 40, 300])
@pytest.mark.parametrize("group", [0, 5, 11])
def test_a_logit_that_overflows(group, N, how):
    """Item b has one at key b of a group of 16: rows whose logit is +infinity become NaNs (0 / 0), for those of -infinity the key is not there."""
    rng = np.random.default_rng(group + N)
    S, d, Bq = 200, 64, 16
    q, k, v = (torch.from_numpy(rng.standard_normal((Bq, 1, n, d))).to(torch.bfloat16).cuda() for n in (N, S, S))
    sign = torch.where(torch.arange(N, device="cuda") % 2 == 0, 1.0, -1.0)
    k[..., 0] = 0.0
    at = 16 * group + np.arange(Bq)
    q[..., 0] = sign * (1.0 if how == "infinity" else 2.0 ** 100)
    k[torch.arange(Bq), 0, at, 0] = float("inf") if how == "infinity" else 2.0 ** 100
    o, lse = _cross(q, k, v, None, None)
    assert torch.isnan(o[:, :, ::2]).all() and torch.isnan(lse[:, :, ::2]).all()
    q[..., 0], k[..., 0] = 0.0, 0.0
    for b in range(Bq):
        want = K.attention(_f64(q)[b, 0, 1::2], _f64(k)[b, 0], _f64(v)[b, 0], np.arange(S) != at[b], d ** -0.5)
        _compare(_f64(o)[b, 0, 1::2], _f64(lse)[b, 0, 1::2], want, 2.0 ** -8, d, _f64(v)[b, 0])


@pytest.mark.parametrize("what", ["q", "first", "all"])
@pytest.mark.parametrize("N,S", [(2, 6000), (64, 6000)])
def test_not_a_number_in_parts_of_a_split_axis(N, S, what):
    """A row whose every part, whose first or of which each key is a NaN: NaNs, not the zeros of a row without keys."""
    rng = np.random.default_rng(N)
    q, k, v = (torch.from_numpy(rng.standard_normal((1, 1, n, 64))).to(torch.bfloat16).cuda() for n in (N, S, S))
    assert B.cross_attn_workspace_bytes(B.make_cross_attn(q, k, v, q)) > 0
    if what == "q":
        q[0, 0, 1, 5] = float("nan")
    else:
        k[0, 0, :1 if what == "first" else S, 5] = float("nan")
    o, lse = _cross(q, k, v, None, None)
    rows = slice(1, 2) if what == "q" else slice(None)
    assert torch.isnan(o[0, 0, rows]).all() and torch.isnan(lse[0, 0, rows]).all()
    assert what != "q" or torch.isfinite(o[0, 0, 2:]).all() and torch.isfinite(o[0, 0, 0]).all()


@pytest.mark.parametrize("M", [2, 40, 300])
@pytest.mark.parametrize("group", [0, 5, 11])
def test_a_logit_over_cached_keys_that_overflows(group, M):
    """The same by way of a page's scale."""
    rng = np.random.default_rng(group + M)
    d, Bq, n = 128, 16, 200
    x = Cached(rng, Bq, 1, 1, M, d, 16, [n] * Bq, True)
    x.codes[0][..., 0] = 0
    sign = torch.where(torch.arange(M, device="cuda") % 2 == 0, 1.0, -1.0)
    x.q.zero_()
    x.q[..., 0] = sign * 2.0 ** 60
    for b in range(Bq):
        page = x.ids[b][group]
        x.scales[0][page] = 2.0 ** 63
        x.codes[0][page] = 0
        x.codes[0][page, 0, b, 0] = K.e4m3_bytes(np.array(448.0))
    x.run(False, None)
    assert torch.isnan(x.o[:, :, ::2]).all() and torch.isnan(x.lse[:, :, ::2]).all()
    for b in range(Bq):
        v = K.gathered(x.codes[1], x.scales[1], x.ids[b].tolist(), n, 16)[0]
        want = K.attention(np.zeros((M // 2, d)), v * 0, v, np.arange(n) != 16 * group + b, d ** -0.5)
        _compare(_f64(x.o)[b, 0, 1::2], _f64(x.lse)[b, 0, 1::2], want, 2.0 ** -11, d, v)
    assert int(x.status) == 0


BAD = [("k", float("nan")), ("v", float("nan")), ("k", float("inf")), ("v", float("inf")), ("kv", float("nan"))]


@pytest.mark.parametrize("which,value", BAD)
@pytest.mark.parametrize("Hq,H,M,d,keys", [(1, 1, 3, 64, 194), (4, 2, 3, 128, 194), (2, 1, 20, 128, 194), (2, 2, 140, 64, 194), (2, 2, 140, 128, 258),
                                           (1, 1, 2, 128, 20001), (2, 1, 64, 128, 6001)])
def test_a_page_that_is_not_a_number_and_queries_before_it(Hq, H, M, d, keys, which, value):
    """Causal: the last page of a sequence is spoilt; the queries before it do not see it.  (The last two: split key axes.)"""
    page = 16
    rng = np.random.default_rng(M + keys)
    x = Cached(rng, 1, Hq, H, M, d, page, [keys], True)
    bad, first = x.ids[0][keys // page], keys // page * page
    clean = [(c.copy(), s.copy()) for c, s in zip(x.codes, x.scales)]
    for i, name in enumerate("kv"):
        if name in which:
            x.scales[i][bad, H - 1] = value
            x.codes[i][bad, H - 1] = 0x7f
    x.run(True, None)
    sees = keys - M + np.arange(M) >= first
    assert sees.any() and not sees.all()
    o, lse = _f64(x.o)[0], _f64(x.lse)[0]
    k, v = (K.gathered(c, s, x.ids[0].tolist(), keys, page) for c, s in clean)
    there = np.arange(keys)[None] <= keys - M + np.arange(M)[:, None]
    for h in range(Hq):
        rows = ~sees if h // (Hq // H) == H - 1 else np.ones(M, bool)
        assert np.isnan(o[h, ~rows]).all() and np.isnan(lse[h, ~rows]).all()
        want = K.attention(_f64(x.q)[0, h, rows], k[h // (Hq // H)], v[h // (Hq // H)], there[rows], d ** -0.5)
        _compare(o[h, rows], lse[h, rows], want, 2.0 ** -11, d, v[h // (Hq // H)])
    assert int(x.status) == 0


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("M", [4, 70])
def test_a_token_that_is_not_a_number(M, bad):
    """The same as a user meets it: a chunk with a NaN (an infinity) in its last token is appended, and attended to in causal form."""
    H, d, page, held = 2, 64, 16, 47                       # (the chunk's last token begins a page)
    n = held + M - (held + M - 1) % page
    M = n - held
    rng = np.random.default_rng(M)
    x = torch.from_numpy(rng.standard_normal((1, n, H, d))).to(torch.bfloat16).cuda().transpose(1, 2)
    q = torch.from_numpy(rng.standard_normal((1, M, H, d))).to(torch.bfloat16).cuda().transpose(1, 2)
    pages = -(-n // page)
    arrays = [[torch.zeros(pages, H, page, d, dtype=torch.uint8, device="cuda"), torch.zeros(pages, H, device="cuda")] for _ in range(2)]
    c, table, status = B.make_kv_cache(*arrays, format="e4m3_page"), torch.arange(pages, dtype=torch.int32, device="cuda")[None].contiguous(), _i32([0])
    spoilt = x.clone()
    spoilt[0, :, n - 1, 3] = bad
    B.kv_cache_append(c, spoilt[:, :, :held], spoilt[:, :, :held], table, _i32([0]), status=status)
    B.kv_cache_append(c, spoilt[:, :, held:], spoilt[:, :, held:], table, _i32([held]), status=status)
    o, lse = torch.empty_like(q), torch.empty(1, H, M, device="cuda")
    p = B.make_cached_attn(c, q, o, table, True)
    ws = torch.empty(max(256, B.cached_attn_workspace_bytes(p)), dtype=torch.uint8, device="cuda")
    B.cached_attn_fwd(p, q, table, _i32([n]), o, None, lse, status, ws)
    assert torch.isnan(o[0, :, M - 1]).all() and torch.isnan(lse[0, :, M - 1]).all() and int(status) == 0
    kv = K.gathered(arrays[0][0].cpu().numpy(), arrays[0][1].cpu().numpy().astype(np.float64), table[0].tolist(), n, page)[:, :n - 1]
    there = np.arange(n - 1)[None] <= held + np.arange(M - 1)[:, None]
    for h in range(H):
        want = K.attention(_f64(q)[0, h, :M - 1], kv[h], kv[h], there, d ** -0.5)
        _compare(_f64(o)[0, h, :M - 1], _f64(lse)[0, h, :M - 1], want, 2.0 ** -11, d, kv[h])


@pytest.mark.parametrize("M", [1, 3, 140])
def test_scales_next_to_zero(M):
    """Keys whose scale times the row's is no number of fp32 but 0, and a length that ends within a tile: logits of 0, not NaNs."""
    x = Cached(np.random.default_rng(21), 1, 2, 1, M, 64, 16, [203], True)
    x.scales[0][:] = np.float32(1e-44)
    x.scales[0][x.ids[0][::3]] = 0.0
    x.codes[0][x.ids[0][::3]] = 0
    x.q *= 1e-3
    x.run(True, None)
    x.check(True, None)
    x.run(False, None)
    x.check(False, None)


@pytest.mark.parametrize("M", [1, 140])
def test_a_sequence_longer_than_its_table_is_reported(M):
    """It counts as long as its table has pages for; the call says so, as the append does."""
    x = Cached(np.random.default_rng(17), 2, 1, 1, M, 128, 16, [160, 160], True)
    c, p, table, ws = x.run(True, None)
    assert int(x.status) == 0
    o, lse, status = x.o.clone(), x.lse.clone(), _i32([0])
    B.cached_attn_fwd(p, x.q, table, _i32([160, 161]), x.o, None, x.lse, status, ws)
    assert torch.equal(o, x.o) and torch.equal(lse, x.lse) and int(status) == B.SVA_DEV_BAD_INDEX


@pytest.mark.parametrize("N,S", [(2, 77), (2, 3000), (40, 77), (64, 3000)])
def test_values_that_are_infinite(N, S):
    """An infinity among the values a row sees is the row's output in its channel, two of unlike sign are a NaN; what is left out has no part in it."""
    gen = torch.Generator("cuda").manual_seed(N + S)
    q, k, v = (torch.randn(1, 2, n, 64, generator=gen, device="cuda").to(torch.bfloat16) for n in (N, S, S))
    lengths = _i32([S - 5])
    clean, clean_lse = _cross(q, k, v, lengths, None)
    inf = float("inf")
    v[0, 0, 20, 3], v[0, 0, 31, 4], v[0, 0, 40, 5], v[0, 0, 50, 5], v[0, 1, S - 2, 6] = inf, -inf, inf, -inf, inf
    o, lse = _cross(q, k, v, lengths, None)
    assert (o[0, 0, :, 3] == inf).all() and (o[0, 0, :, 4] == -inf).all() and torch.isnan(o[0, 0, :, 5]).all()
    same = torch.ones(64, dtype=torch.bool, device="cuda")
    same[3:6] = False
    assert torch.equal(o[0, 0][:, same], clean[0, 0][:, same]) and torch.equal(o[0, 1], clean[0, 1]) and torch.equal(lse, clean_lse)
