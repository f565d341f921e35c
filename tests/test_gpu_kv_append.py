"""Appending to the cache with a scale per page and head, against the fp64 oracle: bytes and scales exactly."""
import numpy as np
import pytest
import torch

from oracle import keys as K
from oracle.layer import e4m3_values, f32
from paper_2606_23743_b200 import binding as B

pytestmark = pytest.mark.gpu


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _f64(t):
    return t.float().cpu().numpy().astype(np.float64)


def _rows(rng, shape, first, spread=1.0):
    b, h, t, d = shape
    x = rng.standard_normal((b, t, h, d) if first else shape)
    x *= np.exp(spread * rng.standard_normal(x.shape[:-1]))[..., None]
    x = torch.from_numpy(x).to(torch.bfloat16).cuda()
    return x.transpose(1, 2) if first else x


def _cache(pages, H, page, d, fill=0x11, scale=0.5):
    arrays = [[torch.full((pages, H, page, d), fill, dtype=torch.uint8, device="cuda"), torch.full((pages, H), scale, device="cuda")] for _ in range(2)]
    return B.make_kv_cache(*arrays, format="e4m3_page"), arrays


def _expect(arrays, x, table, lengths, counts, page):
    codes, scale = arrays[0].cpu().numpy().copy(), arrays[1].cpu().numpy().astype(np.float64)
    K.append(codes, scale, _f64(x), table, lengths, counts, page)
    return codes, scale


def _same(arrays, want):
    np.testing.assert_array_equal(arrays[0].cpu().numpy(), want[0])
    np.testing.assert_array_equal(arrays[1].cpu().numpy().astype(np.float64), want[1])


CASES = [
    # B, H, d, page, tokens first, (lengths, counts) of calls that follow one another; T is the largest count
    (1, 1, 64, 16, False, [([0], [1]), ([1], [1])]),
    (3, 4, 128, 64, True, [([0, 0, 0], [70, 64, 1]), ([70, 64, 1], [1, 1, 1]), ([71, 65, 2], [0, 130, 63])]),
    (2, 3, 128, 48, False, [([0, 0], [47, 100]), ([47, 100], [2, 0]), ([49, 100], [95, 44])]),
    (2, 2, 64, 1024, True, [([0, 0], [1030, 700]), ([1030, 700], [900, 1300])]),
    (1, 5, 128, 512, False, [([0], [300]), ([300], [700])]),
    (5, 1, 64, 32, True, [([0] * 5, [31, 32, 33, 0, 64]), ([31, 32, 33, 0, 64], [1] * 5)]),
]


@pytest.mark.parametrize("Bq,H,d,page,first,calls", CASES)
def test_append(Bq, H, d, page, first, calls):
    rng = np.random.default_rng(page + d + H)
    per = max(-(-(n + m) // page) for at, cnt in calls for n, m in zip(at, cnt))
    pages = Bq * per + 2
    table = rng.permutation(pages)[:Bq * per].reshape(Bq, per)
    c, arrays = _cache(pages, H, page, d)
    status = _i32([0])
    for at, cnt in calls:
        x = [_rows(rng, (Bq, H, max(cnt), d), first) for _ in range(2)]
        want = [_expect(a, t, table.tolist(), at, cnt, page) for a, t in zip(arrays, x)]
        B.kv_cache_append(c, *x, _i32(table), _i32(at), _i32(cnt), status)
        for a, w in zip(arrays, want):
            _same(a, w)
    assert int(status) == 0


def test_what_is_read_back_is_what_the_codes_stand_for():
    rng = np.random.default_rng(5)
    Bq, H, d, page, N = 2, 3, 128, 48, 100
    c, arrays = _cache(7, H, page, d)
    table = _i32([[5, 1, 2], [0, 6, 3]])
    x = [_rows(rng, (Bq, H, N, d), True) for _ in range(2)]
    B.kv_cache_append(c, *x, table, _i32([0, 0]), _i32([100, 77]))
    out = [torch.full((Bq, H, N, d), 9.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    B.kv_cache_read(c, table, _i32([100, 77]), *out)
    for a, o in zip(arrays, out):
        codes, scale = a[0].cpu().numpy(), a[1].cpu().numpy().astype(np.float64)
        for b, n in ((0, 100), (1, 77)):
            want = torch.from_numpy(f32(K.gathered(codes, scale, table[b].tolist(), n, page))).to(torch.bfloat16)
            assert torch.equal(o[b, :, :n].cpu(), want) and not o[b, :, n:].any()


def test_values_far_out():
    """Zeros, values near the ends of bf16, scales that are denormal or have a significand of ones; NaN and infinity spoil their page and head alone."""
    H, d, page = 9, 64, 16
    x = torch.zeros(1, H, 16, d, dtype=torch.bfloat16, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(3)
    noise = torch.randn(16, d, generator=gen, device="cuda")
    x[0, 1] = 3.0e38 * (noise / noise.abs().max())
    x[0, 2] = 1e-38 * noise
    x[0, 3] = 1e-40 * noise
    x[0, 4] = noise
    x[0, 4, 3, 7] = float("nan")
    x[0, 5] = noise
    x[0, 5, 9, 1] = -float("inf")
    x[0, 6] = 448.0 * 2.0 ** -70 * (noise / noise.abs().max())
    x[0, 7, 4, 2] = -0.0
    x[0, 8] = noise
    c, arrays = _cache(2, H, page, d)
    B.kv_cache_append(c, x, x, _i32([[1]]), _i32([0]))
    for codes, scale in arrays:
        want_codes, want_scale = np.full((2, H, page, d), 0x11, np.uint8), np.full((2, H), 0.5)
        K.append(want_codes, want_scale, _f64(x), [[1]], [0], [16], page)
        np.testing.assert_array_equal(scale.cpu().numpy().astype(np.float64), want_scale)
        value = e4m3_values(codes.cpu().numpy()) * want_scale[:, :, None, None]
        np.testing.assert_array_equal(value, e4m3_values(want_codes) * want_scale[:, :, None, None])
        assert np.isnan(value[1, 4]).all() and np.isnan(value[1, 5]).all() and not np.isnan(value[1, 8]).any()


def test_a_larger_value_makes_a_new_scale_for_what_is_there():
    """A page of zeros takes the scale of what comes after it; a page of values is re-expressed once a larger one comes, and not for a smaller."""
    H, d, page = 1, 64, 16
    c, arrays = _cache(1, H, page, d)
    rng = np.random.default_rng(8)
    want = [(a[0].cpu().numpy().copy(), a[1].cpu().numpy().astype(np.float64)) for a in arrays]
    for n, size in enumerate((0.0, 1e-3, 1e-4, 2.0, 1.0, 300.0, 1e-6)):
        x = torch.from_numpy(rng.standard_normal((1, H, 1, d)) * size).to(torch.bfloat16).cuda()
        before = arrays[0][0].clone()
        B.kv_cache_append(c, x, x, _i32([[0]]), _i32([n]))
        for a, w in zip(arrays, want):
            K.append(*w, _f64(x), [[0]], [n], [1], page)
            _same(a, w)
        if size in (1e-4, 1.0, 1e-6):
            assert torch.equal(arrays[0][0][0, 0, :n], before[0, 0, :n])


def test_bad_pages_and_counts():
    H, d, page = 2, 64, 16
    rng = np.random.default_rng(9)
    c, arrays = _cache(4, H, page, d)
    x = [_rows(rng, (4, H, 40, d), False) for _ in range(2)]
    table, at, cnt = [[0, 9, -1], [1, 2, 3], [-5, -1, -1], [3, 3, 3]], [3, 30, 0, -7], [40, 90, 0, -2]
    status = _i32([0])
    real = [40, 40, 0, 0]                                                       # (as they count)
    want = [_expect(a, t, table, [3, 30, 0, 0], real, page) for a, t in zip(arrays, x)]
    B.kv_cache_append(c, *x, _i32(table), _i32(at), _i32(cnt), status)
    for a, w in zip(arrays, want):
        _same(a, w)
    assert int(status) == B.SVA_DEV_BAD_INDEX


def test_captured_and_on_another_stream():
    H, d, page = 2, 128, 32
    rng = np.random.default_rng(10)
    x = [_rows(rng, (1, H, 50, d), True) for _ in range(2)]
    c, arrays = _cache(3, H, page, d)
    table, at = _i32([[2, 0, 1]]), _i32([0])
    want = [_expect(a, t, table.tolist(), [0], [50], page) for a, t in zip(arrays, x)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        B.kv_cache_append(c, *x, table, at)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            B.kv_cache_append(c, *x, table, at)
        side.synchronize()
        for a, w in zip(arrays, want):
            _same(a, w)
            a[0].fill_(0x11)
            a[1].fill_(0.5)
        at.fill_(7)                                                            # what a replay reads is what is there then
        graph.replay()
    side.synchronize()
    for a, t in zip(arrays, x):
        fresh = [torch.full_like(a[0], 0x11), torch.full_like(a[1], 0.5)]
        _same(a, _expect(fresh, t, table.tolist(), [7], [50], page))


@pytest.mark.parametrize("d,page,calls", [(64, 2048, [(0, 1500), (1500, 1700)]), (128, 1040, [(0, 1040), (1040, 7), (1047, 1500)]), (64, 1040, [(3, 1037)])])
def test_pages_beyond_what_the_registers_hold(d, page, calls):
    """A call's rows of one page beyond those that stay in registers (1 024 of 64 channels, 512 of 128): the page's largest value is one of them."""
    rng = np.random.default_rng(d + page)
    H = 2
    pages = -(-sum(calls[-1]) // page) + 1
    table = rng.permutation(pages)[None]
    c, arrays = _cache(pages, H, page, d)
    status = _i32([0])
    for at, cnt in calls:
        x = [_rows(rng, (1, H, cnt, d), True) for _ in range(2)]
        last = min(page - at % page, cnt) - 1                                  # the call's last row in its first page
        for n, t in enumerate(x):
            t[0, n, last, 5] = 3000.0 * (1 + at)
        want = [_expect(a, t, table.tolist(), [at], [cnt], page) for a, t in zip(arrays, x)]
        B.kv_cache_append(c, *x, _i32(table), _i32([at]), _i32([cnt]), status)
        for a, w in zip(arrays, want):
            _same(a, w)
    assert int(status) == 0
