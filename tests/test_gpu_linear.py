"""e4m3 linear layers against the fp64 oracle: codes and scales exactly, products within a bound that is derived here."""
import numpy as np
import pytest
import torch

from oracle import layer as L
from paper_2606_23743_b200 import binding as B

pytestmark = pytest.mark.gpu


def _bf16(rng, *shape, spread=True):
    x = rng.standard_normal(shape)
    if spread:
        x = x * np.exp(rng.standard_normal(shape[-1]))
    return torch.from_numpy(x).to(torch.bfloat16)


def _padded(rows, cols, dtype, fill, extra=0):
    """A [rows, cols] view of a buffer whose rows are whole 16-byte pieces, and the buffer."""
    per = 16 // torch.empty(0, dtype=dtype).element_size()
    buf = torch.full((rows, (-(-cols // per) + extra) * per), fill, dtype=dtype, device="cuda")
    return buf[:, :cols], buf


def _layer(rng, M, N, K, act="none", bias=False, residual=False, extra=0):
    """Inputs on the device, quantised by the library, and the plan."""
    x, xbuf = _padded(M, K, torch.bfloat16, 0, extra)
    w, wbuf = _padded(N, K, torch.bfloat16, 0, extra)
    x.copy_(_bf16(rng, M, K))
    w.copy_(_bf16(rng, N, K, spread=False) / np.sqrt(K))
    x8, w8 = (torch.full((n, (-(-K // 16) + extra) * 16), 0x55, dtype=torch.uint8, device="cuda") for n in (M, N))
    G = -(-K // 128)
    xs = torch.full((G, M + extra), 9.0, device="cuda")
    ws = torch.full((-(-N // 128), G + extra), 9.0, device="cuda")
    out, obuf = _padded(M, N, torch.bfloat16, 5.0, extra)
    r = None
    if residual:
        r, _ = _padded(M, N, torch.bfloat16, 0, extra)
        r.copy_(_bf16(rng, M, N))
    b = torch.from_numpy(rng.standard_normal(N)).float().cuda() if bias else None
    p = B.make_linear(x, x8, xs, w8, ws, out, act, r, w=w)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.quantize_rows_fp8(p, x, x8, xs)
    B.quantize_tiles_fp8(p, w, w8, ws)
    return dict(p=p, x=x, w=w, x8=x8, w8=w8, xs=xs, ws=ws, out=out, obuf=obuf, bias=b, residual=r, status=status, act=act)


def _product(s):
    B.linear_fp8(s["p"], s["x8"], s["xs"], s["w8"], s["ws"], s["out"], s["bias"], s["residual"], s["status"])
    torch.cuda.synchronize()
    assert int(s["status"].item()) == 0
    return s["out"].float().cpu().numpy().astype(np.float64)


def _f64(t):
    return None if t is None else t.detach().float().cpu().numpy().astype(np.float64)


def _check(s, got):
    """|error| <= half a bf16 step of the result, plus what fp32 sums may lose: a group of 128 is at most eight additions whose operands are
    aligned to 2^-22 of the largest, the groups one addition each (K/128 * 2^-24 <= 2^-18 here), all relative to the sum of
    magnitudes A: under 2^-16 A; the activations' slopes are below 1.2, their own fp32 steps under 2^-18 of the result; the residual's
    addition is one fp32 rounding."""
    K = s["p"].K
    x8, w8 = s["x8"][:, :K].cpu().numpy(), s["w8"][:, :K].cpu().numpy()
    M, G = s["p"].M, -(-K // 128)
    ref, A = L.linear(x8, _f64(s["xs"][:, :M]), w8, _f64(s["ws"][:, :G]), _f64(s["bias"]), s["act"], _f64(s["residual"]))
    step = 2.0 ** -8 * np.abs(ref) + 2.0 ** -133
    bound = step + 1.2 * 2.0 ** -16 * (A + (0 if s["bias"] is None else np.abs(_f64(s["bias"])))) + 2.0 ** -18 * (
        np.abs(ref) + (0 if s["residual"] is None else 2 * np.abs(_f64(s["residual"]))))
    worst = np.max(np.abs(got - ref) / bound)
    assert worst <= 1.0, worst


@pytest.mark.parametrize("M,K,extra", [(1, 1, 0), (1, 128, 0), (3, 127, 1), (33, 129, 0), (70, 1000, 2), (4, 2047, 0), (700, 1160, 0), (1, 4096, 0)])
def test_codes_and_scales_are_the_oracles(M, K, extra):
    rng = np.random.default_rng(M * 1000 + K)
    s = _layer(rng, M, 200, K, extra=extra)
    torch.cuda.synchronize()
    codes, scale = L.quantize_rows(_f64(s["x"]))
    np.testing.assert_array_equal(s["x8"][:, :K].cpu().numpy(), codes)
    np.testing.assert_array_equal(_f64(s["xs"][:, :M]), scale)
    codes, scale = L.quantize_tiles(_f64(s["w"]))
    np.testing.assert_array_equal(s["w8"][:, :K].cpu().numpy(), codes)
    np.testing.assert_array_equal(_f64(s["ws"][:, :-(-K // 128)]), scale)
    upto = -(-K // 16) * 16
    assert (s["x8"][:, K:upto] == 0).all() and (s["w8"][:, K:upto] == 0).all()                     # whole 16-byte pieces
    assert (s["x8"][:, upto:] == 0x55).all() and (s["xs"][:, M:] == 9.0).all() and (s["ws"][:, -(-K // 128):] == 9.0).all()


def test_quantisers_at_the_ends_of_the_range():
    """Zero groups, tiny and huge magnitudes (where the reciprocal's way to the quotient does not serve), signed zeros, ties."""
    K = 128 * 6
    x = torch.zeros(3, K)
    x[0, 128:256] = torch.linspace(-1, 1, 128) * 1e-37
    x[0, 256:384] = torch.linspace(-1, 1, 128) * 3e38
    x[0, 384:512] = -0.0
    x[1, :128] = torch.arange(128) * 0.25                          # amax 31.75
    x[1, 128:256] = torch.linspace(0, 448, 128).round()            # scale 1: ties of the format
    x[1, 255] = 448
    x[2, 5] = 9.2e-41                                              # a denormal alone
    x = x.to(torch.bfloat16).cuda()
    x8, xs = torch.zeros(3, K, dtype=torch.uint8, device="cuda"), torch.zeros(6, 3, device="cuda")
    p = B.make_linear(x, x8, xs, w8=x8)
    B.quantize_rows_fp8(p, x, x8, xs)
    codes, scale = L.quantize_rows(_f64(x))
    np.testing.assert_array_equal(_f64(xs), scale)
    np.testing.assert_array_equal(x8.cpu().numpy(), codes)


SIZES = [(1, 8, 16), (1, 2048, 2048), (2, 1000, 4096), (3, 128, 128), (16, 136, 640), (17, 2056, 1000), (31, 384, 8192), (33, 520, 136), (64, 1024, 513),
         (65, 264, 2048), (100, 24, 100), (128, 128, 1), (129, 1000, 127), (200, 4100, 384), (333, 2051, 1031), (512, 512, 512), (1000, 1544, 904),
         (2050, 2304, 256), (1, 24576, 256), (5, 40, 16384), (9473, 520, 264), (1024, 5000, 1160), (200, 1000, 2048), (257, 515, 1500),
         (400, 1544, 4096), (65, 8, 16384)]


@pytest.mark.parametrize("M,N,K", SIZES)
def test_products(M, N, K):
    rng = np.random.default_rng(M + 7 * N + K)
    s = _layer(rng, M, N, K)
    _check(s, _product(s))
    N8 = s["obuf"].shape[1]
    if N8 > N:
        assert (s["obuf"][:, N:] == 5.0).all()                     # columns that do not exist are not written


@pytest.mark.parametrize("act", ["none", "gelu", "silu"])
@pytest.mark.parametrize("bias,residual", [(True, False), (False, True), (True, True)])
@pytest.mark.parametrize("M,N,K,extra", [(2, 333, 300, 1), (40, 260, 520, 0), (300, 1155, 384, 3), (1111, 2500, 200, 0), (5003, 1155, 384, 3), (130, 523, 2100, 1), (70, 1031, 900, 0)])
def test_epilogues(M, N, K, extra, bias, residual, act):
    rng = np.random.default_rng(M + N)
    s = _layer(rng, M, N, K, act, bias, residual, extra)
    _check(s, _product(s))
    if extra:
        assert (s["obuf"][:, N:] == 5.0).all()


@pytest.mark.parametrize("M,N,K", [(7, 256, 512), (300, 640, 512), (300, 640, 2500), (2500, 2048, 256)])
def test_residual_in_place_and_repeatable(M, N, K):
    rng = np.random.default_rng(5)
    s = _layer(rng, M, N, K, "none", True, True)
    first = s["residual"].clone()
    want = _product(s)
    s["out"] = s["residual"]
    got = _product(s)                                              # the sum replaces the residual stream
    np.testing.assert_array_equal(got, want)
    s["residual"].copy_(first)
    np.testing.assert_array_equal(_product(s), want)               # the same bytes again


@pytest.mark.parametrize("M", [3, 300])
def test_scales_and_codes_from_elsewhere(M):
    """Codes of a checkpoint: any finite byte, scales of any size and sign."""
    rng = np.random.default_rng(6)
    N, K = 300, 400
    s = _layer(rng, M, N, K)
    bytes_ = rng.integers(0, 127, (N, 400)) + 128 * rng.integers(0, 2, (N, 400))
    s["w8"].copy_(torch.from_numpy(bytes_.astype(np.uint8)))
    s["ws"].copy_(torch.from_numpy(rng.standard_normal(tuple(s["ws"].shape)) * 10.0 ** rng.integers(-6, 6, tuple(s["ws"].shape))).float())
    _check(s, _product(s))


@pytest.mark.parametrize("M", [3, 300])
def test_bytes_beyond_a_row_do_not_count(M):
    """Rows of codes whose last piece goes on with something else (NaN codes) behind the K inputs."""
    rng = np.random.default_rng(7)
    s = _layer(rng, M, 300, 395)
    want = _product(s)
    s["x8"][:, 395:] = 0x7F
    s["w8"][:, 395:] = 0x7F
    np.testing.assert_array_equal(_product(s), want)


@pytest.mark.parametrize("M", [2, 200])
def test_a_nan_code_stays_with_its_outputs(M):
    rng = np.random.default_rng(8)
    s = _layer(rng, M, 264, 300)
    want = _product(s)
    s["x8"][1, 7] = 0x7F
    s["w8"][200, 299] = 0xFF
    got = _product(s)
    bad = np.zeros(got.shape, bool)
    bad[1, :], bad[:, 200] = True, True
    assert np.isnan(got[bad]).all()
    np.testing.assert_array_equal(got[~bad], want[~bad])


@pytest.mark.parametrize("act", ["gelu", "silu"])
@pytest.mark.parametrize("M", [2, 200, 2500])
def test_activations_far_out(M, act):
    """Sums from the bias alone, far to both sides, infinities and a NaN, which stays alone.  What is left of a value far to the negative side
    may be 2^-54."""
    N = 2048
    b = torch.linspace(-60, 60, N, dtype=torch.float64)
    b[::16] = torch.tensor([-1e38, -1e30, -1e18, -1e4, -100.0, 0.0, 100.0, 1e4, 1e18, 1e30, 1e38, -0.5, 1e-30, -1e-30, -64.0, -65.0] * (N // 256))
    b[5], b[700], b[1501] = float("nan"), float("inf"), float("-inf")
    x8, w8 = torch.zeros(M, 128, dtype=torch.uint8, device="cuda"), torch.zeros(N, 128, dtype=torch.uint8, device="cuda")
    xs, ws = torch.ones(1, M, device="cuda"), torch.ones(N // 128, 1, device="cuda")
    out = torch.empty(M, N, dtype=torch.bfloat16, device="cuda")
    p = B.make_linear(None, x8, xs, w8, ws, out, act, K=128)
    B.linear_fp8(p, x8, xs, w8, ws, out, b.float().cuda())
    got = _f64(out)
    assert (got == got[:1])[:, ~np.isnan(got[0])].all()                 # every row is the same
    with np.errstate(all="ignore"):
        ref = L.activation(b.float().double().numpy(), act)
    ref[1501] = 0.0
    assert np.isnan(got[:, 5]).all() and np.isnan(got).sum() == M and got[0, 700] == np.inf
    at = np.isfinite(ref)
    got, ref = got[0][at], ref[at]
    assert (np.abs(got - ref) <= 2.0 ** -8 * np.abs(ref) + 2.0 ** -18 * np.abs(ref) + 2.0 ** -53).all()


def test_on_a_side_stream_and_captured():
    rng = np.random.default_rng(9)
    s = _layer(rng, 37, 520, 512, "silu", True)
    want = _product(s)
    side = torch.cuda.Stream()
    s["out"].fill_(0)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        B.quantize_rows_fp8(s["p"], s["x"], s["x8"], s["xs"])
        B.linear_fp8(s["p"], s["x8"], s["xs"], s["w8"], s["ws"], s["out"], s["bias"], status=s["status"])
    side.synchronize()
    np.testing.assert_array_equal(_f64(s["out"]), want)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        B.quantize_rows_fp8(s["p"], s["x"], s["x8"], s["xs"])
        B.linear_fp8(s["p"], s["x8"], s["xs"], s["w8"], s["ws"], s["out"], s["bias"], status=s["status"])
    s["out"].fill_(0)
    s["x8"].fill_(0)
    g.replay()
    torch.cuda.synchronize()
    np.testing.assert_array_equal(_f64(s["out"]), want)


@pytest.mark.parametrize("M,N,K", [(3, 520, 2048), (40, 300, 1000), (1500, 4096, 400), (200, 300, 2048)])
def test_without_clusters(M, N, K):
    """As on a part of a device that holds none: nothing is split, no pairs."""
    rng = np.random.default_rng(11)
    s = _layer(rng, M, N, K, "gelu", True, True)
    try:
        B.debug_set_mode(64)
        _check(s, _product(s))
    finally:
        B.debug_set_mode(0)


@pytest.mark.parametrize("M,N,K", [(4, 512, 2048), (300, 512, 2048), (1500, 4096, 1024)])
def test_a_starved_product_gives_up(M, N, K):
    """Inputs after the first 128 are withheld: the waits run out, every role leaves, the call after it is whole."""
    rng = np.random.default_rng(10)
    s = _layer(rng, M, N, K)
    want = _product(s)
    try:
        B.debug_set_wait_limit(100_000_000)                        # about 50 ms
        B.debug_set_mode(1024)
        B.linear_fp8(s["p"], s["x8"], s["xs"], s["w8"], s["ws"], s["out"], s["bias"], s["residual"], s["status"])
        torch.cuda.synchronize()
    finally:
        B.debug_set_mode(0)
        B.debug_set_wait_limit(0)
    assert int(s["status"].item()) == B.SVA_DEV_TIMEOUT
    s["status"].zero_()
    np.testing.assert_array_equal(_product(s), want)


def test_weights_of_very_many_rows():
    """More than 65 535 tiles of 128 outputs."""
    rng = np.random.default_rng(12)
    N, K = 65536 * 128 + 5, 24
    w, w8 = torch.zeros(N, K, dtype=torch.bfloat16, device="cuda"), torch.full((N, 32), 0x55, dtype=torch.uint8, device="cuda")
    ws = torch.full((65537, 1), 9.0, device="cuda")
    w[-133:], w[:128] = _bf16(rng, 133, K).cuda(), _bf16(rng, 128, K).cuda()
    B.quantize_tiles_fp8(B.make_linear(w8=w8, w_scale=ws, w=w), w, w8, ws)
    for at, tiles in ((np.s_[:128], np.s_[:1]), (np.s_[-133:], np.s_[-2:])):
        codes, scale = L.quantize_tiles(_f64(w[at]))
        np.testing.assert_array_equal(w8[at][:, :K].cpu().numpy(), codes)
        np.testing.assert_array_equal(_f64(ws[tiles]), scale)
    assert bool((w8[:, K:] == 0).all()) and bool((w8[128:-133] == 0).all()) and bool((ws[1:-2] == 1.0).all())


def _chose(form):
    names = {1: "few tokens", 2: "single CTAs", 3: "split inputs", 4: "pairs"}
    got = B.debug_last_choice()
    assert got == form, f"these sizes are for {names[form]}, and {names.get(got, got)} took them"


# Sizes that pairs of CTAs take: several tiles per pair, rings and accumulators that come round, one or two groups of inputs, rows and columns that end
# within a tile, a single row or column of tiles.
PAIRS = [(5003, 2500, 1160), (2500, 3001, 2309), (130, 33003, 1030), (33000, 130, 264), (1800, 5003, 100), (3000, 3001, 130)]


@pytest.mark.parametrize("M,N,K", PAIRS)
def test_products_in_pairs(M, N, K):
    rng = np.random.default_rng(M + 7 * N + K)
    s = _layer(rng, M, N, K, extra=1)
    got = _product(s)
    _chose(4)
    _check(s, got)
    assert (s["obuf"][:, N:] == 5.0).all()


@pytest.mark.parametrize("act", ["none", "gelu", "silu"])
@pytest.mark.parametrize("bias,residual", [(True, False), (False, True), (True, True)])
def test_epilogues_in_pairs(bias, residual, act):
    M, N, K = 5003, 2501, 1160
    rng = np.random.default_rng(13)
    s = _layer(rng, M, N, K, act, bias, residual, 1)
    got = _product(s)
    _chose(4)
    _check(s, got)
    assert (s["obuf"][:, N:] == 5.0).all()


@pytest.mark.parametrize("M,N,K", [(5003, 2501, 1160), (2500, 3000, 256)])
def test_residual_in_place_and_repeatable_in_pairs(M, N, K):
    rng = np.random.default_rng(14)
    s = _layer(rng, M, N, K, "silu", True, True)
    first = s["residual"].clone()
    want = _product(s)
    s["out"] = s["residual"]
    got = _product(s)
    _chose(4)
    np.testing.assert_array_equal(got, want)
    s["residual"].copy_(first)
    np.testing.assert_array_equal(_product(s), want)


def test_a_nan_code_stays_with_its_outputs_in_pairs():
    rng = np.random.default_rng(15)
    s = _layer(rng, 5003, 2501, 1160)
    want = _product(s)
    s["x8"][4999, 7] = s["x8"][300, 1159] = 0x7F
    s["w8"][2400, 1159] = s["w8"][130, 640] = 0xFF
    got = _product(s)
    _chose(4)
    bad = np.zeros(got.shape, bool)
    bad[[300, 4999], :], bad[:, [130, 2400]] = True, True
    assert np.isnan(got[bad]).all()
    np.testing.assert_array_equal(got[~bad], want[~bad])


@pytest.mark.parametrize("act", ["gelu", "silu"])
def test_activations_far_out_in_pairs(act):
    """Two values share a reciprocal: a NaN or an infinity beside one leaves it alone."""
    M, N = 2500, 3008
    b = torch.linspace(-60, 60, N, dtype=torch.float64)
    b[5], b[700], b[1501] = float("nan"), float("inf"), float("-inf")
    b[::32], b[1::32] = -1e38, 1e38
    x8, w8 = torch.zeros(M, 128, dtype=torch.uint8, device="cuda"), torch.zeros(N, 128, dtype=torch.uint8, device="cuda")
    xs, ws = torch.ones(1, M, device="cuda"), torch.ones(-(-N // 128), 1, device="cuda")
    out = torch.empty(M, N, dtype=torch.bfloat16, device="cuda")
    p = B.make_linear(None, x8, xs, w8, ws, out, act, K=128)
    B.linear_fp8(p, x8, xs, w8, ws, out, b.float().cuda())
    _chose(4)
    got = _f64(out)
    assert (got == got[:1])[:, ~np.isnan(got[0])].all()
    with np.errstate(all="ignore"):
        ref = L.activation(b.float().double().numpy(), act)
    ref[1501] = 0.0
    assert np.isnan(got[:, 5]).all() and np.isnan(got).sum() == M and got[0, 700] == np.inf
    at = np.isfinite(ref)
    got, ref = got[0][at], ref[at]
    assert (np.abs(got - ref) <= 2.0 ** -8 * np.abs(ref) + 2.0 ** -18 * np.abs(ref) + 2.0 ** -53).all()


@pytest.mark.parametrize("M,N,K,form", [(2500, 3000, 400, 4), (200, 300, 4000, 3)])
def test_what_needs_clusters_goes_without(M, N, K, form):
    rng = np.random.default_rng(16)
    s = _layer(rng, M, N, K, "gelu", True, True)
    _product(s)
    _chose(form)
    try:
        B.debug_set_mode(64)
        got = _product(s)
        _chose(2)
    finally:
        B.debug_set_mode(0)
    _check(s, got)


def test_starved_pairs_give_up():
    rng = np.random.default_rng(17)
    s = _layer(rng, 5003, 2500, 1160, "none", True, True)
    want = _product(s)
    try:
        B.debug_set_wait_limit(100_000_000)                        # about 50 ms
        B.debug_set_mode(1024)
        B.linear_fp8(s["p"], s["x8"], s["xs"], s["w8"], s["ws"], s["out"], s["bias"], s["residual"], s["status"])
        torch.cuda.synchronize()
        _chose(4)
    finally:
        B.debug_set_mode(0)
        B.debug_set_wait_limit(0)
    assert int(s["status"].item()) == B.SVA_DEV_TIMEOUT
    s["status"].zero_()
    np.testing.assert_array_equal(_product(s), want)


@pytest.mark.parametrize("M,N,K,form", [(64, 520, 1030, 1), (65, 520, 1030, 2), (1111, 1501, 1030, 2), (65, 4096, 4096, 3)])
def test_the_other_forms_are_reached(M, N, K, form):
    rng = np.random.default_rng(18)
    s = _layer(rng, M, N, K)
    got = _product(s)
    _chose(form)
    _check(s, got)


@pytest.mark.parametrize("K", [129, 330, 650, 1000, 1100])
def test_codes_and_scales_of_many_rows(K):
    """Four groups of inputs per thread: 2, 3, 6, 8 and 9 groups, rows and inputs that end within a block."""
    M = 4801
    rng = np.random.default_rng(K)
    x, xbuf = _padded(M, K, torch.bfloat16, 0, 1)
    x.copy_(_bf16(rng, M, K))
    xbuf[:, K:] = 7.0                                              # (not inputs)
    G, row = -(-K // 128), -(-K // 16) * 16
    x8, xs = torch.full((M, row + 16), 0x55, dtype=torch.uint8, device="cuda"), torch.full((G, M + 3), 9.0, device="cuda")
    B.quantize_rows_fp8(B.make_linear(x, x8, xs), x, x8, xs)
    assert B.debug_last_choice() == 4
    codes, scale = L.quantize_rows(_f64(x))
    np.testing.assert_array_equal(x8[:, :K].cpu().numpy(), codes)
    np.testing.assert_array_equal(_f64(xs[:, :M]), scale)
    assert (x8[:, K:row] == 0).all() and (x8[:, row:] == 0x55).all() and (xs[:, M:] == 9.0).all()


@pytest.mark.parametrize("M", [5, 200, 4801])
def test_nan_and_infinities_in_the_inputs(M):
    """A NaN is left out of its scale and stays with its own token or output; an infinity takes its token, or the 128 outputs of its tile, with it.
    What is left is as if a zero stood there."""
    N, K = 300, 1000
    rng = np.random.default_rng(19)
    s = _layer(rng, M, N, K)
    s["x"][1, 7] = s["x"][3, 990] = 0.0
    s["w"][5, 130] = s["w"][290, 999] = 0.0
    B.quantize_rows_fp8(s["p"], s["x"], s["x8"], s["xs"])
    B.quantize_tiles_fp8(s["p"], s["w"], s["w8"], s["ws"])
    want = _product(s)
    s["x"][1, 7], s["x"][3, 990] = float("nan"), -float("inf")
    s["w"][5, 130], s["w"][290, 999] = -float("nan"), float("inf")
    B.quantize_rows_fp8(s["p"], s["x"], s["x8"], s["xs"])
    assert B.debug_last_choice() == (4 if M == 4801 else 1)
    B.quantize_tiles_fp8(s["p"], s["w"], s["w8"], s["ws"])
    for x, x8, xs, (codes, scale) in ((s["x"], s["x8"], s["xs"], L.quantize_rows(_f64(s["x"]))), (s["w"], s["w8"], s["ws"], L.quantize_tiles(_f64(s["w"])))):
        got, nan = x8[:, :K].cpu().numpy(), codes == 127
        assert nan.sum() == 2
        np.testing.assert_array_equal(got[~nan], codes[~nan])
        assert ((got[nan] & 127) == 127).all()
        np.testing.assert_array_equal(_f64(xs), scale)
    got = _product(s)
    bad = np.zeros(got.shape, bool)
    bad[[1, 3], :], bad[:, 5], bad[:, 256:] = True, True, True      # (the tile of outputs 256 to 299)
    assert np.isnan(got[bad]).all()
    np.testing.assert_array_equal(got[~bad], want[~bad])


def test_rows_of_nan_alone():
    x = torch.full((3, 256), float("nan"), dtype=torch.bfloat16, device="cuda")
    x[1, :128] = 1.0
    x8, xs = torch.zeros(3, 256, dtype=torch.uint8, device="cuda"), torch.zeros(2, 3, device="cuda")
    B.quantize_rows_fp8(B.make_linear(x, x8, xs), x, x8, xs)
    assert ((x8 & 127) == 127).sum() == 5 * 128 and (x8[1, :128] == 126).all()
    assert xs.tolist() == [[1.0, pytest.approx(1 / 448), 1.0], [1.0, 1.0, 1.0]]
