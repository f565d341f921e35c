"""Host side of the linear, rotary and cache calls: arguments that are refused before any launch, empty calls, the frequency ladder."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import layer as L
from paper_2606_23743_b200 import binding as B
from paper_2606_23743_b200 import build as build_mod

OK, INVALID, UNSUPPORTED, ALIGNMENT = 0, 1, 2, 5
ONE = C.c_void_p(256)                                     # non-null, aligned, never dereferenced: validation fails first


@pytest.fixture(scope="module")
def lib():
    build_mod.build()
    return B.lib()


def _linear(**kw):
    p = B.Linear(M=64, N=256, K=512, act=0, x_stride=512, w_stride=512, out_stride=256, residual_stride=256, x8_stride=512, w8_stride=512,
                 x_scale_stride=64, w_scale_stride=4)
    for k, v in kw.items():
        setattr(p, k, v)
    return p


def test_linear_refuses(lib):
    def call(p, x8=ONE, xs=ONE, w8=ONE, ws=ONE, out=ONE, bias=None, residual=None):
        return lib.sva_linear_fp8(C.byref(p), x8, xs, w8, ws, out, bias, residual, None, None)
    assert call(_linear(M=0)) == OK                       # nothing to do
    assert call(_linear(M=-1)) == call(_linear(N=0)) == call(_linear(K=0)) == INVALID
    assert call(_linear(act=3)) == call(_linear(act=-1)) == INVALID
    assert call(_linear(M=2 ** 31 - 1)) == UNSUPPORTED
    for name in ("x8", "xs", "w8", "ws", "out"):
        assert call(_linear(), **{name: None}) == INVALID
        assert call(_linear(), **{name: C.c_void_p(257)}) == ALIGNMENT
    assert call(_linear(x8_stride=511)) == call(_linear(w8_stride=496)) == call(_linear(out_stride=255)) == INVALID
    assert call(_linear(x_scale_stride=63)) == call(_linear(w_scale_stride=3)) == INVALID
    assert call(_linear(x8_stride=520)) == call(_linear(w8_stride=520)) == call(_linear(out_stride=257)) == ALIGNMENT
    assert call(_linear(residual_stride=8), residual=ONE) == INVALID
    assert call(_linear(residual_stride=260), residual=ONE) == ALIGNMENT
    assert call(_linear(), bias=C.c_void_p(258)) == ALIGNMENT
    assert lib.sva_linear_fp8(None, ONE, ONE, ONE, ONE, ONE, None, None, None, None) == INVALID


def test_linear_quantisers_refuse(lib):
    rows = lambda p, x=ONE, x8=ONE, s=ONE: lib.sva_quantize_rows_fp8(C.byref(p), x, x8, s, None)      # noqa: E731
    tiles = lambda p, w=ONE, w8=ONE, s=ONE: lib.sva_quantize_tiles_fp8(C.byref(p), w, w8, s, None)    # noqa: E731
    assert rows(_linear(M=0)) == OK
    assert rows(_linear(M=-1)) == rows(_linear(K=0)) == tiles(_linear(N=0)) == INVALID
    for call in (rows, tiles):
        assert call(_linear(), None) == call(_linear(), ONE, None) == call(_linear(), ONE, ONE, None) == INVALID
        assert call(_linear(), C.c_void_p(264)) == call(_linear(), ONE, C.c_void_p(264)) == call(_linear(), ONE, ONE, C.c_void_p(258)) == ALIGNMENT
    assert rows(_linear(x_stride=504)) == rows(_linear(x8_stride=500)) == rows(_linear(x_scale_stride=3)) == INVALID
    assert tiles(_linear(w_stride=504)) == tiles(_linear(w8_stride=500)) == tiles(_linear(w_scale_stride=3)) == INVALID
    assert rows(_linear(x_stride=516)) == tiles(_linear(w_stride=516)) == ALIGNMENT


def _rope(**kw):
    st = (C.c_int64 * 3)(4 * 100 * 128, 100 * 128, 128)
    p = B.Rope(B=2, Hq=4, Hk=2, N=100, d=128, rotary_dim=64, layout=0, axis_pairs=(C.c_int32 * 3)(32, 0, 0), inverse=0, factor=1.0, q_stride=st,
               k_stride=st, q_out_stride=st, k_out_stride=st, pos_stride=(C.c_int64 * 2)(100, 0))
    for k, v in kw.items():
        setattr(p, k, v)
    return p


def test_rope_refuses(lib):
    def call(p, q=ONE, k=ONE, steps=ONE, pos=ONE, qo=ONE, ko=ONE):
        return lib.sva_rope(C.byref(p), q, k, steps, pos, qo, ko, None)
    three = C.c_int32 * 3
    assert call(_rope(N=0)) == OK
    for kw in (dict(B=0), dict(Hq=0), dict(Hk=0), dict(N=-1), dict(d=0), dict(rotary_dim=0), dict(rotary_dim=63), dict(rotary_dim=130), dict(layout=2),
               dict(axis_pairs=three(31, 0, 0)), dict(axis_pairs=three(33, -1, 0)), dict(axis_pairs=three(32, 1, 0)),
               dict(pos_stride=(C.c_int64 * 2)(-1, 0))):
        assert call(_rope(**kw)) == INVALID, kw
    assert call(_rope(d=132)) == call(_rope(d=264)) == UNSUPPORTED
    for name in ("q", "qo", "steps", "pos"):
        assert call(_rope(), **{name: None}) == INVALID
        assert call(_rope(), **{name: C.c_void_p(258)}) == ALIGNMENT
    assert call(_rope(), k=None) == call(_rope(), ko=None) == INVALID
    bad = (C.c_int64 * 3)(4 * 100 * 128, 100 * 128, 132)
    for f in ("q_stride", "k_stride", "q_out_stride", "k_out_stride"):
        assert call(_rope(**{f: bad})) == ALIGNMENT


def test_rope_steps(lib):
    for pairs, kw in (([64], {}), ([22, 21, 21], dict(base=256.0)), ([32], dict(scaling="linear", factor=3.0)), ([32], dict(scaling="ntk", factor=8.0)),
                      ([1], dict(scaling="ntk", factor=8.0)), ([64], dict(scaling="parts", factor=16.0, trained_length=4096, base=500000.0))):
        steps, factor = B.rope_steps(2 * sum(pairs), pairs, **kw)
        # fractions of a turn against the oracle's radians: a 53-bit quotient's error, and half a unit
        got = steps.numpy().astype(np.uint64).astype(np.float64) / 2.0 ** 64 * 2 * np.pi
        np.testing.assert_allclose(got, L.frequencies(pairs, **kw), rtol=1e-14, atol=2.0 ** -62)
        assert factor == (pytest.approx(0.1 * np.log(16.0) + 1.0) if kw.get("scaling") == "parts" else 1.0)
    for kw in (dict(base=0.5), dict(base=float("inf")), dict(factor=0.5), dict(scaling="parts", beta_fast=1.0), dict(axis_pairs=[16])):
        with pytest.raises(B.SvaError) as e:
            B.rope_steps(64, **{"axis_pairs": [32], **kw})
        assert e.value.status == INVALID
    with pytest.raises(B.SvaError):
        B.rope_steps(63, [31])


def _cache(**kw):
    c = B.KvCache(H=4, d=128, page=16, pages=10, format=0, k_codes=256, v_codes=256, k_scale=256, v_scale=256, k_sf=256, v_sf=256)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def test_cache_refuses(lib):
    st = (C.c_int64 * 3)(4 * 50 * 128, 50 * 128, 128)
    bad = (C.c_int64 * 3)(4 * 50 * 128, 50 * 128, 132)

    def write(c, k=ONE, v=ONE, ks=st, vs=st, Bq=2, T=50, slots=ONE):
        return lib.sva_kv_cache_write(C.byref(c), k, v, ks, vs, Bq, T, slots, None, None)

    def read(c, k=ONE, v=ONE, ks=st, vs=st, Bq=2, T=50, table=ONE, lengths=ONE, stride=4, most=4):
        return lib.sva_kv_cache_read(C.byref(c), table, stride, most, lengths, Bq, T, k, v, ks, vs, None, None)
    for call in (write, read):
        assert call(_cache(), T=0) == OK
        for kw in (dict(H=0), dict(d=0), dict(page=0), dict(pages=0), dict(format=2), dict(k_codes=None), dict(v_scale=None),
                   dict(format=1, v_sf=None)):
            assert call(_cache(**kw)) == INVALID, kw
        assert call(_cache(d=96)) == call(_cache(page=1 << 16, pages=1 << 15)) == UNSUPPORTED
        assert call(_cache(k_codes=264)) == call(_cache(v_scale=258)) == ALIGNMENT
        assert call(_cache(), Bq=0) == call(_cache(), T=-1) == call(_cache(), k=None) == call(_cache(), v=None) == INVALID
        assert call(_cache(), k=C.c_void_p(264)) == call(_cache(), ks=bad) == call(_cache(), vs=bad) == ALIGNMENT
    assert write(_cache(), slots=None) == read(_cache(), table=None) == read(_cache(), lengths=None) == INVALID
    assert read(_cache(), most=0) == read(_cache(), stride=3) == INVALID
    assert write(_cache(), slots=C.c_void_p(258)) == read(_cache(), table=C.c_void_p(258)) == ALIGNMENT


def test_the_binding_refuses_tensors_that_do_not_match(lib):
    x, w8 = torch.zeros(4, 64, dtype=torch.bfloat16), torch.zeros(8, 64, dtype=torch.uint8)
    B.make_linear(x, w8=w8)
    with pytest.raises(AssertionError):
        B.make_linear(x, w8=w8[:, :32])                   # codes shorter than the inputs
    with pytest.raises(AssertionError):
        B.make_linear(x, w8=w8, out=torch.zeros(4, 9, dtype=torch.bfloat16))
    with pytest.raises(AssertionError):
        B.make_linear(x, w8=w8, x_scale=torch.zeros(1, 3))
    q = torch.zeros(2, 4, 6, 64, dtype=torch.bfloat16)
    with pytest.raises(AssertionError):
        B.make_rope(q, None, q, None, torch.zeros(1, 2, 5, dtype=torch.int32), 64)
    codes, scale = torch.zeros(3, 4, 16, 64, dtype=torch.uint8), torch.zeros(3, 4, 16)
    c = B.make_kv_cache([codes, scale], [codes, scale])
    assert (c.pages, c.H, c.page, c.d) == (3, 4, 16, 64)
    with pytest.raises(AssertionError):
        B.make_kv_cache([codes, scale[:2]], [codes, scale])
    with pytest.raises(AssertionError):
        B.kv_cache_write(c, q, q, torch.zeros(2, 5, dtype=torch.int32))


def test_more_heads_than_can_be_shared_out_are_refused(lib):
    st = (C.c_int64 * 3)(0, 0, 128)
    for n in (2 ** 24 + 1, 2 ** 31 - 1):
        for p in (_rope(Hq=n), _rope(Hk=n)):
            assert lib.sva_rope(C.byref(p), ONE, ONE, ONE, ONE, ONE, ONE, None) == UNSUPPORTED
        assert lib.sva_kv_cache_write(C.byref(_cache(H=n)), ONE, ONE, st, st, 1, 1, ONE, None, None) == UNSUPPORTED
        assert lib.sva_kv_cache_read(C.byref(_cache(H=n)), ONE, 1, 1, ONE, 1, 1, ONE, ONE, st, st, None, None) == UNSUPPORTED


def test_codes_that_end_within_a_piece_are_refused(lib):
    """The quantisers write whole pieces of 16 bytes: a row of codes has room for them, also where it is the only one or the last."""
    x = torch.zeros(3, 100, dtype=torch.bfloat16)
    s = torch.zeros(1, 3)
    padded, big = torch.zeros(3, 112, dtype=torch.uint8), torch.zeros(1000, dtype=torch.uint8)
    B.make_linear(x, x8=padded, x_scale=s)
    assert B.make_linear(x, x8=padded[:, :100], x_scale=s).x8_stride == 112          # (what is behind a row is its own)
    assert B.make_linear(x[:1], x8=padded[:1, :100], x_scale=s[:, :1]).x8_stride == 112
    for codes in (torch.zeros(1, 100, dtype=torch.uint8), big[:100][None], big[16:116].expand(1, 100)):
        with pytest.raises(AssertionError):
            B.make_linear(x[:1], x8=codes, x_scale=s[:, :1])
        with pytest.raises(AssertionError):
            B.make_linear(w=x[:1], w8=codes, w_scale=s[:, :1])
        B.make_linear(x8=codes, x_scale=s[:, :1], w8=codes, K=100)                   # (read only)
    with pytest.raises(AssertionError):
        B.make_linear(x, x8=torch.zeros(324, dtype=torch.uint8).as_strided((3, 100), (112, 1)), x_scale=s)


def test_token_indices_that_do_not_match_are_refused(lib):
    """Indices are read as B x M int32 side by side: a shared row that is spread over the batch, or 64 bits, would be read past its end."""
    x, part = torch.zeros(2, 3, 50, 16, dtype=torch.bfloat16), torch.zeros(2, 3, 9, 16, dtype=torch.bfloat16)
    idx = torch.zeros(2, 9, dtype=torch.int32)
    bad = [(idx.long(), part), (idx[:1].expand(2, 9), part), (idx[:1], part), (torch.zeros(2, 18, dtype=torch.int32)[:, ::2], part), (idx[0], part),
           (idx, part[:, :, :8]), (idx, part[:1]), (idx, part[:, :2]), (idx, part[..., :8]), (idx, part.float())]
    for i, p in bad:
        with pytest.raises(AssertionError):
            B.gather_tokens(x, i, p)
        with pytest.raises(AssertionError):
            B.scatter_tokens(p, i, x)


def _refused(call, *args):
    with pytest.raises(AssertionError):
        call(*args)


def test_calls_refuse_tensors_that_are_not_their_plans(lib):
    """Sizes below the plan's, and memory that is not the GPU's, end before the C call (which here, without a device, would answer with
    an error of its own)."""
    bf, u8 = torch.bfloat16, torch.uint8
    x, x8, xs, w, w8, ws = (torch.zeros(4, 64, dtype=bf), torch.zeros(4, 64, dtype=u8), torch.zeros(1, 4), torch.zeros(8, 64, dtype=bf),
                            torch.zeros(8, 64, dtype=u8), torch.zeros(1, 1))
    out, r, bias = torch.zeros(4, 8, dtype=bf), torch.zeros(4, 8, dtype=bf), torch.zeros(8)
    p = B.make_linear(x, x8, xs, w8, ws, out, residual=r, w=w)
    _refused(B.quantize_rows_fp8, p, x, x8, xs)                                      # not on the GPU
    _refused(B.quantize_tiles_fp8, p, w, w8, ws)
    _refused(B.linear_fp8, p, x8, xs, w8, ws, out, bias, r)
    x, x8, xs, w, w8, ws, out, r = (_OnGpu(t) for t in (x, x8, xs, w, w8, ws, out, r))
    p = B.make_linear(x, x8, xs, w8, ws, out, residual=r, w=w)
    for call, args in ((B.quantize_rows_fp8, (x, x8, xs)), (B.quantize_tiles_fp8, (w, w8, ws)), (B.linear_fp8, (x8, xs, w8, ws, out, _OnGpu(bias), r))):
        for i, t in enumerate(args):
            for other in (t.t[..., :-1], t.t[:0]):
                _refused(call, p, *args[:i], _OnGpu(other), *args[i + 1:])
    _refused(B.linear_fp8, p, x8, xs, w8, ws, out, bias, r)
    _refused(B.linear_fp8, p, x8, xs, w8, ws, out, None, r, torch.zeros(1, dtype=torch.int32))
    q, pos = torch.zeros(2, 4, 6, 64, dtype=bf), torch.zeros(1, 2, 6, dtype=torch.int32)
    steps, _ = B.rope_steps(64)                                                      # (on the CPU unless a device is named)
    _refused(B.rope, B.make_rope(q, q, q, q, pos, 64), q, q, _OnGpu(steps), pos, q, q)
    q, pos = _OnGpu(q), _OnGpu(pos)
    p = B.make_rope(q, q, q, q, pos, 64)
    _refused(B.rope, p, q, q, steps, pos, q, q)
    args = (q, q, _OnGpu(steps), pos, q, q)
    for i, t in enumerate(args):
        for other in (t.t[..., :-1], t.t[:0]):
            _refused(B.rope, p, *args[:i], _OnGpu(other), *args[i + 1:])
    codes, scale, q = torch.zeros(3, 4, 16, 64, dtype=u8), torch.zeros(3, 4, 16), q.t
    c = B.make_kv_cache([codes, scale], [codes, scale])
    slots, table, lengths = torch.zeros(2, 6, dtype=torch.int32), torch.zeros(2, 1, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    _refused(B.kv_cache_write, c, q, q, slots)
    _refused(B.kv_cache_read, c, table, lengths, q, q)


class _OnGpu:
    """A tensor that says it is on the GPU."""

    def __init__(self, t):
        self.t, self.is_cuda = t, True

    def __getattr__(self, name):
        return getattr(self.t, name)


@pytest.mark.parametrize("kw", [dict(trained_length=float("inf"), beta_fast=float("inf")), dict(beta_fast=float("nan")), dict(beta_slow=float("nan")),
                                dict(trained_length=float("nan"))])
def test_rope_steps_refuse_what_gives_no_number(lib, kw):
    with pytest.raises(B.SvaError) as e:
        B.rope_steps(64, [32], **{"scaling": "parts", "factor": 4.0, "trained_length": 4096.0, **kw})
    assert e.value.status == INVALID


def test_rope_steps_at_the_limits_of_the_rule_by_parts(lib):
    """Endlessly long training: every pair stays; an endless fast end: every pair is slowed down."""
    plain, linear = (B.rope_steps(64, [32], scaling=s, factor=4.0)[0] for s in ("none", "linear"))
    for kw, want in ((dict(trained_length=float("inf")), plain), (dict(trained_length=4096.0, beta_fast=float("inf")), linear)):
        assert torch.equal(B.rope_steps(64, [32], scaling="parts", factor=4.0, **kw)[0], want)


def test_calls_refuse_other_strides_than_those_of_a_plan_with_gaps(lib):
    """A plan of views that leave something out between their rows reaches further than their bytes."""
    bf, u8 = torch.bfloat16, torch.uint8
    x, x8, xs = _OnGpu(torch.zeros(4, 96, dtype=bf)[:, :64]), _OnGpu(torch.zeros(4, 80, dtype=u8)[:, :64]), _OnGpu(torch.zeros(1, 9)[:, :4])
    w8, ws, out = _OnGpu(torch.zeros(8, 80, dtype=u8)[:, :64]), _OnGpu(torch.zeros(1, 1)), _OnGpu(torch.zeros(4, 16, dtype=bf)[:, :8])
    r, w = _OnGpu(torch.zeros(4, 24, dtype=bf)[:, :8]), _OnGpu(torch.zeros(8, 72, dtype=bf)[:, :64])
    p = B.make_linear(x, x8, xs, w8, ws, out, residual=r, w=w)
    assert set(p.gaps) == {"x", "x8", "w8", "out", "residual", "w"}                  # (one row of scales has no gap)
    for call, args, of in ((B.quantize_rows_fp8, (x, x8, xs), (0, 1)), (B.quantize_tiles_fp8, (w, w8, ws), (0, 1)),
                           (B.linear_fp8, (x8, xs, w8, ws, out, None, r), (0, 2, 4, 6))):
        for i in of:
            _refused(call, p, *args[:i], _OnGpu(args[i].t.contiguous()), *args[i + 1:])
    qkv, pos, steps = torch.zeros(2, 6, 3, 4, 64, dtype=bf), _OnGpu(torch.zeros(1, 2, 6, dtype=torch.int32)), _OnGpu(B.rope_steps(64)[0])
    q, k, o = _OnGpu(qkv[:, :, 0].transpose(1, 2)), _OnGpu(qkv[:, :, 1].transpose(1, 2)), _OnGpu(torch.zeros(2, 6, 4, 64, dtype=bf).transpose(1, 2))
    p = B.make_rope(q, k, o, o, pos, 64)
    assert set(p.gaps) == {"q", "k"}                                                 # (a transposed whole has none)
    _refused(B.rope, p, _OnGpu(q.t.contiguous()), k, steps, pos, o, o)
    _refused(B.rope, p, q, _OnGpu(k.t.contiguous()), steps, pos, o, o)
