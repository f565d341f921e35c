"""What the calls for keys of their own refuse, on the host: nothing is launched."""
import ctypes as C

import pytest
import torch

from paper_2606_23743_b200 import binding as B

OK, INVALID, UNSUPPORTED, WORKSPACE, ALIGNMENT = 0, 1, 2, 3, 5
ONE, OFF = C.c_void_p(256), C.c_void_p(258)


@pytest.fixture(scope="module")
def lib():
    return B.lib()


def _cache(**kw):
    c = B.KvCache(H=4, d=128, page=16, pages=10, format=8, k_codes=256, v_codes=256, k_scale=256, v_scale=256)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


BAD_CACHES = [(dict(H=0), INVALID), (dict(d=0), INVALID), (dict(page=0), INVALID), (dict(pages=0), INVALID), (dict(format=2), INVALID), (dict(format=9), INVALID),
              (dict(k_codes=None), INVALID), (dict(v_scale=None), INVALID), (dict(d=96), UNSUPPORTED), (dict(page=1 << 16, pages=1 << 15), UNSUPPORTED),
              (dict(page=24), UNSUPPORTED), (dict(H=2 ** 24 + 1), UNSUPPORTED), (dict(k_codes=264), ALIGNMENT), (dict(v_scale=258), ALIGNMENT)]
ST, BAD = (C.c_int64 * 3)(4 * 50 * 128, 50 * 128, 128), (C.c_int64 * 3)(4 * 50 * 128, 50 * 128, 132)


def test_append_refuses(lib):
    def call(c, k=ONE, v=ONE, ks=ST, vs=ST, Bq=2, T=50, table=ONE, stride=4, most=4, lengths=ONE, counts=None):
        return lib.sva_kv_cache_append(C.byref(c), k, v, ks, vs, Bq, T, table, stride, most, lengths, counts, None, None)
    assert call(_cache(), T=0) == OK
    for kw, rc in BAD_CACHES:
        assert call(_cache(**kw)) == rc, kw
    for form in (0, 1):
        assert call(_cache(format=form, k_sf=256, v_sf=256)) == UNSUPPORTED
    assert call(_cache(), Bq=0) == call(_cache(), T=-1) == call(_cache(), k=None) == call(_cache(), v=None) == INVALID
    assert call(_cache(), table=None) == call(_cache(), lengths=None) == call(_cache(), most=0) == call(_cache(), stride=3) == INVALID
    assert call(_cache(), k=OFF) == call(_cache(), ks=BAD) == call(_cache(), vs=BAD) == call(_cache(), counts=OFF) == call(_cache(), table=OFF) == ALIGNMENT
    # the call that knows single tokens only
    assert lib.sva_kv_cache_write(C.byref(_cache()), ONE, ONE, ST, ST, 2, 50, ONE, None, None) == UNSUPPORTED


def _plan(**kw):
    p = B.CachedAttn(B=2, Hq=8, M=50, max_pages=4, causal=0, softmax_scale=0.0, table_stride=4, q_stride=ST, o_stride=ST)
    for k, v in kw.items():
        setattr(p, k, v)
    return p


def test_cached_attn_refuses(lib):
    def call(c=None, q=ONE, table=ONE, lengths=ONE, counts=None, o=ONE, lse=None, ws=None, n=0, **kw):
        return lib.sva_cached_attn_fwd(C.byref(c or _cache()), C.byref(_plan(**kw)), q, table, lengths, counts, o, lse, None, ws, n, None)
    assert call(M=0) == OK
    for kw, rc in BAD_CACHES:
        assert call(_cache(**kw)) == rc, kw
        assert lib.sva_cached_attn_workspace_bytes(C.byref(_cache(**kw)), C.byref(_plan())) == 0
    assert call(_cache(format=0)) == UNSUPPORTED
    for kw in (dict(B=0), dict(Hq=0), dict(Hq=6), dict(M=-1), dict(max_pages=0), dict(causal=2), dict(causal=-1), dict(table_stride=3)):
        assert call(**kw) == INVALID, kw
    for kw in (dict(M=2 ** 30, Hq=16), dict(max_pages=2 ** 27), dict(Hq=2 ** 24 + 4)):
        assert call(**kw) == UNSUPPORTED, kw
    assert call(q=None) == call(o=None) == call(table=None) == call(lengths=None) == INVALID
    assert call(q=OFF) == call(o=OFF) == call(table=OFF) == call(lengths=OFF) == call(counts=OFF) == call(lse=OFF) == call(q_stride=BAD) == \
        call(o_stride=BAD) == ALIGNMENT
    # few rows over a long axis are cut into splits, which need a workspace
    long = dict(M=1, max_pages=2000, table_stride=2000)
    need = lib.sva_cached_attn_workspace_bytes(C.byref(_cache(pages=2000)), C.byref(_plan(**long)))
    assert need > 0
    assert call(_cache(pages=2000), **long) == call(_cache(pages=2000), ws=ONE, n=need - 1, **long) == WORKSPACE
    assert call(_cache(pages=2000), ws=C.c_void_p(264), n=need, **long) == ALIGNMENT


def _cross(**kw):
    p = B.CrossAttn(B=2, Hq=8, Hk=4, N=50, S=50, d=128, q_stride=ST, k_stride=ST, v_stride=ST, o_stride=ST)
    for k, v in kw.items():
        setattr(p, k, v)
    return p


def test_cross_attn_refuses(lib):
    def call(q=ONE, k=ONE, v=ONE, lengths=None, mask=None, o=ONE, lse=None, ws=None, n=0, **kw):
        return lib.sva_cross_attn_fwd(C.byref(_cross(**kw)), q, k, v, lengths, mask, o, lse, None, ws, n, None)
    assert call(N=0) == OK
    for kw in (dict(B=0), dict(Hq=0), dict(Hk=0), dict(Hq=6), dict(N=-1), dict(S=-1)):
        assert call(**kw) == INVALID, kw
        assert lib.sva_cross_attn_workspace_bytes(C.byref(_cross(**kw))) == 0
    for kw in (dict(d=96), dict(d=256), dict(N=2 ** 31 - 1), dict(S=2 ** 31 - 1), dict(Hq=2 ** 25, Hk=2 ** 25)):
        assert call(**kw) == UNSUPPORTED, kw
    assert call(q=None) == call(k=None) == call(v=None) == call(o=None) == call(mask=ONE, mask_stride=-1) == INVALID
    assert call(q=OFF) == call(k=OFF) == call(v=OFF) == call(o=OFF) == call(lengths=OFF) == call(lse=OFF) == ALIGNMENT
    for name in ("q_stride", "k_stride", "v_stride", "o_stride"):
        assert call(**{name: BAD}) == ALIGNMENT
        assert call(**{name: (C.c_int64 * 3)(-8, 8, 128)}) == INVALID
    long = dict(N=1, S=40000)
    need = lib.sva_cross_attn_workspace_bytes(C.byref(_cross(**long)))
    assert need > 0 and call(**long) == call(ws=ONE, n=need - 1, **long) == WORKSPACE


def test_pages_refuse(lib):
    def take(c, refs=ONE, table=ONE, stride=4, rows=3, most=4, lengths=ONE, counts=ONE):
        return lib.sva_kv_pages_take(C.byref(c), refs, table, stride, rows, most, lengths, counts, None, None)

    def fork(c, refs=ONE, table=ONE, stride=4, rows=3, most=4, lengths=ONE, a=ONE, b=ONE, n=2):
        return lib.sva_kv_pages_fork(C.byref(c), refs, table, stride, rows, most, lengths, a, b, n, None, None)

    def free(c, refs=ONE, table=ONE, stride=4, rows=3, most=4, lengths=ONE, a=ONE, b=None, n=2):
        return lib.sva_kv_pages_free(C.byref(c), refs, table, stride, rows, most, lengths, a, b, n, None, None)

    def compact(c, refs=ONE, table=ONE, stride=4, rows=3, most=4, live=None, ws=ONE, n=1 << 20):
        return lib.sva_kv_pages_compact(C.byref(c), refs, table, stride, rows, most, live, None, ws, n, None)

    def copy(c, src=ONE, dst=ONE, n=2):
        return lib.sva_kv_pages_copy(C.byref(c), src, dst, n, None, None)
    for call in (take, fork, free, compact, copy):
        for kw, rc in BAD_CACHES:
            assert call(_cache(**kw)) == rc, kw
        assert call(_cache(format=1)) == INVALID and call(_cache(format=1, k_sf=258, v_sf=256)) == ALIGNMENT
    for call in (take, fork, free, compact):
        assert call(_cache(), refs=None) == call(_cache(), table=None) == call(_cache(), most=0) == call(_cache(), stride=3) == call(_cache(), rows=-1) == INVALID
        assert call(_cache(), refs=OFF) == call(_cache(), table=OFF) == ALIGNMENT
        assert call(_cache(), most=2 ** 20 + 1, stride=2 ** 21) == UNSUPPORTED
    assert take(_cache(), rows=0) == fork(_cache(), n=0) == free(_cache(), n=0) == copy(_cache(), n=0) == OK
    assert take(_cache(), lengths=None) == take(_cache(), counts=None) == fork(_cache(), a=None) == fork(_cache(), b=None) == fork(_cache(), lengths=None) == \
        free(_cache(), a=None) == free(_cache(), lengths=None) == fork(_cache(), n=-1) == free(_cache(), n=-1) == copy(_cache(), n=-1) == \
        copy(_cache(), src=None) == copy(_cache(), dst=None) == INVALID
    assert take(_cache(), counts=OFF) == fork(_cache(), a=OFF) == free(_cache(), b=OFF) == copy(_cache(), src=OFF) == compact(_cache(), live=OFF) == \
        compact(_cache(), ws=C.c_void_p(264)) == ALIGNMENT
    need = lib.sva_kv_pages_compact_workspace_bytes(C.byref(_cache()))
    assert need > 0 and compact(_cache(), n=need - 1) == compact(_cache(), ws=None) == WORKSPACE


def _refused(call, *args, **kw):
    with pytest.raises(AssertionError):
        call(*args, **kw)


def test_the_binding_refuses_tensors_that_do_not_match(lib):
    codes, scale = torch.zeros(6, 4, 16, 64, dtype=torch.uint8), torch.zeros(6, 4)
    c = B.make_kv_cache([codes, scale], [codes, scale], "e4m3_page")
    assert (c.pages, c.H, c.page, c.d, c.format) == (6, 4, 16, 64, 8)
    _refused(B.make_kv_cache, [codes, torch.zeros(6, 4, 16)], [codes, scale], "e4m3_page")
    _refused(B.make_kv_cache, [codes, scale.double()], [codes, scale], "e4m3_page")
    x, table, n = torch.zeros(2, 4, 5, 64, dtype=torch.bfloat16), torch.zeros(2, 3, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    # (nothing here is on the GPU: the last of these is refused for that alone)
    for args in ((x[:, :3], x, table, n), (x, x[..., :32], table, n), (x.float(), x, table, n), (x, x, table.long(), n), (x, x, table[:1], n),
                 (x, x, table, n[:1]), (x, x, table, n.long()), (x, x, table, n, n.float()), (x, x, table, n)):
        _refused(B.kv_cache_append, c, *args)
    q = torch.zeros(2, 8, 5, 64, dtype=torch.bfloat16)
    p = B.make_cached_attn(c, q, q, table)
    assert (p.B, p.Hq, p.M, p.max_pages, p.table_stride) == (2, 8, 5, 3, 3)
    for args in ((q[:, :6], q[:, :6], table), (q, q[:, :, :4], table), (q.float(), q, table), (q, q, table[:1]), (q, q, table.long()),
                 (q[..., :32], q[..., :32], table)):
        _refused(B.make_cached_attn, c, *args)
    wide = torch.zeros(2, 8, 5, 72, dtype=torch.bfloat16)[..., :64]
    for args in ((q, table, n, q[:, :, :4]), (q[:1], table, n, q), (wide, table, n, q), (q, table, n, wide), (q, table[:, :2], n, q), (q, table, n, q)):
        _refused(B.cached_attn_fwd, p, *args)
    k = torch.zeros(2, 4, 7, 64, dtype=torch.bfloat16)
    p = B.make_cross_attn(q, k, k, q)
    assert (p.Hq, p.Hk, p.N, p.S, p.d) == (8, 4, 5, 7, 64)
    for args in ((q, k, k[:, :, :6], q), (q[:, :6], k, k, q[:, :6]), (q, k.float(), k, q), (q, k[..., :32], k, q), (q, k[:1], k[:1], q)):
        _refused(B.make_cross_attn, *args)
    for args in ((q, k, k[:, :, :6], q), (wide, k, k, q), (q, k, k, q)):
        _refused(B.cross_attn_fwd, p, *args)
    refs = torch.zeros(6, dtype=torch.int32)
    for args in ((refs[:5], table, n, n), (refs.long(), table, n, n), (refs, table.long(), n, n), (refs, table, n[:1], n), (refs, table, n, n)):
        _refused(B.kv_pages_take, c, *args)
        _refused(B.kv_pages_fork, c, args[0], args[1], args[2], n, n)
        _refused(B.kv_pages_free, c, args[0], args[1], args[2], n)
    _refused(B.kv_pages_copy, c, n, n[:1])
    _refused(B.kv_pages_compact, c, refs, table, torch.zeros(1000, dtype=torch.uint8))
