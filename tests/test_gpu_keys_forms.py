"""Forms of attention over keys of their own beside those that most calls take: a split key axis of the many-row kernel where rows see unequal parts of it or
splits hold nothing, and the few-row kernels over many rows.  Tolerances as in test_gpu_keys."""
import numpy as np
import pytest
import torch

from oracle import keys as K
from paper_2606_23743_b200 import binding as B
from test_gpu_keys import Cached, _cross, _cross_check, _heads, _i32

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("Hq,H,M,d,page,keys,counts,causal", [
    (2, 1, 64, 64, 64, [6000, 300, 0, 64], None, True),
    (2, 1, 64, 128, 16, [5999, 1, 129], [64, 64, 3], True),        # (the second: 63 queries come before its only token)
    (4, 1, 33, 128, 48, [40, 7000], [33, 0], False),
    (3, 1, 200, 64, 32, [2500, 201], [200, 130], True),
    (1, 1, 600, 128, 64, [3000], None, True),                      # (rows of an item whose own splits are empty)
])
def test_many_rows_over_a_split_axis(Hq, H, M, d, page, keys, counts, causal):
    rng = np.random.default_rng(M + d + sum(keys))
    x = Cached(rng, len(keys), Hq, H, M, d, page, keys, True)
    _, p, _, ws = x.run(causal, counts)
    assert B.debug_last_choice() == 128 and B.cached_attn_workspace_bytes(p) > 0
    x.check(causal, counts)


@pytest.mark.parametrize("Hq,Hk,N,S,d,lengths,part", [(2, 1, 64, 6000, 64, [6000, 10, 0], None), (1, 1, 150, 4000, 128, [4000, 513], 0.2), (4, 2, 40, 3000, 64, None, 0.01)])
def test_many_rows_over_a_split_axis_of_given_keys(Hq, Hk, N, S, d, lengths, part):
    rng = np.random.default_rng(N + S)
    Bq = len(lengths) if lengths else 2
    q, k, v = _heads(rng, (Bq, Hq, N, d), True), _heads(rng, (Bq, Hk, S, d), False), _heads(rng, (Bq, Hk, S, d), False)
    there = np.ones((Bq, S), bool) if lengths is None else np.arange(S)[None] < np.array(lengths)[:, None]
    mask = None
    if part is not None:
        on = rng.random((Bq, S)) < part
        mask, there = torch.from_numpy(on).cuda(), there & on
    assert B.cross_attn_workspace_bytes(B.make_cross_attn(q, k, v, q)) > 0
    o, lse = _cross(q, k, v, None if lengths is None else _i32(lengths), mask)
    assert B.debug_last_choice() == 128
    _cross_check(q, k, v, there, o, lse)


@pytest.mark.parametrize("Hq,H,M,d,keys,causal", [(160, 1, 5, 64, [70, 33], True), (260, 2, 3, 128, [300], False), (129, 1, 2, 64, [2000], True)])
def test_more_heads_than_a_tile_has_rows(Hq, H, M, d, keys, causal):
    rng = np.random.default_rng(Hq)
    x = Cached(rng, len(keys), Hq, H, M, d, 16, keys, True)
    x.run(causal, None)
    assert B.debug_last_choice() == 8
    x.check(causal, None)


@pytest.mark.parametrize("what", ["q", "heads", "keys", "group"])
@pytest.mark.parametrize("d,S", [(64, 300), (128, 2100)])
def test_given_keys_that_no_tensor_map_describes(what, d, S):
    """Strides of 0 along Q's tokens or heads, along the keys' tokens; more than 128 query heads per key head: the few-row kernel, over many rows."""
    rng = np.random.default_rng(S)
    Hq, N = (130, 3) if what == "group" else (3, 100)
    q, k, v = _heads(rng, (2, Hq, N, d), True), _heads(rng, (2, 1, S, d), True), _heads(rng, (2, 1, S, d), True)
    q2, k2 = q, k
    if what == "q":
        q2 = q[:, :, :1].expand(2, Hq, N, d)
    elif what == "heads":
        q2 = q[:, :1].expand(2, Hq, N, d)
    elif what == "keys":
        k2 = k[:, :, :1].expand(2, 1, S, d)
    o, lse = torch.full_like(q, 7.0), torch.full(q.shape[:3], 7.0, device="cuda")
    p = B.make_cross_attn(q2, k2, v, o)
    ws = torch.full((max(256, B.cross_attn_workspace_bytes(p)),), 0xff, dtype=torch.uint8, device="cuda")
    B.cross_attn_fwd(p, q2, k2, v, o, _i32([S, S - 5]), None, lse, None, ws)
    assert B.debug_last_choice() == 16
    _cross_check(q2, k2, v, np.arange(S)[None] < np.array([[S], [S - 5]]), o, lse)


@pytest.mark.parametrize("d,S", [(64, 77), (128, 512), (128, 3000)])
def test_probabilities_of_few_rows_over_given_keys(d, S):
    """They count with 16 bits: what is left of an output's error is its own rounding, 2^-8 of it, and 2^-16 of the weights' mean magnitude of v (with the
    logits' errors as in test_gpu_keys)."""
    rng = np.random.default_rng(S)
    q, k, v = _heads(rng, (2, 4, 4, d), True, 0.5), _heads(rng, (2, 2, S, d), True), _heads(rng, (2, 2, S, d), True)
    o, lse = _cross(q, k, v, None, None)
    assert B.debug_last_choice() == 16
    q, k, v, o = (t.float().cpu().numpy().astype(np.float64) for t in (q, k, v, o))
    for b in range(2):
        for h in range(4):
            want, _, size, top = K.attention(q[b, h], k[b, h // 2], v[b, h // 2], np.ones(S, bool), d ** -0.5)
            e = (d + 8) * 2.0 ** -23 * top + 2.0 ** -20
            assert (np.abs(o[b, h] - want) <= 2.0 ** -8 * np.abs(want) + (2.0 ** -16 + 2 * e) * size).all()
