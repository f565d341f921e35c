"""Rotary positions against the fp64 oracle."""
import numpy as np
import pytest
import torch

from oracle import layer as L
from paper_2606_23743_b200 import binding as B

pytestmark = pytest.mark.gpu


def _f64(t):
    return t.float().cpu().numpy().astype(np.float64)


def _tensor(rng, shape, tokens_first):
    Bq, H, N, d = shape
    x = torch.from_numpy(rng.standard_normal((Bq, N, H, d) if tokens_first else shape)).to(torch.bfloat16).cuda()
    return x.transpose(1, 2) if tokens_first else x


def _pairs(R, axes):
    side = (R // 2) // axes
    return [R // 2 - side * (axes - 1)] + [side] * (axes - 1)


def _check(got, x, theta, pos, pairs, R, layout, factor=1.0, inverse=False):
    """Half a bf16 step, plus the fp32 rotation: the phase is off by 2^-32 turns and one fp32 rounding (2^-24 pi rad), sincospi by two units,
    each product and the sum by one rounding: together under 2^-20 of |a| + |b|."""
    ref = L.rope(x, theta, pos, pairs, R, layout, factor, inverse)
    size = L.rope(np.abs(x), 0 * theta, pos, pairs, R, layout)           # |a|, |b| in their own places
    half = R // 2
    both = size.copy()
    if layout == "half":
        both[..., :half] = both[..., half:R] = size[..., :half] + size[..., half:R]
    else:
        both[..., 0:R:2] = both[..., 1:R:2] = size[..., 0:R:2] + size[..., 1:R:2]
    bound = 2.0 ** -8 * np.abs(ref) + 2.0 ** -20 * factor * both + 2.0 ** -133
    bound[..., R:] = 0.0                                                 # what is not rotated passes through
    assert (np.abs(got - ref) <= bound).all(), np.max(np.abs(got - ref) - bound)


CASES = [
    # B, Hq, Hk, N, d, R, axes, layout, tokens first, start
    (1, 1, 1, 1, 64, 64, 1, "half", False, 0),
    (1, 3, 1, 1, 128, 128, 1, "interleaved", True, 7),
    (9, 32, 8, 1, 128, 128, 1, "half", True, 1 << 20),
    (2, 5, 2, 77, 128, 64, 1, "half", False, 100),
    (2, 5, 5, 77, 128, 64, 1, "interleaved", True, 100),
    (1, 24, 24, 130, 128, 128, 3, "interleaved", False, 0),
    (1, 7, 3, 333, 128, 128, 3, "half", True, 0),
    (1, 4, 4, 45, 64, 20, 1, "half", False, 5),                          # halves that are no whole vectors
    (2, 9, 2, 45, 128, 74, 1, "half", True, 5),
    (1, 4, 2, 45, 128, 74, 1, "interleaved", True, 5),                   # a vector that ends in the middle of the rotated part
    (1, 2, 2, 19, 128, 2, 1, "half", False, 3),
    (1, 2, 2, 19, 128, 2, 1, "interleaved", False, 3),
    (1, 3, 3, 50, 80, 80, 1, "half", False, 0),                          # other head sizes
    (1, 3, 3, 50, 96, 48, 3, "interleaved", True, 0),
    (1, 3, 1, 50, 256, 256, 1, "half", True, 2 ** 31 - 60),              # the last positions there are
    (1, 2, 2, 50, 8, 6, 1, "half", False, 1),
    (1, 2, 1, 40, 248, 246, 3, "half", False, 1),
]


@pytest.mark.parametrize("inverse", [False, True], ids=["forward", "inverse"])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(str(v) for v in c))
def test_rotation(case, inverse):
    Bq, Hq, Hk, N, d, R, axes, layout, first, start = case
    rng = np.random.default_rng(N + d + R)
    q, k = _tensor(rng, (Bq, Hq, N, d), first), _tensor(rng, (Bq, Hk, N, d), first)
    pairs = _pairs(R, axes)
    shared = axes == 3
    pos = np.minimum(start + (np.arange(N) if not shared else rng.integers(0, 60, (axes, 1, N))), 2 ** 31 - 1)
    pos = np.broadcast_to(pos, (axes, 1, N)) if not shared else pos
    if not shared:
        pos = np.minimum(pos + np.arange(Bq)[:, None] * (13 if start < 2 ** 30 else 0), 2 ** 31 - 1)      # sequences at places of their own
    positions = torch.from_numpy(np.ascontiguousarray(pos).astype(np.int32)).cuda()
    steps, _ = B.rope_steps(R, pairs, 10000.0, device="cuda")
    theta = L.frequencies(pairs)
    qo, ko = torch.full_like(q, 3.0), torch.full_like(k, 3.0)
    p = B.make_rope(q, k, qo, ko, positions, R, layout, pairs, 1.25, inverse)
    B.rope(p, q, k, steps, positions, qo, ko)
    torch.cuda.synchronize()
    for x, y in ((q, qo), (k, ko)):
        _check(_f64(y), _f64(x), theta, pos, pairs, R, layout, 1.25, inverse)
    # in place, and q alone
    q2 = q.clone(memory_format=torch.preserve_format)
    p = B.make_rope(q2, None, q2, None, positions, R, layout, pairs, 1.25, inverse)
    B.rope(p, q2, None, steps, positions, q2, None)
    assert torch.equal(q2, qo)


@pytest.mark.parametrize("layout,R", [("half", 64), ("half", 20), ("interleaved", 64), ("interleaved", 74)])
def test_what_is_not_rotated_keeps_its_bits(layout, R):
    """Infinities, NaN and negative zeros behind the rotated channels, and an infinity among them that stays with its pair."""
    q = torch.randn(1, 3, 10, 128, device="cuda").to(torch.bfloat16)
    q[..., R::3], q[..., R + 1::3] = float("inf"), -0.0
    q[0, 0, 0, 100], q[0, 1, 4, 0] = float("nan"), float("inf")
    positions = torch.arange(1, 11, dtype=torch.int32, device="cuda")[None, None]
    steps, _ = B.rope_steps(R, device="cuda")
    out = torch.empty_like(q)
    B.rope(B.make_rope(q, None, out, None, positions, R, layout), q, None, steps, positions, out, None)
    assert torch.equal(out[..., R:].contiguous().view(torch.int16), q[..., R:].contiguous().view(torch.int16))
    bad = ~torch.isfinite(out[..., :R])
    assert int(bad.sum()) == 2 and bad[0, 1, 4, 0] and bad[0, 1, 4, R // 2 if layout == "half" else 1]


def test_negative_positions():
    rng = np.random.default_rng(1)
    q = _tensor(rng, (1, 2, 9, 64), False)
    pos = np.arange(-5, 4)[None, None]
    positions = torch.from_numpy(pos.astype(np.int32)).cuda()
    steps, _ = B.rope_steps(64, device="cuda")
    out = torch.empty_like(q)
    B.rope(B.make_rope(q, None, out, None, positions, 64), q, None, steps, positions, out, None)
    _check(_f64(out), _f64(q), L.frequencies([32]), pos, [32], 64, "interleaved")


@pytest.mark.parametrize("scaling", ["linear", "ntk", "parts"])
def test_long_contexts(scaling):
    """A million positions, frequencies scaled."""
    rng = np.random.default_rng(2)
    kw = dict(base=10000.0, scaling=scaling, factor=8.0, trained_length=4096)
    q = _tensor(rng, (1, 2, 64, 128), False)
    pos = (1_000_000 + 977 * np.arange(64))[None, None]
    positions = torch.from_numpy(pos.astype(np.int32)).cuda()
    steps, factor = B.rope_steps(128, [64], device="cuda", **kw)
    out = torch.empty_like(q)
    B.rope(B.make_rope(q, None, out, None, positions, 128, "half", factor=factor), q, None, steps, positions, out, None)
    want = 0.1 * np.log(8.0) + 1.0 if scaling == "parts" else 1.0
    _check(_f64(out), _f64(q), L.frequencies([64], **kw), pos, [64], 128, "half", want)


def test_packed_projection_in_place():
    """Q and K where a projection of [tokens, 3 H d] left them; V is not touched."""
    rng = np.random.default_rng(3)
    N, H, d = 200, 6, 128
    qkv = torch.from_numpy(rng.standard_normal((1, N, 3, H, d))).to(torch.bfloat16).cuda()
    before = qkv.clone()
    q, k = qkv[:, :, 0].transpose(1, 2), qkv[:, :, 1].transpose(1, 2)
    pos = np.arange(N)[None, None]
    positions = torch.from_numpy(pos.astype(np.int32)).cuda()
    steps, _ = B.rope_steps(128, device="cuda")
    B.rope(B.make_rope(q, k, q, k, positions, 128, "half"), q, k, steps, positions, q, k)
    theta = L.frequencies([64])
    for i, x in enumerate((q, k)):
        _check(_f64(x), _f64(before[:, :, i].transpose(1, 2)), theta, pos, [64], 128, "half")
    assert torch.equal(qkv[:, :, 2], before[:, :, 2])


def test_gradient_by_differences():
    """L = <g, R x> has the gradient R^T g: the inverse call against differences of the oracle's loss."""
    rng = np.random.default_rng(4)
    x, g = rng.standard_normal((1, 2, 4, 64)), _tensor(rng, (1, 2, 4, 64), False)
    pos = np.array([[[3, 1000, 70000, 5]]])
    positions = torch.from_numpy(pos.astype(np.int32)).cuda()
    steps, _ = B.rope_steps(48, [24], device="cuda")
    theta, args = L.frequencies([24]), ([24], 48, "half", 1.1)
    grad = torch.empty_like(g)
    B.rope(B.make_rope(g, None, grad, None, positions, 48, "half", [24], 1.1, True), g, None, steps, positions, grad, None)
    grad, g64, h = _f64(grad), _f64(g), 1e-4
    for at in [(0, 0, 0, 0), (0, 1, 1, 30), (0, 0, 2, 23), (0, 1, 3, 47), (0, 1, 2, 60)]:
        e = np.zeros_like(x)
        e[at] = h
        diff = ((g64 * L.rope(x + e, theta, pos, *args)).sum() - (g64 * L.rope(x - e, theta, pos, *args)).sum()) / (2 * h)
        assert abs(grad[at] - diff) <= 2.0 ** -8 * abs(diff) + 1e-5        # (half a bf16 step; cancellation in the differences)


def test_captured():
    rng = np.random.default_rng(5)
    q = _tensor(rng, (1, 2, 33, 128), False)
    positions = torch.arange(33, dtype=torch.int32, device="cuda")[None, None]
    steps, _ = B.rope_steps(128, device="cuda")
    out, again = torch.empty_like(q), torch.empty_like(q)
    p = B.make_rope(q, None, out, None, positions, 128)
    B.rope(p, q, None, steps, positions, out, None)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        B.rope(p, q, None, steps, positions, again, None)
    again.zero_()
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, again)


@pytest.mark.parametrize("d,R", [(64, 8), (64, 24), (128, 40), (72, 72), (8, 8), (256, 200)])
@pytest.mark.parametrize("N", [1, 33])
def test_halves_of_whole_pieces_of_four(d, R, N):
    """Half layout, halves of four channels times an odd number, and even ones; heads beyond those that a CTA takes; what is behind keeps its bits."""
    rng = np.random.default_rng(d + R + N)
    q, k = _tensor(rng, (2, 18, N, d), True), _tensor(rng, (2, 5, N, d), False)
    q[0, 1, 0, R:] = float("nan")
    pos = np.broadcast_to(np.arange(N) + 1000, (1, 2, N))
    steps, _ = B.rope_steps(R, device="cuda")
    positions = torch.from_numpy(np.ascontiguousarray(pos).astype(np.int32)).cuda()
    qo, ko = torch.empty_like(q), torch.empty_like(k)
    B.rope(B.make_rope(q, k, qo, ko, positions, R, "half"), q, k, steps, positions, qo, ko)
    assert torch.equal(qo[..., R:].contiguous().view(torch.int16), q[..., R:].contiguous().view(torch.int16))
    for x, y in ((q[..., :R], qo[..., :R]), (k, ko)):
        _check(_f64(y), _f64(x), L.frequencies([R // 2]), pos, [R // 2], R, "half")


@pytest.mark.parametrize("first", [False, True])
@pytest.mark.parametrize("layout,d,R,axes", [("interleaved", 128, 128, 3), ("interleaved", 96, 50, 1), ("half", 128, 64, 1), ("half", 128, 74, 1),
                                             ("half", 64, 64, 1)])
def test_more_heads_than_a_thread_has_in_flight(layout, d, R, axes, first):
    """Twenty heads per CTA, 18 and 5 of them there: passes of four, the last one short; out of place and in place."""
    Bq, Hq, Hk, N = 2, 18, 5, 2500
    rng = np.random.default_rng(d + R)
    q, k = _tensor(rng, (Bq, Hq, N, d), first), _tensor(rng, (Bq, Hk, N, d), first)
    pairs = _pairs(R, axes)
    pos = rng.integers(0, 5000, (axes, Bq, N))
    positions = torch.from_numpy(pos.astype(np.int32)).cuda()
    steps, _ = B.rope_steps(R, pairs, device="cuda")
    qo, ko = torch.full_like(q, 3.0), torch.full_like(k, 3.0)
    B.rope(B.make_rope(q, k, qo, ko, positions, R, layout, pairs), q, k, steps, positions, qo, ko)
    assert B.debug_last_choice() == 20
    for x, y in ((q, qo), (k, ko)):
        _check(_f64(y), _f64(x), L.frequencies(pairs), pos, pairs, R, layout)
    q2, k2 = q.clone(memory_format=torch.preserve_format), k.clone(memory_format=torch.preserve_format)
    B.rope(B.make_rope(q2, k2, q2, k2, positions, R, layout, pairs), q2, k2, steps, positions, q2, k2)
    assert B.debug_last_choice() == 20 and torch.equal(q2, qo) and torch.equal(k2, ko)
