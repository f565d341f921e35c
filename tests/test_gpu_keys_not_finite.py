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
