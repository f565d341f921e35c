"""The give-up path of the many-row kernel over keys of their own: its key tiles after the first are withheld (test switch), the bounded waits run out, and
every role of both CTAs leaves.  Nothing faults or hangs."""
import pytest
import torch

from paper_2606_23743_b200 import binding as B

pytestmark = pytest.mark.gpu


def _cross():
    gen = torch.Generator(device="cuda").manual_seed(1)
    q, k, v = (torch.randn(1, 2, n, 128, generator=gen, device="cuda").to(torch.bfloat16) for n in (700, 640, 640))

    def call():
        o, status = torch.full_like(q, 7.0), torch.zeros(1, dtype=torch.int32, device="cuda")
        p = B.make_cross_attn(q, k, v, o)
        B.cross_attn_fwd(p, q, k, v, o, status=status, workspace=torch.empty(max(256, B.cross_attn_workspace_bytes(p)), dtype=torch.uint8, device="cuda"))
        torch.cuda.synchronize()
        return o, int(status)
    return call


def _cached():
    gen = torch.Generator(device="cuda").manual_seed(2)
    q, k = (torch.randn(1, 2, n, 64, generator=gen, device="cuda").to(torch.bfloat16) for n in (700, 640))
    c = B.make_kv_cache(*([torch.zeros(10, 2, 64, 64, dtype=torch.uint8, device="cuda"), torch.zeros(10, 2, device="cuda")] for _ in range(2)), format="e4m3_page")
    table, n = torch.arange(10, dtype=torch.int32, device="cuda")[None].contiguous(), torch.tensor([640], dtype=torch.int32, device="cuda")
    B.kv_cache_append(c, k, k, table, n * 0)

    def call():
        o, status = torch.full_like(q, 7.0), torch.zeros(1, dtype=torch.int32, device="cuda")
        p = B.make_cached_attn(c, q, o, table)
        B.cached_attn_fwd(p, q, table, n, o, status=status, workspace=torch.empty(max(256, B.cached_attn_workspace_bytes(p)), dtype=torch.uint8, device="cuda"))
        torch.cuda.synchronize()
        return o, int(status)
    return call


@pytest.mark.parametrize("make", [_cross, _cached])
def test_a_starved_pair_is_reported_and_not_stored(make):
    call = make()
    want, status = call()
    assert status == 0 and B.debug_last_choice() == 128
    try:
        B.debug_set_wait_limit(100_000_000)                                   # about 50 ms
        B.debug_set_mode(2048)
        o, status = call()
    finally:
        B.debug_set_mode(0)
        B.debug_set_wait_limit(0)
    assert status == B.SVA_DEV_TIMEOUT and (o == 7.0).all()
    o, status = call()                                                        # the context and the next call are intact
    assert status == 0 and torch.equal(o, want)
