"""Plans of the calls over keys of their own are read by calls, never written: threads may share them."""
import ctypes as C

import pytest
import torch

from paper_2606_23743_b200 import binding as B


class _Lib:
    """Stands for the library: keeps what the calls hand over."""

    def sva_cross_attn_fwd(self, p, *args):
        self.plan = C.string_at(C.addressof(p), C.sizeof(p))
        self.mask_stride = p.mask_stride
        return 0


@pytest.mark.parametrize("Bq", [1, 3])
def test_a_mask_leaves_the_plan_as_it_is(monkeypatch, Bq):
    q, k = torch.zeros(Bq, 2, 5, 64, dtype=torch.bfloat16), torch.zeros(Bq, 1, 7, 64, dtype=torch.bfloat16)
    p = B.make_cross_attn(q, k, k, q)
    lib = _Lib()
    monkeypatch.setattr(B, "_lib", lib)
    monkeypatch.setattr(B, "_all_on", lambda *a: True)
    monkeypatch.setattr(B, "_stream", lambda: 0)
    made = bytes(p)
    own, apart = torch.ones(Bq, 7, dtype=torch.bool), torch.ones(Bq, 9, dtype=torch.uint8)[:, :7]
    for mask, stride in ((own, 7), (own[:1].expand(Bq, 7), 0), (apart, 9), (own, 7), (None, None)):
        B.cross_attn_fwd(p, q, k, k, q, None, mask)
        assert bytes(p) == made
        if Bq > 1 and mask is not None:
            assert lib.mask_stride == stride
            # (everything else is the plan's)
            there = B.CrossAttn.from_buffer_copy(lib.plan)
            there.mask_stride = p.mask_stride
            assert bytes(there) == made
