"""The 4-bit verify's workspace is memory of the call's device (a launch writes to it)."""
import pytest
import torch

import paper_2603_19610_amd as pv

pytestmark = pytest.mark.gpu


class Elsewhere:
    def get(self, nbytes):
        return torch.zeros(nbytes, dtype=torch.uint8)


@pytest.mark.parametrize("ragged", [False, True])
def test_a_workspace_of_another_device_is_refused(ragged):
    from test_parity_q4 import empty_cache, i32

    q, cache = torch.zeros((2, 1, 4, 64), dtype=torch.bfloat16, device="cuda"), empty_cache((2, 2, 32), 64)
    n, kw = i32([0, 3]), dict(n_new=i32([1, 0])) if ragged else {}
    with pytest.raises(ValueError, match="ws"):
        pv.verify_attn_q4(q, *cache, n, ws=Elsewhere(), **kw)
    with pytest.raises(ValueError, match="ws"):
        pv.verify_attn_q4_paged(q, *cache, i32([[0], [1]]), n, ws=Elsewhere(), **kw)
    pv.verify_attn_q4(q, *cache, n, ws=pv.Workspace(), **kw)
    assert pv.synchronize() == 0
