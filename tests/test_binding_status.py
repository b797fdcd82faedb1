"""The status word that the page-table, slot, rotary and 4-bit calls take: kernels write to
it, so what is no word of the call's device is refused before anything is launched."""
import pytest
import torch

import paper_2603_19610_amd as pv


@pytest.mark.parametrize("bad,err", [
    (torch.zeros(1, dtype=torch.int32), ValueError), (torch.zeros(1, dtype=torch.int64), ValueError),
    (torch.zeros(0, dtype=torch.int32), ValueError), (4096, TypeError), ([0], TypeError),
], ids=["host", "int64", "empty", "address", "list"])
def test_status_on_the_host_is_refused(bad, err):
    with pytest.raises(err, match="status"):
        pv._flags(bad, torch.device("cuda", 0))


@pytest.mark.gpu
def test_status_that_does_not_fit_is_refused_by_every_call():
    from test_parity_q4 import empty_cache, i32

    bf = lambda *s: torch.zeros(s, dtype=torch.bfloat16, device="cuda")
    z = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")
    rot, slots = pv.Rotary(rot_dim=64, base=1e4), torch.zeros(2, dtype=torch.int64, device="cuda")
    slots[1] = -1
    cache, table = empty_cache((2, 2, 32), 64), i32([[0, 1], [1, 0]])
    rows, q, kv = (bf(2, 4, 64), bf(2, 2, 64), bf(2, 2, 64), z(2), slots), bf(2, 1, 4, 64), bf(2, 2, 8, 64)
    e = z(2, 0)
    calls = [
        lambda st: pv.pages_resize(z(2), z(2), table, z(9), z(1), page_size=32, status=st),
        lambda st: pv.slot_map(z(2), z(2), 2, page_size=32, n_pages=2, page_table=table, status=st),
        lambda st: pv.rotary_append(*rows, bf(2, 2, 32, 64), bf(2, 2, 32, 64), rotary=rot, status=st),
        lambda st: pv.rotary_append_q4(*rows, *cache, rotary=rot, status=st),
        lambda st: pv.quantize_kv_q4(kv, kv, z(2), *cache, status=st),
        lambda st: pv.quantize_kv_q4_paged(kv, kv, z(2), *cache, table, status=st),
        lambda st: pv.verify_attn_q4(q, *cache, z(2), status=st),
        lambda st: pv.verify_attn_q4_paged(q, *cache, table, z(2), status=st),
        lambda st: pv.verify_attn_q4(q, *cache, z(2), n_new=z(2), status=st),
        lambda st: pv.gather_kv_q4(*cache, e, z(2), z(2), z(2), 32, status=st),
        lambda st: pv.gather_kv_q4_paged(*cache, table, e, z(2), z(2), z(2), 32, status=st),
    ]
    for call in calls:
        for bad in (torch.zeros(1, dtype=torch.int32), z(1).long(), z(0), z(1).float()):
            with pytest.raises(ValueError, match="status"):
                call(bad)
        with pytest.raises(TypeError, match="status"):
            call(1)
    words = z(4)
    for call in calls:      # (the first word of a tensor, and one in the midst of others)
        call(words)
        call(words[2:3])
    torch.cuda.synchronize()
    assert not words.any()
