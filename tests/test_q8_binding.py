"""The 8-bit calls' binding without a GPU (not gpu)."""
import torch

import paper_2603_19610_amd as pv


def test_a_captured_call_takes_memory_of_its_graph(monkeypatch):
    """Graphs captured on one stream may be replayed on two at once: their calls do not share the stream's workspace."""
    monkeypatch.setattr(pv, "_default_ws", lambda kind: shared)
    shared = pv.Workspace(torch.device("cpu"))
    mine = pv.Workspace(torch.device("cpu"))
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: True)
    bufs = [pv._ws_buffer("verify_q8", None, 1000, "cpu") for _ in range(2)]
    assert len({b.data_ptr() for b in bufs + [shared.buf]}) == 3
    assert all(b.numel() >= 1000 for b in bufs)
    assert pv._ws_buffer("verify_q8", None, 0, "cpu").numel() > 0      # (a refused call's size; a pointer all the same)
    assert pv._ws_buffer("verify_q8", mine, 1000, "cpu") is mine.buf
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    assert pv._ws_buffer("verify_q8", None, 1000, "cpu") is shared.buf
    assert pv._ws_buffer("verify_q8", mine, 1000, "cpu") is mine.buf


def test_launch_limits_are_refused_as_documented():
    L, F = pv.lib(), 4096
    SHAPE = 2

    def quantize(D, rows):
        return L.pvlm_quantize_kv(pv.PVLM_BF16, 1, 1, 1, D, rows, F, F, F, rows, F, F, F, F, None, None)

    def gather(D, rows):
        return L.pvlm_gather_kv_q8(pv.PVLM_E4M3, 1, 1, 1, D, 64, F, F, F, F, F, F, 4, F, F, rows, 0, F, F, F, F,
                                   None, None)

    def verify(B, Hkv, ctx):
        return L.pvlm_verify_attn_q8(pv.PVLM_BF16, B, 1, Hkv, Hkv, 128, 1 << 30, ctx, 0.1, F, F, F, F, F, F, F, None,
                                     None, F, 0, None, None)
    for D, most in ((128, 1 << 28), (64, 1 << 29)):
        assert quantize(D, most) == SHAPE and quantize(D, 1 << 30) == SHAPE
        assert gather(D, 2 * most) == SHAPE
    assert verify(1, 16, (1 << 30) - 64) == SHAPE                # 4 * 16 * 2^25 blocks
    assert verify(15, 1, (1 << 30) - 64) != SHAPE                # (no workspace, or no device)
    assert verify(1 << 12, 1 << 11, 0) == SHAPE                  # 2^23 rows of queries
