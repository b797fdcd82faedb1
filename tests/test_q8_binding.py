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
