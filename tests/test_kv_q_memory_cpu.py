"""What the 4-bit cache's calls do with memory, without a GPU: where it is taken from, and what may follow a call."""
import contextlib
import os

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
needs_lib = pytest.mark.skipif(not os.path.exists(os.path.join(ROOT, "paper_2510_11331_amd", "libsd.so")), reason="libsd.so not built")


@needs_lib
@pytest.mark.parametrize("where", ["stream", "device", "here"])
def test_rope_table_takes_memory_on_its_stream(where, monkeypatch):
    """The table's memory is of the stream that writes it: taken of another one, it may still be in use there, or be given
    away there before it is written."""
    from paper_2510_11331_amd import kv_q
    inside, seen = [], []

    @contextlib.contextmanager
    def context():
        inside.append(where)
        yield
        inside.pop()

    class Lib:
        @staticmethod
        def sd_rope_table(n_pos, head_dim, theta, out, stream):
            seen.append(("write", list(inside)))
            return 0

    empty = torch.empty

    def take(*a, **k):
        seen.append(("take", list(inside)))
        return empty(*a, **{**k, "device": "cpu"})

    monkeypatch.setattr(kv_q, "lib", lambda: Lib)
    monkeypatch.setattr(kv_q, "_elsewhere", lambda t, stream: None if inside or where == "here" else context())
    monkeypatch.setattr(kv_q, "_raw_stream", lambda index: None)
    monkeypatch.setattr(torch, "empty", take)
    monkeypatch.setattr(torch.cuda, "stream", lambda s: context())
    monkeypatch.setattr(torch.cuda, "device", lambda d: context())
    monkeypatch.setattr(kv_q, "_current_device", lambda: 1 if where == "device" and not inside else 0)
    given = type("Stream", (), {"device": torch.device("cuda", 0)})() if where == "stream" else None
    out = kv_q.rope_table(4, 64, device="cuda:0", stream=given)
    assert out.shape == (4, 32, 2)
    want = [] if where == "here" else [where]
    assert seen == [("take", want), ("write", want)]
