"""Which workspace ``PagedCache.attend`` hands to the library: one a stream, another for captured calls."""
import pytest
import torch

from paper_2505_18719_gb300 import build as B
from paper_2505_18719_gb300 import paged as P


def test_streams_and_captures_have_workspaces_of_their_own(monkeypatch):
    B.build()
    cache = P.PagedCache(2, 4, 16, 2, 2, 64, 64, device="cpu")
    rows = P.Rows(*(torch.zeros(2, dtype=torch.int32) for _ in range(3)), torch.zeros(3, dtype=torch.int32))
    q = torch.zeros(2, 2, 64)
    seen = []

    def attn(*a):
        *_, ws, nbytes, stream = a
        seen.append((stream, ws, nbytes))
        return 0

    at = {"stream": 0, "capturing": False}
    monkeypatch.setattr(P, "_on_gpu", lambda *t: None)
    monkeypatch.setattr(P, "_stream", lambda: at["stream"])
    monkeypatch.setattr(P, "_capturing", lambda: at["capturing"], raising=False)
    monkeypatch.setattr(P.V, "vla_paged_attn", attn)
    for stream, capturing in ((0, False), (7, False), (0, False), (7, False), (9, True), (0, True), (0, False)):
        at.update(stream=stream, capturing=capturing)
        for layer in (0, 1):
            cache.attend(layer, q, rows)
    first = {}
    for stream, ws, nbytes in seen[:8] + seen[12:]:
        assert first.setdefault(stream, ws) == ws and nbytes == P.V.vla_paged_attn_workspace_bytes(64)
    captured = {ws for _, ws, _ in seen[8:12]}
    assert len(captured) == 1 and len({*first.values(), *captured}) == 3
    with pytest.raises(ValueError):
        cache.attend(0, q[:1], rows)
