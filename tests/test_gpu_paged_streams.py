"""Two streams that attend over one cache at the same time."""
import pytest
import torch

from paper_2505_18719_gb300 import paged as P

pytestmark = pytest.mark.gpu


def test_two_streams_attend_over_one_cache():
    # one long context whose items all CTAs cut, and other queries over it on another stream: results as one after the other
    g = torch.Generator(device="cuda").manual_seed(0)
    n, heads, hd = 20000, 4, 128
    cache = P.PagedCache(1, n // 16 + 1, 16, 1, heads, hd, n + 16)
    rows = cache.plan(torch.full((1,), n, dtype=torch.int32, device="cuda"), n)
    k, v = (torch.randn(n, heads, hd, generator=g, device="cuda") for _ in range(2))
    cache.append(0, torch.zeros(n, heads, hd, device="cuda"), k, v, rows)
    last = P.Rows(*(t[-1:] for t in rows[:3]), rows.start)
    queries = [torch.randn(1, heads, hd, generator=g, device="cuda") for _ in range(2)]
    want = [cache.attend(0, q, last) for q in queries]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    out = [[], []]
    for _ in range(50):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                out[i].append(cache.attend(0, queries[i], last))
    torch.cuda.synchronize()
    for i in range(2):
        for x in out[i]:
            assert torch.equal(x, want[i])
    cache.check()
    assert len({t.data_ptr() for t in (cache.workspace, *cache._stream_workspaces.values())}) == 4
