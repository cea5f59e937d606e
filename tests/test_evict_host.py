"""csd_cache_evict's Python call: counts beyond 31 bits, which a C int would take modulo 2^32.  No GPU: the library is a recorder."""

from types import SimpleNamespace

import pytest
import torch

from paper_2604_13634_b200 import CsdError, decode


@pytest.fixture
def call(monkeypatch):
    seen = []
    monkeypatch.setattr(decode, "_lib", lambda: SimpleNamespace(csd_cache_evict=lambda *a: seen.append(a) or 0))
    monkeypatch.setattr(decode, "_stream_ptr", lambda stream, device: 0)
    cache = SimpleNamespace(rows=2, max_pages=3, page_size=16, _device=-1, _ref=None)
    buf = SimpleNamespace(keep=20, ws_bytes=64, kept=torch.zeros(2, 20, dtype=torch.int32), evicted=torch.zeros(2, dtype=torch.int32),
                          workspace=torch.zeros(64, dtype=torch.uint8))

    def run(keep, **kw):
        decode.csd_cache_evict(cache, torch.zeros(2, 48), keep, buf, **kw)
        _, _, _, keep, rows, sinks, recent, *_ = seen[-1]
        return keep, rows is not None, sinks, recent

    return run


def test_counts_are_not_taken_modulo(call):
    assert call(20, sinks=3, recent=4) == (20, False, 3, 4)
    assert call(20, sinks=2 ** 32, recent=2 ** 40 + 1) == (20, False, 2 ** 31 - 1, 2 ** 31 - 1)
    assert call(torch.zeros(2, dtype=torch.int32), recent=2 ** 33)[1:] == (True, 0, 2 ** 31 - 1)
    for keep, kw in ((2 ** 32, {}), (2 ** 32 + 5, {}), (21, {}), (-1, {}), (-2 ** 32, {}), (5, dict(sinks=-2 ** 32)), (5, dict(recent=-2 ** 32 + 1))):
        with pytest.raises(CsdError):
            call(keep, **kw)
