"""The stream that the binding hands to a search, without a GPU."""
import types

import pytest
import torch

from paper_2608_23553_amd import Index


@pytest.mark.parametrize("device", [0, 3])
def test_no_stream_is_the_current_one_of_the_index_own_gpu(device, monkeypatch):
    """Not that of the current GPU: a stream of another device is nothing to launch on."""
    handles = {i: types.SimpleNamespace(cuda_stream=1000 + i) for i in range(4)}

    def current_stream(d=None):
        return handles[2 if d is None else torch.device(d).index if not isinstance(d, int) else d]

    monkeypatch.setattr(torch.cuda, "current_stream", current_stream)
    idx, asked = Index.__new__(Index), []
    idx._info = {"device": device, "ndocs": 5}
    Q = types.SimpleNamespace(shape=(1, 2, 128), data_ptr=lambda: 16)
    results = types.SimpleNamespace(data_ptr=lambda: 32)
    monkeypatch.setattr(Index, "_q", lambda self, Q, stream: (Q, 0))
    monkeypatch.setattr(Index, "_results", lambda self, *a: (results, results))

    class Library:
        def __getattr__(self, name):
            return lambda *a: asked.append((name, getattr(a[-1], "value", a[-1]))) or 0

    monkeypatch.setattr("paper_2608_23553_amd.chimera.lib", Library)
    idx._h = None
    idx.search_pages(types.SimpleNamespace(_h=None), Q, 1, 2, 3)
    idx.search(Q, 1, 2, 3)
    idx.search(Q, 1, 2, 3, refine=1)
    idx.search_collab(Q, 1, 2, 3, 1, 3)
    assert [s for _, s in asked] == [1000 + device] * 4, asked
    asked.clear()
    idx.search_pages(types.SimpleNamespace(_h=None), Q, 1, 2, 3, stream=handles[1])
    assert asked == [("chimera_search_pages", 1001)]
