"""What is no PagedCache is refused by that name by the calls around a cache in pages, whatever was called before (no GPU)."""
import types

import pytest
import torch

import paper_2409_10516_amd as ra
from paper_2409_10516_amd import binding as B


class _Short:
    """Compiled checks that must not be reached."""
    def __getattr__(self, name):
        raise AssertionError(name)


@pytest.mark.parametrize("loaded", [False, True])
@pytest.mark.parametrize("given", [False, True])
@pytest.mark.parametrize("cache", [None, torch.zeros(3), (torch.zeros(3), torch.zeros(3)), types.SimpleNamespace(_core=None)])
@pytest.mark.parametrize("call", [lambda c, **kw: ra.ra_append_tokens_paged(torch.zeros(1, 1, 1, 128), None, None, None, c, **kw),
                                  lambda c, **kw: ra.ra_gather_paged(c, **kw),
                                  lambda c, **kw: ra.ra_full_attention_paged(torch.zeros(1, 1, 128), c, **kw),
                                  lambda c, **kw: ra.ra_attend_paged(torch.zeros(1, 1, 128), c, 0, 0, torch.zeros((1, 1, 1), dtype=torch.int32), **kw)])
def test_other_things_than_caches(call, cache, given, loaded, monkeypatch):
    monkeypatch.setattr(B, "_short", _Short() if loaded else None)
    with pytest.raises(TypeError, match="PagedCache"):
        call(cache, **(dict(stream=types.SimpleNamespace(cuda_stream=0, device_index=0)) if given else {}))
