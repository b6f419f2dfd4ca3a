"""The calls around a cache in pages where their compiled checks have not been built, and caches that are none."""
import pytest
import torch

import paper_2409_10516_amd as ra
from paper_2409_10516_amd import binding as B
from tests.test_gpu_paged import DEV, Cache, ints, queries

pytestmark = pytest.mark.gpu


def _all(cache):
    q, n = queries(2, 4, torch.bfloat16, 3).to(DEV), ints([100, 40])
    ids = torch.arange(12, dtype=torch.int32, device=DEV).expand(2, 4, -1).contiguous()
    x = queries(2, 6 * 8, torch.bfloat16, 4).to(DEV).view(2, 6, 8, 128)
    qx, k, v = x.split((4, 2, 2), dim=2)
    got = [ra.ra_append_tokens_paged(qx, k, v, ints([90, 30]), cache), ra.ra_gather_paged(cache), ra.ra_gather_paged(cache, values=True)]
    got += [*ra.ra_full_attention_paged(q, cache, n), *ra.ra_attend_paged(q, cache, 2, 20, ids, n)]
    return [torch.nan_to_num(t) for t in got]


def test_the_calls_are_the_same_without_them(monkeypatch, tmp_path):
    ref = _all(Cache([100, 40], 2, 16, torch.bfloat16, seed=2).gpu)
    monkeypatch.setattr(B, "CALLS_PATH", str(tmp_path / "_calls.so"))
    monkeypatch.setattr(B, "_short", None)
    cache = Cache([100, 40], 2, 16, torch.bfloat16, seed=2).gpu
    assert cache._core is None
    assert all(torch.equal(a, b) for a, b in zip(_all(cache), ref))
    with pytest.raises(ValueError, match="other memory"):
        cache.K.set_(torch.zeros_like(cache.K))
        ra.ra_gather_paged(cache)
