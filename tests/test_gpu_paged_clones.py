"""Tensors that share memory until one of them is written to (torch's lazy clones), as results and pools of the calls around a cache in pages."""
import pytest
import torch

import paper_2409_10516_amd as ra

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
CALLS = ["append", "gather", "full", "attend"]


def _calls(cache):
    """-> by name: the call, its arguments, its results."""
    ones = lambda *shape: torch.ones(shape, device=DEV)  # noqa: E731
    x, q = ones(1, 2, 4, 128), ones(1, 4, 128)
    k = 2.0 * ones(1, 2, 2, 128)
    ids, n = torch.full((1, 4, 3), 4, dtype=torch.int32, device=DEV), torch.full((1,), 9, dtype=torch.int32, device=DEV)
    res = lambda: dict(out=5.0 * ones(1, 4, 128), lse=5.0 * ones(1, 4))  # noqa: E731
    return {"append": (ra.ra_append_tokens_paged, dict(q=x, k=k, v=k, first=n - 9, cache=cache), dict(q_out=5.0 * ones(1, 4, 2, 128))),
            "gather": (ra.ra_gather_paged, dict(cache=cache, rows=3), dict(out=5.0 * ones(1, 2, 3, 128))),
            "full": (ra.ra_full_attention_paged, dict(q=q, cache=cache, n_tokens=n), res()),
            "attend": (ra.ra_attend_paged, dict(q=q, cache=cache, sink=1, window=2, ids=ids, n_tokens=n), res())}


def _cache():
    g = torch.Generator(device=DEV).manual_seed(1)
    K, V = (torch.randn((3, 2, 8, 128), device=DEV, generator=g) for _ in range(2))
    return ra.PagedCache(K, V, torch.tensor([[2, 0]], dtype=torch.int32, device=DEV))


@pytest.mark.parametrize("given", [False, True])
@pytest.mark.parametrize("name", CALLS)
def test_results_are_written_to_the_given_tensor_alone(name, given):
    cache = _cache()
    call, args, res = _calls(cache)[name]
    others = {k: torch._lazy_clone(t) for k, t in res.items()}
    st = dict(stream=torch.cuda.current_stream()) if given else {}
    call(**args, **res, **st)
    fresh = call(**args)
    fresh = fresh if isinstance(fresh, tuple) else (fresh,)
    for k, want in zip(res, fresh):
        assert torch.equal(res[k], want), k
        assert (others[k] == 5.0).all(), k


@pytest.mark.parametrize("given", [False, True])
@pytest.mark.parametrize("which", ["K", "V"])
@pytest.mark.parametrize("name", CALLS)
def test_pools_that_have_come_to_be_shared_are_refused(name, which, given):
    """A pool that has been cloned since has other memory as soon as it may be written to."""
    cache = _cache()
    call, args, res = _calls(cache)[name]
    pool = getattr(cache, which)
    before, other = pool.clone(), torch._lazy_clone(pool)
    st = dict(stream=torch.cuda.current_stream()) if given else {}
    with pytest.raises(ValueError, match="other memory"):
        call(**args, **res, **st)
    assert torch.equal(other, before) and torch.equal(pool, before)
