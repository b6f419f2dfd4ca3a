"""What the binding of the calls around a cache in pages refuses where there is a GPU: tensors, streams and caches of elsewhere."""
import pytest
import torch

import paper_2409_10516_amd as ra

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _good():
    """Arguments of calls that go through, by name."""
    ints = lambda: torch.zeros(1, dtype=torch.int32, device=DEV)  # noqa: E731
    x, q = torch.zeros((1, 1, 4, 128), device=DEV), torch.zeros((1, 4, 128), device=DEV)
    K, V = (torch.zeros((3, 2, 8, 128), device=DEV) for _ in range(2))
    table = torch.zeros((1, 2), dtype=torch.int32, device=DEV)
    cache = ra.PagedCache(K, V, table)
    res = lambda: dict(workspace=torch.zeros(1 << 16, dtype=torch.uint8, device=DEV), out=torch.zeros((1, 4, 128), device=DEV),  # noqa: E731
                       lse=torch.zeros((1, 4), device=DEV))
    return {
        "cache": (ra.PagedCache, dict(K=K, V=V, table=table)),
        "append": (ra.ra_append_tokens_paged, dict(q=x, k=x[:, :, :2].contiguous(), v=x[:, :, :2].contiguous(), first=ints(), cache=cache, n_new=ints() + 1,
                                                   q_weight=torch.ones(128, device=DEV), k_weight=torch.ones(128, device=DEV),
                                                   inv_freq=torch.ones(64, device=DEV), q_out=torch.zeros((1, 4, 1, 128), device=DEV))),
        "gather": (ra.ra_gather_paged, dict(cache=cache, first=ints(), rows=3, out=torch.zeros((1, 2, 3, 128), device=DEV))),
        "full": (ra.ra_full_attention_paged, dict(q=q, cache=cache, n_tokens=ints() + 5, **res())),
        "attend": (ra.ra_attend_paged, dict(q=q, cache=cache, sink=1, window=1, ids=torch.full((1, 4, 3), 4, dtype=torch.int32, device=DEV),
                                            n_tokens=ints() + 9, n_indexed=ints() + 7, **res())),
    }


TENSORS = [(n, a) for n, args in (("cache", "K V table"), ("append", "q k v first n_new q_weight k_weight inv_freq q_out"), ("gather", "first out"),
                                  ("full", "q n_tokens workspace out lse"), ("attend", "q ids n_tokens n_indexed workspace out lse")) for a in args.split()]


@pytest.mark.parametrize("name", ["cache", "append", "gather", "full", "attend"])
def test_calls_that_are_changed_below_go_through(name):
    call, args = _good()[name]
    call(**args)
    torch.cuda.synchronize()


@pytest.mark.parametrize("name,which", TENSORS)
def test_host_tensors_are_refused(name, which):
    call, args = _good()[name]
    with pytest.raises(ValueError):
        call(**(args | {which: args[which].cpu()}))


@pytest.mark.parametrize("name,which", TENSORS)
def test_other_types_and_shapes_are_refused(name, which):
    call, args = _good()[name]
    t = args[which]
    if which != "workspace":
        with pytest.raises((TypeError, ValueError)):
            call(**(args | {which: t.to(torch.float64 if t.is_floating_point() else torch.int64)}))
        if which != "table":                             # (fewer pages are another table)
            with pytest.raises((TypeError, ValueError, ra.RaError)):
                call(**(args | {which: t[..., :-1]}))
        if t.numel() == 1:                               # (one value always lies side by side)
            return
        with pytest.raises((TypeError, ValueError)):
            call(**(args | {which: t.repeat(*([2] * t.dim()))[(slice(None, None, 2),) * t.dim()]}))      # (of the right shape, but not side by side)
    else:
        with pytest.raises(ra.RaError):
            call(**(args | {which: t[:128]}))


class _Elsewhere:
    """What a stream of another device looks like."""
    cuda_stream, device_index = 0, 7


@pytest.mark.parametrize("name", ["append", "gather", "full", "attend"])
def test_streams_of_another_device_are_refused(name):
    call, args = _good()[name]
    with pytest.raises(ValueError, match="current GPU"):
        call(**args, stream=_Elsewhere())


@pytest.mark.parametrize("name", ["append", "gather", "full", "attend"])
def test_caches_whose_memory_has_changed_are_refused(name):
    call, args = _good()[name]
    K = args["cache"].K
    K.set_(torch.zeros((3, 2, 8, 128), device=DEV))
    with pytest.raises(ValueError, match="other memory"):
        call(**args)


def test_other_refusals():
    K = torch.zeros((3, 2, 8, 128), device=DEV)
    table = torch.zeros((1, 2), dtype=torch.int32, device=DEV)
    cache = ra.PagedCache(K, K.clone(), table)
    for bad in ((K, K.bfloat16(), table), (K.half(), K.half(), table)):
        with pytest.raises(TypeError):
            ra.PagedCache(*bad)
    for bad in ((K, K[:2], table), (K.transpose(1, 2), K, table), (K, K, table[0]), (K, K, table.expand(2, 2)), (K, K, table.long()), (None, None, table)):
        with pytest.raises(ValueError):
            ra.PagedCache(*bad)
    with pytest.raises(ra.RaError, match="power of two"):
        ra.ra_gather_paged(ra.PagedCache(K[:, :, :6].contiguous(), None, table))
    q = torch.zeros((1, 4, 128), device=DEV)
    with pytest.raises(TypeError):
        ra.ra_full_attention_paged(q.bfloat16(), cache)
    with pytest.raises(ValueError):
        ra.ra_full_attention_paged(q.expand(2, 4, 128).contiguous(), cache)
    with pytest.raises(ra.RaError):
        ra.ra_full_attention_paged(q, cache, N=17)
    with pytest.raises(ra.RaError):
        ra.ra_full_attention_paged(q[:, :3].contiguous(), cache)
    with pytest.raises(ra.RaError):
        ra.ra_attend_paged(q, cache, -1, 0, torch.zeros((1, 4, 1), dtype=torch.int32, device=DEV))
    with pytest.raises(ra.RaError):
        ra.ra_attend_paged(q, cache, 1, 0, torch.zeros((1, 4, 0), dtype=torch.int32, device=DEV))
    x = torch.zeros((1, 1, 4, 128), device=DEV)
    with pytest.raises(ValueError):
        ra.ra_append_tokens_paged(x, x, None, None, cache)                       # four KV heads
    with pytest.raises(ValueError):
        ra.ra_append_tokens_paged(None, None, None, None, cache)
    with pytest.raises(TypeError):
        ra.ra_append_tokens_paged(x.bfloat16(), None, None, None, cache)
    with pytest.raises(ra.RaError):
        ra.ra_append_tokens_paged(x, None, None, None, cache, inv_freq=torch.ones(12, device=DEV))
