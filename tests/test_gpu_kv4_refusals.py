"""What the binding of the calls around a 4-bit cache refuses where there is a GPU: tensors, streams and handles of elsewhere."""
import pytest
import torch

import paper_2409_10516_amd as ra

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _x4(device=DEV):
    return tuple(torch.zeros((1, 2, 8, n), dtype=torch.uint8, device=device) for n in (64, 4))


def _index():
    return ra.ra_index_import(torch.full((4, 8, 2), -1, dtype=torch.int32), torch.zeros(4, dtype=torch.int32), 1, 4, 2)


def _good():
    """Arguments of calls that go through, by name."""
    idx = _index()
    x, ints = torch.zeros((1, 1, 4, 128), device=DEV), lambda: torch.zeros(1, dtype=torch.int32, device=DEV)
    q = torch.zeros((1, 4, 128), device=DEV)
    return {
        "append": (ra.ra_append_tokens, dict(q=x, k=x[:, :, :2].contiguous(), v=x[:, :, :2].contiguous(), first=ints(), n_new=ints() + 1,
                                             q_weight=torch.ones(128, device=DEV), k_weight=torch.ones(128, device=DEV),
                                             inv_freq=torch.ones(64, device=DEV), q_out=torch.zeros((1, 4, 1, 128), device=DEV),
                                             K=torch.zeros((1, 2, 8, 128), device=DEV), V=torch.zeros((1, 2, 8, 128), device=DEV), k4=_x4(), v4=_x4())),
        "quantize": (ra.ra_quantize_kv4, dict(X=torch.zeros((1, 2, 3, 128), device=DEV), first=ints(), n_new=ints() + 3, out=_x4())),
        "dequantize": (ra.ra_dequantize_kv4, dict(x4=_x4(), dtype=torch.float32, first=ints(), rows=3, out=torch.zeros((1, 2, 3, 128), device=DEV))),
        "full": (ra.ra_full_attention_q4, dict(q=q, k4=_x4(), v4=_x4(), n_tokens=ints() + 5, workspace=torch.zeros(1 << 16, dtype=torch.uint8, device=DEV),
                                               out=torch.zeros((1, 4, 128), device=DEV), lse=torch.zeros((1, 4), device=DEV))),
        "attend": (ra.ra_attend_q4, dict(q=q, idx=idx, k4=_x4(), v4=_x4(), sink=1, window=1, ids=torch.full((1, 4, 3), 4, dtype=torch.int32, device=DEV),
                                         out=torch.zeros((1, 4, 128), device=DEV), lse=torch.zeros((1, 4), device=DEV))),
    }


TENSORS = [(n, a) for n, args in (("append", "q k v first n_new q_weight k_weight inv_freq q_out K V k4 v4"), ("quantize", "X first n_new out"),
                                  ("dequantize", "x4 first out"), ("full", "q k4 v4 n_tokens workspace out lse"),
                                  ("attend", "q k4 v4 ids out lse")) for a in args.split()]


@pytest.mark.parametrize("name", ["append", "quantize", "dequantize", "full", "attend"])
def test_calls_that_are_changed_below_go_through(name):
    call, args = _good()[name]
    call(**args)
    torch.cuda.synchronize()


@pytest.mark.parametrize("name,which", TENSORS)
def test_host_tensors_are_refused(name, which):
    call, args = _good()[name]
    t = args[which]
    for there in ([t.cpu()] if torch.is_tensor(t) else [(t[0].cpu(), t[1]), (t[0], t[1].cpu())]):
        with pytest.raises(ValueError):
            call(**(args | {which: there}))


class _Elsewhere:
    """What a stream of another device looks like."""
    cuda_stream, device_index = 0, 7


@pytest.mark.parametrize("name", ["append", "quantize", "dequantize", "full", "attend"])
def test_streams_of_another_device_are_refused(name):
    call, args = _good()[name]
    with pytest.raises(ValueError, match="current GPU"):
        call(**args, stream=_Elsewhere())


def test_a_handle_of_another_device_is_refused():
    call, args = _good()["attend"]
    idx = args["idx"]
    assert idx.device == torch.cuda.current_device() and idx.info(12) == idx.device
    call(**args)
    idx.__dict__["device"] = 7                      # (kept for a handle's life once it has been asked for)
    with pytest.raises(ValueError, match="current GPU"):
        call(**args)


@pytest.mark.parametrize("n_kv", [32767, 65535])
def test_conversions_take_as_many_heads_as_they_say(n_kv):
    """n_seq x n_kv_heads up to 65535; one more is refused."""
    X = torch.randn((1, n_kv, 2, 128), generator=torch.Generator(device=DEV).manual_seed(n_kv), device=DEV)
    x4 = ra.ra_quantize_kv4(X)
    back = ra.ra_dequantize_kv4(x4, torch.float32)
    for h in (0, 1, n_kv // 2, n_kv - 1):
        one = ra.ra_quantize_kv4(X[:, h:h + 1].contiguous())
        assert all(torch.equal(a[:, h:h + 1], b) for a, b in zip(x4, one))
        assert torch.equal(ra.ra_dequantize_kv4(one, torch.float32), back[:, h:h + 1])
    with pytest.raises(ra.RaError, match="65535"):
        ra.ra_quantize_kv4(torch.zeros((2, 32768, 1, 128), device=DEV))
