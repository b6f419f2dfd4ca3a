"""What the calls around a 4-bit cache refuse, before anything touches a device (no GPU)."""
import ctypes as C

import pytest
import torch

import paper_2409_10516_amd as ra


def _p(at=0x10000):
    return C.c_void_p(at)       # non-null; never dereferenced when validation fails first


GOOD = dict(q_in=_p(), k_in=_p(), v_in=_p(), dt=1, n_seq=2, n_q=4, n_kv=2, T=3, d=128, q_row=512, k_row=256, v_row=256, qw=None, kw=None,
            eps=1e-6, inv_freq=_p(), rot=128, inter=0, first=None, n_new=None, stride=9, stride4=9, stream=None, q_out=_p(), K=_p(), V=_p(),
            K4=None, K4s=None, V4=None, V4s=None)


@pytest.mark.parametrize("change,status,needle", [
    (dict(dt=5), 3, "dtype"), (dict(n_seq=0), 1, "positive"), (dict(n_q=3), 1, "multiple"), (dict(d=64), 6, "d = 128"),
    (dict(T=0), 1, "positive"), (dict(T=1 << 31), 6, "large"), (dict(stride=0), 1, "positive"), (dict(K4=_p(), K4s=_p(), stride4=0), 1, "positive"), (dict(stride=1 << 31), 6, "large"), (dict(q_in=None), 1, "together"),
    (dict(q_out=None), 1, "together"), (dict(q_in=None, k_in=None, v_in=None), 1, "no input"), (dict(K=None), 1, "k_in"),
    (dict(k_in=None), 1, "k_in"), (dict(v_in=None), 1, "v_in"), (dict(K4=_p()), 1, "together"), (dict(V4s=_p()), 1, "together"),
    (dict(K4=_p(0x10008), K4s=_p()), 1, "aligned"), (dict(K4=_p(), K4s=_p(0x10002)), 1, "aligned"), (dict(rot=24), 6, "16"),
    (dict(rot=144), 1, "rot_dim"), (dict(rot=-16), 1, "rot_dim"), (dict(inv_freq=None), 1, "inv_freq"), (dict(q_row=511), 2, "apart"),
    (dict(k_row=0), 2, "apart"), (dict(q_row=513), 6, "16 bytes"), (dict(q_in=_p(0x10008)), 1, "aligned"), (dict(V=_p(0x10004)), 1, "aligned"),
    (dict(qw=_p(), eps=-1.0), 1, "eps"), (dict(kw=_p(), eps=float("nan")), 1, "eps"), (dict(qw=_p(0x10001)), 1, "aligned"),
    (dict(T=1 << 23, n_seq=2, q_row=512), 6, "tokens"), (dict(n_q=(1 << 31) - 2, q_row=1 << 38), 6, "heads"),
    (dict(q_in=None, q_out=None, k_in=None, K=None, inv_freq=None), 1, "inv_freq"),    # (values alone are not rotated, but a length is given)
    (dict(n_q=1 << 24, q_row=1 << 31), 6, "heads"), (dict(n_q=1 << 23, n_seq=120, T=1, q_row=1 << 30), 6, "heads"),
])
def test_append_refuses(change, status, needle):
    L = ra.lib()
    assert L.ra_append_tokens(*(GOOD | change).values()) == status
    assert needle in L.ra_last_error().decode()


@pytest.mark.parametrize("args,status,needle", [
    # X, dt, n_seq, n_kv, T, d, first, n_new, stride, stream, codes, scale
    ((None, 1, 1, 1, 4, 128, None, None, 4, None, _p(), _p()), 1, "NULL"),
    ((_p(), 2, 1, 1, 4, 128, None, None, 4, None, _p(), _p()), 3, "dtype"),
    ((_p(), 1, 1, 1, 4, 96, None, None, 4, None, _p(), _p()), 6, "d = 128"),
    ((_p(), 1, 0, 1, 4, 128, None, None, 4, None, _p(), _p()), 1, "positive"),
    ((_p(), 1, 1, 1, 0, 128, None, None, 4, None, _p(), _p()), 1, "positive"),
    ((_p(), 1, 1, 1, 4, 128, None, None, 0, None, _p(), _p()), 1, "positive"),
    ((_p(), 1, 1, 1, 4, 128, None, None, 4, None, None, _p()), 1, "NULL"),
    ((_p(), 1, 1, 1, 4, 128, None, None, 4, None, _p(), None), 1, "NULL"),
    ((_p(0x10002), 1, 1, 1, 4, 128, None, None, 4, None, _p(), _p()), 1, "aligned"),
    ((_p(), 1, 1, 1, 4, 128, None, None, 4, None, _p(), _p(0x10001)), 1, "aligned"),
    ((_p(), 1, 70000, 1, 4, 128, None, None, 4, None, _p(), _p()), 6, "65535"),
])
def test_quantize_and_dequantize_refuse(args, status, needle):
    L = ra.lib()
    assert L.ra_quantize_kv4(*args) == status
    assert needle in L.ra_last_error().decode()
    X, dt, n_seq, n_kv, T, d, first, _, stride, stream, codes, scale = args
    assert L.ra_dequantize_kv4(codes, scale, dt, n_seq, n_kv, T, d, first, stride, stream, X) == status
    assert needle in L.ra_last_error().decode()


FULL = dict(q=_p(), dt=1, K4=_p(), K4s=_p(), V4=_p(), V4s=_p(), n_seq=1, n_q=4, n_kv=2, N=100, stride=128, d=128, n_tokens=None, ws=_p(),
            ws_bytes=1 << 30, stream=None, out=_p(), lse=_p())


@pytest.mark.parametrize("change,status,needle", [
    (dict(q=None), 1, "NULL"), (dict(out=None), 1, "NULL"), (dict(ws=None), 1, "NULL"), (dict(dt=2), 3, "dtype"), (dict(n_q=5), 1, "multiple"),
    (dict(n_kv=0), 1, "positive"), (dict(d=256), 6, "d = 128"), (dict(K4=None), 1, "K"), (dict(V4s=None), 1, "V"),
    (dict(V4=_p(0x10004)), 1, "aligned"), (dict(N=0), 1, "positive"), (dict(N=1 << 31, stride=1 << 31), 6, "large"), (dict(stride=99), 2, "below"),
    (dict(q=_p(0x10002)), 1, "aligned"), (dict(ws=_p(0x10004)), 1, "aligned"), (dict(ws_bytes=8), 2, "workspace"),
    (dict(n_q=(1 << 31) - 1, n_kv=1), 6, "too many heads"), (dict(n_seq=1 << 23, n_q=4, n_kv=4), 6, "too many heads"),
])
def test_full_attention_refuses(change, status, needle):
    L = ra.lib()
    assert L.ra_full_attention_q4(*(FULL | change).values()) == status
    assert needle in L.ra_last_error().decode()


@pytest.mark.parametrize("N,n_q,needle", [((1 << 24) + 1, 16 * 1024, "too many heads"), ((1 << 30) - 1, 16 * 2047, "too many heads")])
def test_full_attention_refuses_stretches_past_31_bits(N, n_q, needle):
    """Rows that a workgroup would take of one head, with 64 bytes of codes each."""
    L = ra.lib()
    assert L.ra_full_attention_q4(*(FULL | dict(n_q=n_q, n_kv=1, N=N, stride=N)).values()) == 6
    assert needle in L.ra_last_error().decode()


def test_workspace_sizes():
    L = ra.lib()
    size = L.ra_full_attention_q4_workspace_bytes
    assert size(1, 1, 32, 8, 131072) > 0 and size(0, 16, 32, 8, 1) > 0
    assert size(1, 1, 32, 7, 1000) == 0 and size(2, 1, 32, 8, 1000) == 0 and size(1, 1, 32, 8, 0) == 0
    assert size(1, 1, 32, 8, 1 << 31) == 0


def test_attend_refuses_without_a_handle():
    L = ra.lib()
    args = [_p(), None, 1, _p(), _p(), _p(), _p(), 100, 128, 4, 8, 10, _p(), None, _p(), _p(), None, None, None, None]
    assert L.ra_attend_q4(*args) == 1 and "handle" in L.ra_last_error().decode()
    args[0] = None
    assert L.ra_attend_q4(*args) == 1 and "NULL" in L.ra_last_error().decode()


def test_binding_refuses_tensors_that_are_not_on_the_gpu():
    x, c, s = torch.zeros(1, 2, 1, 128), torch.zeros(1, 1, 4, 64, dtype=torch.uint8), torch.zeros(1, 1, 4, 4, dtype=torch.uint8)
    with pytest.raises((ValueError, RuntimeError, AssertionError)):
        ra.ra_append_tokens(x, None, None, None)
    with pytest.raises(ValueError):
        ra.ra_append_tokens(None, None, None, None)
    with pytest.raises((ValueError, RuntimeError, AssertionError)):
        ra.ra_quantize_kv4(torch.zeros(1, 1, 4, 128))
    with pytest.raises((ValueError, RuntimeError, AssertionError)):
        ra.ra_dequantize_kv4((c, s), torch.float32)
    with pytest.raises((ValueError, RuntimeError, AssertionError)):
        ra.ra_full_attention_q4(torch.zeros(1, 1, 128), (c, s), (c, s))
