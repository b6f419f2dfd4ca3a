"""A decoded token of a batch that keeps its cache in 4 bits only: append, then attention over all of it, each against float64."""
import numpy as np
import pytest
import torch

import paper_2409_10516_amd as ra
from oracle import kv4 as OK
from tests.test_gpu_kv4 import _inv_freq, _row_close
from tests.test_gpu_q4 import _cache, _check
from tests.util import to_np

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n_q,n_kv,cap", [(8, 2, 3001), (4, 4, 700)])
def test_token_of_a_batch(dtype, n_q, n_kv, cap):
    """Sequences of unequal length, one that has no new token, one that is empty before, one whose cache ends with the token."""
    first, n_new = [cap // 2, 40, 0, cap - 1], [1, 0, 1, 1]
    n_seq, lens = 4, [a + b for a, b in zip(first, n_new)]
    k4, v4, _, _ = _cache(n_seq, n_kv, cap, seed=cap, junk=first)
    g = torch.Generator().manual_seed(cap)
    x = torch.randn((n_seq, 1, n_q + 2 * n_kv, 128), generator=g).to(dtype)
    w = [(1 + 0.2 * torch.randn(128, generator=g)).to(dtype) for _ in range(2)]
    f = _inv_freq(128)
    q, k, v = x.to(DEV).split((n_q, n_kv, n_kv), dim=2)
    dev = lambda a: torch.tensor(a, dtype=torch.int32, device=DEV)  # noqa: E731
    out_q = ra.ra_append_tokens(q, k, v, dev(first), n_new=dev(n_new), q_weight=w[0].to(DEV), k_weight=w[1].to(DEV),
                                inv_freq=torch.from_numpy(f).to(DEV), k4=k4, v4=v4).squeeze(2)
    out, lse = (t.cpu().numpy() for t in ra.ra_full_attention_q4(out_q, k4, v4, dev(lens)))
    X = to_np(x)[:, 0]
    for s in range(n_seq):
        K, V = (OK.dequantize_rows(*(t[s].cpu().numpy() for t in c)) for c in (k4, v4))
        if n_new[s]:
            ref, size = OK.head_rows(X[s:s + 1, :n_q], [first[s]], to_np(w[0]), 1e-6, f)
            _row_close(to_np(out_q[s])[None], ref, size, dtype)
            assert np.array_equal(V[:, first[s]], OK.dequantize_rows(*OK.quantize_rows(X[s, n_q + n_kv:])))
            # (a key is within its rounding to 4 bits, half a step of at most a third of its block's largest value)
            ref, _ = OK.head_rows(X[s:s + 1, n_q:n_q + n_kv], [first[s]], to_np(w[1]), 1e-6, f)
            top = np.repeat(np.abs(ref[0]).reshape(n_kv, 4, 32).max(axis=-1), 32, axis=-1)
            assert (np.abs(K[:, first[s]] - ref[0]) <= (1 / 3 + 2.0 ** -7) * top).all()
        for h in range(n_q):
            _check(out[s, h], lse[s, h], to_np(out_q[s, h]), K[h // (n_q // n_kv)], V[h // (n_q // n_kv)], np.arange(lens[s]), dtype)
