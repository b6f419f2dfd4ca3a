"""What the weights of the softmax keep of their 24 bits where values meet them (ra_full_attention_q4)."""
import numpy as np
import pytest
import torch

import paper_2409_10516_amd as ra
from oracle import kv4 as OK

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
ROWS = 8


def _bf16(x):
    return torch.tensor(x, dtype=torch.float64).to(torch.bfloat16).double().numpy()


def _queries():
    """First dimensions of 16 queries, each of 8 bits, whose rows of key -1 have a weight that loses most of what it can lose in
    two terms of 8 bits each -> (values, weights, the weights in two terms)."""
    x = np.unique(_bf16(np.linspace(0.5, 8.0, 4000)))
    w = np.exp(-x / np.sqrt(128.0))
    first = _bf16(w)
    two = first + _bf16(w - first)
    far = np.argsort(-np.abs(two / w - 1.0))[:16]
    return x[far], w[far], two[far]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n_q", [8, 16])
@pytest.mark.parametrize("cap", [ROWS, 20000])
def test_weights_meet_values_with_24_bits(dtype, n_q, cap):
    """One row with logit 0 and value 1, seven with logit -x / sqrt(128) and value 0: out = 1 / (1 + 7 w). Logits are exact. w: the
    exponent x log2(e) / sqrt(128) <= 1.03 is off by its factor's and its own rounding (1.1 x 2^-24 of w after the factor ln 2), the
    exponential by a step of the last place (2 x 2^-24). Its terms have 8 bits, so that sums of seven equal ones are exact and what is rounded is
    one sum per term (a step each: 6 x 2^-24), one over the columns' groups (1 x 2^-24) and the division (a step and a half: 3 x 2^-24).
    Together below 14 x 2^-24. In a list of rows (cap 20000) the same rows are one record."""
    x, w, two = (v[:n_q] for v in _queries())
    ref, bound = 1.0 / (1.0 + 7.0 * w), 14 * U
    assert (np.abs((1.0 + 7.0 * w) / (1.0 + 7.0 * two) - 1.0) > 1.5 * bound).all()      # (weights of 16 bits would show)
    K, V = np.zeros((2, 1, 1, cap, 128), np.float32)
    K[0, 0, 1:ROWS, 0], V[0, 0, 0, :] = -1.0, 1.0
    k4, v4 = (tuple(torch.from_numpy(t).to(DEV) for t in OK.quantize_rows(y[:, :, :ROWS])) for y in (K, V))
    if cap > ROWS:
        k4, v4 = (tuple(torch.nn.functional.pad(t, (0, 0, 0, cap - ROWS)) for t in y) for y in (k4, v4))
    q = torch.zeros((1, n_q, 128), dtype=dtype)
    q[0, :, 0] = torch.from_numpy(x).to(dtype)
    out, lse = ra.ra_full_attention_q4(q.to(DEV), k4, v4, torch.tensor([ROWS], dtype=torch.int32, device=DEV))
    got = out[0].double().cpu().numpy()
    assert (np.abs(got / ref[:, None] - 1.0) <= bound).all(), np.abs(got / ref[:, None] - 1.0).max() / U
    assert (np.abs(lse[0].double().cpu().numpy() + np.log(ref)) <= 14 * U * (1.0 - np.log(ref))).all()
