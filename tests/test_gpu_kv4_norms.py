"""Norms of rows at the ends of float32's range (ra_append_tokens), where 1 / sqrt(mean(x^2) + eps) is no normal float32."""
import numpy as np
import pytest
import torch

import paper_2409_10516_amd as ra
from oracle import kv4 as OK
from tests.test_gpu_kv4 import _inv_freq, _row_close
from tests.util import to_np

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rot", [0, 128])
def test_norms_of_tiny_and_huge_rows(dtype, rot):
    """eps 0: rows of subnormal numbers have a norm like any other. Sizes 2^-140 .. 2^124, in one batch with ordinary rows; the
    bounds are those of any row (each operation rounds once, and none to a subnormal number)."""
    g = torch.Generator().manual_seed(17)
    sizes = [-140, -133, -128, -127, -126, -100, 0, 90, 100, 120, 124, 126]
    x = torch.randn((1, len(sizes), 3, 128), generator=g, dtype=torch.float64).clamp(-3.9, 3.9)
    x = (x * torch.tensor([2.0 ** (e - (2 if e > 0 else 0)) for e in sizes], dtype=torch.float64).view(1, -1, 1, 1)).to(dtype)
    w = (1 + 0.3 * torch.randn(128, generator=g)).to(dtype)
    f = _inv_freq(rot) if rot else None
    out = ra.ra_append_tokens(x.to(DEV), None, None, None, q_weight=w.to(DEV), eps=0.0, inv_freq=None if f is None else torch.from_numpy(f).to(DEV))
    X = to_np(x)[0]
    some = np.abs(X).max(axis=-1) > 0                # (bfloat16 ends at 2^-133: the rows of 2^-140 are zero there, nothing over nothing)
    assert np.isfinite(X).all() and some[1:].all() and some[0].all() == (dtype == torch.float32)
    with np.errstate(invalid="ignore"):
        ref, size = OK.head_rows(X, np.arange(len(sizes)), to_np(w), 0.0, f)
    got = to_np(out)[0].transpose(1, 0, 2)
    assert np.isnan(got[~some]).all()
    _row_close(got[some], ref[some], size[some], dtype)


def test_norm_of_zero_rows():
    """Nothing over nothing with eps 0, zeroes with any other; the neighbouring heads have their norms."""
    x = torch.ones((1, 2, 3, 128))
    x[0, 0, 1] = 0
    w = torch.ones(128, device=DEV)
    out = ra.ra_append_tokens(x.to(DEV), None, None, None, q_weight=w, eps=0.0).cpu()
    assert torch.isnan(out[0, 1, 0]).all() and (out[0, 1, 1] == 1).all() and (out[0, 0] == 1).all() and (out[0, 2] == 1).all()
    out = ra.ra_append_tokens(x.to(DEV), None, None, None, q_weight=w, eps=1e-30).cpu()
    assert (out[0, 1, 0] == 0).all() and (out[0, 1, 1] == 1).all()
