"""The largest sizes that the calls around a 4-bit cache take are the ones that include/ra.h gives, refused before a launch (no GPU)."""
import pytest

import paper_2409_10516_amd as ra
from tests.test_kv4_host import FULL, GOOD, _p


@pytest.mark.parametrize("change,needle", [
    (dict(n_q=1, n_kv=1, n_seq=1 << 24, N=1, stride=1), "2^24 tiles"),
    (dict(n_q=16, n_kv=1, n_seq=1 << 21, N=(1 << 24) + 1, stride=1 << 25), "2^21 tiles"),
    (dict(n_q=16 * 1024, n_kv=1, N=(1 << 24) + 1, stride=1 << 25), "2^24 rows"),
])
def test_full_attention_says_which_limit(change, needle):
    L = ra.lib()
    assert L.ra_full_attention_q4(*(FULL | dict(ws_bytes=1 << 50) | change).values()) == 6
    assert needle in L.ra_last_error().decode()


def test_workgroups_that_combine_records_fit_a_launch():
    """128 threads for each query head of records: below 2^32 in all. From 2^21 tiles of 16 on no records are left, up to 2^24 tokens."""
    size = ra.lib().ra_full_attention_q4_workspace_bytes
    for N in (40000, 1 << 24):
        assert size(1, 1, 1 << 25, 1, N) == 256 and size(1, 1, (1 << 25) - 16, 1, N) > 1 << 30


def test_limits_of_append_and_of_the_conversions():
    L = ra.lib()
    args = GOOD | dict(T=(1 << 24) // 2, n_seq=2)
    assert L.ra_append_tokens(*args.values()) == 6 and "2^24 - 1 tokens" in L.ra_last_error().decode()
    for n_seq, n_kv in ((1, 65536), (256, 256), (1 << 16, 1)):
        assert L.ra_quantize_kv4(_p(), 1, n_seq, n_kv, 1, 128, None, None, 1, None, _p(), _p()) == 6
        assert "65535" in L.ra_last_error().decode()
        assert L.ra_dequantize_kv4(_p(), _p(), 0, n_seq, n_kv, 1, 128, None, 1, None, _p()) == 6
        assert "65535" in L.ra_last_error().decode()
