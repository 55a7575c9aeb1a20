"""Launch rules of cross attention at sizes whose both sides were timed."""
import pytest

from paper_2511_13198_amd import pdyattn as P


def shapes(n, q, k, prefix, hq, hkv, d, causal=True):
    return P.cross_launch_shapes(prefix, n * q, n * k, n, q, k, hq, hkv, d, causal)


@pytest.mark.parametrize("n,q,k,prefix,hq,hkv,d,apart", [
    # two (sequence, kv head) pairs a CU: whole up to some shared keys, more for more rows
    (64, 1, 100, 700, 32, 8, 128, False), (64, 1, 400, 700, 32, 8, 128, False),
    (64, 1, 100, 900, 32, 8, 128, True), (64, 1, 100, 700, 8, 8, 128, True),
    (128, 1, 100, 900, 32, 4, 128, False), (64, 16, 200, 700, 32, 8, 128, False),
    # over four: the rounds that fused takes against the partial results that apart writes
    (512, 1, 30, 128, 32, 8, 64, True), (512, 1, 30, 256, 32, 8, 64, True),
    (512, 1, 30, 256, 8, 8, 128, True), (512, 1, 30, 128, 32, 8, 128, False),
    (256, 32, 200, 400, 16, 8, 128, False), (256, 32, 200, 700, 16, 8, 64, False),
    (256, 16, 200, 256, 8, 8, 64, False),
])
def test_shared_keys_apart_or_with_each_sequence(n, q, k, prefix, hq, hkv, d, apart):
    assert shapes(n, q, k, prefix, hq, hkv, d)["apart"] == apart
