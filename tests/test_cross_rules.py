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


@pytest.mark.parametrize("n,q,k,longest,hq,hkv,d,cut", [
    (512, 1, 1000, 131072, 32, 8, 128, True), (512, 1, 1000, 8192, 32, 8, 128, True),
    (512, 1, 1000, 4096, 32, 8, 128, False), (512, 1, 1000, 32768, 32, 8, 64, True),
    (32, 64, 300, 16384, 16, 16, 128, True), (32, 64, 300, 2048, 16, 16, 64, True),
    (32, 64, 300, 1024, 16, 16, 128, False), (512, 1, 1000, 1000, 32, 8, 128, False),
])
def test_one_long_cache_among_short_ones_is_cut(n, q, k, longest, hq, hkv, d, cut):
    s = P.cross_launch_shapes(0, n * q, (n - 1) * k + longest, n, q, max(k, longest), hq, hkv, d, False)
    assert (s["cross_fwd_kernel"][2] > 1) == cut and (s["cross_dq_kernel"][2] > 1) == cut


@pytest.mark.parametrize("n,q,longest,k,hq,hkv,d,cut", [
    (300, 16, 8192, 60, 8, 1, 128, True), (300, 16, 128, 60, 8, 1, 64, True),
    (256, 16, 512, 16, 32, 8, 128, True), (256, 16, 128, 16, 32, 8, 128, False),
    (32, 16, 2048, 1000, 8, 8, 64, True), (32, 16, 512, 1000, 8, 8, 64, False),
    (300, 16, 16, 60, 8, 1, 128, False),
])
def test_keys_that_one_long_sequence_sees_are_cut(n, q, longest, k, hq, hkv, d, cut):
    s = P.cross_launch_shapes(0, (n - 1) * q + longest, n * k, n, longest, k, hq, hkv, d, False)
    assert (s["cross_dkdv_kernel"][2] > 1) == cut
