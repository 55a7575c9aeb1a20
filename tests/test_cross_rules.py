"""Launch rules of cross attention at sizes whose both sides were timed."""
import math
import random

import pytest

from paper_2511_13198_amd import pdyattn as P
from tests import test_gpu_cross, test_gpu_cross_plans


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
    (140, 1, 6000, 120, 8, 8, 64, False), (140, 1, 6000, 250, 8, 8, 128, False),
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


def plans(prefix, tq, tk, n, mq, mk, hq, hkv, d, causal):
    """(kernel, waves, groups, d, plan, shared keys or not, a list or not) of each launch."""
    s = P.cross_launch_shapes(prefix, tq, tk, n, mq, mk, hq, hkv, d, causal)
    out = set()
    for kernel, first in (("fwd", "fwd_whole_first"), ("dq", "dq_whole_first"), ("dkdv", None)):
        w, g, parts = s[f"cross_{kernel}_kernel"]
        plan = "parts" if parts > 1 else "whole"
        if first:
            plan = "apart" if s["apart"] else "whole first" if s[first] else plan
        out.add((kernel, w, g, d, plan, prefix > 0, n > 64))
    return out


def test_the_gpu_cases_reach_what_random_sizes_reach():
    """Every kernel, tile shape and plan together, not one by one."""
    seen = set()
    for lq, lk, _, prefix, hq, hkv, d, causal in test_gpu_cross.CASES + test_gpu_cross_plans.CASES:
        seen |= plans(prefix, sum(lq) + 3, sum(lk) + 3, len(lq), max(lq), max(lk), hq, hkv, d, causal)
    rng = random.Random(0)

    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    reached = set()
    for _ in range(20000):
        n, hkv, d = log(1, rng.choice([64, 3000])), rng.choice([1, 2, 4, 8, 16]), rng.choice([64, 128])
        hq, q, k = rng.choice([1, 2, 3, 4, 8, 16]) * hkv, log(1, 3000), log(1, 30000)
        prefix = log(1, 30000) if rng.random() < 0.5 else 0
        tq = max(q, int(n * q * rng.choice([1, 1, 0.6, 0.3, 0.05])))
        tk = max(k, int(n * k * rng.choice([1, 1, 0.6, 0.3, 0.05])))
        if max((tq + n) * hq, (tk + prefix) * hkv) < 1 << 31:
            reached |= plans(prefix, tq, tk, n, q, k, hq, hkv, d, rng.random() < 0.5)
    assert len(reached) > 170 and not reached - seen, sorted(map(str, reached - seen))
