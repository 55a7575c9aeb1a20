"""Cross attention where few batches go: plans and tile shapes that the other cases do not
bring together."""
import pytest

from tests import cross_util as cu
from tests import test_gpu_cross as gpu

pytestmark = pytest.mark.gpu

# (query lengths, key lengths, used or None, prefix, Hq, Hkv, d, causal)
CASES = [
    # one long sequence among many short ones: whole by their number, so cut
    ([1] * 512, [(7 * i) % 40 for i in range(511)] + [3000], None, 0, 8, 8, 128, False),
    ([1] * 520, [3000] + [(5 * i) % 30 for i in range(519)], None, 0, 16, 8, 64, True),
    ([64] * 15 + [50] + [64] * 16, [(9 * i) % 70 for i in range(31)] + [3001], None, 0, 16, 16, 128, True),
    ([33] * 40, [(9 * i) % 70 for i in range(20)] + [2500] + [11] * 19, None, 0, 16, 16, 64, False),
    ([1 + i % 2 for i in range(259)] + [310], [i % 6 for i in range(260)], None, 0, 8, 1, 128, False),
    ([400] + [1 + i % 2 for i in range(259)], [1 + i % 6 for i in range(260)], None, 0, 8, 1, 64, True),
    ([16] * 20 + [700] + [16] * 11, [150] * 32, [i * 4 for i in range(32)], 0, 8, 8, 64, False),
]


def lengths(n, most, part):
    """n lengths: `most`, and from none up to a `part`th of it (1: all alike)."""
    return [most] + [most if part == 1 else most // part * (37 * i % 64) // 63 for i in range(1, n)]


# (sequences, longest queries and part, longest keys and part, prefix, Hq, Hkv, d, causal):
# with the cases above and those of test_gpu_cross every kernel in every tile shape and
# plan, with shared keys and without, for up to 64 sequences and more, at both head
# dimensions
SPREAD = [
    (1, 12, 16, 8455, 2, 13400, 6, 3, 64, True), (1, 1, 4, 13913, 1, 9629, 6, 3, 128, False),
    (2, 225, 16, 19990, 1, 27, 4, 2, 128, True), (8, 869, 2, 17391, 1, 3, 4, 2, 128, True),
    (1, 1, 4, 1406, 1, 1, 4, 2, 64, True), (20, 1260, 4, 7104, 4, 0, 6, 3, 128, False),
    (1, 1721, 1, 2729, 1, 4, 4, 2, 64, False), (1, 2384, 1, 1, 1, 0, 8, 2, 128, True),
    (1, 2728, 2, 2, 2, 3, 8, 2, 128, False), (1, 2959, 1, 1, 16, 0, 9, 3, 64, False),
    (1, 2965, 16, 3, 16, 1, 10, 2, 64, False), (1, 2813, 1, 1, 1, 0, 12, 4, 64, True),
    (3, 2784, 1, 7, 1, 1, 4, 2, 64, False), (3, 2882, 1, 2, 16, 0, 4, 2, 128, True),
    (1, 2813, 2, 20, 1, 9, 12, 3, 128, True), (1, 2804, 2, 596, 4, 1974, 6, 3, 128, True),
    (3, 2365, 1, 2229, 4, 0, 6, 2, 128, True), (5, 2959, 1, 2452, 4, 19, 4, 2, 128, True),
    (8, 1855, 1, 3927, 16, 0, 4, 2, 64, True), (8, 1959, 1, 4963, 16, 113, 4, 2, 64, True),
    (3, 2444, 1, 3225, 16, 0, 9, 3, 128, True), (12, 2553, 1, 3933, 4, 0, 4, 2, 64, True),
    (8, 2981, 1, 3908, 16, 0, 8, 2, 64, True), (65, 1, 2, 2, 2, 1, 4, 2, 64, False),
    (65, 2, 16, 2, 1, 693, 4, 2, 128, False), (65, 99, 1, 2, 4, 1, 4, 2, 64, True),
    (65, 1, 16, 1506, 2, 6, 4, 2, 64, True), (65, 9, 4, 9976, 16, 55, 4, 2, 128, True),
    (65, 1283, 16, 7832, 4, 0, 4, 2, 64, True), (65, 93, 1, 2926, 2, 2, 4, 2, 128, True),
    (65, 962, 2, 3260, 2, 0, 2, 2, 128, False), (70, 1148, 2, 4356, 1, 0, 2, 1, 128, True),
    (70, 273, 1, 5303, 1, 5, 2, 1, 128, False), (12, 451, 1, 2474, 16, 0, 16, 8, 128, True),
    (50, 46, 1, 7277, 1, 0, 4, 2, 64, True), (50, 50, 1, 2, 16, 8306, 4, 2, 64, False),
    (20, 469, 1, 3497, 16, 4, 12, 3, 64, False), (1, 1, 2, 526, 1, 32, 4, 2, 128, True),
    (1, 26, 2, 370, 16, 679, 4, 2, 64, False), (1, 29, 4, 12, 1, 716, 4, 2, 128, True),
    (65, 2, 16, 61, 16, 758, 4, 2, 64, False), (65, 342, 2, 4, 1, 0, 4, 2, 64, True),
    (65, 2378, 16, 1, 1, 0, 4, 2, 64, True), (65, 93, 1, 21, 4, 4, 4, 2, 64, False),
    (65, 429, 4, 2, 1, 0, 4, 2, 128, True), (65, 365, 2, 29, 16, 2, 4, 2, 128, False),
    (65, 441, 4, 4547, 4, 2, 4, 2, 64, False), (65, 95, 1, 5226, 4, 0, 2, 2, 128, True),
    (65, 1145, 4, 5317, 4, 223, 2, 1, 128, True), (65, 102, 1, 2, 16, 4100, 2, 2, 64, True),
    (1, 2052, 1, 21, 2, 4049, 6, 2, 64, True), (65, 64, 1, 8307, 1, 0, 4, 2, 64, True),
    (20, 2007, 2, 3727, 4, 38, 8, 8, 128, True), (65, 2, 2, 1, 16, 8, 4, 2, 128, False),
    (65, 19, 4, 985, 16, 6, 4, 2, 128, True), (65, 21, 4, 609, 4, 0, 4, 2, 128, False),
    (65, 24, 16, 1575, 4, 4969, 4, 2, 64, True), (65, 21, 16, 55, 16, 16450, 4, 2, 128, True),
    (65, 1878, 16, 18410, 16, 4, 4, 2, 64, True), (65, 199, 1, 8, 1, 9, 2, 1, 64, True),
    (65, 107, 1, 4637, 2, 0, 4, 2, 64, True), (100, 1175, 1, 1766, 16, 1, 8, 8, 128, True),
    (50, 697, 1, 488, 4, 791, 16, 16, 128, False),
    (31, 1024, 16, 10049, 16, 5, 16, 4, 128, False), (20, 893, 1, 2183, 2, 0, 2, 2, 64, True),
    (12, 1777, 1, 4152, 16, 0, 4, 4, 64, False), (8, 842, 1, 2238, 16, 46, 6, 2, 64, False),
    (5, 1682, 1, 4403, 4, 5, 16, 2, 64, False), (65, 402, 16, 1313, 4, 0, 4, 4, 128, False),
    (257, 3000, 5, 3, 1, 0, 8, 4, 128, True),
]


def spread(i, n, q, q_part, k, k_part, prefix, hq, hkv, d, causal):
    lk = lengths(n, k, k_part)
    # (every third with keys not in use)
    used = [x - x // 3 * (j % 3) for j, x in enumerate(lk)] if i % 3 == 0 else None
    return lengths(n, q, q_part), lk, used, prefix, hq, hkv, d, causal


CASES += [spread(i, *s) for i, s in enumerate(SPREAD)]


@pytest.mark.parametrize("case", CASES, ids=gpu.case_id)
def test_forward_and_gradients(case):
    import torch
    x, ref, args, len_k = gpu.setup(case, 7)
    t, tk = sum(case[0]), sum(case[1])
    o, lse = torch.full_like(x["q"], 7.0), torch.full((case[4], t + 3), 7.0, device="cuda")
    gpu.forward(x, args, len_k, out=o, lse=lse)
    cu.check("o", o[:t], tuple(r[:t] for r in ref["o"]))
    cu.check("lse", lse[:, :t], tuple(r[:, :t] for r in ref["lse"]))
    assert (o[t:] == 7.0).all() and (lse[:, t:] == 7.0).all()
    got = gpu.backward(x, o, lse, args, len_k, **gpu.empties(x, torch.float32, 7.0))
    for name, g in zip(gpu.GRADS, got):
        end = t if name == "dq" else g.shape[0] if name.endswith("p") else tk
        cu.check(name, g[:end], tuple(r[:end] for r in ref[name]))
        assert (g[end:] == 7.0).all(), f"{name}: rows of no sequence were written"
