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
