"""Cross attention where the sizes that a call is given and the offsets that it reads
part: rows and keys of no sequence alone, longest lengths that are too small, offsets
that are wrong."""
import math

import pytest

from tests import cross_util as cu
from tests import test_gpu_cross as gpu

pytestmark = pytest.mark.gpu


def filled(shape, dtype, value=7.0):
    import torch
    return torch.full(shape, value, dtype=dtype, device="cuda")


@pytest.mark.parametrize("n", [2, 70])
def test_keys_of_no_sequence_alone(n):
    """Sequences without keys beside rows of k and v that belong to none: dq = 0, dk and dv
    stay as they were, with queries and without."""
    import torch
    from paper_2511_13198_amd import pdyattn
    k = filled((9, 2, 64), torch.bfloat16)
    ck = cu.offsets([0] * n, "cuda")
    for rows in (3, 0):
        q = filled((n * rows, 4, 64), torch.bfloat16)
        cq = cu.offsets([rows] * n, "cuda")
        o, lse = pdyattn.attn_cross_fwd(q, k, k, cq, ck)
        assert (o == 0).all() and (lse == -math.inf).all()
        dk, dv = filled(k.shape, torch.float32), filled(k.shape, torch.float32)
        dq, _, _ = pdyattn.attn_cross_bwd(q, k, k, o, lse, q, cq, ck, dk=dk, dv=dv)
        assert (dq == 0).all() and (dk == 7).all() and (dv == 7).all()


@pytest.mark.parametrize("prefix", [0, 5])
def test_rows_of_no_sequence_alone(prefix):
    """Sequences without queries beside rows of q that belong to none, the longest length
    left to the call: o, lse and dq stay as they were, the keys' gradients are 0."""
    import torch
    from paper_2511_13198_amd import pdyattn
    q, k = filled((5, 4, 64), torch.bfloat16), filled((6, 2, 64), torch.bfloat16)
    kp = filled((prefix, 2, 64), torch.bfloat16)
    cq, ck = cu.offsets([0, 0], "cuda"), cu.offsets([4, 2], "cuda")
    o, dq = filled(q.shape, torch.bfloat16), filled(q.shape, torch.float32)
    lse = filled((4, 5), torch.float32)
    if prefix:
        pdyattn.attn_prefix_fwd(q, k, k, kp, kp, cq, ck, out=o, lse=lse)
        grads = pdyattn.attn_prefix_bwd(q, k, k, kp, kp, o, lse, q, cq, ck, dq=dq)
    else:
        pdyattn.attn_cross_fwd(q, k, k, cq, ck, out=o, lse=lse)
        grads = pdyattn.attn_cross_bwd(q, k, k, o, lse, q, cq, ck, dq=dq)
    assert (o == 7).all() and (lse == 7).all() and (dq == 7).all()
    assert all((g == 0).all() for g in grads[1:])


# (query lengths, key lengths, used or None, prefix, Hq, Hkv, d, causal)
BOUNDS = [
    # padded batches and caches, the longest length that of the keys in use
    ([1, 5, 1, 3], [1024] * 4, [300, 7, 0, 299], 0, 8, 2, 128, True),
    ([30, 200, 8, 100], [1500] * 4, [900, 11, 64, 650], 0, 4, 4, 64, False),
    ([40, 1, 300], [700] * 3, [1, 90, 33], 200, 4, 2, 128, True),
    ([1 + i % 3 for i in range(80)], [300] * 80, [i % 50 for i in range(80)], 0, 4, 1, 64, True),
]


@pytest.mark.parametrize("case", BOUNDS, ids=gpu.case_id)
def test_the_longest_length_of_the_keys_in_use_will_do(case):
    """With seqlens_k a max_seqlen_k that bounds these alone gives every result, zeros for
    the keys not in use among them."""
    import torch
    x, ref, args, len_k = gpu.setup(case, 4)
    args = (*args[:3], max(case[2]), *args[4:])
    o, lse = gpu.forward(x, args, len_k)
    got = gpu.backward(x, o, lse, args, len_k, **gpu.empties(x, torch.float32, 7.0))
    t, tk = sum(case[0]), sum(case[1])
    cu.check("o", o[:t], tuple(r[:t] for r in ref["o"]))
    for name, g in zip(gpu.GRADS, got):
        end = t if name == "dq" else g.shape[0] if name.endswith("p") else tk
        cu.check(name, g[:end], tuple(r[:end] for r in ref[name]))
        assert (g[end:] == 7.0).all(), f"{name}: rows of no sequence were written"


# (the first sequence is the one that is longer than it was said to be)
SHORT = [
    ([40, 1, 30, 9], [300] * 4, None, 0, 8, 2, 128, True),
    ([600, 90, 100, 33], [500, 600, 2, 90], None, 0, 4, 4, 64, False),
    ([700, 300, 290], [900, 650, 400], None, 150, 2, 2, 128, True),
    ([9, 2, 1, 2], [40, 10, 0, 3], None, 1100, 4, 4, 128, True),
    ([200] + [3] * 75, [90] + [60] * 75, None, 0, 4, 2, 128, True),
    ([5] + [1] * 99, [90] + [6] * 99, None, 1300, 8, 2, 64, True),
]


@pytest.mark.parametrize("case", SHORT, ids=gpu.case_id)
def test_a_longest_query_length_too_small_costs_its_own_sequence_alone(case):
    """Every other sequence has its results; of the longer one the first max_seqlen_q rows
    have theirs, and no row of none is written."""
    import torch
    x, ref, args, len_k = gpu.setup(case, 5)
    most, first, t, tk = max(case[0][1:]), case[0][0], sum(case[0]), sum(case[1])
    args = (*args[:2], most, *args[3:])
    o, lse = filled(x["q"].shape, torch.bfloat16), filled((case[4], t + 3), torch.float32)
    gpu.forward(x, args, len_k, out=o, lse=lse)
    keep = torch.tensor([i for i in range(t) if i < most or i >= first], device="cuda")
    cu.check("o", o, ref["o"], keep)
    cu.check("lse", lse.T, tuple(r.T for r in ref["lse"]), keep)
    assert (o[t:] == 7).all() and (lse[:, t:] == 7).all()
    dq, dk, dv = gpu.backward(x, o, lse, args, len_k, **gpu.empties(x, torch.float32, 7.0))[:3]
    cu.check("dq", dq, ref["dq"], keep)
    for name, g in (("dk", dk), ("dv", dv)):
        cu.check(name, g, ref[name], torch.arange(case[1][0], tk, device="cuda"))
        assert (g[tk:] == 7).all()
    assert (dq[t:] == 7).all()


@pytest.mark.parametrize("case", [c for c in SHORT if c[1][0] > max(c[1][1:])] +
                         [([9, 4, 30], [1000, 260, 300], None, 0, 4, 2, 64, True)], ids=gpu.case_id)
def test_a_longest_key_length_too_small_costs_its_own_gradients_alone(case):
    """Rows attend to all keys whatever the bound; dk and dv of the longer sequence's first
    max_seqlen_k keys and of all others are there."""
    import torch
    x, ref, args, len_k = gpu.setup(case, 6)
    most, first, t, tk = max(case[1][1:]), case[1][0], sum(case[0]), sum(case[1])
    args = (*args[:3], most, *args[4:])
    o, lse = gpu.forward(x, args, len_k)
    cu.check("o", o[:t], tuple(r[:t] for r in ref["o"]))
    got = gpu.backward(x, o, lse, args, len_k, **gpu.empties(x, torch.float32, 7.0))
    keep = torch.tensor([i for i in range(tk) if i < most or i >= first], device="cuda")
    for name, g in zip(gpu.GRADS, got):
        cu.check(name, g[:t] if name == "dq" else g,
                 tuple(r[:t] for r in ref[name]) if name == "dq" else ref[name],
                 keep if name in ("dk", "dv") else None)
        if name in ("dk", "dv"):
            assert (g[tk:] == 7).all()


def no_rows(offsets, total):
    """The rows that offsets cannot mean: of no sequence, and not before the last offset."""
    rows = set(range(total)) - set(range(min(offsets[-1], total)))
    for a, b in zip(offsets, offsets[1:]):
        rows -= set(range(min(max(a, 0), total), min(b, total)))
    return sorted(rows)


# (queries, keys, prefix, Hq, Hkv, longest queries, longest keys, cu_seqlens_q, cu_seqlens_k)
FEW_Q = [[0, 40, 20], [0, 20, 5000], [50, 20, 10], [0, 1, -7], [10 ** 9, -10 ** 9, 30]]
FEW_K = [[0, 100, 300], [0, 9000, 9000], [300, 20, 100], [250, 0, -1], [-5, 2 ** 31 - 1, 7]]
MANY_Q = [[(37 * i) % 90 - 10 for i in range(101)], [60 - i for i in range(101)], [0] * 100 + [70],
          [0, 60] * 50 + [20]]
MANY_K = [[(53 * i) % 400 - 40 for i in range(101)], [300] + [0, 290] * 50,
          [5 * i for i in range(101)], [400 - 3 * i for i in range(101)]]
LONG_Q = [[0, 380, 90, 800], [400, 1, 399, -1], [0, 10 ** 9, 0, 350]]
LONG_K = [[8000, 0, 9000, 20], [-1, 10 ** 9, 5000, 9000], [0, 7000, 3000, 8999]]
WRONG = [(50, 300, p, hq, hkv, mq, 200, q, k)
         for q, k in zip(FEW_Q, FEW_K)
         for p, hq, hkv, mq in ((0, 4, 2, 30), (0, 4, 4, 2), (30, 2, 2, 50), (1200, 8, 2, 5))]
WRONG += [(60, 300, p, hq, hkv, mq, mk, q, k)
          for q, k in zip(MANY_Q, MANY_K)
          for p, hq, hkv, mq, mk in ((0, 4, 2, 3, 9), (0, 4, 1, 60, 300), (20, 2, 2, 40, 200),
                                     (1500, 8, 1, 2, 30))]
WRONG += [(400, 9000, p, 8, 4, 380, mk, q, k)
          for q, k in zip(LONG_Q, LONG_K) for p, mk in ((0, 9000), (0, 300), (700, 8000))]


@pytest.mark.parametrize("d,used", [(64, False), (128, True)])
@pytest.mark.parametrize("case", range(len(WRONG)))
def test_wrong_offsets_write_nothing_but_their_rows(case, d, used):
    """Offsets that fall, leave the tensors or contradict the longest lengths give some
    result, in the outputs and the workspace alone, and rows that they cannot mean stay."""
    import torch
    from paper_2511_13198_amd import pdyattn as P
    tq, tk, prefix, hq, hkv, mq, mk, cq, ck = WRONG[case]
    n, band = len(cq) - 1, 4096
    guards = []

    def guarded(shape, dtype, value):
        size = math.prod(shape)
        whole = torch.full((size + 2 * band,), value, dtype=dtype, device="cuda")
        guards.append((whole, size, value))
        return whole[band:band + size].view(shape)

    g = torch.Generator(device="cuda").manual_seed(case)
    q, do = (torch.randn((tq, hq, d), generator=g, device="cuda").bfloat16() for _ in range(2))
    k, v = (torch.randn((tk, hkv, d), generator=g, device="cuda").bfloat16() for _ in range(2))
    kp, vp = (torch.randn((prefix, hkv, d), generator=g, device="cuda").bfloat16()
              for _ in range(2))
    off = [torch.tensor(c, dtype=torch.int32, device="cuda") for c in (cq, ck)]
    len_k = torch.tensor([(10 ** 9, -7, 12)[i % 3] for i in range(n)], dtype=torch.int32,
                         device="cuda") if used else None
    sizes = (prefix, tq, tk, n, mq, mk, hq, hkv, d)
    o, lse = guarded((tq, hq, d), torch.bfloat16, 7.0), guarded((hq, tq), torch.float32, 7.0)
    grads = [guarded((t, h, d), torch.float32, 7.0) for t, h in
             ((tq, hq), (tk, hkv), (tk, hkv), (prefix, hkv), (prefix, hkv))]
    rest = (*off, mq, mk, True)
    P.attn_prefix_fwd(q, k, v, kp, vp, *rest, seqlens_k=len_k, out=o, lse=lse,
                      workspace=guarded((P.prefix_fwd_workspace_size(*sizes),), torch.uint8, 7))
    P.attn_prefix_bwd(q, k, v, kp, vp, o, lse, do, *rest, seqlens_k=len_k, dq=grads[0], dk=grads[1],
                      dv=grads[2], dk_prefix=grads[3], dv_prefix=grads[4],
                      workspace=guarded((P.prefix_bwd_workspace_size(*sizes),), torch.uint8, 7))
    torch.cuda.synchronize()
    for whole, size, value in guards:
        assert (whole[:band] == value).all() and (whole[band + size:] == value).all()
    stay = no_rows(cq, tq)
    assert (o[stay] == 7).all() and (lse[:, stay] == 7).all() and (grads[0][stay] == 7).all()
    stay = no_rows(ck, tk)
    assert (grads[1][stay] == 7).all() and (grads[2][stay] == 7).all()
