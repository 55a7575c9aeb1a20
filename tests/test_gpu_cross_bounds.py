"""Cross attention where the sizes that a call is given and the offsets that it reads
part: rows and keys of no sequence alone, longest lengths that are too small, offsets
that are wrong."""
import math

import pytest

from tests import cross_util as cu

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
    o, lse, dq = filled(q.shape, torch.bfloat16), filled((4, 5), torch.float32), filled(q.shape, torch.float32)
    if prefix:
        pdyattn.attn_prefix_fwd(q, k, k, kp, kp, cq, ck, out=o, lse=lse)
        grads = pdyattn.attn_prefix_bwd(q, k, k, kp, kp, o, lse, q, cq, ck, dq=dq)
    else:
        pdyattn.attn_cross_fwd(q, k, k, cq, ck, out=o, lse=lse)
        grads = pdyattn.attn_cross_bwd(q, k, k, o, lse, q, cq, ck, dq=dq)
    assert (o == 7).all() and (lse == 7).all() and (dq == 7).all()
    assert all((g == 0).all() for g in grads[1:])
