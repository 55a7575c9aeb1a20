"""Cross attention and shared-prefix attention on the GPU against the definition in
64 bits: lengths from none to thousands, odd sizes, grouped heads, both masks,
padded keys, rows that see nothing, rows of no sequence, streams and graphs."""
import math

import pytest

from tests import cross_util as cu

pytestmark = pytest.mark.gpu

# (query lengths, key lengths, used or None, prefix, Hq, Hkv, d, causal)
CASES = [
    # one token a sequence: packed keys, a cache with room, a group of 8, of 3, of 1
    ([1] * 4, [150] * 4, None, 0, 8, 8, 64, False),
    ([1] * 7, [600] * 7, [600, 1, 0, 33, 512, 129, 65], 0, 32, 8, 128, True),
    ([1] * 3, [4000] * 3, [4000, 3999, 64], 0, 8, 1, 128, True),
    ([1, 1], [1, 2], None, 0, 3, 1, 64, False),
    ([1], [20000], None, 0, 8, 8, 64, False),
    # several tokens: 15, 24, 40, 100 packed rows; causal aligned at the end
    ([5, 1, 0, 3], [300, 64, 10, 0], None, 0, 6, 2, 128, True),
    ([3] * 5, [1000] * 5, [7, 1000, 3, 2, 1], 0, 32, 4, 64, True),
    ([10, 7], [2500, 90], None, 0, 4, 1, 128, True),
    ([25, 3, 17], [700, 31, 129], None, 0, 8, 2, 64, False),
    # more queries than keys under the causal mask: early rows see nothing
    ([40, 9], [12, 9], None, 0, 4, 2, 128, True),
    # long rows: tiles of 256, split keys and not
    ([300, 0, 515], [777, 5, 2049], None, 0, 4, 4, 128, False),
    ([1200], [3000], None, 0, 6, 2, 64, True),
    ([70] * 60, [129] * 60, None, 0, 5, 1, 64, False),
    # more sequences than lanes
    ([1 + i % 3 for i in range(150)], [(37 * i) % 90 for i in range(150)], None, 0, 2, 1, 128, True),
    # shared keys: few rows behind many of them (apart), others; one key, no own keys
    ([1] * 5, [40] * 5, [1, 40, 17, 0, 8], 333, 8, 2, 128, True),
    ([1] * 64, [9] * 64, None, 1000, 4, 4, 64, True),
    ([1] * 9, [700] * 9, [700, 0, 1, 64, 128, 129, 650, 2, 90], 2500, 16, 2, 128, True),
    ([16, 3, 0, 9], [20, 3, 1, 300], None, 900, 8, 2, 64, True),
    ([20] * 12, [20] * 12, None, 600, 6, 2, 128, False),
    ([2, 1, 4], [2, 1, 4], None, 1, 8, 8, 64, True),
    ([4, 8, 1], [0, 0, 0], None, 130, 8, 4, 128, False),
    ([100, 33, 1, 250], [100, 33, 1, 250], None, 200, 8, 2, 128, True),
    ([300, 129], [300, 400], None, 1, 3, 1, 64, True),
    ([90, 120], [64, 64], [10, 64], 65, 2, 2, 128, True),
]


def make(lq, lk, prefix, hq, hkv, d, seed=0, behind=3):
    """Inputs on the GPU; `behind` rows of no sequence after the last."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(n, h):
        return torch.randn((n, h, d), generator=g, device="cuda").to(torch.bfloat16)

    x = dict(q=normal(sum(lq) + behind, hq), k=normal(sum(lk) + behind, hkv),
             v=normal(sum(lk) + behind, hkv), do=normal(sum(lq) + behind, hq))
    if prefix:
        x["kp"], x["vp"] = normal(prefix, hkv), normal(prefix, hkv)
    return x


def spoil(x, lk, used):
    """NaN and infinities where no key is in use."""
    at = 0
    for s, n in enumerate(lk):
        u = n if used is None else used[s]
        for t, bad in ((x["k"], math.inf), (x["v"], math.nan)):
            t[at + u:at + n] = bad
        at += n
    x["k"][at:], x["v"][at:] = math.nan, -math.inf


def setup(case, seed=0):
    import torch
    lq, lk, used, prefix, hq, hkv, d, causal = case
    x = make(lq, lk, prefix, hq, hkv, d, seed)
    ref = cu.reference(x["q"], x["k"], x["v"], cu.offsets(lq), cu.offsets(lk), causal,
                       1 / math.sqrt(d), used, x.get("kp"), x.get("vp"), x["do"])
    spoil(x, lk, used)
    x["q"][sum(lq):] = math.nan
    x["do"][sum(lq):] = math.nan
    args = (cu.offsets(lq, "cuda"), cu.offsets(lk, "cuda"), max(lq), max(lk), causal,
            1 / math.sqrt(d))
    len_k = None if used is None else torch.tensor(used, dtype=torch.int32, device="cuda")
    return x, ref, args, len_k


def forward(x, args, len_k, **kw):
    from paper_2511_13198_amd import pdyattn
    if "kp" in x:
        return pdyattn.attn_prefix_fwd(x["q"], x["k"], x["v"], x["kp"], x["vp"], *args,
                                       seqlens_k=len_k, **kw)
    return pdyattn.attn_cross_fwd(x["q"], x["k"], x["v"], *args, seqlens_k=len_k, **kw)


def case_id(c):
    return f"q{sum(c[0])}k{sum(c[1])}p{c[3]}h{c[4]}kv{c[5]}d{c[6]}"


@pytest.mark.parametrize("case", CASES, ids=case_id)
def test_forward(case):
    import torch
    x, ref, args, len_k = setup(case)
    t = sum(case[0])
    o = torch.full_like(x["q"], 7.0)
    lse = torch.full((case[4], x["q"].shape[0]), 7.0, device="cuda")
    forward(x, args, len_k, out=o, lse=lse)
    torch.cuda.synchronize()
    cu.check("o", o[:t], tuple(r[:t] for r in ref["o"]))
    cu.check("lse", lse[:, :t], tuple(r[:, :t] for r in ref["lse"]))
    assert (o[t:] == 7.0).all() and (lse[:, t:] == 7.0).all(), "rows of no sequence were written"


def backward(x, o, lse, args, len_k, **kw):
    from paper_2511_13198_amd import pdyattn
    if "kp" in x:
        return pdyattn.attn_prefix_bwd(x["q"], x["k"], x["v"], x["kp"], x["vp"], o, lse, x["do"],
                                       *args, seqlens_k=len_k, **kw)
    return pdyattn.attn_cross_bwd(x["q"], x["k"], x["v"], o, lse, x["do"], *args,
                                  seqlens_k=len_k, **kw)


GRADS = ("dq", "dk", "dv", "dkp", "dvp")


def empties(x, dtype, value):
    """Gradient tensors holding `value`, as the backward's keywords."""
    import torch
    names = {"dq": "q", "dk": "k", "dv": "v"}
    if "kp" in x:
        names.update(dk_prefix="kp", dv_prefix="vp")
    return {n: torch.full_like(x[of], value, dtype=dtype) for n, of in names.items()}


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("case", CASES, ids=case_id)
def test_gradients(case, dtype):
    import torch
    x, ref, args, len_k = setup(case, 1)
    o, lse = forward(x, args, len_k)
    out = empties(x, getattr(torch, dtype), 7.0)
    got = backward(x, o, lse, args, len_k, **out)
    torch.cuda.synchronize()
    t, tk = sum(case[0]), sum(case[1])
    for name, g in zip(GRADS, got):
        end = t if name == "dq" else g.shape[0] if name.endswith("p") else tk
        cu.check(name, g[:end], tuple(r[:end] for r in ref[name]))
        assert (g[end:] == 7.0).all(), f"{name}: rows of no sequence were written"
