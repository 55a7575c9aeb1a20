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
    ([20, 9, 1], [300, 700, 65], None, 0, 4, 2, 64, True),
    # enough key tiles to fill the chip: short rows, long ones
    ([30, 1, 17, 8, 30, 30, 2, 9], [500] * 8, [500, 499, 1, 0, 256, 128, 300, 500], 0, 16, 16, 128, False),
    ([600, 700], [9000, 7500], None, 0, 16, 16, 128, True),
    ([530, 601], [9100, 7401], None, 0, 16, 16, 64, False),
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
    # many heads to a group, and a prime number of them
    ([3, 9, 1], [40, 300, 7], None, 20, 64, 1, 64, True),
    ([40, 5], [100, 260], None, 0, 48, 1, 128, True),
    ([70, 12], [90, 150], [90, 0], 0, 7, 1, 64, False),
    # a little more than whole rounds of tiles: the last items alone in parts, tiles that
    # end inside a token's heads
    ([864, 500, 1, 735, 600], [864, 500, 1, 735, 600], None, 1500, 24, 8, 128, True),
    ([384, 200, 10, 303, 384, 95, 300, 250, 384, 90], [390, 200, 0, 303, 700, 95, 1, 250, 384, 90], None,
     1200, 48, 16, 64, True),
    ([480, 200, 10, 303, 480, 300, 400, 227], [480, 200, 10, 303, 480, 300, 400, 227], None, 1500, 48, 16,
     64, True),
    # more sequences than lanes: shared keys with them and apart, long rows, a list of
    # three levels
    ([1 + i % 2 for i in range(300)], [i % 20 for i in range(300)], None, 700, 4, 2, 64, True),
    ([1] * 65, [3] * 65, [i % 4 for i in range(65)], 1500, 8, 1, 128, True),
    ([i % 90 for i in range(100)], [(i * 7) % 160 for i in range(100)], None, 40, 4, 2, 128, True),
    ([0] * 66 + [200, 0, 31], [9] * 66 + [1500, 0, 1], None, 0, 2, 2, 64, False),
    ([i % 3 for i in range(4200)], [(i * 5) % 4 for i in range(4200)], None, 0, 2, 2, 64, False),
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


def test_results_repeat_bit_for_bit():
    import torch
    for case in (CASES[2], CASES[11], CASES[-5]):
        x, _, args, len_k = setup(case, 2)
        runs = []
        for _ in range(3):
            o, lse = forward(x, args, len_k)
            runs.append((o, lse) + backward(x, o, lse, args, len_k))
        t, tk = sum(case[0]), sum(case[1])
        for a in runs[1:]:
            for i, (p, r) in enumerate(zip(a, runs[0])):
                n = (slice(None), slice(0, t)) if i == 1 else slice(0, tk if i in (3, 4) else t if i < 3 else None)
                assert torch.equal(p[n], r[n])


def test_nothing_in_use():
    """No queries: gradients of the keys are zero.  No keys at all: o = 0, lse = -inf."""
    import torch
    from paper_2511_13198_amd import pdyattn
    k = torch.randn(40, 2, 64, device="cuda").to(torch.bfloat16)
    none = torch.empty(0, 4, 64, dtype=torch.bfloat16, device="cuda")
    lse0 = torch.empty(4, 0, device="cuda")
    cq, ck = cu.offsets([0, 0], "cuda"), cu.offsets([30, 10], "cuda")
    dq, dk, dv, dkp, dvp = pdyattn.attn_prefix_bwd(none, k, k, k, k, none, lse0, none, cq, ck,
                                                   dk=torch.full_like(k, 7.0))
    assert dq.shape == none.shape
    for g in (dk, dv, dkp, dvp):
        assert (g == 0).all()
    q = torch.randn(5, 4, 64, device="cuda").to(torch.bfloat16)
    nokeys = torch.empty(0, 2, 64, dtype=torch.bfloat16, device="cuda")
    cq, ck = cu.offsets([2, 3], "cuda"), cu.offsets([0, 0], "cuda")
    o, lse = pdyattn.attn_cross_fwd(q, nokeys, nokeys, cq, ck)
    assert (o == 0).all() and (lse == -math.inf).all()
    dq, dk, dv = pdyattn.attn_cross_bwd(q, nokeys, nokeys, o, lse, q, cq, ck)
    assert (dq == 0).all() and dk.shape == nokeys.shape


def test_not_a_number_and_infinite_logits():
    """A row that sees a NaN or +inf logit gets o = NaN, lse = -inf, whole or in parts;
    one whose logits are all -inf sees nothing; other rows are as without."""
    import torch
    from paper_2511_13198_amd import pdyattn
    for lk in (100, 9000):
        x = make([4], [lk], 0, 2, 2, 128, 3, behind=0)
        cq, ck = cu.offsets([4], "cuda"), cu.offsets([lk], "cuda")
        clean = pdyattn.attn_cross_fwd(x["q"], x["k"], x["v"], cq, ck)
        x["q"][1, 0, 5] = math.nan
        x["q"][2, 1] = math.inf
        o, lse = pdyattn.attn_cross_fwd(x["q"], x["k"], x["v"], cq, ck)
        for t, h in ((1, 0), (2, 1)):
            assert torch.isnan(o[t, h]).all() and lse[h, t] == -math.inf
            o[t, h], lse[h, t] = clean[0][t, h], clean[1][h, t]
        assert torch.equal(o, clean[0]) and torch.equal(lse, clean[1])
        k = x["k"].clone()
        k[:, 0] = -math.inf
        q = x["q"].clone()
        q[:, 0] = 1.0
        o, lse = pdyattn.attn_cross_fwd(q, k, x["v"], cq, ck)
        assert (o[:, 0] == 0).all() and (lse[0] == -math.inf).all()


def test_wrong_offsets_stay_inside():
    """Offsets that fall, leave the tensors or contradict max_seqlen give some result,
    without touching the rows they cannot mean."""
    import torch
    from paper_2511_13198_amd import pdyattn
    x = make([20, 30], [100, 200], 0, 4, 2, 64, 4, behind=0)
    for cq, ck in (([0, 40, 20], [0, 100, 300]), ([0, 20, 5000], [0, 100, 9000]),
                   ([0, -5, 50], [50, 20, 300]), ([0, 1, 50], [0, 0, -1])):
        cq = torch.tensor(cq, dtype=torch.int32, device="cuda")
        ck = torch.tensor(ck, dtype=torch.int32, device="cuda")
        used = torch.tensor([10 ** 9, -7], dtype=torch.int32, device="cuda")
        for len_k in (None, used):
            o, lse = pdyattn.attn_cross_fwd(x["q"], x["k"], x["v"], cq, ck, 30, 200, True,
                                            seqlens_k=len_k)
            pdyattn.attn_cross_bwd(x["q"], x["k"], x["v"], x["q"], torch.zeros_like(lse), x["do"],
                                   cq, ck, 30, 200, True, seqlens_k=len_k)
        torch.cuda.synchronize()


def test_cache_beyond_32_bit_offsets():
    """Keys whose element offsets pass 2^31, at the cache's end."""
    import torch
    from paper_2511_13198_amd import pdyattn
    hkv, d, slots, n = 8, 128, 1 << 18, 9  # 2.4e9 elements
    free, _ = torch.cuda.mem_get_info()
    if free < 24 << 30:
        pytest.skip("needs 24 GiB of device memory")
    k = torch.zeros((n * slots, hkv, d), dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    g = torch.Generator(device="cuda").manual_seed(8)
    used = [3, 0, 5, 1, 0, 0, 0, 7, 700]
    for s, u in enumerate(used):
        for t in (k, v):
            t[s * slots:s * slots + u] = torch.randn((u, hkv, d), generator=g, device="cuda").to(
                torch.bfloat16)
    q = torch.randn((n, 16, d), generator=g, device="cuda").to(torch.bfloat16)
    do = torch.randn((n, 16, d), generator=g, device="cuda").to(torch.bfloat16)
    cq, ck = cu.offsets([1] * n, "cuda"), cu.offsets([slots] * n, "cuda")
    len_k = torch.tensor(used, dtype=torch.int32, device="cuda")
    o, lse = pdyattn.attn_cross_fwd(q, k, v, cq, ck, 1, slots, True, seqlens_k=len_k)
    at = torch.cat([torch.arange(s * slots, s * slots + u) for s, u in enumerate(used)]).cuda()
    ref = cu.reference(q, k[at], v[at], cu.offsets([1] * n), cu.offsets(used), True, d ** -0.5,
                       do=do)
    cu.check("o", o, ref["o"])
    cu.check("lse", lse, ref["lse"])
    dq, dk, dv = pdyattn.attn_cross_bwd(q, k, v, o, lse, do, cq, ck, 1, slots, True,
                                        seqlens_k=len_k, grad_dtype=torch.bfloat16)
    cu.check("dq", dq, ref["dq"])
    cu.check("dk", dk[at], ref["dk"])
    cu.check("dv", dv[at], ref["dv"])
    dk[at] = 0
    assert not dk.any()


@pytest.mark.parametrize("prefix", [0, 1])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("rows", [(3, 1, 17), (300, 2, 70)])
def test_a_row_with_one_key_has_no_gradient(rows, d, prefix):
    """Its P is 1 whatever the key, so dS = P (dP - D) is 0: what is left is P's own
    distance from 1.  The exponent is the difference of the logit m (base 2) and of LSE,
    two products from each other and back, five roundings of 2^-24 |m|; with the power's
    2^-22 and the sum's 2^-24 that is under (1 + |m| / 4) 2^-20 of dP, and dS enters the
    product rounded to bf16.  (With D from a bf16 O it would be up to 2^-8.)"""
    import torch
    from paper_2511_13198_amd import pdyattn
    lk = [0] * len(rows) if prefix else [1] * len(rows)
    hq, hkv, g = 4, 2, 2
    x = make(rows, lk, prefix, hq, hkv, d, seed=d + prefix, behind=0)
    rest = (cu.offsets(rows, "cuda"), cu.offsets(lk, "cuda"), max(rows), max(1, max(lk)) if not prefix
            else 0)
    scale = 1 / math.sqrt(d)
    if prefix:
        ins = (x["q"], x["k"], x["v"], x["kp"], x["vp"])
        o, lse = pdyattn.attn_prefix_fwd(*ins, *rest, scale=scale)
        dq = pdyattn.attn_prefix_bwd(*ins, o, lse, x["do"], *rest, scale=scale)[0]
        key, val = x["kp"][:1].expand(len(rows), -1, -1), x["vp"][:1].expand(len(rows), -1, -1)
    else:
        ins = (x["q"], x["k"], x["v"])
        o, lse = pdyattn.attn_cross_fwd(*ins, *rest, scale=scale)
        dq = pdyattn.attn_cross_bwd(*ins, o, lse, x["do"], *rest, scale=scale)[0]
        key, val = x["k"], x["v"]
    at = torch.repeat_interleave(torch.arange(len(rows)), torch.tensor(rows)).cuda()
    k, v = (t[at].double().repeat_interleave(g, 1) for t in (key, val))
    m = (x["q"].double() * k).sum(2) * scale / math.log(2)
    dp = (x["do"].double() * v).sum(2)
    bound = scale * dp.abs() * (1 + m.abs() / 4) * 2.0 ** -20 * (1 + 2.0 ** -8)
    off = dq.double().abs() / (bound[:, :, None] * k.abs()).clamp_min(1e-30)
    print(f"    worst {float(off.max()):.3f} of its bound", flush=True)
    assert float(off.max()) <= 1.0


def test_no_keys_at_all():
    """Empty k and v: o = 0, lse = -inf, dq = 0."""
    import torch
    from paper_2511_13198_amd import pdyattn
    q = torch.ones((5, 4, 64), dtype=torch.bfloat16, device="cuda")
    k = torch.empty((0, 2, 64), dtype=torch.bfloat16, device="cuda")
    cq, ck = cu.offsets([2, 3], "cuda"), cu.offsets([0, 0], "cuda")
    o, lse = pdyattn.attn_cross_fwd(q, k, k, cq, ck)
    assert not bool(o.any()) and bool((lse == -math.inf).all())
    dq, dk, dv = pdyattn.attn_cross_bwd(q, k, k, o, lse, q, cq, ck)
    assert not bool(dq.any()) and dk.shape == dv.shape == k.shape
