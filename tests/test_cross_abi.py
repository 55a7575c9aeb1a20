"""Cross attention, shared-prefix attention and rotary positions without a GPU: what the
calls refuse, sizes and shapes of launches, and the tests' own reference."""
import ctypes
import math

import pytest
import torch

from paper_2511_13198_amd import pdyattn as P
from tests import cross_util as cu
from tests import test_gpu_cross as gpu

FAKE = 0x10000  # aligned, never dereferenced: every call below fails validation first
FWD = dict(q=FAKE, k=FAKE, v=FAKE, kp=FAKE, vp=FAKE, cu_q=FAKE, cu_k=FAKE, len_k=0, prefix=100,
           n=2, tq=64, tk=500, mq=40, mk=300, hq=8, hkv=2, d=128, causal=1, scale=0.1, o=FAKE,
           lse=FAKE, ws=FAKE, wsb=1 << 40, stream=None)
BWD = dict(FWD, do=FAKE, bf16=1, dq=FAKE, dk=FAKE, dv=FAKE, dkp=FAKE, dvp=FAKE)


def call(kind, name, **kw):
    a = dict(FWD if kind == "fwd" else BWD, **kw)
    pre = name == "prefix"
    args = [a["q"], a["k"], a["v"]] + ([a["kp"], a["vp"]] if pre else [])
    if kind == "bwd":
        args += [a["o"], a["lse"], a["do"]]
    args += [a["cu_q"], a["cu_k"], a["len_k"]] + ([a["prefix"]] if pre else [])
    args += [a[x] for x in ("n", "tq", "tk", "mq", "mk", "hq", "hkv", "d", "causal", "scale")]
    if kind == "bwd":
        args += [a["bf16"], a["dq"], a["dk"], a["dv"]] + ([a["dkp"], a["dvp"]] if pre else [])
    else:
        args += [a["o"], a["lse"]]
    return getattr(P.lib(), f"attn_{name}_{kind}")(*args, a["ws"], a["wsb"], a["stream"])


BAD = [
    (dict(tq=-1), "total_q"), (dict(tk=-1), "total_q"), (dict(n=0), "num_seqs"),
    (dict(mq=65), "max_seqlen_q"), (dict(mq=0), "max_seqlen_q"), (dict(mk=501), "max_seqlen_k"),
    (dict(mk=-1), "max_seqlen_k"), (dict(hq=6, hkv=4), "multiple"), (dict(hkv=0), "head counts"),
    (dict(causal=2), "causal"), (dict(scale=0.0), "scale"), (dict(scale=math.inf), "scale"),
    (dict(cu_q=0), "cu_seqlens_q"), (dict(cu_k=FAKE + 2), "cu_seqlens_k"),
    (dict(len_k=FAKE + 1), "seqlens_k"), (dict(q=0), "q is NULL"), (dict(k=FAKE + 8), "aligned"),
    (dict(v=0), "v is NULL"), (dict(o=0), "o is NULL"), (dict(lse=FAKE + 4), "aligned"),
    (dict(ws=0), "workspace"), (dict(tq=1 << 27, hq=32), "too large"),
    (dict(hq=1 << 17, hkv=2), "too many heads"), (dict(hq=1 << 15, hkv=1 << 15), "too many heads"),
    (dict(n=1 << 25), "too large"),
]
BAD_BWD = [(dict(do=0), "dout is NULL"), (dict(dq=FAKE + 2), "aligned"), (dict(dk=0), "dk is NULL"),
           (dict(dv=0), "dv is NULL"), (dict(bf16=2), "grad_bf16")]
BAD_PREFIX = [(dict(prefix=-1), "prefix_len"), (dict(kp=0), "k_prefix"), (dict(vp=FAKE + 8), "v_prefix")]


@pytest.mark.parametrize("name", ["cross", "prefix"])
@pytest.mark.parametrize("kind", ["fwd", "bwd"])
def test_refusals(kind, name):
    bad = BAD + (BAD_BWD if kind == "bwd" else []) + (BAD_PREFIX if name == "prefix" else [])
    if kind == "bwd" and name == "prefix":
        bad = bad + [(dict(dkp=0), "dk_prefix"), (dict(dvp=0), "dv_prefix")]
    for kw, text in bad:
        assert call(kind, name, **kw) == P.PDY_ERR_INVALID_ARG, (kw, P.last_error())
        assert text in P.last_error(), (kw, P.last_error())
    assert call(kind, name, d=96) == P.PDY_ERR_UNSUPPORTED and "head_dim" in P.last_error()
    assert call(kind, name, wsb=16) == P.PDY_ERR_WORKSPACE and f"attn_{name}_{kind}" in P.last_error()


def test_nothing_to_do():
    for name in ("cross", "prefix"):
        assert call("fwd", name, tq=0, mq=0, q=0, o=0, ws=0) == P.PDY_OK
    assert call("bwd", "cross", tq=0, mq=0, tk=0, mk=0, q=0, dq=0, ws=0) == P.PDY_OK
    assert call("bwd", "prefix", prefix=0, tq=0, mq=0, tk=0, mk=0, q=0, dq=0, ws=0) == P.PDY_OK


def test_sizes_without_queries_or_keys():
    for prefix in (0, 40, 4000):
        for tq, tk in ((0, 0), (0, 50), (50, 0)):
            sizes = (tq, tk, 2, min(tq, 30), min(tk, 30), 8, 2, 128)
            assert P.prefix_fwd_workspace_size(prefix, *sizes) >= 256
            assert P.prefix_bwd_workspace_size(prefix, *sizes) >= 256
            s = P.cross_launch_shapes(prefix, *sizes)
            assert (s["cross_dq_kernel"] == (0, 0, 0)) == (tq == 0)
            assert (s["cross_dkdv_kernel"] == (0, 0, 0)) == (tk + prefix == 0)


def test_workspace_sizes():
    size = P.cross_fwd_workspace_size
    assert size(64, 500, 2, 40, 300, 8, 2, 128) >= 256
    assert size(64, 500, 2, 65, 300, 8, 2, 128) == 0 and size(64, 500, 2, 40, 300, 8, 3, 128) == 0
    # many rows need none, few rows their partial results: under 260 MiB
    assert size(65536, 65536, 8, 8192, 8192, 32, 8, 128) == 256
    for args in ((64, 1 << 20, 64, 1, 16384, 32, 8, 128), (1024, 1 << 20, 32, 32, 16384, 32, 8, 128),
                 (1, 1 << 20, 1, 1, 1 << 20, 8, 8, 64)):
        assert 256 < size(*args) < 260 << 20
    # D, counts and partial gradients: under D + 780 MiB
    for prefix in (0, 1000, 32768):
        for args in ((64, 1 << 16, 64, 1, 4096, 32, 8, 128), (16384, 16384, 16, 2048, 2048, 32, 8, 128),
                     (8, 1 << 20, 2, 4, 1 << 20, 8, 8, 64)):
            need = P.prefix_bwd_workspace_size(prefix, *args)
            d = args[5] * args[0] * 4
            assert d <= need < d + (780 << 20)
    # a prefix whose rows' partial results would be larger stays with each sequence
    assert not P.cross_launch_shapes(4000, 1 << 20, 1 << 20, 1 << 20, 1, 1, 8, 8, 128)["apart"]


def test_shapes_of_launches_and_what_the_gpu_cases_cover():
    """The rules' two sides, and that the GPU tests' cases reach every kernel and
    combining path at both head dimensions."""
    def shape(n, q, k, hq, hkv, d, pre=0, causal=False):
        return P.cross_launch_shapes(pre, n * q, n * k, n, q, k, hq, hkv, d, causal)

    # up to 64 rows the smallest tile that holds them; a group's heads are rows
    for rows, fwd, dq in ((32, (4, 4), (4, 2)), (33, (4, 2), (4, 2)), (64, (4, 2), (4, 2))):
        s = shape(2, rows, 500, 4, 4, 128)
        assert s["cross_fwd_kernel"][:2] == fwd and s["cross_dq_kernel"][:2] == dq
        assert shape(2, rows // 4, 500, 16, 4, 128)["cross_fwd_kernel"][:2] == few(rows // 4 * 4)
    # then by the estimate: small tiles for launches that do not fill the chip, the
    # largest, whole, for those that do, parts where few rows see many keys
    assert shape(4, 300, 600, 3, 1, 128)["cross_fwd_kernel"] == (4, 2, 1)
    assert shape(50, 80, 464, 16, 16, 128)["cross_fwd_kernel"] == (4, 1, 1)
    assert shape(64, 512, 512, 32, 32, 128)["cross_fwd_kernel"] == (8, 1, 1)
    assert shape(1, 200, 30000, 16, 16, 128)["cross_fwd_kernel"][2] > 8
    # shared keys apart for few rows behind many of them; not where all keys are few, nor
    # (more of them) where the sequences fill the chip several times
    assert shape(4, 1, 200, 8, 2, 128, 513)["apart"] and not shape(4, 1, 200, 8, 2, 128, 512)["apart"]
    assert not shape(4, 1, 100, 8, 2, 128, 540)["apart"] and shape(4, 1, 101, 8, 2, 128, 540)["apart"]
    assert shape(300, 1, 10, 8, 4, 128, 257)["apart"] and not shape(200, 1, 10, 8, 4, 128, 257)["apart"]
    assert not shape(4, 17, 100, 8, 2, 128, 4000)["apart"]
    seen = set()
    for lq, lk, used, prefix, hq, hkv, d, causal in gpu.CASES:
        s = P.cross_launch_shapes(prefix, sum(lq) + 3, sum(lk) + 3, len(lq), max(lq), max(lk), hq,
                                  hkv, d, causal)
        for kernel in ("cross_fwd_kernel", "cross_dq_kernel", "cross_dkdv_kernel"):
            w, g, parts = s[kernel]
            seen |= {(kernel, w, g, d), (kernel, "parts" if parts > 1 else "whole", d)}
        seen |= {("apart", s["apart"], d), ("fwd whole first", s["fwd_whole_first"], d),
                 ("dq whole first", s["dq_whole_first"], d)}
    want = {("cross_fwd_kernel", *s, d) for s in ((4, 4), (4, 2), (4, 1), (8, 1)) for d in (64, 128)}
    want |= {("cross_dq_kernel", *s, d) for s in ((4, 2), (4, 1), (8, 1)) for d in (64, 128)}
    want |= {("cross_dkdv_kernel", *s, d) for s in ((4, 1), (8, 2)) for d in (64, 128)}
    want.add(("cross_dkdv_kernel", 8, 1, 128))
    want |= {(k, p, d) for k in ("cross_fwd_kernel", "cross_dq_kernel", "cross_dkdv_kernel")
             for p in ("parts", "whole") for d in (64, 128)}
    want |= {(what, a, d) for a in (True, False) for d in (64, 128)
             for what in ("apart", "fwd whole first", "dq whole first")}
    assert not want - seen, sorted(map(str, want - seen))


def few(rows):
    return (4, 4) if rows <= 32 else (4, 2)


def test_shape_query_refusals():
    with pytest.raises(P.PdyError):
        P.cross_launch_shapes(0, 10, 10, 2, 11, 5, 8, 8, 128)
    assert P.lib().pdy_cross_launch_shapes(0, 10, 10, 2, 5, 5, 8, 8, 128, 0, None) == P.PDY_ERR_INVALID_ARG
    assert set(P.cross_launch_shapes(0, 0, 0, 2, 0, 0, 8, 8, 128).values()) == {(0, 0, 0), False}


def test_binding_refuses_host_tensors_types_and_shapes():
    q, k = torch.zeros(4, 2, 64, dtype=torch.bfloat16), torch.zeros(6, 2, 64, dtype=torch.bfloat16)
    cq, ck = cu.offsets([1, 3]), cu.offsets([2, 4])
    with pytest.raises(ValueError, match="device tensor"):
        P.attn_cross_fwd(q, k, k, cq, ck)
    with pytest.raises(TypeError, match="q must be"):
        P.attn_cross_fwd(q.float(), k, k, cq, ck)
    with pytest.raises(ValueError, match="needs k_prefix"):
        P.attn_prefix_fwd(q, k, k, None, None, cq, ck)
    with pytest.raises(ValueError, match="needs k_prefix"):
        P.attn_prefix_bwd(q, k, k, k, None, q, None, q, cq, ck)
    with pytest.raises(ValueError, match="device tensor"):
        P.attn_rotary(q, k, torch.zeros(4, 1, dtype=torch.int32), (32,))
    with pytest.raises(ValueError, match="needs q or k"):
        P.attn_rotary(None, None, torch.zeros(4, 1, dtype=torch.int32), (32,))
    with pytest.raises(TypeError, match="bfloat16 or torch.float32"):
        P.attn_rotary(q.half(), None, torch.zeros(4, 1, dtype=torch.int32), (32,))
    with pytest.raises(ValueError, match="out_k without k"):
        P.attn_rotary(q, None, torch.zeros(4, 1, dtype=torch.int32), (32,), out_k=k)


def rotary(**kw):
    turns, axes = (ctypes.c_uint64 * 32)(), (ctypes.c_int32 * 32)()
    for i, x in enumerate(kw.pop("axis", [0] * 32)):
        axes[i] = x
    a = dict(q=FAKE, k=FAKE, pos=FAKE, t=10, axes=1, hq=4, hkv=2, d=64, pairs=32,
             turns=ctypes.addressof(turns), pa=ctypes.addressof(axes), inter=0, inv=0, inf=0,
             outf=0, qo=FAKE, ko=FAKE, stream=None)
    a.update(kw)
    return P.lib().attn_rotary(*a.values())


@pytest.mark.parametrize("kw,text", [
    (dict(t=-1), "total_tokens"), (dict(t=1 << 26), "total_tokens"), (dict(axes=0), "num_axes"), (dict(axes=5), "num_axes"),
    (dict(hq=0, hkv=0), "head counts"), (dict(hq=-1), "head counts"), (dict(pairs=33), "num_pairs"),
    (dict(pairs=12), "num_pairs"), (dict(pairs=0), "num_pairs"), (dict(pairs=40), "num_pairs"),
    (dict(inter=2), "interleaved"), (dict(inv=-1), "inverse"), (dict(turns=None), "turns"),
    (dict(pa=None), "pair_axes"), (dict(axis=[0] * 31 + [1]), "pair_axes"), (dict(q=0), "q is NULL"),
    (dict(ko=FAKE + 8), "aligned"), (dict(pos=0), "positions"), (dict(pos=FAKE + 2), "positions"),
    (dict(inf=1, outf=0), "in place"),
])
def test_rotary_refusals(kw, text):
    assert rotary(**kw) == P.PDY_ERR_INVALID_ARG, P.last_error()
    assert text in P.last_error()


def test_rotary_unsupported_and_nothing_to_do():
    assert rotary(d=96) == P.PDY_ERR_UNSUPPORTED and rotary(outf=1) == P.PDY_ERR_UNSUPPORTED
    assert rotary(t=0, q=0, k=0, pos=0, qo=0, ko=0) == P.PDY_OK
    assert P.lib().attn_rotary_turns(None, 3, None) == P.PDY_ERR_INVALID_ARG
    for bad in (math.nan, math.inf):
        with pytest.raises(P.PdyError, match="not finite"):
            P._rotary_tables((8,), 10000.0, (bad,) * 8)
    with pytest.raises(ValueError, match="freqs must have"):
        P._rotary_tables((8,), 10000.0, (1.0,) * 7)
    with pytest.raises(ValueError, match="sections"):
        P._rotary_tables((9, -1), 10000.0, None)


@pytest.mark.parametrize("w", [0.0, 1.0, -1.0, 1e-12, 3.7e5, -0.3, 2 * math.pi, 1e300])
def test_turns_are_the_frequencies_modulo_a_turn(w):
    from fractions import Fraction
    x, y = (ctypes.c_double * 1)(w), (ctypes.c_uint64 * 1)()
    assert P.lib().attn_rotary_turns(x, 1, y) == P.PDY_OK
    if abs(w) > 1e15:
        return  # (a step of such a number is many turns: any fraction does)
    pi = Fraction(3141592653589793238462643383279502884197, 10 ** 39)
    turns = Fraction(w) / (2 * pi) % 1
    off = abs(Fraction(y[0], 2 ** 64) - turns)
    # half a step of the quotient in 64 bits, and the fraction's own last bit
    assert min(off, 1 - off) <= Fraction(max(1, int(abs(w)))) / 2 ** 62


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("prefix", [0, 3])
def test_reference_gradients_are_differences(causal, prefix):
    """The reference's gradients against central differences of sum(dout * o), in 64
    bits, for every input, grouped heads and rows without keys among them."""
    g = torch.Generator().manual_seed(3)
    lq, lk, used = [3, 0, 2], [4, 2, 1], [2, 2, 1]
    rnd = lambda n, h: torch.randn((n, h, 2), generator=g, dtype=torch.float64)  # noqa: E731
    x = {"q": rnd(5, 4), "k": rnd(7, 2), "v": rnd(7, 2)}
    if prefix:
        x.update(kp=rnd(prefix, 2), vp=rnd(prefix, 2))
    do = rnd(5, 4)

    def run(do=None):
        return cu.reference(x["q"], x["k"], x["v"], cu.offsets(lq), cu.offsets(lk), causal, 0.7,
                            used, x.get("kp"), x.get("vp"), do)

    grads = run(do)
    for name, t in x.items():
        got = grads["d" + name][0]
        for i in range(t.numel()):
            flat, h = t.view(-1), 1e-5
            keep = float(flat[i])
            flat[i] = keep + h
            up = float((run()["o"][0] * do).sum())
            flat[i] = keep - h
            down = float((run()["o"][0] * do).sum())
            flat[i] = keep
            assert abs((up - down) / (2 * h) - float(got.view(-1)[i])) < 1e-7, (name, i)


def test_a_planted_mistake_is_seen():
    """A lost key, a shifted mask and a wrong scale are far outside the bounds."""
    g = torch.Generator().manual_seed(5)
    rnd = lambda n, h: torch.randn((n, h, 64), generator=g).to(torch.bfloat16)  # noqa: E731
    q, k, v = rnd(40, 2), rnd(300, 1), rnd(300, 1)
    cq, ck = cu.offsets([40]), cu.offsets([300])
    ref = cu.reference(q, k, v, cq, ck, True, 0.125)["o"]
    cu.check("o", ref[0].to(torch.bfloat16), ref)
    for other in (cu.reference(q, k, v, cq, ck, True, 0.125, [299]),
                  cu.reference(q, k, v, cq, ck, False, 0.125),
                  cu.reference(q, k, v, cq, ck, True, 0.13)):
        with pytest.raises(AssertionError):
            cu.check("o", other["o"][0].to(torch.bfloat16), ref)
