"""The paged key/value cache without a GPU: what the calls refuse, sizes of workspaces, the
built kernels' waits and registers, and the tests' own reference."""
import math
import os
import re

import pytest
import torch

from paper_2511_13198_amd import pdyattn as P
from tests import cross_util as cu
from tests import paged_util as pg
from tests import test_gpu_paged as gpu
from tests import test_isa_lds_waits as isa

FAKE = 0x10000  # aligned, never dereferenced: every call below fails validation first
POOL = dict(n=2, pages=40, page=32, width=10, hkv=2, d=128, e4m3=0)
WRITE = dict(POOL, k=FAKE, v=FAKE, cu=FAKE, table=FAKE, len=FAKE, ks=0, vs=0, t=5, kp=FAKE, vp=FAKE,
             scores=FAKE, stream=None)
FWD = dict(POOL, q=FAKE, kp=FAKE, vp=FAKE, table=FAKE, cu=FAKE, len=FAKE, ks=0, vs=0, t=5, mq=3,
           mk=300, hq=8, causal=1, scale=0.1, o=FAKE, lse=FAKE, scores=FAKE, ws=FAKE, wsb=1 << 40,
           stream=None)
EVICT = dict(POOL, kp=FAKE, vp=FAKE, scores=FAKE, table=FAKE, len=FAKE, new=FAKE + 64, nwidth=4,
             mk=300, budget=100, recent=10, first=4, kept=FAKE, lens=FAKE, ws=FAKE, wsb=1 << 40,
             stream=None)
ORDER = {
    "write": "k v cu table len ks vs n t pages page width hkv d e4m3 kp vp scores stream",
    "fwd": "q kp vp table cu len ks vs n t pages page width mq mk hq hkv d e4m3 causal scale o lse "
           "scores ws wsb stream",
    "evict": "kp vp scores table len new n pages page width nwidth mk hkv d e4m3 budget recent first "
             "kept lens ws wsb stream",
}
ARGS = {"write": WRITE, "fwd": FWD, "evict": EVICT}


def call(kind, **kw):
    a = dict(ARGS[kind], **kw)
    return getattr(P.lib(), f"attn_paged_{kind}")(*[a[x] for x in ORDER[kind].split()])


BAD = [
    (dict(n=0), "num_seqs"), (dict(hkv=0), "head counts"), (dict(page=0), "page_size"),
    (dict(page=24), "page_size"), (dict(page=-16), "page_size"), (dict(pages=-1), "num_pages"),
    (dict(width=-1), "max_pages"), (dict(pages=1 << 30), "too many pages"),
    (dict(width=1 << 26, page=16), "too many pages"), (dict(e4m3=2), "cache_e4m3"),
    (dict(len=0), "seqlens_k"), (dict(len=FAKE + 2), "seqlens_k"), (dict(table=0), "page_table"),
    (dict(kp=0), "k_pages"), (dict(vp=FAKE + 8), "v_pages"), (dict(scores=FAKE + 4), "scores"),
    (dict(hkv=1 << 15), "too many heads"),
]
SCALES = [(dict(e4m3=1), "k_scale"), (dict(e4m3=1, ks=FAKE), "v_scale"), (dict(vs=FAKE), "e4m3 cache"),
          (dict(e4m3=1, ks=FAKE, vs=FAKE + 1), "v_scale")]
OWN = {
    "write": SCALES + [(dict(t=-1), "total_tokens"), (dict(t=1 << 26), "total_tokens"),
                       (dict(cu=0), "cu_seqlens"), (dict(k=0), "k is NULL"), (dict(v=FAKE + 2), "aligned")],
    "fwd": SCALES + [
        (dict(t=-1), "total_q"), (dict(mq=6), "max_seqlen_q"), (dict(mq=0), "max_seqlen_q"),
        (dict(mk=-1), "max_seqlen_k"), (dict(mk=321), "max_seqlen_k"), (dict(hq=3), "multiple"),
        (dict(hq=0), "multiple"), (dict(causal=2), "causal"), (dict(scale=0.0), "scale"),
        (dict(scale=math.nan), "scale"), (dict(cu=FAKE + 1), "cu_seqlens_q"), (dict(q=0), "q is NULL"),
        (dict(o=0), "o is NULL"), (dict(lse=FAKE + 4), "aligned"), (dict(ws=0), "workspace"),
        (dict(t=1 << 28, mq=1), "too large"), (dict(hq=1 << 18), "too many heads")],
    "evict": [
        (dict(budget=0), "budget"), (dict(recent=-1), "recent"), (dict(first=-1), "recent"),
        (dict(recent=97), "recent"), (dict(nwidth=3), "new_table"), (dict(new=0), "new_table"),
        (dict(new=FAKE), "other pages"), (dict(scores=0), "scores"), (dict(kept=0), "kept"),
        (dict(lens=FAKE + 2), "new_lens"), (dict(ws=0), "workspace"), (dict(mk=321), "max_seqlen_k"),
        (dict(budget=1 << 30, nwidth=1 << 26), "too large"), (dict(n=1 << 22), "too large"),
        (dict(n=70000), "too many")],
}


@pytest.mark.parametrize("kind", sorted(ARGS))
def test_refusals(kind):
    for kw, text in BAD + OWN[kind]:
        assert call(kind, **kw) == P.PDY_ERR_INVALID_ARG, (kw, P.last_error())
        assert text in P.last_error(), (kw, P.last_error())
    assert call(kind, d=96) == P.PDY_ERR_UNSUPPORTED and "head_dim" in P.last_error()
    if kind != "write":
        assert call(kind, wsb=16) == P.PDY_ERR_WORKSPACE and f"attn_paged_{kind}" in P.last_error()


def test_nothing_to_do_and_sizes():
    assert call("write", t=0, k=0, v=0, cu=0) == P.PDY_OK
    assert call("fwd", t=0, mq=0, q=0, o=0, ws=0) == P.PDY_OK
    size = P.paged_fwd_workspace_size
    for scores in (False, True):
        assert size(0, 2, 0, 300, 8, 2, 128, scores) >= 256
        assert size(5, 2, 6, 300, 8, 2, 128, scores) == 0 == size(5, 2, 3, 300, 8, 3, 128, scores)
    assert P.paged_evict_workspace_size(2, 300, 2, 100) >= 256
    assert P.paged_evict_workspace_size(2, 300, 2, 0) == 0


def test_shapes_of_launches_and_what_the_gpu_cases_cover():
    """The rules' two sides, and that the GPU tests' cases reach every kernel."""
    def shape(n, q, k, hq, hkv, d, e4m3=False, scores=False):
        return tuple(P.paged_launch_shapes(n * q, n, q, k, hq, hkv, d, e4m3, scores).values())

    # the smallest tile that holds a sequence's rows; few keys whole, more waves where a step
    # is short and a CU has one workgroup at most
    assert shape(4, 1, 1024, 8, 8, 128) == (4, 16, 1, False)
    assert shape(4, 1, 1025, 8, 8, 128)[2] > 1 and shape(8, 1, 2048, 8, 8, 128)[2] == 1
    assert shape(4, 1, 1024, 8, 8, 128, True) == (8, 16, 1, False) == shape(4, 1, 2048, 8, 8, 64)
    assert shape(33, 1, 1024, 8, 8, 128, True)[0] == 4 == shape(4, 1, 4000, 8, 8, 64)[0]
    assert [shape(2, q, 500, 4, 4, 64)[1] for q in (16, 17, 32, 33, 500)] == [16, 32, 32, 64, 64]
    # up to 16 rows leave their logits, while these fit
    assert shape(4, 4, 5000, 16, 4, 64, scores=True)[3] and not shape(4, 5, 5000, 16, 4, 64, scores=True)[3]
    assert not shape(4, 1, 1 << 24, 16, 4, 64, scores=True)[3]
    for bad in (dict(max_seqlen_q=6), dict(max_seqlen_k=-1), dict(hkv=3), dict(d=96)):
        with pytest.raises(P.PdyError):
            P.paged_launch_shapes(**dict(dict(total_q=5, num_seqs=2, max_seqlen_q=3, max_seqlen_k=9,
                                              hq=4, hkv=2, d=64), **bad))
    seen = set()
    for case, (_, _, _, _, d, _, _) in enumerate(gpu.ATTEND):
        for e4m3 in (False, True):
            for scores in (False, True):
                s = gpu.shapes_of(case, e4m3, scores)
                whole = "parts" if s["parts"] > 1 else "whole"
                seen |= {(d, e4m3, s["rows"], whole, s["waves"], scores and s["logits"])}
    want = {(d, e4m3, rows, how, 4, False) for d in (64, 128) for e4m3 in (False, True)
            for rows in (16, 32, 64) for how in ("parts", "whole")}
    want |= {(d, e4m3, 16, how, 4, True) for d in (64, 128) for e4m3 in (False, True)
             for how in ("parts", "whole")}
    want |= {(d, e4m3, 16, "whole", 8, logits) for logits in (False, True)
             for d, e4m3 in ((64, False), (64, True), (128, True))}
    assert not want - seen, sorted(map(str, want - seen))


def test_binding_refuses_host_tensors_types_and_shapes():
    kp = torch.zeros(6, 2, 16, 64, dtype=torch.bfloat16)
    k8 = kp.to(torch.float8_e4m3fn)
    table, lens = torch.zeros(3, 4, dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    q, off = torch.zeros(3, 4, 64, dtype=torch.bfloat16), cu.offsets([1, 1, 1])
    scores, one = torch.zeros(6, 2, 16), torch.ones(2)
    with pytest.raises(TypeError, match="float8_e4m3fn"):
        P.attn_paged_fwd(q, kp.float(), kp, table, off, lens)
    for f in (lambda: P.attn_paged_fwd(q, kp, kp, table, off, lens),
              lambda: P.attn_paged_write(q, q, k8, k8, table, off, lens, one, one),
              lambda: P.attn_paged_evict(kp, kp, scores, table, lens, table, 5)):
        with pytest.raises(ValueError, match="device tensor"):
            f()
    with pytest.raises(ValueError, match="needs scores"):
        P.attn_paged_evict(kp, kp, None, table, lens, table, 5)


def hazards_along_branches(body):
    """isa.lds_wait_hazards along every path of one kernel: a read that is issued in front of
    a branch may be waited for behind it.  Also the number of LDS reads."""
    lines = [x.split(";", 1)[0].rstrip() for x in body.splitlines()]
    lines = [x for x in lines if x.strip() and (re.match(r"^\.LBB\w+:", x) or not x.strip().startswith("."))]
    at = {x[:-1]: i for i, x in enumerate(lines) if x.endswith(":")}
    lgkm = [isa.WAIT.match(x) and isa.LGKM.search(x) for x in lines]
    reads = [isa.LDS_READ.match(x) for x in lines]
    dest = {i: isa._regs(m.group(2)) for i, m in enumerate(reads) if m}
    used = [isa._regs(x[m.end():]) if m else isa._regs(x) for x, m in zip(lines, reads)]
    state = [None] * (len(lines) + 1)  # of the reads in flight: later ones at least
    state[0] = {}
    todo, hazards = [0], set()
    while todo:
        i = todo.pop()
        if i >= len(lines):
            continue
        x, now = lines[i].strip(), dict(state[i])
        for r in now:
            if dest[r] & (used[i] | dest.get(i, set())) and not lgkm[i]:
                hazards.add((lines[r].strip(), x))
        if lgkm[i]:
            n = int(lgkm[i].group(1))
            now = {r: k for r, k in now.items() if k < n}
        if x.startswith("ds_"):  # (writes count as well, and end in order with the reads)
            now = {r: k + 1 for r, k in now.items()}
        if reads[i]:
            now[i] = 0
        to = re.match(r"s_c?branch\w*\s+(\S+)", x)
        after = [at[to.group(1)]] if to else []
        if not x.startswith(("s_branch", "s_endpgm")):
            after.append(i + 1)
        for j in after:
            old = state[j]
            new = dict(now) if old is None else dict(old)
            for r, k in now.items():
                new[r] = min(k, new.get(r, k))
            if new != old:
                state[j] = new
                todo.append(j)
    return sorted(hazards), len(dest)


def test_lds_waits_and_no_scratch():
    asm = isa.device_asm(os.path.join(os.path.dirname(isa.SRC), "paged.hip"))
    kernels = re.findall(r"^_Z\w+:.*?^\.Lfunc_end", asm, re.M | re.S)
    checked = 0
    for body in kernels:
        hazards, reads = hazards_along_branches(body)
        assert not hazards, (body.split(":")[0], hazards[:10])
        checked += reads
    assert checked >= 200 and len(kernels) >= 40
    sizes = re.findall(r"^\s*\.private_segment_fixed_size:\s*(\d+)", asm, re.M)
    assert len(sizes) >= 20 and not any(int(x) for x in sizes)


def test_the_walk_follows_branches():
    """A read whose wait stands behind a branch backwards is covered by it; a path around
    the wait, and a use in front of it, are found."""
    body = """_Z1kv:
.LBB0_1:
    s_waitcnt lgkmcnt({n})
    v_mov_b32 v20, v5
.LBB0_2:
    {first}
    ds_read_b128 v[4:7], v1
    {between}
    s_cbranch_scc1 .LBB0_1
    s_endpgm
"""
    def found(n=0, first="v_mov_b32 v9, v8", between="v_mov_b32 v9, v8"):
        return hazards_along_branches(body.format(n=n, first=first, between=between))[0]

    assert not found()
    assert any("v20" in x[1] for x in found(n=1))
    assert found(between="v_mov_b32 v9, v6") and found(between="v_mov_b32 v4, v8")
    assert found(between="s_cbranch_vccz .LBB0_2")
    assert hazards_along_branches(body)[1] == 1


@pytest.mark.parametrize("e4m3", [False, True])
def test_the_reference_against_the_plain_cache(e4m3):
    """A pool read page by page is the sequence that was written, and the attention over it
    that of the sequence laid out in one piece."""
    lens, lq = [40, 0, 17, 3], [2, 1, 17, 1]
    c = pg.Cache(lens, 2, 64, 16, e4m3, seed=4)
    q, off = pg.queries(lq, 4, 64, seed=4)
    got = pg.attention(c, q, lq, True, 0.125)
    K = torch.zeros(sum(lens), 2, 64, dtype=torch.float64)
    V = torch.zeros_like(K)
    a = 0
    for i, n in enumerate(lens):
        for h in range(2):
            K[a:a + n, h], V[a:a + n, h] = c.keys(i, h)[:2]
        a += n
    want = cu.reference(q, K, V, off, cu.offsets(lens), True, 0.125)
    for name in ("o", "lse"):
        assert torch.allclose(got[name][0], want[name][0], rtol=1e-12, atol=1e-12)
        seen = torch.isfinite(want[name][1])
        assert torch.allclose(got[name][1][seen], want[name][1][seen], rtol=1e-6, atol=1e-12)
    # weights: a row's are 1 together
    rows = sum(4 * min(a, b) if b else 0 for a, b in zip(lq, lens))
    assert abs(float(got["scores"][0].sum()) - rows) < 1e-9
    k, _ = pg.queries(lq, 2, 64, seed=9)
    new = pg.write(c, k, k, lq)
    c.k = new[0]
    at = 0
    for i, (n, m) in enumerate(zip(lens, lq)):
        for t in range(max(0, m - n), m):
            row = c.keys(i, 1)[0][n - m + t]
            x = k[at + t, 1].double()
            step = 2.0 ** -4 * x.abs() + 2.0 ** -10 * float(c.ks[1]) if e4m3 else 0.0
            assert bool(((row - x).abs() <= step).all())
        at += m
    kept, new_lens = pg.evict(c, 10, 3, 2)
    assert new_lens.tolist() == [10, 0, 10, 3]
    assert kept[0, 0, :2].tolist() == [0, 1] and kept[0, 0, -3:].tolist() == [37, 38, 39]
    assert kept[3, 1].tolist() == [0, 1, 2] + [-1] * 7
