"""The paged key/value cache on the GPU against its definitions in 64 bits: writing,
attention of one to many rows a sequence, the keys' weights, eviction, and a run of all of
them."""
import math

import pytest
import torch

from paper_2511_13198_amd import pdyattn as P
from tests import cross_util as cu
from tests import paged_util as pg

pytestmark = pytest.mark.gpu

# (new rows, keys in use of the sequences, Hq, Hkv, d, page, causal)
ATTEND = [
    ([1], [1], 1, 1, 64, 16, True),
    ([1, 1], [16, 17], 4, 4, 128, 16, True),
    ([1, 1, 1, 1], [0, 1500, 31, 33], 8, 8, 64, 16, True),
    ([1] * 5, [700, 4096, 1, 0, 2049], 32, 8, 128, 16, True),
    ([1, 1, 1], [5000, 3, 20000], 8, 1, 128, 128, True),
    ([1, 3, 5, 2], [900, 77, 2500, 2], 24, 8, 128, 48, True),
    ([2, 0, 4], [1, 100, 3], 6, 2, 64, 80, True),          # rows without a key
    ([4, 4], [200, 0], 8, 2, 128, 32, False),
    ([7, 1, 8], [300, 64, 1030], 16, 4, 64, 256, True),
    ([5, 6], [640, 33], 7, 1, 128, 112, True),             # 42 packed rows
    ([33, 1, 64], [500, 129, 64], 4, 2, 128, 64, True),    # several tiles of rows
    ([40, 70], [90, 3000], 3, 3, 64, 16, False),
    ([100], [777], 28, 4, 64, 48, True),
    ([1] * 130, [(37 * i) % 211 for i in range(130)], 4, 2, 64, 16, True),
    ([(i % 3) for i in range(300)], [(53 * i) % 90 + 3 for i in range(300)], 2, 1, 128, 32, True),
    ([1], [66000], 4, 2, 64, 64, True),
    ([6, 2, 8], [3000, 100, 5000], 8, 2, 128, 16, True),   # 32 rows, in parts
    ([30, 17], [6000, 2100], 3, 3, 64, 32, True),
    ([12, 40], [7000, 333], 8, 2, 128, 48, True),          # 64 rows and more, in parts
    ([64, 3], [5000, 9000], 1, 1, 64, 128, False),
    ([1] * 40, [(103 * i) % 1500 for i in range(40)], 16, 8, 128, 16, True),  # whole, 4 waves
    ([2, 1], [900, 700], 16, 2, 64, 16, True),             # 16 rows
    ([8, 3], [900, 500], 8, 2, 128, 16, True),             # 32 rows, whole
    # past the caches (more keys than these hold), 32 and 64 rows
    ([30, 32, 20, 1], [16000, 9100, 12345, 3], 16, 16, 64, 64, True),
    ([16, 9], [40000, 28000], 32, 8, 128, 128, True),
]


def run(c, q, cuq, lq, causal, scale=None, scores=None, out=None, **kw):
    hq = q.shape[1]
    lse = torch.full((hq, q.shape[0]), 7.0, device="cuda")
    if out is None:
        out = torch.full_like(q, 7.0)
    return P.attn_paged_fwd(q, c.k, c.v, c.table, cuq, c.len, max(lq), max(max(c.lens), 1),
                            causal=causal, scale=scale, **c.scales(), scores=scores, out=out,
                            lse=lse, **kw)


def shapes_of(case, e4m3, scores):
    """The launch of a case's call, as below."""
    lq, lk, hq, hkv, d, page, causal = ATTEND[case]
    return P.paged_launch_shapes(sum(lq) + 2, len(lq), max(lq), max(max(lk), 1), hq, hkv, d, e4m3,
                                 scores)


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("case", range(len(ATTEND)))
def test_attention_and_weights(case, e4m3):
    lq, lk, hq, hkv, d, page, causal = ATTEND[case]
    c = pg.Cache(lk, hkv, d, page, e4m3, "cuda", seed=case)
    q, cuq = pg.queries(lq, hq, d, "cuda", seed=case, spare=2)
    scale = 0.9 / math.sqrt(d)
    want = pg.attention(c, q, lq, causal, scale)
    T = sum(lq)
    o, lse = run(c, q, cuq, lq, causal, scale)
    before = c.scores.clone()
    o2, lse2 = run(c, q, cuq, lq, causal, scale, scores=c.scores)
    torch.cuda.synchronize()
    print(f"  case {case} e4m3={e4m3}", flush=True)
    # rows of no sequence stay
    assert bool((o[T:] == 7).all()) and bool((lse[:, T:] == 7).all())
    # (the launch that also sums weights may cut the keys otherwise)
    for x, y in ((o, lse), (o2, lse2)):
        cu.check("o", x[:T], [z[:T] for z in want["o"]])
        cu.check("lse", y[:, :T], [z[:, :T] for z in want["lse"]])
    live = c.live.cuda()[:, None].expand_as(before)
    added = c.scores[live].double() - before[live].double()
    cu.check("scores", added, (want["scores"][0][live], want["scores"][1][live]))
    assert pg.same_bits(c.scores[~live], before[~live])


@pytest.mark.parametrize("e4m3,d", [(False, 64), (False, 128), (True, 64), (True, 128)])
@pytest.mark.parametrize("n,most", [(40, 9000), (6, 1000), (300, 1000)])
def test_attention_is_the_same_again_and_beside_the_weights(n, most, e4m3, d):
    """Bit for bit, while the memory is busy: in parts, whole, by 4 and 8 waves."""
    lens = [(977 * i) % most + 1 for i in range(n)]
    c = pg.Cache([1], 8, d, 16, e4m3, "cuda")
    used = [-(-x // 16) for x in lens]
    g = torch.Generator(device="cuda").manual_seed(3)
    shape = (sum(used), 8, 16, d)
    for name in ("k", "v"):
        x = torch.randn(shape, generator=g, device="cuda")
        setattr(c, name, (x * 50).clamp(-448, 448).to(pg.E4M3) if e4m3 else x.to(torch.bfloat16))
    order = torch.randperm(sum(used), generator=g, device="cuda").int()
    c.table = torch.zeros((n, max(used)), dtype=torch.int32, device="cuda")
    at = 0
    for i, x in enumerate(used):
        c.table[i, :x] = order[at:at + x]
        at += x
    c.lens, c.len = lens, torch.tensor(lens, dtype=torch.int32, device="cuda")
    c.scores = torch.zeros(shape[:3], device="cuda")
    q, cuq = pg.queries([1] * n, 32, d, "cuda")
    first = run(c, q, cuq, [1] * n, True)
    runs = [run(c, q, cuq, [1] * n, True, scores=c.scores if i % 2 else None) for i in range(30)]
    for o, lse in runs:
        assert torch.equal(o, first[0]) and torch.equal(lse, first[1])
    again = torch.zeros_like(c.scores)
    for _ in range(15):
        run(c, q, cuq, [1] * n, True, scores=again)
    assert torch.equal(again, c.scores)
    # a row's weights are 1 together
    total = 15.0 * 32 * n
    assert abs(float(again.double().sum()) - total) < 1e-4 * total


@pytest.mark.parametrize("e4m3", [False, True])
def test_weights_of_few_rows_from_the_keys(e4m3):
    """A bound of the lengths for which no logits are left: from the keys, as of many rows."""
    lens, lq, wide = [700, 33, 2100], [1, 0, 3], 1 << 20
    c = pg.Cache(lens, 2, 64, 16, e4m3, "cuda", seed=8)
    table = torch.full((3, wide), -7, dtype=torch.int32, device="cuda")
    table[:, :c.table.shape[1]] = c.table
    c.table = table
    q, cuq = pg.queries(lq, 8, 64, "cuda")
    assert not P.paged_launch_shapes(4, 3, 3, 16 * wide, 8, 2, 64, e4m3, True)["logits"]
    before = c.scores.clone()
    o, lse = P.attn_paged_fwd(q, c.k, c.v, c.table, cuq, c.len, 3, **c.scales(), scores=c.scores)
    want = pg.attention(c, q, lq, True, 0.125)
    cu.check("o", o, want["o"])
    cu.check("lse", lse, want["lse"])
    live = c.live.cuda()[:, None].expand_as(before)
    cu.check("scores", c.scores[live].double() - before[live].double(),
             [x[live] for x in want["scores"]])


WRITE = [
    ([1], [1], 1, 64, 16), ([1, 1, 1], [700, 16, 17], 8, 128, 16), ([3, 0, 5, 1], [3, 9, 900, 48], 3, 64, 48),
    ([300, 1, 77], [1000, 1, 77], 4, 128, 80), ([9, 2], [4, 2], 2, 128, 32),  # tokens in front of key 0
    ([1] * 200, [(31 * i) % 97 + 1 for i in range(200)], 2, 64, 16), ([2500, 1800], [2600, 1800], 1, 64, 256),
]


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("case", range(len(WRITE)))
def test_write(case, e4m3):
    lq, lk, hkv, d, page = WRITE[case]
    c = pg.Cache(lk, hkv, d, page, e4m3, "cuda", seed=case)
    (k, cuq), (v, _) = (pg.queries(lq, hkv, d, "cuda", seed=s, spare=2) for s in (1, 2))
    if case == 1:  # beyond the largest number, infinite, tiny, none, -0
        k[0, 0, :8] = torch.tensor([1e4, -1e4, math.inf, -math.inf, math.nan, 0.0, -0.0, 1e-30])
    want = pg.write(c, k, v, lq)
    P.attn_paged_write(k, v, c.k, c.v, c.table, cuq, c.len, **c.scales(), scores=c.scores)
    for x, y in zip((c.k, c.v, c.scores), want):
        if case == 1:  # (which NaN a NaN becomes is not said)
            x, y = torch.nan_to_num(x.float(), 3.5), torch.nan_to_num(y.float(), 3.5)
        assert pg.same_bits(x, y)
    P.attn_paged_write(k, v, c.k, c.v, c.table, cuq, c.len, **c.scales())
    if case != 1:
        assert pg.same_bits(c.k, want[0])


EVICT = [
    ([100], 1, 64, 16, 50, 0, 0), ([100, 50, 51, 0, 1], 3, 128, 16, 50, 10, 4),
    ([3000, 2048, 2049], 4, 128, 48, 2048, 64, 4), ([17, 40], 2, 64, 32, 1, 0, 0),
    ([17, 40], 2, 64, 32, 1, 1, 0), ([500, 300], 2, 128, 80, 32, 16, 16),  # nothing by score
    ([20000, 7], 2, 64, 128, 4097, 0, 1), ([70000], 1, 64, 256, 100, 3, 0),
    ([9000, 300], 2, 64, 32, 120, 7, 2), ([9000, 300, 12000], 1, 128, 16, 2000, 0, 3),
    # as many keys that may go as a kernel's threads hold, and one more
    ([4112], 1, 64, 16, 400, 16, 0), ([4128], 2, 64, 16, 400, 15, 16),
    ([32800, 32784], 1, 64, 16, 100, 16, 19), ([32800, 32784], 1, 64, 16, 100, 15, 19),
]


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("scores", ["random", "equal", "special"])
@pytest.mark.parametrize("case", range(len(EVICT)))
def test_evict(case, scores, e4m3):
    lens, hkv, d, page, budget, recent, first = EVICT[case]
    c = pg.Cache(lens, hkv, d, page, e4m3, "cuda", seed=case, extra=-(-budget // page))
    if scores == "equal":
        c.scores.fill_(0.5)
    elif scores == "special":
        pick = torch.randint(0, 9, c.scores.shape, device="cuda")
        some = torch.tensor([math.nan, math.inf, -math.inf, 0.0, -0.0, -1.0, 1e-40, 1.0, 1.0000001])
        c.scores.copy_(some.cuda()[pick])
    before = [x.clone() for x in (c.k, c.v, c.scores)]
    host = pg.Cache(lens, hkv, d, page, e4m3, "cpu", seed=case, extra=-(-budget // page))
    host.scores = c.scores.cpu()
    want, lens_want = pg.evict(host, budget, recent, first)
    kept, new = P.attn_paged_evict(c.k, c.v, c.scores, c.table, c.len, c.new_table, budget,
                                   recent=recent, first=first)
    assert torch.equal(kept.cpu(), want) and torch.equal(new.cpu(), lens_want)
    for x, old in zip((c.k, c.v, c.scores), before):
        y = old.clone()
        a, b = (t.view(torch.uint8) if t.dtype == pg.E4M3 else t for t in (y, old))
        for i, n in enumerate(lens):
            m = min(n, budget)
            if not m:
                continue
            j = torch.arange(m, device="cuda")
            p = torch.tensor([r[0] for r in c.rows[i]], device="cuda")
            s = torch.tensor([r[1] for r in c.rows[i]], device="cuda")
            for h in range(hkv):
                idx = kept[i, h, :m].long()
                a[c.new_table[i].long()[j // page], h, j % page] = b[p[idx], h, s[idx]]
        assert pg.same_bits(x, y)


def test_refusals_of_tensors():
    c = pg.Cache([20, 5], 2, 64, 16, False, "cuda", extra=1)
    e = pg.Cache([20, 5], 2, 64, 16, True, "cuda", extra=1)
    q, cu_q = pg.queries([1, 2], 4, 64, "cuda")
    k, _ = pg.queries([1, 2], 2, 64, "cuda")

    def fwd(q=q, k=c.k, v=c.v, table=c.table, off=cu_q, lens=c.len, **kw):
        P.attn_paged_fwd(q, k, v, table, off, lens, 2, 20, **kw)

    def write(k=k, v=k, **kw):
        P.attn_paged_write(k, v, c.k, c.v, c.table, cu_q, c.len, **kw)

    def evict(table=c.new_table, budget=10, **kw):
        P.attn_paged_evict(c.k, c.v, c.scores, c.table, c.len, table, budget, **kw)

    for f, kw, kind, text in [
            (fwd, dict(table=c.table.long()), TypeError, "page_table must be"),
            (fwd, dict(v=e.v), TypeError, "v_pages must be"),
            (fwd, dict(k=c.k.transpose(1, 2), v=c.v.transpose(1, 2)), ValueError, "contiguous"),
            (fwd, dict(v=c.v[:-1]), ValueError, "k_pages' shape"),
            (fwd, dict(lens=c.len[:1]), ValueError, "rows each"),
            (fwd, dict(off=cu_q[:2]), ValueError, "offsets"),
            (fwd, dict(q=q.float()), TypeError, "q must be"),
            (fwd, dict(q=q[:, :, :32].contiguous()), ValueError, "head dimension"),
            (fwd, dict(q=q[:, :3].contiguous()), P.PdyError, "multiple"),
            (fwd, dict(k=e.k, v=e.v), ValueError, "needs k_scale"),
            (fwd, dict(k=e.k, v=e.v, k_scale=e.ks, v_scale=e.vs[:1]), ValueError, "one value"),
            (fwd, dict(k_scale=e.ks, v_scale=e.vs), ValueError, "bf16 one has none"),
            (fwd, dict(scores=c.scores[:, :1].contiguous()), ValueError, "scores must be"),
            (fwd, dict(scores=c.scores.double()), TypeError, "scores must be"),
            (fwd, dict(out=q[:1]), ValueError, "q's shape"),
            (fwd, dict(workspace=torch.empty(64, dtype=torch.uint8, device="cuda")), P.PdyError,
             "workspace"),
            (write, dict(k=q, v=q), ValueError, "pages' Hkv"),
            (write, dict(v=k[:2]), ValueError, "pages' Hkv"),
            (write, dict(k=k.half()), TypeError, "k must be"),
            (evict, dict(table=c.new_table[:1]), ValueError, "num_seqs rows"),
            (evict, dict(table=c.table), P.PdyError, "other pages"),
            (evict, dict(budget=0), P.PdyError, "budget"),
            (evict, dict(budget=17), P.PdyError, "room"),
            (evict, dict(recent=8, first=3), P.PdyError, "together"),
            (evict, dict(kept=torch.empty(2, 2, 9, dtype=torch.int32, device="cuda")), ValueError,
             "kept must be")]:
        with pytest.raises(kind, match=text):
            f(**kw)
