"""The paged key/value cache beside what it may not touch: wrong lengths and tables between
guards, evictions that write the lengths in place, the weights of many sequences."""
import math

import pytest
import torch

from paper_2511_13198_amd import pdyattn as P
from tests import cross_util as cu
from tests import paged_util as pg

pytestmark = pytest.mark.gpu


class Guarded:
    """Tensors that lie between stretches of a pattern, which must be there at the end."""

    def __init__(self):
        self.all = []

    def __call__(self, x):
        n, edge = x.nbytes, 4096
        room = torch.full((2 * edge + -(-n // 256) * 256,), 0xA5, dtype=torch.uint8, device="cuda")
        inner = room[edge:edge + n]
        inner.copy_(x.contiguous().view(-1).view(torch.uint8))
        self.all.append((room, edge, n))
        return inner.view(x.dtype).view(x.shape)

    def check(self):
        for room, edge, n in self.all:
            assert bool((room[:edge] == 0xA5).all()) and bool((room[edge + n:] == 0xA5).all())


@pytest.mark.parametrize("most", [None, 2540])
@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("lq", [[1] * 5, [9, 1, 5, 4, 12]])
def test_wrong_lengths_and_tables_between_guards(lq, e4m3, most):
    """Lengths beyond the bound or below 0, pages that do not exist: the other sequences'
    outputs, weights, keys and evictions are theirs, everything else stays."""
    lens, hkv, d, page = [700, 1000, 2500, 64, 333], 2, 64, 16
    ok = (0, 4)
    c = pg.Cache(lens, hkv, d, page, e4m3, "cuda", spare=3, extra=7)
    q, off = pg.queries(lq, 4, d, "cuda", spare=3)
    want = pg.attention(c, q, lq, True, 1 / math.sqrt(d))
    c.len.copy_(torch.tensor([700, 1 << 30, 2500, -5, 333]))
    c.table[2, 5:9] = torch.tensor([1 << 30, -(1 << 31), c.k.shape[0], -1])
    g = Guarded()
    c.k, c.v, c.scores, c.table, c.len = (g(x) for x in (c.k, c.v, c.scores, c.table, c.len))
    before = c.scores.clone()
    width = c.table.shape[1] * page
    o, lse = g(torch.full_like(q, 7.0)), g(torch.full((4, q.shape[0]), 7.0, device="cuda"))
    ws = g(torch.zeros(P.paged_fwd_workspace_size(q.shape[0], 5, max(lq), most or width, 4, hkv, d,
                                                  True), dtype=torch.uint8, device="cuda"))
    P.attn_paged_fwd(q, c.k, c.v, c.table, off, c.len, max(lq), most, **c.scales(),
                     scores=c.scores, out=o, lse=lse, workspace=ws)
    g.check()
    at = off.tolist()
    for i in ok:
        rows = slice(at[i], at[i + 1])
        cu.check("o", o[rows], [x[rows] for x in want["o"]])
        cu.check("lse", lse[:, rows], [x[:, rows] for x in want["lse"]])
        _, _, p, s = c.keys(i, 0)
        for h in range(hkv):
            cu.check("scores", (c.scores[p, h, s] - before[p, h, s]).double(),
                     [x[p, h, s] for x in want["scores"]])
    assert bool((o[at[3]:at[4]] == 0).all()) and bool((lse[:, at[3]:at[4]] == -math.inf).all())
    assert bool((o[at[5]:] == 7).all()) and bool((lse[:, at[5]:] == 7).all())
    # no other weights: what is free or in no sequence's use, and the one without keys
    rest = ~c.live.cuda()
    for i, free in ((1, False), (2, False), (3, True)):
        rest[sorted({p for p, _ in c.rows[i]})] = free
    assert pg.same_bits(c.scores.transpose(1, 2)[rest], before.transpose(1, 2)[rest])

    # writing: what the intact sequences write, and the last of the third, whose page exists
    k, v = (g(pg.queries(lq, hkv, d, "cuda", seed=s, spare=3)[0]) for s in (5, 6))
    pools = [x.clone() for x in (c.k, c.v, c.scores)]
    P.attn_paged_write(k, v, c.k, c.v, c.table, off, c.len, **c.scales(), scores=c.scores)
    g.check()
    whole = pg.write(c, k, v, lq)  # (of all sequences as they would be)
    for i in (0, 2, 4):
        for j in range(lens[i] - lq[i], lens[i]):
            p, s = c.rows[i][j]
            for x, y in zip(pools, whole):
                x, y = (t.view(torch.uint8) if t.dtype == pg.E4M3 else t for t in (x, y))
                x[p, :, s] = y[p, :, s]
    for x, y in zip((c.k, c.v, c.scores), pools):
        assert pg.same_bits(x, y)

    # evicting: the intact sequences' keys to their new pages, the broken ones' to none
    budget, new = 100, c.new_table.clone()
    new[1], new[2], new[3] = -3, 1 << 30, c.k.shape[0]
    kept, lens_out = g(torch.full((5, hkv, budget), 9, dtype=torch.int32, device="cuda")), g(c.len.clone())
    ws = g(torch.zeros(P.paged_evict_workspace_size(5, most or width, hkv, budget),
                       dtype=torch.uint8, device="cuda"))
    c.scores.nan_to_num_()
    pools = [x.clone() for x in (c.k, c.v, c.scores)]
    c.lens = lens
    rank = pg.evict(c, budget, 7, 3)[0]
    P.attn_paged_evict(c.k, c.v, c.scores, c.table, c.len, g(new), budget, recent=7, first=3,
                       max_seqlen_k=most, kept=kept, new_lens=lens_out, workspace=ws)
    g.check()
    assert lens_out.tolist() == [100, 100, 100, 0, 100]
    for i in ok:
        assert torch.equal(kept[i].cpu(), rank[i])
        p, s = (torch.tensor(x, device="cuda") for x in zip(*c.rows[i]))
        j = torch.arange(budget, device="cuda")
        for x in pools:
            bits = x.view(torch.uint8) if x.dtype == pg.E4M3 else x
            for h in range(hkv):
                idx = kept[i, h].long()
                bits[new[i].long()[j // page], h, j % page] = bits[p[idx], h, s[idx]]
    for x, y in zip((c.k, c.v, c.scores), pools):
        assert pg.same_bits(x, y)


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("lens,hkv,d,page,budget,recent,first", [
    ([100, 50, 51, 0, 1], 3, 128, 16, 50, 10, 4),       # (as many would be one launch)
    ([17, 40], 2, 64, 32, 1, 0, 0), ([500, 300], 2, 128, 80, 32, 16, 16),
    ([3000, 2048, 2049], 4, 128, 48, 2048, 64, 4), ([9000, 300], 2, 64, 32, 120, 7, 2),
])
def test_an_eviction_that_writes_the_lengths_in_place(lens, hkv, d, page, budget, recent, first,
                                                      e4m3):
    """kept, pages and lengths are those of the call with lengths of its own, and that is the
    definition's."""
    def make():
        return pg.Cache(lens, hkv, d, page, e4m3, "cuda", seed=2, extra=-(-budget // page))

    def evict(c, **kw):
        return P.attn_paged_evict(c.k, c.v, c.scores, c.table, c.len, c.new_table, budget,
                                  recent=recent, first=first, **kw)

    host = pg.Cache(lens, hkv, d, page, e4m3, seed=2, extra=-(-budget // page))
    want, lens_want = pg.evict(host, budget, recent, first)
    a, b = make(), make()
    kept, new = evict(a)
    kept2, new2 = evict(b, new_lens=b.len)
    assert new2 is b.len and a.len.tolist() == lens
    for x, y in ((kept, kept2), (new, new2)):
        assert torch.equal(x, y)
    assert torch.equal(kept.cpu(), want) and torch.equal(new.cpu(), lens_want)
    for x, y in zip((a.k, a.v, a.scores), (b.k, b.v, b.scores)):
        assert pg.same_bits(x, y)
    j = torch.arange(budget, device="cuda")
    for i, n in enumerate(lens):
        m = min(n, budget)
        if not m:
            continue
        p, s = (torch.tensor(x, device="cuda") for x in zip(*host.rows[i]))
        to = b.new_table[i].long()[j[:m] // page], j[:m] % page
        for h in range(hkv):
            idx = kept2[i, h, :m].long()
            for x, old in ((b.k, host.k), (b.v, host.v), (b.scores, host.scores)):
                got, was = x[to[0], h, to[1]], old.cuda()[p[idx], h, s[idx]]
                assert pg.same_bits(got, was)


def test_weights_of_many_sequences():
    """More sequences than a workgroup has threads: the sums of some of them, of one row's
    total all."""
    n = 3000
    lens = [(61 * i) % 150 for i in range(n - 1)] + [40000]
    c = pg.Cache(lens, 1, 64, 16, False, "cuda")
    q, off = pg.queries([1] * n, 2, 64, "cuda")
    before = c.scores.clone()
    P.attn_paged_fwd(q, c.k, c.v, c.table, off, c.len, 1, 40000, scores=c.scores)
    live = c.live.cuda()
    pick = [0, 1, 17, 1024, 2047, 2998, 2999]
    short = pg.Cache(lens, 1, 64, 16, False, "cuda")
    short.lens, short.rows = [lens[i] for i in pick], [c.rows[i] for i in pick]
    want = pg.attention(short, q[pick].contiguous(), [1] * len(pick), True, 0.125)["scores"]
    for i in pick:
        if lens[i]:
            _, _, p, s = c.keys(i, 0)
            cu.check("scores", (c.scores[p, 0, s] - before[p, 0, s]).double(),
                     [x[p, 0, s] for x in want])
    total = 2.0 * sum(x > 0 for x in lens)
    added = (c.scores.double() - before.double())[live[:, None]]
    assert abs(float(added.sum()) - total) < 1e-4 * total
    assert pg.same_bits(c.scores[~live[:, None]], before[~live[:, None]])
