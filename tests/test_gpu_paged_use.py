"""The paged key/value cache as it is used: a prompt and the tokens after it, evictions on
the way, captured graphs, other streams, pages that sequences share, wrong tables and
lengths, keys that are no numbers, a pool beyond 32 bits."""
import math

import pytest
import torch

from paper_2511_13198_amd import pdyattn as P
from tests import cross_util as cu
from tests import paged_util as pg

pytestmark = pytest.mark.gpu
I32 = torch.int32


def fill(n, hkv, d, page, pages, width, e4m3=False, seed=0):
    """An empty cache (NaN everywhere) for n sequences of up to `width` pages each."""
    c = pg.Cache([0] * n, hkv, d, page, e4m3, "cuda", seed=seed, spare=pages)
    order = torch.randperm(pages, generator=torch.Generator().manual_seed(seed)).int()
    c.table = order[:n * width].view(n, width).contiguous().cuda()
    c.free = order[n * width:].tolist()
    c.rows = [[(int(c.table[i, j // page]), j % page) for j in range(width * page)]
              for i in range(n)]
    c.scores.fill_(math.nan)
    return c


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("d,page", [(128, 16), (64, 48)])
def test_a_prompt_its_tokens_and_evictions(d, page, e4m3):
    """Prompts by attn_fwd into the cache, then tokens: rotated, written, attended to with the
    keys' weights; evictions twice.  Every step against 64 bits from the pages' own keys, and
    the keys against those that were written."""
    hq, hkv, budget, recent, first = 8, 2, 96, 16, 2
    lens, width = [150, 1, 97, 40], 6 if page == 48 else 14
    n = len(lens)
    c = fill(n, hkv, d, page, 2 * n * width, width, e4m3)
    g = torch.Generator().manual_seed(2)
    rnd = lambda t, h: torch.randn((t, h, d), generator=g).to(torch.bfloat16).cuda()  # noqa: E731
    spare = torch.tensor(c.free[:n * width], dtype=I32).view(n, width).cuda()
    T = sum(lens)
    q, k, v = rnd(T, hq), rnd(T, hkv), rnd(T, hkv)
    off = cu.offsets(lens, "cuda")
    pos = torch.cat([torch.arange(x) for x in lens]).int().cuda()
    q, k = P.attn_rotary(q, k, pos, (d // 2,))
    P.attn_fwd(q, k, v, off, max(lens))
    c.len = torch.tensor(lens, dtype=I32, device="cuda")
    P.attn_paged_write(k, v, c.k, c.v, c.table, off, c.len, **c.scales(), scores=c.scores)
    kept = [[list(range(x)) for _ in range(hkv)] for x in lens]  # of the keys ever written
    ever = [[k[int(off[i]):int(off[i + 1]), h] for h in range(hkv)] for i in range(n)]
    # the last rows of every prompt give its keys their first weights
    tail = [min(x, 8) for x in lens]
    rows = torch.cat([torch.arange(int(off[i + 1]) - t, int(off[i + 1])) for i, t in enumerate(tail)])
    step = [(q[rows.cuda()].contiguous(), tail)]
    total = list(lens)
    for turn in range(5):
        if turn:
            q1, k1, v1 = rnd(n, hq), rnd(n, hkv), rnd(n, hkv)
            p1 = torch.tensor(total, dtype=I32, device="cuda")
            q1, k1 = P.attn_rotary(q1, k1, p1, (d // 2,))
            one = cu.offsets([1] * n, "cuda")
            c.len += 1
            P.attn_paged_write(k1, v1, c.k, c.v, c.table, one, c.len, **c.scales(), scores=c.scores)
            for i in range(n):
                for h in range(hkv):
                    kept[i][h].append(total[i])
                    ever[i][h] = torch.cat([ever[i][h], k1[i:i + 1, h]])
                total[i] += 1
            step = [(q1, [1] * n)]
        c.lens = c.len.tolist()
        c.rows = [[(int(c.table[i, j // page]), j % page) for j in range(c.lens[i])]
                  for i in range(n)]
        qs, lq = step[0]
        before = c.scores.clone()
        o, lse = P.attn_paged_fwd(qs, c.k, c.v, c.table, cu.offsets(lq, "cuda"), c.len, max(lq),
                                  **c.scales(), scores=c.scores)
        want = pg.attention(c, qs, lq, True, 1 / math.sqrt(d))
        cu.check("o", o, want["o"])
        cu.check("lse", lse, want["lse"])
        for i in range(n):
            for h in range(hkv):
                K, _, p, s = c.keys(i, h)
                cu.check("scores", (c.scores[p, h, s] - before[p, h, s]).double(),
                         [x[p, h, s] for x in want["scores"]])
                # the pages hold the keys that were written and stayed
                x = ever[i][h][torch.tensor(kept[i][h], device="cuda")].double()
                near = 2.0 ** -4 * x.abs() + 2.0 ** -10 * float(c.ks[h]) if e4m3 else 0 * x
                assert bool(((K - x).abs() <= near).all())
        if turn in (1, 3):
            c2 = [[[float(c.scores[a, h, b]) for a, b in c.rows[i]] for h in range(hkv)]
                  for i in range(n)]
            out, c.len = P.attn_paged_evict(c.k, c.v, c.scores, c.table, c.len, spare, budget,
                                            recent=recent, first=first)
            c.table, spare = spare, c.table
            for i in range(n):
                for h in range(hkv):
                    now = [x for x in out[i, h].tolist() if x >= 0]
                    m = len(c2[i][h])
                    if m <= budget:
                        assert now == list(range(m))
                    else:
                        assert now[:first] == list(range(first))
                        assert now[-recent:] == list(range(m - recent, m)) and len(now) == budget
                        gone = set(range(m)) - set(now)
                        assert max(c2[i][h][j] for j in gone) <= min(c2[i][h][j] for j in now[first:-recent])
                    kept[i][h] = [kept[i][h][j] for j in now]


def decode(c, q, k, v, off, scores, out, lse, ws, most):
    P.attn_paged_write(k, v, c.k, c.v, c.table, off, c.len, scores=scores)
    return P.attn_paged_fwd(q, c.k, c.v, c.table, off, c.len, 1, most, scores=scores, out=out,
                            lse=lse, workspace=ws)


def test_captured_steps_follow_lengths_and_tables():
    """Two graphs that share a workspace, replayed in turn, with eager work on the same
    tensors between them; lengths, tables and tokens change between replays."""
    n, hq, hkv, d, page, width, most = 6, 8, 2, 128, 16, 300, 4800
    c = fill(n, hkv, d, page, n * width + 4, width)
    c.k.zero_(), c.v.zero_(), c.scores.zero_()
    g = torch.Generator(device="cuda").manual_seed(1)
    q, k, v = (torch.zeros((n, h, d), dtype=torch.bfloat16, device="cuda") for h in (hq, hkv, hkv))
    off = cu.offsets([1] * n, "cuda")
    ws = torch.empty(P.paged_fwd_workspace_size(n, n, 1, most, hq, hkv, d, True), dtype=torch.uint8,
                     device="cuda")
    outs = [(torch.zeros_like(q), torch.zeros((hq, n), device="cuda")) for _ in range(2)]
    c.len.fill_(1)
    decode(c, q, k, v, off, c.scores, *outs[0], ws, most)
    torch.cuda.synchronize()
    graphs = []
    for use in (True, False):  # with the weights, without
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            decode(c, q, k, v, off, c.scores if use else None, *outs[use], ws, most)
        graphs.append(graph)
    for turn in range(6):
        c.len.copy_(torch.tensor([(711 * (turn + 1) * (i + 1)) % most + 1 for i in range(n)]))
        c.table.copy_(c.table.view(-1)[torch.randperm(n * width, generator=g, device="cuda")].view(n, width))
        for t in (q, k, v):
            t.copy_(torch.randn(t.shape, generator=g, device="cuda"))
        c.k.copy_(torch.randn(c.k.shape, generator=g, device="cuda"))
        c.v.copy_(torch.randn(c.v.shape, generator=g, device="cuda"))
        c.scores.zero_()
        use = turn % 2 == 0
        graphs[turn % 2].replay()
        got = [x.clone() for x in (*outs[use], c.k, c.scores)]
        ws.fill_(255)
        c.scores.zero_()
        eager = decode(c, q, k, v, off, c.scores if use else None, None, None, None, most)
        for a, b in zip(got, (*eager, c.k, c.scores)):
            assert torch.equal(a, b)
        torch.cuda.synchronize()


def test_on_a_stream_of_the_callers():
    """Calls go to the current stream: behind what stands there, beside the default one."""
    c = pg.Cache([500, 900, 33], 2, 64, 16, False, "cuda")
    q, off = pg.queries([1, 1, 1], 4, 64, "cuda")
    want = P.attn_paged_fwd(q, c.k, c.v, c.table, off, c.len, 1, 900)
    late = torch.zeros_like(q)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        x = torch.randn(4096, 4096, device="cuda")
        for _ in range(20):
            x = x @ x / 64
        late.copy_(q)
        got = P.attn_paged_fwd(late, c.k, c.v, c.table, off, c.len, 1, 900)
    side.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_shared_pages():
    """Sequences with a common beginning read the same pages; their own copies give the same."""
    page, d, hkv = 16, 128, 2
    c = pg.Cache([200, 150, 90], hkv, d, page, False, "cuda", spare=40)
    q, off = pg.queries([1, 2, 1], 8, d, "cuda")
    shared = c.table.clone()
    shared[1, :5] = shared[0, :5]  # 80 keys
    shared[2, :5] = shared[0, :5]
    for i in (1, 2):
        for j in range(80):
            c.rows[i][j] = c.rows[0][j]
    o, lse = P.attn_paged_fwd(q, c.k, c.v, shared, off, c.len, 2)
    want = pg.attention(c, q, [1, 2, 1], True, 1 / math.sqrt(d))
    cu.check("o", o, want["o"])
    cu.check("lse", lse, want["lse"])


@pytest.mark.parametrize("scores", [False, True])
@pytest.mark.parametrize("most", [None, 2540])
def test_wrong_lengths_and_tables_cost_their_own_sequence_alone(most, scores):
    """Lengths beyond the bound or below 0, pages that do not exist: no stray access, the
    other sequences as ever."""
    lens = [700, 1000, 2500, 64]
    c = pg.Cache(lens, 2, 64, 16, False, "cuda", spare=3)
    q, off = pg.queries([1] * 4, 4, 64, "cuda")
    good = P.attn_paged_fwd(q, c.k, c.v, c.table, off, c.len, 1, most)
    before = c.scores.clone()
    c.len.copy_(torch.tensor([700, 1 << 30, 2500, -5]))
    c.table[2, 5:9] = torch.tensor([1 << 30, -(1 << 31), c.k.shape[0], -1])
    o, lse = P.attn_paged_fwd(q, c.k, c.v, c.table, off, c.len, 1, most,
                              scores=c.scores if scores else None)
    torch.cuda.synchronize()
    cu.check("o", o[:1], (good[0][:1].double(), 0.01 * good[0][:1].double().abs() + 1e-2))
    assert bool((o[3] == 0).all()) and bool((lse[:, 3] == -math.inf).all())
    k, _ = pg.queries([1] * 4, 2, 64, "cuda", seed=5)
    pages = c.k.clone()
    P.attn_paged_write(k, k, c.k, c.v, c.table, off, c.len, scores=c.scores)
    p, s = c.rows[0][699]
    assert torch.equal(c.k[p, :, s], k[0])
    c.k[p, :, s] = pages[p, :, s]
    p, s = c.rows[2][2499]
    assert torch.equal(c.k[p, :, s], k[2])
    c.k[p, :, s] = pages[p, :, s]
    # (nothing else: a key in no page, in front of the first, or beyond the table is dropped)
    assert pg.same_bits(c.k, pages)
    kept, new = P.attn_paged_evict(c.k, c.v, before.nan_to_num(), c.table, c.len,
                                   torch.full((4, 10), -3, dtype=I32, device="cuda"), 100,
                                   new_lens=c.len)
    assert pg.same_bits(c.k, pages) and new.tolist() == [100, 100, 100, 0] and new is c.len


@pytest.mark.parametrize("d", [64, 128])
def test_keys_that_are_no_numbers(d):
    """A NaN or infinite key in use makes its rows NaN with lse = -inf, adds no weights, and
    touches no other sequence or head; logits of any size are numbers like others."""
    lens = [300, 5000, 40]
    c = pg.Cache(lens, 2, d, 16, False, "cuda")
    q, off = pg.queries([1] * 3, 4, d, "cuda")
    q[2] *= 300.0
    want = pg.attention(c, q, [1] * 3, True, 1.0)
    p, s = c.rows[0][123]
    c.k[p, 0, s, 3] = math.nan
    p, s = c.rows[1][4321]
    c.k[p, 1, s] = torch.where(q[1, 2] > 0, math.inf, -math.inf)
    before = c.scores.clone()
    o, lse = P.attn_paged_fwd(q, c.k, c.v, c.table, off, c.len, 1, 5000, scale=1.0,
                              scores=c.scores)
    bad = [(0, 0), (0, 1), (1, 2)]
    for t, h in bad:
        assert bool(o[t, h].isnan().all()) and float(lse[h, t]) == -math.inf
    for t, h in [(t, h) for t in range(3) for h in range(4) if (t, h) not in bad and (t, h) != (1, 3)]:
        cu.check("o", o[t, h], [x[t, h] for x in want["o"]])
    for t, e in ((0, 1), (1, 0), (2, 0), (2, 1)):
        _, _, p, s = c.keys(t, e)
        cu.check("scores", (c.scores[p, e, s] - before[p, e, s]).double(),
                 [x[p, e, s] for x in want["scores"]])
    _, _, p, s = c.keys(0, 0)
    assert pg.same_bits(c.scores[p, 0, s], before[p, 0, s])


@pytest.mark.parametrize("e4m3", [False, True])
def test_a_pool_beyond_32_bits(e4m3):
    """Pages whose elements lie beyond 2^32, and a cache of another pool with the same keys."""
    hkv, d, page, lens = 2, 128, 256, [3000, 70, 600]
    small = pg.Cache(lens, hkv, d, page, e4m3, "cuda", seed=6, extra=2)
    far = (1 << 32) // (hkv * d * page) + 5
    pages = far + small.k.shape[0]
    big = pg.Cache(lens, hkv, d, page, e4m3, "cuda", seed=6, extra=2)
    big.k = torch.empty((pages, hkv, page, d), dtype=small.k.dtype, device="cuda")
    big.v = torch.empty_like(big.k)
    big.scores = torch.zeros((pages, hkv, page), device="cuda")
    for name in ("k", "v", "scores"):
        getattr(big, name)[far:].view(torch.uint8).copy_(getattr(small, name).view(torch.uint8))
    big.table, big.new_table = small.table + far, small.new_table + far
    q, off = pg.queries([1, 2, 1], 8, d, "cuda")
    k, _ = pg.queries([1, 2, 1], hkv, d, "cuda", seed=3)
    got = []
    for c in (small, big):
        P.attn_paged_write(k, k, c.k, c.v, c.table, off, c.len, **c.scales(), scores=c.scores)
        o = P.attn_paged_fwd(q, c.k, c.v, c.table, off, c.len, 2, 3000, **c.scales(), scores=c.scores)
        kept = P.attn_paged_evict(c.k, c.v, c.scores, c.table, c.len, c.new_table, 500)
        got.append((*o, *kept))
    for x, y in zip(*got):
        assert torch.equal(x, y)
    for name in ("k", "v", "scores"):
        assert pg.same_bits(getattr(big, name)[far:], getattr(small, name))


def test_many_sequences():
    """More sequences than a workgroup has threads, several times over."""
    n = 3000
    lens = [(61 * i) % 150 for i in range(n - 1)] + [40000]
    c = pg.Cache(lens, 1, 64, 16, False, "cuda")
    q, off = pg.queries([1] * n, 2, 64, "cuda")
    o, lse = P.attn_paged_fwd(q, c.k, c.v, c.table, off, c.len, 1, scores=c.scores)
    short = pg.Cache(lens, 1, 64, 16, False, "cuda")
    pick = [0, 1, 17, 1024, 2047, 2998, 2999]
    short.lens, short.rows = [lens[i] for i in pick], [c.rows[i] for i in pick]
    want = pg.attention(short, q[pick].contiguous(), [1] * len(pick), True, 0.125)
    cu.check("o", o[pick], want["o"])
    cu.check("lse", lse[:, pick], want["lse"])
