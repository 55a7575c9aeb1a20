"""Scales of any size that the header allows: of the logits, and of an 8-bit cache's heads."""
import math

import pytest
import torch

from paper_2511_13198_amd import pdyattn as P
from tests import cross_util as cu
from tests import paged_util as pg

pytestmark = pytest.mark.gpu


# (new rows: 16 and fewer a kv head, whose weights come from the logits; more: from the keys)
@pytest.mark.parametrize("lq,lens", [([1, 2, 1], [40, 3000, 7]), ([40, 5, 1], [90, 3000, 7])])
@pytest.mark.parametrize("scale,ks", [(1e-30, 1e-20), (1e-38, 1e-30), (1e30, 1e10)])
def test_products_of_scales_beyond_the_range(scale, ks, lq, lens):
    """scale * k_scale rounds to 0, or to infinity, in 32 bits: logits of 0 (there with queries
    of 0) make every visible key weigh the same, masked ones nothing."""
    c = pg.Cache(lens, 2, 64, 16, True, "cuda", seed=3)
    c.ks.fill_(ks)
    q, off = pg.queries(lq, 4, 64, "cuda", seed=3)
    if scale > 1:
        q.zero_()
    want = pg.attention(c, q, lq, True, scale)
    before = c.scores.clone()
    o, lse = P.attn_paged_fwd(q, c.k, c.v, c.table, off, c.len, max(lq), max(lens), scale=scale,
                              **c.scales(), scores=c.scores)
    cu.check("o", o, want["o"])
    cu.check("lse", lse, want["lse"])
    live = c.live.cuda()[:, None].expand_as(before)
    cu.check("scores", c.scores[live].double() - before[live].double(),
             [x[live] for x in want["scores"]])


@pytest.mark.parametrize("top", [-126, -123, -100, -63, 0, 100, 126])
def test_writes_by_scales_of_any_size(top):
    """8-bit values are the 32-bit quotients x / scale rounded to the nearest, for scales
    down to the smallest and up to the largest numbers, and quotients next to a border."""
    hkv, d = 512, 64
    g = torch.Generator().manual_seed(top + 200)
    c = pg.Cache([1], hkv, d, 16, True, seed=1)
    new, want = [], []
    for pool in (c.k, c.v):
        x = (2.0 ** top * (1 + torch.rand(hkv, generator=g, dtype=torch.float64))).to(torch.bfloat16)
        # x / s is next to the middle of two 8-bit numbers, on either side
        middle = (2 * torch.randint(8, 16, (hkv,), generator=g) + 1) / 16.0
        s = (x.double() / middle / 2.0 ** (max(top, 0) // 20)).float()
        s = (s.view(torch.int32) + torch.randint(-1, 2, (hkv,), generator=g).int()).view(torch.float32)
        e = torch.arange(d) % 8 - 4
        x = (x[:, None].double() * 2.0 ** e).to(torch.bfloat16) * (1 - 2 * (e % 2)).to(torch.bfloat16)
        x[:, 0], x[:, 1], x[:, 2] = math.inf, -0.0, -math.inf
        new.append((x[None], s))
        y = (x.float() / s[:, None]).clamp(-448, 448).to(pg.E4M3)
        out = pool.clone()
        p, at = c.rows[0][0]
        out.view(torch.uint8)[p, :, at] = y.view(torch.uint8)
        want.append(out)
    (k, ks), (v, vs) = new
    kp, vp = c.k.cuda(), c.v.cuda()
    P.attn_paged_write(k.cuda().contiguous(), v.cuda().contiguous(), kp, vp, c.table.cuda(),
                       cu.offsets([1], "cuda"), c.len.cuda(), ks.cuda(), vs.cuda())
    for x, y in zip((kp, vp), want):
        assert pg.same_bits(x.cpu(), y)


def test_a_quotient_that_meets_a_border_in_32_bits():
    """1 / 0.04: the scale's 32 bits are a little less than 0.04, the exact quotient a little
    over 25; in 32 bits it is 25, the middle of 24 and 26, and goes to the even one, 24."""
    c = pg.Cache([1], 2, 64, 16, True, "cuda", seed=1)
    s = torch.full((2,), 0.04, device="cuda")
    k = torch.ones((1, 2, 64), dtype=torch.bfloat16, device="cuda")
    assert 1.0 / float(s[0].double()) > 25
    P.attn_paged_write(k, -k, c.k, c.v, c.table, cu.offsets([1], "cuda"), c.len, s, s)
    p, at = c.rows[0][0]
    for x, want in ((c.k, 24.0), (c.v, -24.0)):
        assert bool((x.view(torch.uint8)[p, :, at].view(pg.E4M3).float() == want).all())
