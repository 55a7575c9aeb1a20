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
