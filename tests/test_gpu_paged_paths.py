"""Ways through the paged attention that small caches do not take, against the definitions in
64 bits: keys read past the caches, items that are not cut because partial results of the
batch would not fit, rows of more parts than a wave has lanes, groups of many heads."""
import math

import pytest
import torch

from paper_2511_13198_amd import pdyattn as P
from tests import cross_util as cu
from tests import paged_util as pg

pytestmark = pytest.mark.gpu

# (name, new rows, keys in use, Hq, Hkv, d, e4m3, rows of no sequence)
LONG = [40000, 33, 30000, 0, 12345]
CASES = [
    # past the caches, in parts
    ("stream16", [1] * 5, LONG, 16, 8, 128, False, 2),
    ("stream16", [1] * 5, LONG, 16, 8, 128, True, 2),
    ("stream16", [2, 1, 8, 1, 3], LONG, 32, 16, 64, False, 2),
    ("stream16", [2, 1, 8, 1, 3], LONG, 32, 16, 64, True, 2),
    ("stream32", [8, 3, 7], [50000, 30000, 5], 32, 8, 128, False, 2),
    ("stream32", [8, 3, 7], [50000, 30000, 5], 32, 8, 128, True, 2),
    ("stream32", [8, 3, 7], [50000, 30000, 5], 64, 16, 64, True, 2),
    ("stream64", [16, 9], [50000, 30000], 64, 16, 64, False, 2),
    ("stream64", [16, 9], [50000, 30000], 64, 16, 64, True, 2),
    # past the caches, whole: 4 waves, 8 waves
    ("whole4", [1] * 24, [1400 + 27 * i for i in range(24)], 16, 8, 128, False, 2),
    ("whole4", [1] * 40, [1280 + 19 * i for i in range(40)], 16, 8, 128, True, 2),
    ("whole4", [1] * 40, [1280 + 19 * i for i in range(40)], 16, 8, 64, False, 2),
    ("whole4", [1] * 72, [1900 + 2 * i for i in range(72)], 16, 8, 64, True, 2),
    ("whole8", [1] * 32, [2100 + 61 * i for i in range(32)], 16, 8, 64, False, 2),
    # not cut, because of rows that are no sequence's
    ("uncut", [8, 1, 5, 0], [9000, 4097, 33, 500], 32, 16, 128, False, 2100),
    ("uncut", [8, 1, 5, 0], [9000, 4097, 33, 500], 32, 16, 128, True, 2100),
    ("uncut", [8, 1, 5, 0], [9000, 4097, 33, 500], 32, 16, 64, False, 4100),
    ("uncut", [8, 1, 5, 0], [9000, 4097, 33, 500], 32, 16, 64, True, 4100),
    # a wave joins more parts than it has lanes: up to 129, and up to 256
    ("parts", [1] * 17, [70000] + [37 * i for i in range(16)], 32, 8, 128, False, 2),
    ("parts", [1] * 17, [37 * i for i in range(16)] + [70000], 32, 8, 64, True, 2),
    ("parts", [1] * 17, [70000] + [37 * i for i in range(16)], 32, 2, 64, False, 2),
    ("parts", [1] * 17, [70000] + [37 * i for i in range(16)], 32, 2, 128, True, 2),
    # heads of a group: 14 and 24 (odd tiles of 16 and 32), 40, 72 with several tokens
    ("group", [1, 1, 0], [300, 2500, 7], 28, 2, 128, False, 2),
    ("group", [1, 2, 1], [300, 2500, 7], 48, 2, 64, True, 2),
    ("group", [1, 1, 1], [300, 2500, 0], 40, 1, 128, True, 2),
    ("group", [3, 1], [300, 2500], 72, 1, 64, False, 2),
]


def shapes_of(case, scores):
    _, lq, lens, hq, hkv, d, e4m3, spare = case
    return P.paged_launch_shapes(sum(lq) + spare, len(lq), max(lq), max(lens), hq, hkv, d, e4m3,
                                 scores)


def streams(case):
    """Whether the keys in use are more than 128 MB of K and V, where one tile holds a
    sequence's rows."""
    _, lq, lens, hq, hkv, d, e4m3, _ = case
    rows = max(lq) * hq // hkv
    steps = sum(-(-n // 32) for n in lens)
    return rows <= 64 and steps > (128 << 20) // (hkv * 64 * d * (1 if e4m3 else 2))


def most_parts(case):
    """Parts of the longest sequence, by the rule that the kernel follows."""
    _, lq, lens, hq, hkv, d, e4m3, spare = case
    steps = [-(-n // 32) for n in lens]
    entries = -(-1024 // hkv)
    cap = max(8, int(sum(steps) / entries + 1))
    return min(shapes_of(case, False)["parts"], -(-max(steps) // cap))


class Big(pg.Cache):
    """A cache drawn on the GPU."""

    def __init__(self, lens, hkv, d, page, e4m3, seed=0):
        super().__init__([1], hkv, d, page, e4m3, "cuda", seed=seed)  # (for the scales)
        g = torch.Generator(device="cuda").manual_seed(seed)
        used = [-(-n // page) for n in lens]
        pool = sum(used) + 3
        order = torch.randperm(pool, generator=g, device="cuda").int()
        self.lens = list(lens)
        self.len = torch.tensor(lens, dtype=torch.int32, device="cuda")
        self.table = torch.full((len(lens), max(used) + 1), -1, dtype=torch.int32, device="cuda")
        live = torch.zeros((pool, page), dtype=torch.bool, device="cuda")
        self.at = []
        first = 0
        for i, n in enumerate(lens):
            self.table[i, :used[i]] = order[first:first + used[i]]
            j = torch.arange(n, device="cuda")
            self.at.append((self.table[i][j // page].long(), j % page))
            live[self.at[i]] = True
            first += used[i]
        self.live = live
        for name in ("k", "v"):
            x = torch.randn((pool, hkv, page, d), generator=g, device="cuda")
            x = (x * 50).clamp_(-448, 448).to(pg.E4M3) if e4m3 else x.to(torch.bfloat16)
            bits = x.view(torch.uint8) if e4m3 else x.view(torch.int16)
            bits.masked_fill_(~live[:, None, :, None], 0x7f if e4m3 else 0x7fc0)
            setattr(self, name, x)
        w = torch.rand((pool, hkv, page), generator=g, device="cuda")
        self.scores = w.masked_fill_(~live[:, None], math.nan)

    def keys(self, i, h):
        p, s = self.at[i]
        out = []
        for x, scale in ((self.k, self.ks), (self.v, self.vs)):
            y = (x.view(torch.uint8)[p, h, s].view(pg.E4M3) if self.e4m3 else x[p, h, s]).double()
            out.append(y if scale is None else y * scale[h].double())
        return out[0], out[1], p, s


def check_norms(o, want, lq):
    """Of every sequence the error's norm, which the bounds of single elements (sums of
    roundings that all go one way) leave far off over many keys.  A rounding to bf16 of
    either sign is off by at most 2^-8 / sqrt(3) of a value in the mean square; those of P
    against values v of either sign add up to that share of O's norm, and O's own rounding
    to as much: sqrt(2) 2^-8 / sqrt(3) = 3.2e-3 together, a tenth more for the sample."""
    a = 0
    for nq in lq:
        x, y = o[a:a + nq].double(), want[a:a + nq]
        assert float((x - y).norm()) <= 3.5e-3 * float(y.norm())
        a += nq


@pytest.mark.parametrize("case", range(len(CASES)))
def test_attention_and_weights(case):
    kind, lq, lens, hq, hkv, d, e4m3, spare = CASES[case]
    print(f"  case {case} {kind}", flush=True)
    c = Big(lens, hkv, d, 16 if case % 2 else 48, e4m3, seed=case)
    q, off = pg.queries(lq, hq, d, "cuda", seed=case, spare=spare)
    T, scale = sum(lq), 0.9 / math.sqrt(d)
    want = pg.attention(c, q, lq, True, scale)
    before = c.scores.clone()
    live = c.live[:, None].expand_as(before)
    for scores in (None, c.scores):
        o, lse = torch.full_like(q, 7.0), torch.full((hq, q.shape[0]), 7.0, device="cuda")
        P.attn_paged_fwd(q, c.k, c.v, c.table, off, c.len, max(lq), max(lens), scale=scale,
                         **c.scales(), scores=scores, out=o, lse=lse)
        cu.check("o", o[:T], [x[:T] for x in want["o"]])
        check_norms(o, want["o"][0], lq)
        cu.check("lse", lse[:, :T], [x[:, :T] for x in want["lse"]])
        assert bool((o[T:] == 7).all()) and bool((lse[:, T:] == 7).all())
    cu.check("scores", c.scores[live].double() - before[live].double(),
             [x[live] for x in want["scores"]])
    assert pg.same_bits(c.scores[~live], before[~live])
