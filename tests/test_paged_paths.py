"""That the GPU cases of the paged attention's rarer paths take them."""
from tests import test_gpu_paged as usual
from tests import test_gpu_paged_paths as gpu


def test_the_cases_take_their_paths():
    seen = set()
    for case in gpu.CASES:
        kind, lq, lens, hq, hkv, d, e4m3, _ = case
        for scores in (False, True):
            s = gpu.shapes_of(case, scores)
            # (up to 4,096 keys may stay whole; beyond them one part is for want of room)
            long = max(lens) > 4096
            how = "parts" if s["parts"] > 1 else "uncut" if long else "whole"
            seen.add((d, e4m3, s["rows"], how, s["waves"], scores and s["logits"],
                      gpu.streams(case)))
            if kind.startswith(("stream", "whole")):
                assert gpu.streams(case), case
            if kind == "uncut":
                assert how == "uncut" and s["rows"] == 16 and s["logits"] == scores, case
            if kind == "parts":
                assert gpu.most_parts(case) > 64 and s["rows"] == 16 and s["logits"] == scores
                assert (sum(lq) + 2) * hq > 512, "joined by a workgroup a row"
    bools = (False, True)
    want = {(d, e4m3, 16, "parts", 4, x, True) for d in (64, 128) for e4m3 in bools for x in bools}
    want |= {(d, e4m3, 16, "whole", 4, x, True) for d in (64, 128) for e4m3 in bools for x in bools}
    want |= {(64, False, 16, "whole", 8, x, True) for x in bools}
    want |= {(d, e4m3, 16, "uncut", 4, x, False) for d in (64, 128) for e4m3 in bools for x in bools}
    want |= {(128, False, 32, "parts", 4, False, True), (128, True, 32, "parts", 4, False, True),
             (64, True, 32, "parts", 4, False, True), (64, False, 64, "parts", 4, False, True),
             (64, True, 64, "parts", 4, False, True)}
    assert not want - seen, sorted(map(str, want - seen))
    # 32 and 64 rows of the other sizes: the usual cases
    for i, rows, d, e4m3 in ((23, 32, 64, False), (24, 64, 128, False), (24, 64, 128, True)):
        lq, lk, hq, hkv, dim, _, _ = usual.ATTEND[i]
        assert dim == d and usual.shapes_of(i, e4m3, True)["rows"] == rows
        assert gpu.streams(("", lq, lk, hq, hkv, d, e4m3, 2))
    groups = {c[3] // c[4] for c in gpu.CASES}
    assert {14, 24, 40, 72} <= groups
