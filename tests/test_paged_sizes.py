"""Sizes and tensors at the edges of what the paged cache's calls take, without a GPU."""
from paper_2511_13198_amd import pdyattn as P
from tests.test_paged_abi import FAKE, call


def test_workspaces_of_the_largest_sizes():
    """The logits' bytes of the largest sizes pass 64 bits: more than may be left, so none."""
    size = P.paged_fwd_workspace_size
    most = (1 << 30) - 16
    for n in ((1 << 31) - 33, (1 << 27) + 1, 1 << 28, (1 << 30) + 5):
        assert size(16, n, 16, most, 1, 1, 64, True) == size(16, n, 16, most, 1, 1, 64, False)
        assert not P.paged_launch_shapes(16, n, 16, most, 1, 1, 64, with_scores=True)["logits"]
    for scores in (False, True):
        assert size(1 << 20, 1 << 20, 1, most, 256, 256, 64, scores) < (2 << 30)


def test_an_evictions_new_lengths_beside_the_old():
    """All of the old lengths, or none of them: a part would be read after it was written."""
    for off in (-4, 4):
        assert call("evict", len=FAKE + 64, lens=FAKE + 64 + off) == P.PDY_ERR_INVALID_ARG
        assert "new_lens" in P.last_error()
    # (in place, in front of and behind: refused for the next reason)
    for off in (-8, 0, 8):
        assert call("evict", len=FAKE + 64, lens=FAKE + 64 + off, wsb=0) == P.PDY_ERR_WORKSPACE


def test_refused_numbers_of_sequences():
    """As the header has them: 65,535 sequences with scores and of evictions, and the grids."""
    for kw in (dict(n=65536), dict(n=65535, mk=512 * 129, width=4200)):
        assert call("fwd", **kw) == P.PDY_ERR_INVALID_ARG and "too large" in P.last_error()
    assert call("evict", n=65536) == P.PDY_ERR_INVALID_ARG and "too many" in P.last_error()
    for kw in (dict(n=65535, hkv=65), dict(n=65535, hkv=3, budget=1 << 14, nwidth=1 << 9)):
        assert call("evict", **kw) == P.PDY_ERR_INVALID_ARG and "too large" in P.last_error()
