"""Rotary positions with several axes against complex multiplication in 64 bits.

Bounds: an angle is off by about 2^-32 of a turn, its sine and cosine by at most
2^-22 with the roundings of the remainder and the sums; two products and a sum in 32
bits add 2^-23 of their size: 4 2^-22 (|x| + |y|) in all, plus half a step (2^-8 of
the value) of a bf16 output."""
import math

import pytest

pytestmark = pytest.mark.gpu


def reference(x, pos, sections, freqs, interleaved, inverse):
    import torch
    x = x.double()
    out = x.clone()
    pairs = sum(sections)
    size = torch.zeros_like(x)
    axis = [a for a, n in enumerate(sections) for _ in range(n)]
    for p in range(pairs):
        i, j = (2 * p, 2 * p + 1) if interleaved else (p, p + pairs)
        t = pos[:, axis[p]].double() * freqs[p] * (-1 if inverse else 1)
        z = torch.complex(x[..., i], x[..., j]) * torch.polar(torch.ones_like(t), t)[:, None]
        out[..., i], out[..., j] = z.real, z.imag
        size[..., i] = size[..., j] = x[..., i].abs() + x[..., j].abs()
    return out, size


def check(got, x, ref):
    import torch
    val, size = ref
    bound = 2.0 ** -20 * size
    if got.dtype == torch.bfloat16:
        bound = bound + 2.0 ** -8 * val.abs()
    off = (got.double() - val).abs()
    worst = float((off / bound.clamp_min(1e-30)).max()) if off.numel() else 0.0
    print(f"    worst {worst:.3f} of its bound", flush=True)
    assert worst <= 1.0


CASES = [
    # (tokens, Hq, Hkv, d, sections, interleaved, largest position)
    (1, 1, 1, 64, (32,), False, 10),
    (19, 32, 8, 128, (64,), False, 640000),
    (333, 5, 3, 128, (16, 24, 24), False, 4096),
    (1000, 4, 4, 64, (7, 0, 25), False, 2 ** 31 - 1),
    (77, 3, 1, 128, (10, 14), True, 5000),
    (257, 2, 2, 64, (8, 8, 8, 8), True, 100),
    (64, 8, 2, 64, (8,), False, 50),
    (4100, 6, 2, 128, (32, 32), True, 1000),
]


def inputs(case, dtype, seed=0):
    import torch
    t, hq, hkv, d, sections, _, top = case
    g = torch.Generator(device="cuda").manual_seed(seed)
    q = torch.randn((t, hq, d), generator=g, device="cuda").to(dtype)
    k = torch.randn((t, hkv, d), generator=g, device="cuda").to(dtype)
    pos = torch.randint(-top, top, (t, len(sections)), generator=g, device="cuda",
                        dtype=torch.int32)
    return q, k, pos


def spectrum(sections, base=10000.0):
    n = sum(sections)
    return [base ** (-p / n) for p in range(n)]


@pytest.mark.parametrize("inverse", [False, True])
@pytest.mark.parametrize("types", ["bfloat16 bfloat16", "float32 float32", "float32 bfloat16"])
@pytest.mark.parametrize("case", CASES, ids=lambda c: f"t{c[0]}h{c[1]}kv{c[2]}d{c[3]}s{sum(c[4])}")
def test_rotation(case, types, inverse):
    import torch
    from paper_2511_13198_amd import pdyattn
    tin, tout = (getattr(torch, t) for t in types.split())
    q, k, pos = inputs(case, tin)
    sections, inter = case[4], case[5]
    oq = torch.full(q.shape, math.nan, dtype=tout, device="cuda")
    ok = torch.full(k.shape, math.nan, dtype=tout, device="cuda")
    pdyattn.attn_rotary(q, k, pos, sections, interleaved=inter, inverse=inverse, out_q=oq, out_k=ok)
    w = spectrum(sections)
    check(oq, q, reference(q, pos, sections, w, inter, inverse))
    check(ok, k, reference(k, pos, sections, w, inter, inverse))


def test_in_place_own_frequencies_and_one_tensor():
    import torch
    from paper_2511_13198_amd import pdyattn
    q, k, pos = inputs((100, 4, 2, 128, (16,), False, 3000), torch.float32, 3)
    w = [0.0, -1.5, 7.0, 1e-9] + [0.3 / (p + 1) for p in range(12)]
    want = reference(q, pos, (16,), w, False, False)
    x = q.clone()
    got, none = pdyattn.attn_rotary(x, None, pos[:, 0].contiguous(), (16,), freqs=w, out_q=x)
    assert none is None and got is x
    check(x, q, want)
    assert torch.equal(x[..., 32:], q[..., 32:]), "elements behind the pairs"
    # and back: two rotations of an element are within twice the bound of one
    pdyattn.attn_rotary(x, None, pos, (16,), freqs=w, inverse=True, out_q=x)
    size = torch.maximum(want[1], q.abs().double())
    assert float(((x.double() - q.double()).abs() / (2.0 ** -19 * size.clamp_min(1e-30))).max()) < 2
    only_k = pdyattn.attn_rotary(None, k, pos, (16,), freqs=w)[1]
    check(only_k, k, reference(k, pos, (16,), w, False, False))


def test_the_inverse_is_the_gradient():
    """<rotate(dx), g> = <dx, unrotate(g)> for every element's difference dx."""
    import torch
    from paper_2511_13198_amd import pdyattn
    q, _, pos = inputs((3, 1, 1, 64, (20, 12), False, 500), torch.float32, 5)
    g = torch.randn_like(q)
    back = pdyattn.attn_rotary(g, None, pos, (20, 12), inverse=True)[0]
    eye = torch.eye(64, device="cuda")[None, :, :].expand(3, 64, 64).contiguous()
    cols = pdyattn.attn_rotary(eye, None, pos, (20, 12))[0]  # head e: rotate(unit e)
    want = (cols.double() * g.double()).sum(2)
    size = (cols.abs().double() * g.abs().double()).sum(2)
    assert float(((back[:, 0].double() - want).abs() / size.clamp_min(1e-30)).max()) < 2.0 ** -19


def test_not_a_number_stays_in_its_pair():
    import torch
    from paper_2511_13198_amd import pdyattn
    q, k, pos = inputs((40, 4, 2, 128, (32,), False, 900), torch.bfloat16, 7)
    clean = pdyattn.attn_rotary(q, k, pos, (32,))[0]
    q[3, 1, 5], q[3, 2, 100] = math.nan, math.inf
    got = pdyattn.attn_rotary(q, k, pos, (32,))[0]
    assert torch.isnan(got[3, 1, 5]) and torch.isnan(got[3, 1, 37]) and got[3, 2, 100] == math.inf
    got[3, 1, 5], got[3, 1, 37], got[3, 2, 100] = clean[3, 1, 5], clean[3, 1, 37], clean[3, 2, 100]
    assert torch.equal(got, clean)


def test_empty_batch():
    import torch
    from paper_2511_13198_amd import pdyattn
    q = torch.empty((0, 4, 64), dtype=torch.bfloat16, device="cuda")
    pos = torch.empty((0, 1), dtype=torch.int32, device="cuda")
    assert pdyattn.attn_rotary(q, None, pos, (32,))[0].shape == (0, 4, 64)
