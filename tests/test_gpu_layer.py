"""The operators together, as a model's layer and its serving loop use them: rotated
packed attention, shared prefixes, cross attention, token by token over a cache; on
other streams, in captured graphs, and the ring with rotated shards."""
import math

import pytest

from tests import cross_util as cu

pytestmark = pytest.mark.gpu


def normal(g, *shape):
    import torch
    return torch.randn(shape, generator=g, device="cuda").to(torch.bfloat16)


def test_shared_prefix_is_the_packed_batch_with_the_prefix_in_every_sequence():
    """Rows behind shared keys see what the same rows see in a causal batch whose
    sequences all start with them."""
    import torch
    from paper_2511_13198_amd import pdyattn
    g = torch.Generator(device="cuda").manual_seed(1)
    for lens, prefix, hq, hkv, d in (([5, 1, 12], 700, 8, 2, 128), ([200, 33], 130, 4, 4, 64)):
        T = sum(lens)
        q, k, v, do = normal(g, T, hq, d), normal(g, T, hkv, d), normal(g, T, hkv, d), normal(g, T, hq, d)
        qp, kp, vp = normal(g, prefix, hq, d), normal(g, prefix, hkv, d), normal(g, prefix, hkv, d)
        c = cu.offsets(lens, "cuda")
        o, lse = pdyattn.attn_prefix_fwd(q, k, v, kp, vp, c, c)
        grads = pdyattn.attn_prefix_bwd(q, k, v, kp, vp, o, lse, do, c, c)
        full = [prefix + n for n in lens]
        zero = torch.zeros_like(qp)
        cat = lambda x, p: torch.cat([y for s in torch.split(x, lens) for y in (p, s)])  # noqa: E731
        own = torch.cat([torch.arange(a + prefix, a + n) for a, n in
                         zip(cu.offsets(full).tolist(), full)]).cuda()
        cf = cu.offsets(full, "cuda")
        Q, K, V, G = cat(q, qp), cat(k, kp), cat(v, vp), cat(do, zero)
        of, lf = pdyattn.attn_fwd(Q, K, V, cf)
        gf = pdyattn.attn_bwd(Q, K, V, of, lf, G, cf)
        ref = cu.reference(q, k, v, c, c, True, d ** -0.5, None, kp, vp, do)
        for name, a in (("o", o), ("dq", grads[0]), ("dk", grads[1]), ("dv", grads[2])):
            b = of if name == "o" else gf[("dq", "dk", "dv").index(name)]
            cu.check(name, a, ref[name])
            cu.check(name, b[own], ref[name])
        assert float((lse - lf[:, own]).abs().max()) < 1e-4
        first = torch.cat([torch.arange(a, a + prefix) for a in cu.offsets(full).tolist()[:-1]]).cuda()
        for mine, theirs, name in ((grads[3], gf[1], "dkp"), (grads[4], gf[2], "dvp")):
            cu.check(name, mine, ref[name])
            cu.check(name, theirs[first].view(len(lens), prefix, hkv, d).sum(0), ref[name])


def test_tokens_one_by_one_over_a_cache_are_the_prompt():
    """Prompts in one call, and the same tokens one at a time (and three at a time) over
    a cache with room: the same rows, shared prefix or not."""
    import torch
    from paper_2511_13198_amd import pdyattn
    g = torch.Generator(device="cuda").manual_seed(2)
    hq, hkv, d, slots = 8, 2, 128, 40
    lens = [9, 30, 1, 17]
    n, T = len(lens), sum(lens)
    for prefix in (0, 900):
        q, k, v = normal(g, T, hq, d), normal(g, T, hkv, d), normal(g, T, hkv, d)
        kp, vp = (normal(g, prefix, hkv, d) for _ in range(2)) if prefix else (None, None)
        c = cu.offsets(lens, "cuda")
        ref = cu.reference(q, k, v, c, c, True, d ** -0.5, None, kp, vp)["o"]
        run = (lambda qq, kk, vv, *a, **kw: pdyattn.attn_prefix_fwd(qq, kk, vv, kp, vp, *a, **kw)) \
            if prefix else pdyattn.attn_cross_fwd
        whole, _ = run(q, k, v, c, c, causal=True)
        cu.check("o", whole, ref)
        kc = torch.full((n * slots, hkv, d), math.nan, dtype=torch.bfloat16, device="cuda")
        vc = torch.full_like(kc, math.inf)
        ck = cu.offsets([slots] * n, "cuda")
        starts = cu.offsets(lens).tolist()[:-1]
        for step in (1, 3):
            for t0 in range(0, max(lens), step):
                rows = [list(range(t0, min(t0 + step, m))) for m in lens]
                at = torch.tensor([starts[s] + i for s, r in enumerate(rows) for i in r], device="cuda")
                to = torch.tensor([s * slots + i for s, r in enumerate(rows) for i in r], device="cuda")
                kc[to], vc[to] = k[at], v[at]
                used = torch.tensor([min(t0 + step, m) for m in lens], dtype=torch.int32, device="cuda")
                cq = cu.offsets([len(r) for r in rows], "cuda")
                o, _ = run(q[at], kc, vc, cq, ck, step, slots, True, seqlens_k=used)
                cu.check("o", o, (ref[0][at], ref[1][at]))


def layer(x, c_img, c_txt, pos_img, pos_txt, ws):
    """Image patches attend among themselves with rows' and columns' positions; text
    behind a shared prompt attends causally, then to its image; and all the way back."""
    from paper_2511_13198_amd import pdyattn as P
    sec_i, sec_t = (16, 16), (32,)
    img, mi = c_img
    txt, mt = c_txt
    qi, ki = P.attn_rotary(x["qi"], x["ki"], pos_img, sec_i)
    oi, li = P.attn_fwd(qi, ki, x["vi"], img, mi, False, workspace=ws["a"])
    qt, kt = P.attn_rotary(x["qt"], x["kt"], pos_txt, sec_t)
    ot, lt = P.attn_prefix_fwd(qt, kt, x["vt"], x["kp"], x["vp"], txt, txt, mt, mt, workspace=ws["b"])
    oc, lc = P.attn_cross_fwd(ot, oi, x["vi"], txt, img, mt, mi, workspace=ws["c"])
    dot, doi, dvc = P.attn_cross_bwd(ot, oi, x["vi"], oc, lc, x["do"], txt, img, mt, mi,
                                     grad_dtype=ot.dtype, workspace=ws["d"])
    dqt, dkt, dvt, dkp, dvp = P.attn_prefix_bwd(qt, kt, x["vt"], x["kp"], x["vp"], ot, lt, dot, txt,
                                                txt, mt, mt, workspace=ws["e"])
    dqi, dki, dvi = P.attn_bwd(qi, ki, x["vi"], oi, li, doi, img, mi, False, workspace=ws["f"])
    dqt, dkt = P.attn_rotary(dqt, dkt, pos_txt, sec_t, inverse=True, out_q=dqt, out_k=dkt)
    dqi, dki = P.attn_rotary(dqi, dki, pos_img, sec_i, inverse=True, out_dtype=ot.dtype)
    return {"oc": oc, "lc": lc, "ot": ot, "oi": oi, "dqt": dqt, "dkt": dkt, "dvt": dvt, "dkp": dkp,
            "dvp": dvp, "dqi": dqi, "dki": dki, "dvi": dvi, "dvc": dvc}


def layer_inputs(seed, li, lt, prefix=300, hq=4, hkv=4, d=64):
    import torch
    from paper_2511_13198_amd import pdyattn as P
    g = torch.Generator(device="cuda").manual_seed(seed)
    ti, tt, n = sum(li), sum(lt), len(li)
    x = {"qi": normal(g, ti, hq, d), "ki": normal(g, ti, hkv, d), "vi": normal(g, ti, hkv, d),
         "qt": normal(g, tt, hq, d), "kt": normal(g, tt, hkv, d), "vt": normal(g, tt, hkv, d),
         "kp": normal(g, prefix, hkv, d), "vp": normal(g, prefix, hkv, d), "do": normal(g, tt, hq, d)}
    pos_i = torch.stack([torch.arange(ti, device="cuda") // 16, torch.arange(ti, device="cuda") % 16],
                        1).int()
    pos_t = torch.arange(tt, device="cuda", dtype=torch.int32)[:, None].contiguous()
    mi, mt = max(li), max(lt)
    size = {"a": P.fwd_workspace_size(ti, n, mi, hq, hkv, d),
            "b": P.prefix_fwd_workspace_size(prefix, tt, tt, n, mt, mt, hq, hkv, d),
            "c": P.cross_fwd_workspace_size(tt, ti, n, mt, mi, hq, hkv, d),
            "d": P.cross_bwd_workspace_size(tt, ti, n, mt, mi, hq, hkv, d),
            "e": P.prefix_bwd_workspace_size(prefix, tt, tt, n, mt, mt, hq, hkv, d),
            "f": P.bwd_workspace_size(ti, n, mi, hq, hkv, d)}
    ws = {k: torch.empty(max(256, v), dtype=torch.uint8, device="cuda") for k, v in size.items()}
    return x, (cu.offsets(li, "cuda"), mi), (cu.offsets(lt, "cuda"), mt), pos_i, pos_t, ws


def test_a_layer_and_back():
    """Every stage against the definition on what it was given, the rotations against
    complex multiplication."""
    import torch
    from tests.test_gpu_rotary import check, reference, spectrum
    x, ci, ct, pi, pt, ws = layer_inputs(3, [256, 64, 130], [30, 7, 61])
    r = layer(x, ci, ct, pi, pt, ws)
    from paper_2511_13198_amd import pdyattn as P
    qi, ki = P.attn_rotary(x["qi"], x["ki"], pi, (16, 16))
    check(qi, x["qi"], reference(x["qi"], pi, (16, 16), spectrum((16, 16)), False, False))
    qt, kt = P.attn_rotary(x["qt"], x["kt"], pt, (32,))
    own = cu.reference(qi, ki, x["vi"], ci[0], ci[0], False, 0.125)
    cu.check("o", r["oi"], own["o"])
    pre = cu.reference(qt, kt, x["vt"], ct[0], ct[0], True, 0.125, None, x["kp"], x["vp"])
    cu.check("o", r["ot"], pre["o"])
    cross = cu.reference(r["ot"], r["oi"], x["vi"], ct[0], ci[0], False, 0.125, do=x["do"])
    cu.check("o", r["oc"], cross["o"])
    cu.check("dv", r["dvc"], cross["dv"])
    dot, doi = (cross[n][0].to(torch.bfloat16) for n in ("dq", "dk"))
    # (dot and doi as the layer had them are within their bounds of these; the gradients
    # they lead to are linear in them, so their bounds add twice a rounding of each)
    for kind, args, names in (
            ("pre", (qt, kt, x["vt"], ct[0], ct[0], True, 0.125, None, x["kp"], x["vp"], dot),
             {"dv": "dvt", "dkp": "dkp", "dvp": "dvp"}),
            ("own", (qi, ki, x["vi"], ci[0], ci[0], False, 0.125, None, None, None, doi),
             {"dv": "dvi"})):
        ref = cu.reference(*args)
        for name, mine in names.items():
            got, want = r[mine].double(), ref[name][0]
            assert float((got - want).norm() / want.norm()) < 3 * cu.U, (kind, name)
    ref = cu.reference(qt, kt, x["vt"], ct[0], ct[0], True, 0.125, None, x["kp"], x["vp"], dot)
    for name, mine, pos, sec in (("dq", "dqt", pt, (32,)), ("dk", "dkt", pt, (32,))):
        want, _ = reference(ref[name][0], pos, sec, spectrum(sec), False, True)
        assert float((r[mine].double() - want).norm() / want.norm()) < 3 * cu.U, mine


def test_streams_and_graphs():
    """The layer on another stream, and two captured layers replayed in turn and beside
    eager calls, give the eager results bit for bit; each graph has its own workspaces."""
    import torch
    sets = [layer_inputs(s, li, lt) for s, li, lt in
            ((5, [256, 64, 130], [30, 7, 61]), (6, [100, 300, 16], [1, 1, 1]))]
    want = [{k: v.clone() for k, v in layer(*s).items()} for s in sets]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = [layer(*s) for s in sets]
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert all(torch.equal(a[k], b[k]) for k in b)
    graphs, outs = [], []
    for s in sets:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(layer(*s))
        graphs.append(graph)
    for rep in range(4):
        for o in outs:
            for t in o.values():
                t.fill_(7.0)
        for graph in graphs if rep % 2 else graphs[::-1]:
            graph.replay()
        eager = layer_inputs(7 + rep, [64, 90, 33], [12, 1, 40])
        layer(*eager)
        torch.cuda.synchronize()
        for a, b in zip(outs, want):
            for k in b:
                assert torch.equal(a[k], b[k]), (rep, k)


def test_a_graph_follows_the_lengths_it_reads():
    """Offsets, lengths and cached keys change between replays: a captured step of one
    token a sequence over a growing cache gives what eager calls give."""
    import torch
    from paper_2511_13198_amd import pdyattn as P
    g = torch.Generator(device="cuda").manual_seed(9)
    n, hq, hkv, d, slots = 6, 8, 2, 128, 3000
    q, k, v = normal(g, n, hq, d), normal(g, n * slots, hkv, d), normal(g, n * slots, hkv, d)
    cq, ck = cu.offsets([1] * n, "cuda"), cu.offsets([slots] * n, "cuda")
    used = torch.ones(n, dtype=torch.int32, device="cuda")
    ws = torch.empty(P.cross_fwd_workspace_size(n, n * slots, n, 1, slots, hq, hkv, d),
                     dtype=torch.uint8, device="cuda")
    o, lse = torch.empty_like(q), torch.empty(hq, n, device="cuda")
    step = lambda: P.attn_cross_fwd(q, k, v, cq, ck, 1, slots, True, seqlens_k=used, out=o,  # noqa: E731
                                    lse=lse, workspace=ws)
    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for lens in ([1, 2, 3, 4, 5, 6], [3000, 0, 128, 129, 1500, 1], [64] * 6):
        used.copy_(torch.tensor(lens, dtype=torch.int32))
        q.copy_(normal(g, n, hq, d))
        graph.replay()
        torch.cuda.synchronize()
        mine = o.clone(), lse.clone()
        step()
        assert torch.equal(mine[0], o) and torch.equal(mine[1], lse)
        ref = cu.reference(q, k, v, cq, ck, True, d ** -0.5, lens)
        cu.check("o", mine[0], ref["o"])
        cu.check("lse", mine[1], ref["lse"])


@pytest.mark.parametrize("layout", ["contiguous", "zigzag"])
def test_ring_with_rotated_shards(layout):
    """The ring that rotates its shards is the ring on rotated q and k, its gradients
    rotated back."""
    import torch
    from paper_2511_13198_amd import context_parallel as cp
    from paper_2511_13198_amd import pdyattn as P
    g = torch.Generator(device="cuda").manual_seed(11)
    T, hq, hkv, d, p = 1001, 4, 2, 128, 4
    q, k, v, do = normal(g, T, hq, d), normal(g, T, hkv, d), normal(g, T, hkv, d), normal(g, T, hq, d)
    pos = torch.arange(500000, 500000 + T, device="cuda", dtype=torch.int32)[:, None].contiguous()
    rotary = {"positions": pos, "sections": (64,), "base": 1e6}
    o, lses = cp.ring_forward(q, k, v, p, layout=layout, rotary=rotary)
    grads = cp.ring_backward(q, k, v, o, lses, do, p, layout=layout, rotary=rotary)
    qr, kr = P.attn_rotary(q, k, **rotary)
    o2, lses2 = cp.ring_forward(qr, kr, v, p, layout=layout)
    dq, dk, dv = cp.ring_backward(qr, kr, v, o2, lses2, do, p, layout=layout)
    dq, dk = P.attn_rotary(dq, dk, inverse=True, **rotary)
    assert torch.equal(o, o2) and all(torch.equal(lses[r], lses2[r]) for r in lses)
    assert all(torch.equal(a, b) for a, b in zip(grads, (dq, dk, dv)))
    with pytest.raises(ValueError, match="every device"):
        cp.ring_forward(q, k, v, p, layout=layout, rotary=rotary, devices=[0])
