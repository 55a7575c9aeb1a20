"""A paged key/value cache, as timed cases: writing new keys and values, attention of
one or few new tokens over the pages, alone or with the sums of each key's attention
weight, and eviction of the keys of least weight.

A case is one pass through an operator on a batch of sequences.  Pages are
[num_pages, Hkv, page_size, d], in bf16 or in e4m3 with a scale for each key head; a
sequence's pages are anywhere in the pool.

With `own` the pass makes the calls of paper_2511_13198_amd.pdyattn, outputs and
workspaces kept over the passes as a serving loop keeps them.  Without, it computes the
same in elementary torch operations in 32 bits on the padded batch, rounded once at the
end.

The range: 1 to 256 sequences with 1 to 64 new tokens each over 0 to 131,072 cached keys;
1 to 65,536 tokens written; caches of up to 32,768 keys a sequence shortened to between 32
and 4,096; pages of 16 to 256 keys; head dimensions 64 and 128; one to 32 query heads,
grouped or not.
"""
import math
import random

import torch

own = False

BF16, F32, F64, E4M3 = torch.bfloat16, torch.float32, torch.float64, torch.float8_e4m3fn
E4M3_MAX = 448.0


def listed():
    return [
        # one token for each of four requests over 1,500 keys: latency
        _attend("paged_fwd_4x1_k1500_h8_d64", 4, (1, 1), (1500, 1500), 8, 8, 64, 16, "bf16"),
        # serving: one token for each of 64 sequences over caches filled to different
        # lengths
        _attend("paged_fwd_64x1_k16384_h32kv8", 64, (1, 1), (256, 16384), 32, 8, 128, 16, "bf16"),
        # the same with an 8-bit cache and larger pages
        _attend("paged_fwd_64x1_k16384_h32kv8_e4m3", 64, (1, 1), (256, 16384), 32, 8, 128, 64,
                "e4m3"),
        # a few drafted tokens a sequence over caches of odd lengths, three query heads a
        # key head, pages that are no power of two
        _attend("paged_fwd_17x5_k9000_h24kv8", 17, (1, 5), (900, 9000), 24, 8, 128, 48, "bf16"),
        # one very long sequence
        _attend("paged_fwd_1x1_k131072_h32kv8_e4m3", 1, (1, 1), (131072, 131072), 32, 8, 128, 128,
                "e4m3"),
        # many short chats, some without a key: eight query heads a key head
        _attend("paged_fwd_256x1_k2048_h16kv2", 256, (1, 1), (0, 2048), 16, 2, 128, 32, "bf16"),
        # serving with a cache that is kept short: attention and the keys' weights
        _attend("paged_weigh_64x1_k8192_h32kv8", 64, (1, 1), (512, 8192), 32, 8, 128, 16, "bf16",
                weigh=True),
        # the last 32 tokens of six prompts, to see which of their keys matter
        _attend("paged_weigh_6x32_k16384_h16_d64", 6, (32, 32), (4000, 16384), 16, 16, 64, 64,
                "bf16", weigh=True),
        # the next token of 64 sequences: latency
        _write("paged_write_64x1_h8", 64, (1, 1), (256, 16384), 8, 128, 16, "bf16"),
        # prompts, to an 8-bit cache
        _write("paged_write_8x8192_h8_e4m3", 8, (1024, 8192), (1024, 8192), 8, 128, 64, "e4m3"),
        # caches a little over what they may hold
        _evict("paged_evict_64x2304_to_2048_h8", 64, (1900, 2304), 8, 128, 16, "bf16", 2048, 64,
               4),
        # long prompts cut down, 8-bit
        _evict("paged_evict_4x32768_to_4096_h8_e4m3", 4, (8000, 32768), 8, 128, 64, "e4m3", 4096,
               256, 16),
    ]


def _attend(name, n, q, k, hq, hkv, d, page, cache, weigh=False, causal=True, lseed=42):
    """q, k: least and most new tokens and keys in use (the new ones among them) of a
    sequence; k from 0: some sequences have no key."""
    return {"name": name, "op": "attend", "n": n, "q_lo": q[0], "q_hi": q[1], "k_lo": k[0],
            "k_hi": k[1], "hq": hq, "hkv": hkv, "d": d, "page": page, "cache": cache,
            "weigh": weigh, "causal": causal, "lseed": lseed}


def _write(name, n, q, k, hkv, d, page, cache, lseed=42):
    """q: new tokens of a sequence; k: keys in use after them (at least the new ones)."""
    return {"name": name, "op": "write", "n": n, "q_lo": q[0], "q_hi": q[1], "k_lo": k[0],
            "k_hi": k[1], "hkv": hkv, "d": d, "page": page, "cache": cache, "lseed": lseed}


def _evict(name, n, k, hkv, d, page, cache, budget, recent, first, lseed=42):
    """k: keys in use; budget: of these stay, the last `recent` and the `first` ones anyway."""
    return {"name": name, "op": "evict", "n": n, "k_lo": k[0], "k_hi": k[1], "hkv": hkv, "d": d,
            "page": page, "cache": cache, "budget": budget, "recent": recent, "first": first,
            "lseed": lseed}


def _log_int(rng, lo, hi):
    return lo if hi <= lo else int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """A case of the same ranges, at most about half of the largest listed one's cost."""
    d = rng.choice([64, 128, 128])
    hkv = rng.choice([1, 2, 4, 8, 16])
    page = rng.choice([16, 16, 32, 48, 64, 112, 128, 256])
    cache = rng.choice(["bf16", "bf16", "e4m3"])
    op = rng.choice(["attend", "attend", "attend", "attend", "write", "write", "evict", "evict"])
    while True:
        n, lseed = _log_int(rng, 1, 256), rng.randrange(1 << 20)
        if op == "attend":
            group = rng.choice([x for x in (1, 2, 3, 4, 7, 8) if x * hkv <= 32])
            q_hi = rng.choice([1, 1, 1, 1, 3, 8]) if rng.random() < 0.75 else _log_int(rng, 2, 64)
            k_hi = max(q_hi, _log_int(rng, 16, 131072))
            case = _attend("", n, (max(1, q_hi // rng.choice([1, 4])), q_hi),
                           (rng.choice([0, 1, max(1, k_hi // 8)]), k_hi), hkv * group, hkv, d,
                           page, cache, weigh=rng.random() < 0.35, causal=rng.random() < 0.9,
                           lseed=lseed)
            if n * k_hi * hkv * d <= 1 << 30 and n * hkv * group * q_hi * k_hi <= 1 << 30:
                break
        elif op == "write":
            q_hi = 1 if rng.random() < 0.3 else _log_int(rng, 1, 8192)
            k_hi = max(q_hi, _log_int(rng, 1, 16384))
            case = _write("", n, (max(1, q_hi // rng.choice([1, 4, 16])), q_hi), (1, k_hi), hkv, d,
                          page, cache, lseed=lseed)
            if n * q_hi <= 65536 and n * k_hi * hkv * d <= 1 << 30:
                break
        else:
            n = min(n, 64)
            k_hi = _log_int(rng, 64, 32768)
            budget = min(4096, max(32, int(k_hi * rng.choice([0.1, 0.3, 0.6, 0.9]))))
            recent = rng.choice([0, 1, budget // 8, budget // 2])
            case = _evict("", n, (max(1, k_hi // rng.choice([1, 2, 8])), k_hi), hkv, d, page,
                          cache, budget, recent, rng.choice([0, 1, 4, 16]), lseed=lseed)
            if n * k_hi * hkv * d <= 1 << 30:
                break
    del case["name"]
    return case


def _lengths(case):
    """New tokens and keys in use of the sequences; keys from 0 leave some without any."""
    rng = random.Random(case["lseed"])
    n = case["n"]
    q = [_log_int(rng, case["q_lo"], case["q_hi"]) if "q_lo" in case else 0 for _ in range(n)]
    k = [max(a, _log_int(rng, max(1, case["k_lo"]), case["k_hi"])) for a in q]
    if case["k_lo"] == 0:
        k[1:] = [0 if rng.random() < 0.1 else x for x in k[1:]]
    return q, k


def _visible(nq, nk, causal):
    """Visible (query, key) pairs of a sequence; causal: the last query sees every key."""
    if not causal:
        return nq * nk
    full = min(nq, nk)
    return full * nk - full * (full - 1) // 2


def work(case):
    hkv, d = case["hkv"], case["d"]
    size = 2 if case["cache"] == "bf16" else 1
    ql, kl = _lengths(case)
    t, keys = sum(ql), sum(kl)
    if case["op"] == "write":
        return {"bytes": 2 * t * hkv * d * (2 + size), "flops": 2 * t * hkv * d}
    if case["op"] == "evict":
        kept = sum(min(x, case["budget"]) for x in kl) * hkv
        return {"bytes": 4 * keys * hkv + kept * (2 * 2 * d * size + 4 + 4),
                "flops": keys * hkv}
    pairs = sum(_visible(a, b, case["causal"]) for a, b in zip(ql, kl))
    hq = case["hq"]
    nbytes = 2 * keys * hkv * d * size + 2 * 2 * t * hq * d + 4 * t * hq
    if case["weigh"]:
        nbytes += 8 * keys * hkv
    return {"bytes": nbytes, "flops": 4 * d * hq * pairs}


def _pages(k, page):
    return -(-k // page)


def _inputs(case, seed):
    """The pool, its scales and table, and what the call brings."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    hkv, d, page, n = case["hkv"], case["d"], case["page"], case["n"]
    ql, kl = _lengths(case)
    most = _pages(max(max(kl), 1), page) + 1  # (a table has room for more than is in use)
    used = [_pages(x, page) for x in kl]
    kept = _pages(case["budget"], page) if case["op"] == "evict" else 0
    pool = sum(used) + n * kept + 5
    order = torch.randperm(pool, generator=g, device="cuda").int()
    # unused entries name any page
    table = torch.randint(0, pool, (n, most), generator=g, dtype=torch.int32, device="cuda")
    at = 0
    for i, x in enumerate(used):
        table[i, :x] = order[at:at + x]
        at += x
    x = {"table": table, "len_k": torch.tensor(kl, dtype=torch.int32, device="cuda")}
    shape = (pool, hkv, page, d)
    for name in ("k", "v"):
        y = torch.randn(shape, generator=g, dtype=F32, device="cuda")
        if case["cache"] == "bf16":
            x[name + "_pages"], x[name + "_scale"] = y.to(BF16), None
        else:
            # a scale a head, as the largest value met while calibrating sets it
            s = torch.rand(hkv, generator=g, dtype=F32, device="cuda") * 0.004 + 0.01
            y.div_(s[:, None, None]).clamp_(-E4M3_MAX, E4M3_MAX)
            x[name + "_pages"], x[name + "_scale"] = y.to(E4M3), s
        del y

    def normal(t, h):
        return torch.randn((t, h, d), generator=g, dtype=F32, device="cuda").to(BF16)

    if case["op"] == "attend":
        x["q"] = normal(sum(ql), case["hq"])
        if case["weigh"]:
            x["scores"] = torch.rand(shape[:3], generator=g, dtype=F32, device="cuda")
    elif case["op"] == "write":
        x["k"], x["v"] = normal(sum(ql), hkv), normal(sum(ql), hkv)
        x["scores"] = torch.rand(shape[:3], generator=g, dtype=F32, device="cuda")
    else:
        # weights sum up very unevenly; some keys never had any
        y = torch.randn(shape[:3], generator=g, dtype=F32, device="cuda").mul_(3.0).exp_()
        x["scores"] = y.masked_fill_(torch.rand(shape[:3], generator=g, device="cuda") < 0.05, 0.0)
        x["new_table"] = order[at:at + n * kept].view(n, kept).contiguous()
    if case["op"] != "evict":
        cu = [0]
        for y in ql:
            cu.append(cu[-1] + y)
        x["cu_q"] = torch.tensor(cu, dtype=torch.int32, device="cuda")
    return x


def prepare(case, seed):
    s = {"case": case, **_inputs(case, seed)}
    ql, kl = _lengths(case)
    s["max_q"], s["max_k"] = max(ql), max(max(kl), 1)
    if case["op"] == "attend":
        s["scale"] = 1.0 / math.sqrt(case["d"])
        s["o"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty((case["hq"], s["q"].shape[0]), dtype=F32, device="cuda")
    elif case["op"] == "evict":
        s["kept"] = torch.empty((case["n"], case["hkv"], case["budget"]), dtype=torch.int32,
                                device="cuda")
        s["new_len"] = torch.empty_like(s["len_k"])
    return s


def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    from paper_2511_13198_amd import pdyattn
    case = s["case"]
    n, hkv, d = case["n"], case["hkv"], case["d"]
    if case["op"] == "write":
        pdyattn.attn_paged_write(s["k"], s["v"], s["k_pages"], s["v_pages"], s["table"], s["cu_q"],
                                 s["len_k"], k_scale=s["k_scale"], v_scale=s["v_scale"],
                                 scores=s["scores"])
        return {"k": s["k_pages"], "v": s["v_pages"], "scores": s["scores"]}
    if case["op"] == "evict":
        if "ws" not in s:
            s["ws"] = torch.empty(pdyattn.paged_evict_workspace_size(n, s["max_k"], hkv,
                                                                     case["budget"]),
                                  dtype=torch.uint8, device="cuda")
        kept, lens = pdyattn.attn_paged_evict(
            s["k_pages"], s["v_pages"], s["scores"], s["table"], s["len_k"], s["new_table"],
            case["budget"], recent=case["recent"], first=case["first"], max_seqlen_k=s["max_k"],
            kept=s["kept"], new_lens=s["new_len"], workspace=s["ws"])
        return {"k": s["k_pages"], "v": s["v_pages"], "scores": s["scores"], "kept": kept,
                "len": lens}
    scores = s.get("scores")
    if "ws" not in s:
        need = pdyattn.paged_fwd_workspace_size(s["q"].shape[0], n, s["max_q"], s["max_k"],
                                                case["hq"], hkv, d, scores is not None)
        s["ws"] = torch.empty(need, dtype=torch.uint8, device="cuda")
    o, lse = pdyattn.attn_paged_fwd(
        s["q"], s["k_pages"], s["v_pages"], s["table"], s["cu_q"], s["len_k"], s["max_q"],
        s["max_k"], causal=case["causal"], scale=s["scale"], k_scale=s["k_scale"],
        v_scale=s["v_scale"], scores=scores, out=s["o"], lse=s["lse"], workspace=s["ws"])
    return {"o": o, "lse": lse} if scores is None else {"o": o, "lse": lse, "scores": scores}


# ---------------------------------------------------------------------------
# The plain form
# ---------------------------------------------------------------------------
def _run_plain(s):
    return {"attend": _plain_attend, "write": _plain_write, "evict": _plain_evict}[
        s["case"]["op"]](s)


def _bits(x):
    """A tensor to be indexed, whatever its type."""
    return x.view(torch.uint8) if x.dtype is E4M3 else x


def _plain_write(s):
    case = s["case"]
    page = case["page"]
    cu, t = s["cu_q"].long(), s["k"].shape[0]
    i = torch.arange(t, device=cu.device)
    seq = torch.searchsorted(cu, i, right=True) - 1
    at = s["len_k"].long()[seq] - cu[seq + 1] + i  # the sequence's last tokens are its last keys
    pg = s["table"][seq, at // page].long()
    for name in ("k", "v"):
        x = s[name]
        if s[name + "_scale"] is not None:
            x = x.float() / s[name + "_scale"][:, None]
            x = x.clamp(-E4M3_MAX, E4M3_MAX).to(E4M3)
        _bits(s[name + "_pages"])[pg, :, at % page] = _bits(x)
    s["scores"][pg, :, at % page] = 0.0
    return {"k": s["k_pages"], "v": s["v_pages"], "scores": s["scores"]}


def _plain_evict(s):
    case = s["case"]
    n, hkv, page, budget = case["n"], case["hkv"], case["page"], case["budget"]
    table = s["table"].long()
    length = s["len_k"].long()[:, None, None]
    have = table.shape[1] * page
    j = torch.arange(have, device=table.device)
    w = s["scores"][table].transpose(1, 2).reshape(n, hkv, have)
    w = torch.where((j < case["first"]) | (j >= length - case["recent"]), math.inf, w)
    w = torch.where(j < length, w, -math.inf)
    order = torch.sort(w, dim=2, descending=True, stable=True)[1][..., :budget]
    if have < budget:
        order = torch.nn.functional.pad(order, (0, budget - have), value=have)
    order = torch.where(order < length, order, have).sort(dim=2)[0]
    stays = order < length
    src = order.clamp(max=have - 1)
    pg = table.gather(1, (src // page).view(n, -1)).view(n, hkv, budget)
    h = torch.arange(hkv, device=table.device)[:, None]
    to = torch.arange(budget, device=table.device)
    to_pg = s["new_table"].long()[:, to // page][:, None].expand(n, hkv, budget)
    to_h, to_at = h.expand(n, hkv, budget), (to % page).expand(n, hkv, budget)
    for x in (_bits(s["k_pages"]), _bits(s["v_pages"]), s["scores"]):
        new, old = x[pg, h, src % page], x[to_pg, to_h, to_at]
        x[to_pg, to_h, to_at] = torch.where(stays[..., None] if x.dim() == 4 else stays, new, old)
    kept = torch.where(stays, order, -1).int()
    return {"k": s["k_pages"], "v": s["v_pages"], "scores": s["scores"], "kept": kept,
            "len": s["len_k"].clamp(max=budget)}


def _plain_attend(s):
    case, scale = s["case"], s["scale"]
    n, hq, hkv, d, page = case["n"], case["hq"], case["hkv"], case["d"], case["page"]
    g, mq = hq // hkv, s["max_q"]
    cu, nk, table = s["cu_q"].long(), s["len_k"].long(), s["table"].long()
    nq, t = cu.diff(), s["q"].shape[0]
    mk = table.shape[1] * page
    j = torch.arange(mk, device=cu.device)
    i = torch.arange(mq, device=cu.device)
    rows = (cu[:-1, None] + i).clamp_(max=t - 1)

    def keys(name):  # [n, hkv, mk, d] in 32 bits, zero behind the last in use
        x = _bits(s[name + "_pages"])[table].transpose(1, 2)
        x = (x.reshape(n, hkv, mk, d).view(s[name + "_pages"].dtype)).float()
        if s[name + "_scale"] is not None:
            x.mul_(s[name + "_scale"][:, None, None])
        return x.masked_fill_((j >= nk[:, None])[:, None, :, None], 0.0)

    q = s["q"][rows].float().transpose(1, 2).reshape(n, hkv, g * mq, d)
    see = (j < nk[:, None])[:, None] & (i < nq[:, None])[..., None]  # [n, mq, mk]
    if case["causal"]:
        see = see & (j <= i[:, None] + (nk - nq)[:, None, None])
    see = see[:, None, None].expand(n, hkv, g, mq, mk)
    a = q @ keys("k").transpose(2, 3).contiguous()
    a.view(n, hkv, g, mq, mk).mul_(scale).masked_fill_(~see, -math.inf)
    top = a.amax(3, keepdim=True)
    top = top.masked_fill(top == -math.inf, 0.0)
    a = a.sub_(top).exp_()
    total = a.sum(3, keepdim=True)
    a.mul_(torch.where(total > 0, 1.0 / total, 0.0))
    o = a @ keys("v")
    lse = top + total.log()
    # packed rows again
    tok = torch.arange(t, device=cu.device)
    seq = torch.searchsorted(cu, tok, right=True) - 1
    at = tok - cu[seq]
    out = {"o": o.view(n, hq, mq, d)[seq, :, at].to(BF16),
           "lse": lse.view(n, hq, mq)[seq, :, at].t().contiguous()}
    if case["weigh"]:
        # (every place of the table is a page's, so that no place is left out: those not
        # in use get nothing)
        w = a.sum(2).view(n, hkv, -1, page).transpose(1, 2)  # [n, pages, hkv, page]
        at = table[:, :, None] * hkv + torch.arange(hkv, device=cu.device)
        s["scores"].view(-1, page).index_add_(0, at.reshape(-1), w.reshape(-1, page))
        out["scores"] = s["scores"]
    return out


# ---------------------------------------------------------------------------
# The definition, in 64 bits
# ---------------------------------------------------------------------------
def exact(case, seed):
    x = _inputs(case, seed)
    return {"attend": _exact_attend, "write": _exact_write, "evict": _exact_evict}[case["op"]](
        case, x)


def _sequence(x, name, pages, h, nk):
    """The first nk keys of a head in these pages, in 64 bits."""
    pool = x[name]
    y = _bits(pool)[pages, h].view(pool.dtype).double().view(-1, pool.shape[3])[:nk]
    scale = x[name[0] + "_scale"]
    return y if scale is None else y * scale[h].double()


def _exact_attend(case, x):
    hq, hkv, d, page = case["hq"], case["hkv"], case["d"], case["page"]
    g, scale = hq // hkv, 1.0 / math.sqrt(d)
    ql, kl = _lengths(case)
    t, dev = sum(ql), x["q"].device
    o = torch.zeros((t, hq, d), dtype=F64, device=dev)
    lse = torch.full((hq, t), -math.inf, dtype=F64, device=dev)
    scores = x["scores"].double() if case["weigh"] else None
    first = 0
    for i, (nq, nk) in enumerate(zip(ql, kl)):
        pages = x["table"][i, :_pages(nk, page)].long()
        for h in range(hkv if nk else 0):
            k, v = (_sequence(x, w, pages, h, nk) for w in ("k_pages", "v_pages"))
            weight = torch.zeros(pages.numel() * page, dtype=F64, device=dev)
            for e in range(h * g, h * g + g):
                s = (x["q"][first:first + nq, e].double() @ k.t()) * scale
                if case["causal"]:
                    last = torch.arange(nk - nq, nk, device=dev)[:, None]
                    s = s.masked_fill(torch.arange(nk, device=dev) > last, -math.inf)
                z = torch.logsumexp(s, 1)
                p = torch.exp(s - z[:, None])
                o[first:first + nq, e], lse[e, first:first + nq] = p @ v, z
                weight[:nk] += p.sum(0)
            if scores is not None:
                scores[pages, h] += weight.view(-1, page)
        first += nq
    out = {"o": o, "lse": lse}
    if scores is not None:
        out["scores"] = scores
    return out


def _exact_write(case, x):
    """A key's place: the last of a sequence's new tokens is its last key.  In e4m3 the
    number before it is rounded."""
    page = case["page"]
    ql, kl = _lengths(case)
    out = {"k": x["k_pages"].double(), "v": x["v_pages"].double(), "scores": x["scores"].double()}
    first = 0
    for i, (nq, nk) in enumerate(zip(ql, kl)):
        done = 0
        while done < nq:  # page by page
            at = nk - nq + done
            count = min(nq - done, page - at % page)
            p, a, b = int(x["table"][i, at // page]), at % page, at % page + count
            for name in ("k", "v"):
                y = x[name][first + done:first + done + count].double().transpose(0, 1)
                if x[name + "_scale"] is not None:
                    y = (y / x[name + "_scale"].double()[:, None, None]).clamp(-E4M3_MAX, E4M3_MAX)
                out[name][p, :, a:b] = y
            out["scores"][p, :, a:b] = 0.0
            done += count
        first += nq
    return out


def _exact_evict(case, x):
    """Head by head: the number of keys that go, then those of least weight between the
    first and the recent ones, the later of equal ones before the earlier."""
    page, budget = case["page"], case["budget"]
    hkv = case["hkv"]
    _, kl = _lengths(case)
    out = {"k": x["k_pages"].double(), "v": x["v_pages"].double(), "scores": x["scores"].double(),
           "kept": torch.full((case["n"], hkv, budget), -1, dtype=torch.int32, device="cuda"),
           "len": torch.tensor([min(k, budget) for k in kl], dtype=torch.int32, device="cuda")}
    for i, nk in enumerate(kl):
        pages = x["table"][i, :_pages(nk, page)].long()
        into = x["new_table"][i].long()
        for h in range(hkv):
            w = x["scores"][pages, h].reshape(-1)[:nk]
            lo, hi = min(case["first"], nk), max(nk - case["recent"], min(case["first"], nk))
            going = max(0, nk - budget)
            mid = w[lo:hi].flip(0)  # (a stable sort puts the later of equal ones first)
            gone = hi - 1 - torch.sort(mid, stable=True)[1][:going]
            stay = torch.ones(nk, dtype=torch.bool, device=w.device)
            stay[gone] = False
            idx = stay.nonzero()[:, 0]
            to = torch.arange(idx.numel(), device=w.device)
            for name, y in (("k", x["k_pages"]), ("v", x["v_pages"]), ("scores", x["scores"])):
                z = (_bits(y)[pages[idx // page], h, idx % page])
                z = z.view(y.dtype) if y.dtype is E4M3 else z
                out[name][into[to // page], h, to % page] = z.double()
            out["kept"][i, h, :idx.numel()] = idx.int()
    return out
