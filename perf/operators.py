"""Operators of a paged key/value cache: what they are measured on.

Serving several sequences out of one pool of cache pages takes three operators, each with cases here:

``rope``       norm of every query and key head, position rotation, and the write of keys and values into their pages
``attention``  new tokens of a ragged batch (one token, or a chunk of a prompt) over the pages of their sequences; with
               ``weights``, also what every cached position has received of the softmax, added to a running sum
``evict``      of every sequence and key/value head, the positions that weigh most and the most recent ones, copied in
               order to other pages

Heads are 128 wide.  The head counts are those of the repository's blocks (32 and 40 query heads, as many key/value
heads), and the same with fewer key/value heads; 2048-token prompts, caches of up to 131072 positions, activations and
caches with the spread that its synthetic weights give.  ``listed`` gives the named cases, ``draw`` one more of the same
ranges; ``prepare`` makes what a program holds before the call, ``run`` makes the call or computes the plain form,
``exact`` is the definition in 64 bits.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

D = 128
EPS = 1e-5
STD = 0.02 * math.sqrt(4096)  # spread of a projection of a normalised row


# ------------------------------------------------------------------ the cases
def listed():
    return [
        # the smallest call: the token being served of one sequence, 7B-shaped block without norms of its heads
        {"name": "rope_token", "kind": "rope", "heads": 32, "kv_heads": 32, "page": 64, "norm": False, "seqs": 1,
         "new_min": 1, "new_max": 1, "cached_min": 1337, "cached_max": 1337, "ragged": 1},
        # chunks of several prompts in one call, heads normalised, q, k and v as columns of one product
        {"name": "rope_prompts", "kind": "rope", "heads": 32, "kv_heads": 8, "page": 64, "norm": True, "seqs": 9,
         "new_min": 300, "new_max": 2048, "cached_min": 1, "cached_max": 4000, "ragged": 2},
        # one token of one short sequence, a key/value head per query head: latency
        {"name": "token", "kind": "attention", "heads": 32, "kv_heads": 32, "page": 16, "weights": False, "seqs": 1,
         "new_min": 1, "new_max": 1, "cached_min": 330, "cached_max": 330, "ragged": 3},
        # a token of each of many sequences, their lengths from a few to thousands of positions
        {"name": "serving", "kind": "attention", "heads": 32, "kv_heads": 8, "page": 64, "weights": False, "seqs": 64,
         "new_min": 1, "new_max": 1, "cached_min": 17, "cached_max": 4096, "ragged": 4},
        # one token at the end of a very long sequence
        {"name": "long_token", "kind": "attention", "heads": 32, "kv_heads": 8, "page": 256, "weights": False, "seqs": 1,
         "new_min": 1, "new_max": 1, "cached_min": 100002, "cached_max": 100002, "ragged": 5},
        # tokens of running sequences and chunks of new prompts in one call, small pages
        {"name": "mixed_chunks", "kind": "attention", "heads": 40, "kv_heads": 8, "page": 16, "weights": False, "seqs": 11,
         "new_min": 1, "new_max": 300, "cached_min": 1, "cached_max": 3000, "ragged": 6},
        # a whole prompt of one calibration row, nothing cached before it
        {"name": "prompt", "kind": "attention", "heads": 32, "kv_heads": 32, "page": 64, "weights": False, "seqs": 1,
         "new_min": 2048, "new_max": 2048, "cached_min": 0, "cached_max": 0, "ragged": 7},
        # the last chunk of a long document: the largest call
        {"name": "long_chunk", "kind": "attention", "heads": 32, "kv_heads": 8, "page": 128, "weights": False, "seqs": 1,
         "new_min": 2048, "new_max": 2048, "cached_min": 30720, "cached_max": 30720, "ragged": 8},
        # a token of each of several sequences whose caches are to be cut: attention weights are added up
        {"name": "weighed_serving", "kind": "attention", "heads": 40, "kv_heads": 40, "page": 32, "weights": True,
         "seqs": 24, "new_min": 1, "new_max": 1, "cached_min": 100, "cached_max": 2048, "ragged": 9},
        # prompts of such sequences
        {"name": "weighed_prompts", "kind": "attention", "heads": 32, "kv_heads": 8, "page": 128, "weights": True, "seqs": 3,
         "new_min": 301, "new_max": 1501, "cached_min": 1, "cached_max": 200, "ragged": 10},
        # one sequence cut back by a few positions
        {"name": "evict_one", "kind": "evict", "kv_heads": 32, "page": 64, "seqs": 1, "cached_min": 611, "cached_max": 611,
         "keep": 512, "recent": 64, "ragged": 11},
        # a batch of long sequences cut to half and less
        {"name": "evict_many", "kind": "evict", "kv_heads": 8, "page": 64, "seqs": 15, "cached_min": 5000, "cached_max": 9001,
         "keep": 4096, "recent": 500, "ragged": 12},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))))) if hi > lo else lo


# heads and positions as far as the largest listed cases go: bytes of a cache that is read, query-key pairs of a chunk
_MOST_ROWS = 100003 * 8
_MOST_PAIRS = 2048 * 31744 * 32


def draw(rng):
    kind = rng.choice(("rope", "attention", "attention", "attention", "evict"))
    heads, kv = rng.choice(((32, 32), (40, 40), (32, 8), (40, 8), (28, 4), (8, 1)))
    case = {"kind": kind, "kv_heads": kv, "page": rng.choice((16, 32, 64, 128, 256)), "ragged": rng.randrange(1 << 20)}
    if kind == "rope":
        seqs = _log(rng, 1, 64)
        new = 1 if rng.random() < 0.4 else _log(rng, 2, min(2048, 10000 // seqs))
        return dict(case, heads=heads, norm=rng.random() < 0.6, seqs=seqs, new_min=(new + 3) // 4, new_max=new,
                    cached_min=1, cached_max=_log(rng, 2, 4000))
    if kind == "evict":
        seqs = _log(rng, 1, 16)
        most = _log(rng, 40, min(16384, _MOST_ROWS // (2 * kv * seqs)))
        keep = _log(rng, 16, most)
        return dict(case, seqs=seqs, cached_min=(most + 1) // 2, cached_max=most, keep=keep, recent=rng.randint(0, keep))
    case.update(heads=heads, weights=rng.random() < 0.35)
    form = rng.choice(("tokens", "tokens", "chunks", "chunks", "long"))
    if form == "tokens":
        seqs = _log(rng, 1, 64)
        most = _log(rng, 16, min(16384, _MOST_ROWS // (kv * seqs)))
        return dict(case, seqs=seqs, new_min=1, new_max=1, cached_min=(most + 15) // 16, cached_max=most)
    if form == "long":
        most = _log(rng, 16000, _MOST_ROWS // max(kv, 8))
        return dict(case, seqs=1, new_min=1, new_max=1, cached_min=most, cached_max=most)
    seqs = _log(rng, 1, 8)
    new = _log(rng, 2, 2048 // seqs)
    most = max(1, min(_log(rng, 1, 30000), _MOST_PAIRS // (seqs * new * heads) - new, _MOST_ROWS // (kv * seqs)))
    return dict(case, seqs=seqs, new_min=max(1, new // 8), new_max=new, cached_min=1 if rng.random() < 0.5 else most,
                cached_max=most)


def _lengths(case):
    """(new tokens, positions cached before them) of every sequence, from the case alone."""
    rng = random.Random(case["ragged"])
    spread = lambda what: _log(rng, case[what + "_min"], case[what + "_max"]) if case.get(what + "_max") else 0
    return [(spread("new"), spread("cached")) for _ in range(case["seqs"])]


def work(case):
    lengths, kv = _lengths(case), case["kv_heads"]
    if case["kind"] == "evict":
        rows = sum(min(c, case["keep"]) for _, c in lengths) * kv
        seen = sum(c for _, c in lengths) * kv
        return {"bytes": rows * (2 * 4 * D + 4 + 4) + seen * 4, "flops": seen}
    heads, tokens = case["heads"], sum(n for n, _ in lengths)
    if case["kind"] == "rope":
        # each row read and written, a row of the table; norm and rotation
        return {"bytes": tokens * ((heads + 2 * kv) * 4 * D + 4 * D),
                "flops": tokens * (heads + kv) * D * (7 if case["norm"] else 3)}
    pairs = sum(n * c + n * (n + 1) // 2 for n, c in lengths) * heads
    positions = sum(n + c for n, c in lengths) * kv
    nbytes = positions * 4 * D + tokens * heads * 4 * D
    if case["weights"]:
        nbytes += positions * 4 + sum(c for _, c in lengths) * kv * 4 + tokens * heads * 4
    return {"bytes": nbytes, "flops": 4 * D * pairs}


# ------------------------------------------------------------------ inputs
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 1000003 + 29)
    return g


def _normal(g, *shape, std=1.0):
    return (torch.randn(*shape, generator=g, device="cuda") * std).half()


def _tables(lengths, page, seed):
    """Pages of every sequence, dealt from a shuffled pool with a few left over; -1 where a sequence has none."""
    need = [-(-length // page) for length in lengths]
    pages = sum(need) + 3
    order = np.random.default_rng(seed).permutation(pages).astype(np.int32)
    table = np.full((len(lengths), max(max(need), 1)), -1, dtype=np.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    return table, pages


def _angles(positions):
    return torch.arange(positions, device="cuda", dtype=torch.float64)[:, None] * (
        10000.0 ** (-2.0 * torch.arange(D // 2, device="cuda", dtype=torch.float64) / D))


def _inputs(case, seed):
    """The inputs of a case as tensors and host tables; what ``prepare`` and ``exact`` both start from."""
    g, page, kv = _gen(seed), case["page"], case["kv_heads"]
    lengths = _lengths(case)
    total = [n + c for n, c in lengths]
    table, pages = _tables(total, page, seed)
    s = {"case": case, "lengths": lengths, "total": total, "table": table, "pages": pages}
    if case["kind"] == "evict":
        s["k"], s["v"] = _normal(g, pages, kv, page, D, std=STD), _normal(g, pages, kv, page, D, std=STD)
        # sums of attention weights: a few positions hold most of it, some have received nothing
        w = torch.exp(2.0 * torch.randn(case["seqs"], kv, max(total), generator=g, device="cuda"))
        s["weights"] = torch.where(torch.rand(w.shape, generator=g, device="cuda") < 0.1, torch.zeros_like(w), w)
        s["dst_table"], s["dst_pages"] = _tables([min(t, case["keep"]) for t in total], page, seed + 1)
        return s
    heads, tokens = case["heads"], sum(n for n, _ in lengths)
    if case["kind"] == "rope":
        if case["norm"]:  # columns of one product
            qkv = _normal(g, tokens, (heads + 2 * kv) * D, std=STD)
            s["q"], s["kn"], s["vn"] = torch.split(qkv, (heads * D, kv * D, kv * D), 1)
            s["q_gain"], s["k_gain"] = (1.0 + 0.1 * torch.randn(2, D, generator=g, device="cuda")).half().unbind(0)
        else:
            s["q"], s["kn"], s["vn"] = (_normal(g, tokens, h * D, std=STD) for h in (heads, kv, kv))
            s["q_gain"] = s["k_gain"] = None
        a = _angles(max(total))
        s["rope"] = torch.stack((torch.cos(a), torch.sin(a)), -1).float()
        s["k"], s["v"] = (torch.zeros(pages, kv, page, D, dtype=torch.float16, device="cuda") for _ in range(2))
        return s
    s["q"] = _normal(g, tokens, heads * D, std=STD)
    s["k"], s["v"] = _normal(g, pages, kv, page, D, std=STD), _normal(g, pages, kv, page, D, std=STD)
    if case["weights"]:
        s["weights"] = torch.rand(case["seqs"], kv, max(total), generator=g, device="cuda") * 8.0
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    kv, page = case["kv_heads"], case["page"]
    empty = lambda *shape, dtype=torch.float16: torch.zeros(shape, dtype=dtype, device="cuda")
    if case["kind"] == "evict":
        s["k_out"], s["v_out"] = (empty(s["dst_pages"], kv, page, D) for _ in range(2))
        s["kept"] = empty(case["seqs"], kv, case["keep"], dtype=torch.int32)
        s["new_len"] = empty(case["seqs"], dtype=torch.int32)
        s["weights_out"] = empty(case["seqs"], kv, case["keep"], dtype=torch.float32)
    else:
        s["out"] = empty(*s["q"].shape)
        if case["kind"] == "attention" and case["weights"]:
            s["lse"] = empty(s["q"].shape[0], case["heads"], dtype=torch.float32)
            s["weights_out"] = torch.zeros_like(s["weights"])
    if own:
        import paper_2501_07139_amd as fq

        fq.fq_init()
        s["batch"] = fq.PagedBatch([n for n, _ in s["lengths"]], s["total"], s["table"], page, s["pages"])
        if case["kind"] == "attention":
            s["workspace"] = empty(fq.fq_attn_paged_workspace_bytes(s["batch"], case["heads"], kv, case["weights"]),
                                   dtype=torch.uint8)
        if case["kind"] == "evict":
            s["dst"] = torch.from_numpy(s["dst_table"]).cuda()
        return s
    # the plain form indexes with these: page and row of every position of every sequence
    s["pages_of"], s["rows_of"] = [], []
    for b, total in enumerate(s["total"]):
        t = np.arange(total)
        s["pages_of"].append(torch.from_numpy(s["table"][b][t // page].astype(np.int64)).cuda())
        s["rows_of"].append(torch.from_numpy(t % page).cuda())
    if case["kind"] == "evict":
        s["dst_of"] = []
        for b, total in enumerate(s["total"]):
            t = np.arange(min(total, case["keep"]))
            s["dst_of"].append((torch.from_numpy(s["dst_table"][b][t // page].astype(np.int64)).cuda(),
                                torch.from_numpy(t % page).cuda()))
    return s


# ------------------------------------------------------------------ the calls, and the same in elementary operations
def run(s):
    kind = s["case"]["kind"]
    if own:
        return {"rope": _call_rope, "attention": _call_attention, "evict": _call_evict}[kind](s)
    return {"rope": _plain_rope, "attention": _plain_attention, "evict": _plain_evict}[kind](s)


def _call_rope(s):
    import paper_2501_07139_amd as fq

    q = fq.fq_qk_norm_rope(s["q"], s["kn"], s["vn"], s["batch"], s["rope"], s["k"], s["v"], q_gain=s["q_gain"],
                           k_gain=s["k_gain"], eps=EPS, out=s["out"])
    return {"q": q, "k": s["k"], "v": s["v"]}


def _call_attention(s):
    import paper_2501_07139_amd as fq

    if s["case"]["weights"]:
        out = fq.fq_attn_paged(s["q"], s["batch"], s["k"], s["v"], out=s["out"], lse=s["lse"], weights=s["weights"],
                               weights_out=s["weights_out"], workspace=s["workspace"])
        return {"out": out, "lse": s["lse"], "weights": s["weights_out"]}
    return fq.fq_attn_paged(s["q"], s["batch"], s["k"], s["v"], out=s["out"], workspace=s["workspace"])


def _call_evict(s):
    import paper_2501_07139_amd as fq

    kept, new_len = fq.fq_cache_evict(s["batch"], s["weights"], s["k"], s["v"], s["dst"], s["case"]["keep"],
                                      s["case"]["recent"], k_out=s["k_out"], v_out=s["v_out"], kept=s["kept"],
                                      new_len=s["new_len"], weights_out=s["weights_out"])
    return {"kept": kept, "new_len": new_len, "k": s["k_out"], "v": s["v_out"], "weights": s["weights_out"]}


def _plain_rope(s):
    case, at = s["case"], 0
    for b, (n, c) in enumerate(s["lengths"]):
        rows, where = slice(at, at + n), (s["pages_of"][b][c:], s["rows_of"][b][c:])
        cos, sin = s["rope"][c:c + n, None, :, 0], s["rope"][c:c + n, None, :, 1]
        for name, gain in (("q", s["q_gain"]), ("kn", s["k_gain"])):
            x = s[name][rows].float().reshape(n, -1, D)
            if gain is not None:
                x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS) * gain.float()
            even, odd = x[..., 0::2], x[..., 1::2]
            y = torch.stack((even * cos - odd * sin, even * sin + odd * cos), -1).reshape(x.shape).half()
            if name == "q":
                s["out"][rows] = y.reshape(n, -1)
            else:
                s["k"][where[0], :, where[1]] = y
        s["v"][where[0], :, where[1]] = s["vn"][rows].reshape(n, -1, D)
        at += n
    return {"q": s["out"], "k": s["k"], "v": s["v"]}


def _plain_attention(s):
    case, at = s["case"], 0
    heads, kv = case["heads"], case["kv_heads"]
    group = heads // kv
    for b, (n, c) in enumerate(s["lengths"]):
        total = n + c
        keys, values = (s[x][s["pages_of"][b], :, s["rows_of"][b]].float().transpose(0, 1) for x in ("k", "v"))
        q = s["q"][at:at + n].float().reshape(n, kv, group, D).permute(1, 2, 0, 3).reshape(kv, group * n, D)
        scores = (torch.matmul(q, keys.transpose(1, 2).contiguous()) / math.sqrt(D)).view(kv, group, n, total)
        hidden = torch.arange(total, device="cuda") > torch.arange(c, total, device="cuda")[:, None]
        scores.masked_fill_(hidden, -math.inf)
        top = scores.amax(-1, keepdim=True)
        p = torch.exp(scores - top)
        del scores
        norm = p.sum(-1, keepdim=True)
        p /= norm
        out = torch.matmul(p.view(kv, group * n, total), values.contiguous())
        s["out"][at:at + n] = out.view(kv, group, n, D).permute(2, 0, 1, 3).reshape(n, heads * D).half()
        if case["weights"]:
            s["lse"][at:at + n] = (top + torch.log(norm))[..., 0].permute(2, 0, 1).reshape(n, heads)
            got = p.sum((1, 2))
            got[:, :c] += s["weights"][b, :, :c]
            s["weights_out"][b, :, :total] = got
        at += n
    if case["weights"]:
        return {"out": s["out"], "lse": s["lse"], "weights": s["weights_out"]}
    return s["out"]


def _plain_evict(s):
    case = s["case"]
    kv = case["kv_heads"]
    head = torch.arange(kv, device="cuda")[:, None]
    s["kept"].fill_(-1)
    s["weights_out"].zero_()
    for b, total in enumerate(s["total"]):
        m = min(total, case["keep"])
        recent = min(case["recent"], m)
        order = torch.sort(s["weights"][b, :, :total - recent], dim=1, descending=True, stable=True)[1]
        last = torch.arange(total - recent, total, device="cuda").expand(kv, recent)
        kept = torch.sort(torch.cat((order[:, :m - recent], last), 1), dim=1)[0]
        s["kept"][b, :, :m] = kept.int()
        s["new_len"][b] = m
        s["weights_out"][b, :, :m] = torch.gather(s["weights"][b], 1, kept)
        to_page, to_row = s["dst_of"][b]
        from_page, from_row = s["pages_of"][b][kept], s["rows_of"][b][kept]
        for src, dst in (("k", "k_out"), ("v", "v_out")):
            s[dst][to_page[None, :], head, to_row[None, :]] = s[src][from_page, head, from_row]
    return {"kept": s["kept"], "new_len": s["new_len"], "k": s["k_out"], "v": s["v_out"], "weights": s["weights_out"]}


# ------------------------------------------------------------------ the definitions in 64 bits
def _walk(pool, table, total, page):
    """The rows of one sequence, [heads, positions, 128], page after page."""
    used = [pool[int(table[i])] for i in range(-(-total // page))]
    return torch.cat(used, 1)[:, :total].double() if used else pool.new_zeros(pool.shape[1], 0, D).double()


def _exact_rope(s):
    page, kv = s["case"]["page"], s["case"]["kv_heads"]
    phase = torch.polar(torch.ones_like(_angles(max(s["total"]))), _angles(max(s["total"])))
    positions = torch.cat([torch.arange(c, c + n, device="cuda") for n, c in s["lengths"]])

    def turned(x, gain):
        x = x.double().view(x.shape[0], -1, D)
        if gain is not None:
            x = x * torch.rsqrt(x.square().sum(-1, keepdim=True) / D + EPS) * gain.double()
        pairs = torch.view_as_complex(x.reshape(*x.shape[:2], D // 2, 2).contiguous())
        return torch.view_as_real(pairs * phase[positions][:, None]).reshape(x.shape)

    q, new_k = turned(s["q"], s["q_gain"]), turned(s["kn"], s["k_gain"])
    new_v = s["vn"].double().view(-1, kv, D)
    k, v = s["k"].double(), s["v"].double()
    at = 0
    for b, (n, c) in enumerate(s["lengths"]):
        t = c
        while t < c + n:  # the run of tokens that lies in one page
            end = min(c + n, (t // page + 1) * page)
            rows, src, p = slice(t % page, t % page + end - t), slice(at + t - c, at + end - c), int(s["table"][b][t // page])
            k[p, :, rows], v[p, :, rows] = new_k[src].transpose(0, 1), new_v[src].transpose(0, 1)
            t = end
        at += n
    return {"q": q.reshape(q.shape[0], -1), "k": k, "v": v}


def _exact_attention(s):
    case = s["case"]
    heads, kv, page = case["heads"], case["kv_heads"], case["page"]
    group, at = heads // kv, 0
    q = s["q"].double().view(-1, heads, D)
    out, lse = torch.zeros_like(q), torch.zeros(q.shape[:2], dtype=torch.float64, device="cuda")
    sums = s["weights"].double().clone() if case["weights"] else None
    if sums is not None:
        for b, (n, c) in enumerate(s["lengths"]):
            sums[b, :, c:] = 0.0
    for b, (n, c) in enumerate(s["lengths"]):
        keys, values = (_walk(s[x], s["table"][b], n + c, page) for x in ("k", "v"))
        rows = slice(at, at + n)
        visible = torch.tril(torch.ones(n, n + c, dtype=torch.bool, device="cuda"), diagonal=c)
        for h in range(heads):
            logits = (q[rows, h] @ keys[h // group].T) * D ** -0.5
            logits = torch.where(visible, logits, torch.full_like(logits, -math.inf))
            lse[rows, h] = torch.logsumexp(logits, 1)
            p = torch.exp(logits - lse[rows, h, None])
            out[rows, h] = p @ values[h // group]
            if sums is not None:
                sums[b, h // group, :n + c] += p.sum(0)
        at += n
    if sums is None:
        return out.view(-1, heads * D)
    return {"out": out.view(-1, heads * D), "lse": lse, "weights": sums}


def _exact_evict(s):
    case = s["case"]
    kv, page, seqs = case["kv_heads"], case["page"], case["seqs"]
    w = s["weights"].cpu().numpy()
    kept = np.full((seqs, kv, case["keep"]), -1, dtype=np.int32)
    weights = np.zeros((seqs, kv, case["keep"]))
    k = torch.zeros(s["dst_pages"], kv, page, D, dtype=torch.float64, device="cuda")
    v = torch.zeros_like(k)
    for b, total in enumerate(s["total"]):
        m = min(total, case["keep"])
        old = total - min(case["recent"], m)
        rows_k, rows_v = _walk(s["k"], s["table"][b], total, page), _walk(s["v"], s["table"][b], total, page)
        for h in range(kv):
            rank = np.lexsort((np.arange(old), -w[b, h, :old]))  # by weight, then by position
            stays = np.ones(total, dtype=bool)
            stays[rank[m - (total - old):]] = False
            kept[b, h, :m] = np.flatnonzero(stays)
            weights[b, h, :m] = w[b, h, :total][stays]
            index = torch.from_numpy(np.flatnonzero(stays)).cuda()
            for first in range(0, m, page):
                part, p = index[first:first + page], int(s["dst_table"][b][first // page])
                k[p, h, :len(part)], v[p, h, :len(part)] = rows_k[h, part], rows_v[h, part]
    return {"kept": torch.from_numpy(kept).cuda(),
            "new_len": torch.tensor([min(t, case["keep"]) for t in s["total"]], dtype=torch.int32, device="cuda"),
            "k": k, "v": v, "weights": torch.from_numpy(weights).cuda()}


def exact(case, seed):
    s = _inputs(case, seed)
    return {"rope": _exact_rope, "attention": _exact_attention, "evict": _exact_evict}[case["kind"]](s)
