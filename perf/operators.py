"""The work by which the speed of attention and of its 8-bit cache is judged: reading a prompt, writing the cache,
the decode step over it, and moving its pages.

A case is a dict of plain values; `listed()` names twelve, `draw(rng)` makes more of the same kinds:

  prefill   hgf_diff_attention_prefill                (a prompt's differential attention; ragged batches; caps, biases, masks)
  decode    hgf_diff_attention_decode_kv8             (one token per sequence over the paged 8-bit cache)
  append    hgf_kv8_append, then hgf_kv8_gather       (new tokens into the cache, and what the cache then holds)
  fork      hgf_kv8_pages_fork, _copy_pages, _grow    (several continuations of one prompt)
  compact   hgf_kv8_pages_free, _compact, _copy_pages (finished sequences go, the pages in use move together)

Shapes are the paper's own model (d = 512: 8 heads of 32, context 512), the 7B shape (32 heads of 64) and the wide
heads of the attention cases (16 heads of 128).  Heads are those of differential attention: q and k hold 2 `heads`
heads of d_h columns, v `heads`.

With `own` false `run` computes the operators in their plain form, in torch alone."""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

LAMBDA = 0.8
BLOCK = 16                    # positions that share a scale of the cache

# ------------------------------------------------------------------------------------- the cases


def listed():
    return [
        # a prompt of a ragged 500 tokens for the paper's model: few rows, latency
        {"name": "prefill_512_t500", "kind": "prefill", "sequences": 1, "longest": 500, "earlier": 0, "heads": 8, "d_h": 32,
         "causal": True, "prefix": False, "document": 0, "cap": 0.0, "bias": False},
        # a packed batch scored at once: ragged sequences of several documents each, capped scores
        {"name": "prefill_documents", "kind": "prefill", "sequences": 6, "longest": 2048, "earlier": 0, "heads": 16, "d_h": 64,
         "causal": True, "prefix": False, "document": 300, "cap": 30.0, "bias": False},
        # the next turn of three conversations: rows behind earlier keys, a prefix that is read both ways, a distance bias
        {"name": "prefill_turn_d128", "kind": "prefill", "sequences": 3, "longest": 1001, "earlier": 3000, "heads": 16, "d_h": 128,
         "causal": True, "prefix": True, "document": 0, "cap": 0.0, "bias": True},
        # a long prompt of the 7B shape: the largest
        {"name": "prefill_7b_t4096", "kind": "prefill", "sequences": 1, "longest": 4096, "earlier": 0, "heads": 32, "d_h": 64,
         "causal": True, "prefix": False, "document": 0, "cap": 0.0, "bias": False},
        # a decode step of the paper's model for 24 users: launches and latencies
        {"name": "decode_512_b24", "kind": "decode", "sequences": 24, "longest": 512, "heads": 8, "d_h": 32, "page": 64,
         "cap": 0.0, "bias": False},
        # ragged long caches of the 7B shape
        {"name": "decode_7b_b8", "kind": "decode", "sequences": 8, "longest": 4096, "heads": 32, "d_h": 64, "page": 64,
         "cap": 0.0, "bias": False},
        # sixteen users with long caches, wide heads, capped scores and a distance bias, small pages
        {"name": "decode_d128_b16", "kind": "decode", "sequences": 16, "longest": 8192, "heads": 16, "d_h": 128, "page": 16,
         "cap": 50.0, "bias": True},
        # one new token for each of 24 users of the paper's model
        {"name": "append_512_b24", "kind": "append", "sequences": 24, "longest": 512, "new": 1, "heads": 8, "d_h": 32, "page": 64},
        # a prompt of 2048 tokens of the 7B shape into fresh pages
        {"name": "append_7b_t2048", "kind": "append", "sequences": 1, "longest": 2048, "new": 2048, "heads": 32, "d_h": 64, "page": 64},
        # pieces of prompts that begin and end inside blocks, wide heads
        {"name": "append_d128_pieces", "kind": "append", "sequences": 12, "longest": 1500, "new": 301, "heads": 16, "d_h": 128, "page": 128},
        # eight samples from each of four prompts, two layers
        {"name": "fork_512_8x4", "kind": "fork", "sequences": 4, "copies": 8, "longest": 512, "layers": 2, "heads": 8, "d_h": 32, "page": 64},
        # a third of 48 conversations ends and the rest moves together, two layers of the 7B shape
        {"name": "compact_7b_48", "kind": "compact", "sequences": 48, "longest": 600, "layers": 2, "heads": 32, "d_h": 64, "page": 32},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


# the most that one drawn case may do (a little under the largest listed ones)
_MOST_FLOPS, _MOST_BYTES = 1.3e11, 5.0e8


def draw(rng):
    while True:
        case = _draw(rng)
        w = work(case)
        if w["flops"] <= _MOST_FLOPS and w["bytes"] <= _MOST_BYTES:
            return case


def _draw(rng):
    kind = rng.choice(["prefill", "prefill", "decode", "decode", "append", "fork", "compact"])
    heads, d_h = rng.choice([1, 3, 4, 8, 16, 32]), rng.choice([16, 32, 64, 128])
    page = rng.choice([16, 32, 64, 128, 256])
    cap, bias = rng.choice([0.0, 0.0, 20.0, 50.0]), rng.random() < 0.3
    if kind == "prefill":
        return {"kind": kind, "sequences": _log(rng, 1, 16), "longest": _log(rng, 1, 4096),
                "earlier": rng.choice([0, 0, _log(rng, 1, 4096)]), "heads": heads, "d_h": d_h, "causal": rng.random() < 0.85,
                "prefix": rng.random() < 0.25, "document": rng.choice([0, 0, _log(rng, 8, 1000)]), "cap": cap, "bias": bias}
    if kind == "decode":
        return {"kind": kind, "sequences": _log(rng, 1, 64), "longest": _log(rng, 1, 8192), "heads": heads, "d_h": d_h, "page": page,
                "cap": cap, "bias": bias}
    if kind == "append":
        longest = _log(rng, 1, 4096)
        return {"kind": kind, "sequences": _log(rng, 1, 64), "longest": longest, "new": min(longest, rng.choice([1, _log(rng, 1, 2048)])),
                "heads": heads, "d_h": d_h, "page": page}
    if kind == "fork":
        return {"kind": kind, "sequences": _log(rng, 1, 16), "copies": rng.randint(1, 16), "longest": _log(rng, 1, 2048),
                "layers": rng.randint(1, 4), "heads": heads, "d_h": d_h, "page": page}
    return {"kind": kind, "sequences": _log(rng, 2, 64), "longest": _log(rng, 16, 1024), "layers": rng.randint(1, 4), "heads": heads,
            "d_h": d_h, "page": page}


# ------------------------------------------------------------------------------------- sizes that follow from a case


def _ragged(n, longest, salt, least=1):
    """n lengths from `least` to `longest`, the first one full: the same for every seed."""
    return [longest if i == 0 else least + ((i + 977 * salt) * 2654435761 % 4294967296) * (longest - least + 1) // 4294967296 for i in range(n)]


def _prompt(case):
    """Queries and keys of every sequence (the keys: earlier ones, then the queries' own)."""
    lq = _ragged(case["sequences"], case["longest"], 1)
    before = _ragged(case["sequences"], case["earlier"], 2, 0) if case["earlier"] else [0] * len(lq)
    return lq, [a + b for a, b in zip(lq, before)]


def _documents(case, lk):
    """Document numbers of the keys, one array a sequence: lengths about the mean, the last 9 positions of every
    second sequence padding (-1)."""
    r = random.Random(case["document"] * 1000003 + sum(lk))
    out = []
    for b, n in enumerate(lk):
        ids, d = np.empty(n, dtype=np.int32), 0
        at = 0
        while at < n:
            step = max(1, int(case["document"] * (0.3 + 1.4 * r.random())))
            ids[at:at + step] = d
            at, d = at + step, d + 1
        if b % 2 == 1:
            ids[max(0, n - 9):] = -1
        out.append(ids)
    return out


def _prefixes(case, lk):
    return [n // 3 if b % 2 == 0 else min(n, 7) for b, n in enumerate(lk)]


def _visible_pairs(case):
    lq, lk = _prompt(case)
    docs = _documents(case, lk) if case["document"] else None
    pre = _prefixes(case, lk) if case["prefix"] else [0] * len(lk)
    total = 0
    for b, (n, m) in enumerate(zip(lq, lk)):
        p = np.arange(m - n, m)
        if docs is None:
            total += int(np.maximum(p + 1, pre[b]).sum()) if case["causal"] else n * m
            continue
        # (documents follow each other: a key's document begins and ends where its number does)
        d = docs[b]
        real = int((d >= 0).sum())
        q = p[d[p] >= 0]
        lo, hi = np.searchsorted(d[:real], d[q], "left"), np.searchsorted(d[:real], d[q], "right")
        total += int((np.minimum(hi, np.maximum(q + 1, pre[b])) - lo).clip(0).sum() if case["causal"] else (hi - lo).sum())
    return total


def _cache_lengths(case):
    if case["kind"] == "append":
        n = _ragged(case["sequences"], case["longest"], 3)
        new = [min(a, b) for a, b in zip(n, _ragged(case["sequences"], case["new"], 4))]
        return n, new
    return _ragged(case["sequences"], case["longest"], 3), None


def work(case):
    """Bytes and operations of one pass: inputs read once, outputs written once."""
    kind, H, d = case["kind"], case["heads"], case["d_h"]
    if kind == "prefill":
        lq, lk = _prompt(case)
        return {"bytes": 2.0 * d * H * (3 * sum(lq) + 3 * sum(lk)), "flops": 8.0 * d * H * _visible_pairs(case)}
    row = 3 * H * (d + 4.0 / BLOCK)                 # codes and scales of a position
    if kind == "decode":
        n, _ = _cache_lengths(case)
        return {"bytes": sum(n) * row + len(n) * 6.0 * H * d, "flops": 8.0 * d * H * sum(n)}
    if kind == "append":
        n, new = _cache_lengths(case)
        earlier = sum((a - b) % BLOCK for a, b in zip(n, new))
        return {"bytes": sum(new) * (6.0 * H * d + row) + 2.0 * earlier * row + sum(n) * (row + 6.0 * H * d),
                "flops": 2.0 * 3 * H * d * (sum(new) + sum(n))}
    n, _ = _cache_lengths(case)
    page, L = case["page"], case["layers"]
    if kind == "fork":
        moved = case["copies"] * sum(1 for a in n if a % page)
        read = case["copies"] * sum(n)
    else:
        moved = len(_moves(case)[1])
        read = sum(a for i, a in enumerate(n) if i % 3 != 1)
    return {"bytes": L * (2.0 * moved * page * row + read * (row + 6.0 * H * d)), "flops": L * 3.0 * H * d * read}


# ------------------------------------------------------------------------------------- inputs


def _tables(case, n):
    """Page table, sequence numbers of the rows and pages in all: pages in an order as a server's use leaves it."""
    page = case["page"]
    S, W = len(n) + 3, (max(n) + page - 1) // page + 1
    copies = case.get("copies", 0)
    S += len(n) * copies
    used = sum((a + page - 1) // page for a in n)
    spare = 5 + 2 * len(n) * copies
    r = random.Random(used * 7919 + S)
    order = list(range(used + spare))
    r.shuffle(order)
    rows = list(range(S))
    r.shuffle(rows)
    table = np.full((S, W), -1, dtype=np.int32)
    lens, refs = np.zeros(S, dtype=np.int32), np.zeros(used + spare, dtype=np.int32)
    at = 0
    for i, a in enumerate(n):
        k = (a + page - 1) // page
        table[rows[i], :k] = order[at:at + k]
        refs[order[at:at + k]] = 1
        lens[rows[i]] = a
        at += k
    return table, lens, refs, rows


def _moves(case):
    """Pages that are in use behind the place where they would all fit, when every third sequence has gone."""
    n, _ = _cache_lengths(case)
    table, _, refs, rows = _tables(case, n)
    for i in range(len(n)):
        if i % 3 == 1:
            refs[table[rows[i]][table[rows[i]] >= 0]] = 0
    live = int((refs > 0).sum())
    return live, np.nonzero(refs[live:] > 0)[0] + live


class _Maker:
    """Seeded tensors on the GPU."""

    def __init__(self, seed):
        self.gen = torch.Generator(device="cuda")
        self.gen.manual_seed(seed)

    def normal(self, *shape):
        return torch.randn(shape, generator=self.gen, device="cuda")

    def half(self, *shape):
        """fp16 with a few channels that are larger than the others, as projections have them."""
        x = self.normal(*shape)
        x[..., ::11] *= 3.0
        return x.half()

    def pool(self, pages, blocks, heads, d_h):
        """Codes [pages, blocks, heads, 16, d_h] and scales [pages, blocks, heads] of a cache in use."""
        codes = torch.empty((pages, blocks, heads, BLOCK, d_h), dtype=torch.int8, device="cuda")
        step = max(1, (1 << 26) // (blocks * heads * BLOCK * d_h))
        for at in range(0, pages, step):
            part = codes[at:at + step]
            part.copy_((self.normal(*part.shape) * 36.0).round_().clamp_(-127, 127))
        scale = torch.exp2(torch.randint(-6, -3, (pages, blocks, heads), generator=self.gen, device="cuda").float())
        return codes, scale


def _ints(values):
    return torch.tensor(np.ascontiguousarray(values), dtype=torch.int32, device="cuda")


def _data(case, seed):
    """What both sides are given, in plain layouts."""
    mk, H, d = _Maker(seed), case["heads"], case["d_h"]
    if case["kind"] == "prefill":
        lq, lk = _prompt(case)
        s = {"lq": lq, "lk": lk, "q": mk.half(sum(lq), 2 * H, d), "k": mk.half(sum(lk), 2 * H, d), "v": mk.half(sum(lk), H, d)}
        s["slopes"] = torch.exp2(-8.0 * torch.arange(1, 2 * H + 1, device="cuda") / (2 * H)).float() if case["bias"] else None
        s["pre"] = _prefixes(case, lk) if case["prefix"] else None
        s["docs"] = _documents(case, lk) if case["document"] else None
        return s
    n, new = _cache_lengths(case)
    table, lens, refs, rows = _tables(case, n)
    s = {"n": n, "new": new, "table": _ints(table), "lens": _ints(lens), "refs": _ints(refs), "rows": rows}
    blocks = case["page"] // BLOCK
    s["layers"] = [(mk.pool(len(refs), blocks, 2 * H, d), mk.pool(len(refs), blocks, H, d)) for _ in range(case.get("layers", 1))]
    if case["kind"] == "decode":
        s["q"] = mk.half(len(n), 2 * H, d)
        s["slopes"] = torch.exp2(-8.0 * torch.arange(1, 2 * H + 1, device="cuda") / (2 * H)).float() if case["bias"] else None
    if case["kind"] == "append":
        s["k"], s["v"] = mk.half(sum(new), 2 * H, d), mk.half(sum(new), H, d)
    return s


def prepare(case, seed):
    s = _data(case, seed)
    s["case"] = case
    if own:
        from paper_2602_05269_amd import binding as hb
        s["hb"] = hb
    if case["kind"] == "prefill":
        s["cu_q"], s["cu_k"] = _ints(np.cumsum([0] + s["lq"])), _ints(np.cumsum([0] + s["lk"])) if case["earlier"] else None
        s["prefix"] = _ints(s["pre"]) if s["pre"] else None
        s["doc_k"] = s["doc_q"] = None
        if s["docs"]:
            s["doc_k"] = _ints(np.concatenate(s["docs"]))
            s["doc_q"] = _ints(np.concatenate([x[len(x) - n:] for x, n in zip(s["docs"], s["lq"])]))
        s["out"] = torch.empty((sum(s["lq"]), case["heads"], case["d_h"]), dtype=torch.float16, device="cuda")
        return s
    n, H, d, page = s["n"], case["heads"], case["d_h"], case["page"]
    s["seqs"] = _ints(s["rows"][:len(n)])
    s["cu"] = _ints(np.cumsum([0] + n))
    if case["kind"] == "append":
        s["cu_new"] = _ints(np.cumsum([0] + s["new"])) if case["new"] > 1 else None
    if case["kind"] == "fork":
        c = case["copies"]
        s["src"] = _ints(np.repeat(s["rows"][:len(n)], c))
        s["dst"] = _ints(s["rows"][len(n):len(n) * (c + 1)])
        s["ones"] = _ints([1] * (len(n) * c))
        s["cu_dst"] = _ints(np.cumsum([0] + list(np.repeat(n, c))))
    if case["kind"] == "compact":
        s["gone"] = _ints([s["rows"][i] for i in range(len(n)) if i % 3 == 1])
        stay = [i for i in range(len(n)) if i % 3 != 1]
        s["stay"], s["cu_stay"] = _ints([s["rows"][i] for i in stay]), _ints(np.cumsum([0] + [n[i] for i in stay]))
    if case["kind"] in ("fork", "compact"):          # (the engine's own copy of the tables, from which every pass begins)
        s["kept"] = [s[k].clone() for k in ("table", "lens", "refs")]
    if own:
        s["pages"] = hb.Kv8Pages(s["refs"].numel(), page, s["table"].shape[0], s["table"].shape[1])
        s["pages"].table.copy_(s["table"]), s["pages"].lens.copy_(s["lens"]), s["pages"].refs.copy_(s["refs"])
        s["caches"] = []
        while s["layers"]:
            (kc, ks), (vc, vs) = s["layers"].pop(0)
            c = hb.Kv8Cache(s["refs"].numel(), page, H, d)
            c.load(kc, ks, vc, vs)
            s["caches"].append(c)
            del kc, vc
        half = lambda t, h: torch.empty((t, h, d), dtype=torch.float16, device="cuda")
        s["out"] = half(len(n), H)
        if case["kind"] == "decode":
            s["scratch"] = torch.empty(hb.hgf_diff_attention_kv8_workspace_bytes(len(n), s["pages"], H, d), dtype=torch.uint8, device="cuda")
        rows = {"decode": 0, "append": sum(n), "fork": case.get("copies", 0) * sum(n), "compact": sum(n[i] for i in range(len(n)) if i % 3 != 1)}
        s["read"] = [(half(rows[case["kind"]], 2 * H), half(rows[case["kind"]], H)) for _ in s["caches"]]
    return s


# ------------------------------------------------------------------------------------- one pass


def run(s):
    return _own(s) if own else _plain(s)


def _own(s):
    case = s["case"]
    kind, hb = case["kind"], s["hb"]
    if kind == "prefill":
        return hb.hgf_diff_attention_prefill(s["q"], s["k"], s["v"], s["cu_q"], LAMBDA, cu_k=s["cu_k"], causal=case["causal"],
                                             prefix=s["prefix"], doc_q=s["doc_q"], doc_k=s["doc_k"], softcap=case["cap"],
                                             slopes=s["slopes"], out=s["out"])
    pages = s["pages"]
    if kind == "decode":
        return hb.hgf_diff_attention_decode_kv8(s["q"], s["caches"][0], pages, LAMBDA, seqs=s["seqs"], softcap=case["cap"],
                                                slopes=s["slopes"], out=s["out"], workspace=s["scratch"])
    if kind == "append":
        hb.hgf_kv8_append(s["k"], s["v"], s["caches"][0], pages, cu_new=s["cu_new"], seqs=s["seqs"])
        return hb.hgf_kv8_gather(s["caches"][0], pages, s["cu"], *s["read"][0], seqs=s["seqs"])
    pages.table.copy_(s["kept"][0]), pages.lens.copy_(s["kept"][1]), pages.refs.copy_(s["kept"][2])
    if kind == "fork":
        pairs, ok = hb.hgf_kv8_pages_fork(pages, s["src"], s["dst"])
        for c in s["caches"]:
            hb.hgf_kv8_copy_pages(c, pairs)
        read = [hb.hgf_kv8_gather(c, pages, s["cu_dst"], *r, seqs=s["dst"]) for c, r in zip(s["caches"], s["read"])]
        grown = hb.hgf_kv8_pages_grow(pages, s["dst"], s["ones"])
        return [pages.table, pages.lens, pages.refs, pairs, ok, grown, read]
    hb.hgf_kv8_pages_free(pages, s["gone"])
    pairs, count, moved = hb.hgf_kv8_pages_compact(pages)
    for c in s["caches"]:
        hb.hgf_kv8_copy_pages(c, pairs, count=count)
    read = [hb.hgf_kv8_gather(c, pages, s["cu_stay"], *r, seqs=s["stay"]) for c, r in zip(s["caches"], s["read"])]
    return [pages.table, pages.lens, pages.refs, pairs, count, moved, read]


# ------------------------------------------------------------------------------------- the plain forms


def _attend(q, k, v, seen, distance, slopes, cap):
    """Rows of differential attention in 32 bits: q [n, 2H, d], k [m, 2H, d], v [m, H, d]; `seen` and `distance` [n, m]."""
    H, d = v.shape[1], v.shape[2]
    x = torch.matmul(q.transpose(0, 1).contiguous(), k.permute(1, 2, 0).contiguous()) * (1.0 / math.sqrt(d))
    if cap:
        x = cap * torch.tanh(x / cap)
    if slopes is not None:
        x = x - slopes.view(-1, 1, 1) * distance
    if seen is not None:
        x = torch.where(seen, x, float("-inf"))
    top = x.amax(2, keepdim=True)
    x = torch.exp(x - torch.where(top == float("-inf"), 0.0, top))
    total = x.sum(2, keepdim=True)
    w = x / torch.where(total == 0, 1.0, total)
    w = 0.5 * (w[:H] - LAMBDA * w[H:])
    return torch.matmul(w, v.transpose(0, 1).contiguous()).transpose(0, 1)


def _plain_prefill(s):
    case, outs, at_q, at_k = s["case"], [], 0, 0
    plain_mask = not (case["causal"] or s["docs"])
    for b, (n, m) in enumerate(zip(s["lq"], s["lk"])):
        k, v = s["k"][at_k:at_k + m].float(), s["v"][at_k:at_k + m].float()
        j = torch.arange(m, device="cuda")
        for r in range(0, n, 1024):
            rows = slice(at_q + r, at_q + min(n, r + 1024))
            p = m - n + r + torch.arange(rows.stop - rows.start, device="cuda").view(-1, 1)
            seen = None
            if not plain_mask:
                seen = torch.ones((p.shape[0], m), dtype=torch.bool, device="cuda")
                if case["causal"]:
                    seen = j <= p
                    if s["prefix"] is not None:
                        seen = seen | (j < s["prefix"][b])
                if s["docs"]:
                    dq, dk = s["doc_q"][rows].view(-1, 1), s["doc_k"][at_k:at_k + m].view(1, -1)
                    seen = seen & (dq == dk) & (dk >= 0)
            outs.append(_attend(s["q"][rows].float(), k, v, seen, (p - j).abs().float(), s["slopes"], case["cap"]).half())
        at_q, at_k = at_q + n, at_k + m
    return torch.cat(outs)


def _positions(s, pool, table, row, n):
    """[n, heads, d] in 32 bits: the first n positions of a sequence."""
    codes, scale = pool
    page = s["case"]["page"]
    ids = table[row, :(n + page - 1) // page].long()
    x = codes[ids].float() * scale[ids].unsqueeze(-1).unsqueeze(-1)          # [pages, blocks, heads, 16, d]
    return x.transpose(2, 3).reshape(-1, codes.shape[2], codes.shape[4])[:n]


def _plain_decode(s):
    case, outs = s["case"], []
    k_pool, v_pool = s["layers"][0]
    for b, n in enumerate(s["n"]):
        k, v = (_positions(s, p, s["table"], s["rows"][b], n) for p in (k_pool, v_pool))
        distance = (n - 1 - torch.arange(n, device="cuda")).float().view(1, -1)
        outs.append(_attend(s["q"][b:b + 1].float(), k, v, None, distance, s["slopes"], case["cap"]).half())
    return torch.cat(outs)


def _scale_of(amax):
    """The smallest power of two of which 127 reach the magnitude (at least 2^-30)."""
    m, e = torch.frexp(amax)
    e = torch.where(m <= 127.0 / 128.0, e - 7, e - 6)
    return torch.exp2(torch.where(amax == 0, -30, e).clamp_min(-30).float())


def _plain_append(s, x, pool, slot, off, earlier):
    """New rows x [T, heads, d] into their blocks: `slot` names each token's block, `off` its place there, `earlier`
    how many positions of the block were there before."""
    codes, scale = (t.flatten(0, 1) for t in pool)
    x = x.float()
    amax = torch.zeros_like(scale).index_reduce_(0, slot, x.abs().amax(2), "amax")[slot]
    old = torch.where((earlier > 0).view(-1, 1), scale[slot], 0.0)
    new = torch.maximum(old, _scale_of(amax))
    keep = (torch.arange(BLOCK, device="cuda").view(1, -1) < earlier.view(-1, 1)).view(-1, 1, BLOCK, 1)
    block = codes[slot].float()
    block = torch.where(keep, torch.round(block * (old / new).unsqueeze(-1).unsqueeze(-1)), block)
    codes[slot] = block.to(torch.int8)
    scale[slot] = new
    codes[slot, :, off] = torch.round(x / new.unsqueeze(-1)).clamp(-127, 127).to(torch.int8)


def _plain_gather(s, pools, table, rows, n):
    return tuple(torch.cat([_positions(s, p, table, r, m) for r, m in zip(rows, n)]).half() for p in pools)


def _plain_grow(t, lens, refs, seqs, new, page):
    """Pages for sequences that become longer: the lowest free ones, in the order of the list."""
    seqs = seqs.long()
    have, want = (lens[seqs] + page - 1) // page, (lens[seqs] + new + page - 1) // page
    need = want - have
    upto = need.cumsum(0)
    free = torch.argsort((refs != 0).int(), stable=True)
    ok = (need == 0) | (upto <= (refs == 0).sum())
    i = torch.arange(t.shape[1], device="cuda").view(1, -1)
    fill = ok.view(-1, 1) & (i >= have.view(-1, 1)) & (i < want.view(-1, 1))
    pick = free[((upto - need).view(-1, 1) + i - have.view(-1, 1)).clamp(0, len(free) - 1)].int()
    t[seqs] = torch.where(fill, pick, t[seqs])
    count = torch.zeros_like(refs).index_add_(0, pick.long().flatten(), fill.int().flatten())
    refs += count
    lens[seqs] += torch.where(ok, new, 0)
    return ok.int()


def _plain_fork(t, lens, refs, src, dst, page):
    """dst shares src's full pages and gets a fresh one for the last, if that is not full: (from, to) pairs to copy."""
    src, dst = src.long(), dst.long()
    n = lens[src]
    full, need = n // page, (n % page != 0).int()
    upto = need.cumsum(0)
    free = torch.argsort((refs != 0).int(), stable=True)
    ok = (need == 0) | (upto <= (refs == 0).sum())
    fresh = free[(upto - 1).clamp(0, len(free) - 1)].int()
    last = t[src].gather(1, full.clamp_max(t.shape[1] - 1).long().view(-1, 1)).view(-1)
    i = torch.arange(t.shape[1], device="cuda").view(1, -1)
    share = ok.view(-1, 1) & (i < full.view(-1, 1))
    own_page = ok & (need == 1)
    t[dst] = torch.where(share, t[src], torch.where(own_page.view(-1, 1) & (i == full.view(-1, 1)), fresh.view(-1, 1), t[dst]))
    refs.index_add_(0, t[src].clamp_min(0).long().flatten(), share.int().flatten())
    refs.index_add_(0, fresh.long(), own_page.int())
    lens[dst] = torch.where(ok, n, 0)
    pairs = torch.stack([torch.where(own_page, last, -1), torch.where(own_page, fresh, -1)], 1)
    return pairs.int(), ok.int()


def _plain_copy(pools, pairs):
    """Contents of the pages that the pairs name; pairs of -1 copy nothing (they copy page 0 to itself)."""
    src, dst = (torch.where(pairs[:, i] >= 0, pairs[:, i], 0).long() for i in (0, 1))
    for pool in pools:
        for x in pool:
            part = x[src]
            zero = x[:1].clone()
            x[dst] = part
            hit = ((pairs[:, 1] == 0).long() * torch.arange(1, len(pairs) + 1, device="cuda")).amax(0)
            x[0] = torch.where(hit > 0, part[(hit - 1).clamp_min(0)], zero[0])


def _plain_compact(t, lens, refs, gone, page):
    gone = gone.long()
    used = torch.arange(t.shape[1], device="cuda").view(1, -1) < ((lens[gone] + page - 1) // page).view(-1, 1)
    refs.index_add_(0, t[gone].clamp_min(0).long().flatten(), -used.int().flatten())
    t[gone], lens[gone] = -1, 0
    at = torch.arange(len(refs), device="cuda")
    live = refs > 0
    count = live.sum()
    hole, mover = ~live & (at < count), live & (at >= count)
    room = max(1, len(refs) // 2)
    holes = torch.argsort((~hole).int(), stable=True)
    movers = torch.argsort((~mover).int(), stable=True)
    moves = mover.sum()
    there = torch.arange(room, device="cuda") < moves
    size = min(room, len(refs))
    pairs = torch.full((room, 2), -1, dtype=torch.int32, device="cuda")
    pairs[:size, 0] = torch.where(there[:size], movers[:size], -1).int()
    pairs[:size, 1] = torch.where(there[:size], holes[:size], -1).int()
    moved = torch.where(live, torch.where(mover, holes[(mover.cumsum(0) - 1).clamp_min(0)], at), -1).int()
    refs.copy_(torch.where(at < count, torch.where(hole, refs[movers[(hole.cumsum(0) - 1).clamp_min(0)]], refs), 0))
    used = torch.arange(t.shape[1], device="cuda").view(1, -1) < ((lens + page - 1) // page).view(-1, 1)
    t.copy_(torch.where(used, moved[t.clamp_min(0).long()], t))
    return pairs, moves.int().view(1), moved


def _plain(s):
    case = s["case"]
    kind = case["kind"]
    if kind == "prefill":
        return _plain_prefill(s)
    if kind == "decode":
        return _plain_decode(s)
    page, t, lens, refs = case["page"], s["table"], s["lens"], s["refs"]
    n, rows = s["n"], s["rows"]
    if kind == "append":
        cu = s["cu_new"] if s["cu_new"] is not None else torch.arange(len(n) + 1, device="cuda", dtype=torch.int32)
        i = torch.arange(sum(s["new"]), device="cuda", dtype=torch.int32)
        b = torch.searchsorted(cu, i, right=True) - 1
        seq = s["seqs"][b].long()
        start = lens[seq] - (cu[b + 1] - cu[b])
        pos = start + i - cu[b]
        slot = t[seq, (pos // page).long()].long() * (page // BLOCK) + pos % page // BLOCK
        earlier = (start - pos // BLOCK * BLOCK).clamp(0, BLOCK)
        for x, pool in zip((s["k"], s["v"]), s["layers"][0]):
            _plain_append(s, x, pool, slot, (pos % BLOCK).long(), earlier)
        return _plain_gather(s, [p for p in s["layers"][0]], t, rows, n)
    t.copy_(s["kept"][0]), lens.copy_(s["kept"][1]), refs.copy_(s["kept"][2])
    if kind == "fork":
        pairs, ok = _plain_fork(t, lens, refs, s["src"], s["dst"], page)
        for pools in s["layers"]:
            _plain_copy(pools, pairs)
        c = case["copies"]
        dst, m = rows[len(n):len(n) * (c + 1)], [x for x in n for _ in range(c)]
        read = [_plain_gather(s, p, t, dst, m) for p in s["layers"]]
        grown = _plain_grow(t, lens, refs, s["dst"], s["ones"], page)
        return [t, lens, refs, pairs, ok, grown, read]
    pairs, count, moved = _plain_compact(t, lens, refs, s["gone"], page)
    for pools in s["layers"]:
        _plain_copy(pools, pairs)
    stay = [i for i in range(len(n)) if i % 3 != 1]
    read = [_plain_gather(s, p, t, [rows[i] for i in stay], [n[i] for i in stay]) for p in s["layers"]]
    return [t, lens, refs, pairs, count, moved, read]


# ------------------------------------------------------------------------------------- the same in 64 bits


def _softmax_rows(x, m):
    """Weights of the scores x [n, m] where the mask m allows; zeros where it allows nothing."""
    e = torch.exp(x - x.masked_fill(~m, -1e300).amax(1, keepdim=True)).masked_fill(~m, 0.0)
    return e / e.sum(1, keepdim=True).clamp_min(1e-300)


def _heads64(q, k, v, m, away, slopes, cap):
    """Head by head from the definition: out[h] = (softmax(s_h) - lambda softmax(s_{H+h})) v_h / 2."""
    H, d = v.shape[1], v.shape[2]
    out = torch.empty((q.shape[0], H, d), dtype=torch.float64, device="cuda")
    for h in range(H):
        w = []
        for g in (h, H + h):
            x = (q[:, g].double() @ k[:, g].double().t().contiguous()) / d ** 0.5
            if cap:
                x = cap * torch.tanh(x / cap)
            if slopes is not None:
                x = x - slopes[g].double() * away
            w.append(_softmax_rows(x, m))
        out[:, h] = ((w[0] - LAMBDA * w[1]) / 2) @ v[:, h].double().contiguous()
    return out


def _values64(pool, ids, n):
    """[n, heads, d] of the pages `ids` in 64 bits."""
    codes, scale = pool
    parts = [codes[i].double() * scale[i].double()[..., None, None] for i in ids]
    return torch.cat([b.transpose(0, 1) for x in parts for b in x])[:n]


def _exact_blocks(old, scale, x, start):
    """One head's codes and block scales after the rows x [n, d] came behind `start` rows; exact in 64 bits."""
    codes, scale = list(old), list(scale)
    for first in range(start // BLOCK * BLOCK, start + x.shape[0], BLOCK):
        part = x[max(0, first - start):first + BLOCK - start]
        b, before = first // BLOCK, max(0, start - first)
        amax = part.abs().amax((0, 2))                                     # [heads]
        want = torch.where(amax > 0, torch.exp2(torch.ceil(torch.log2(amax.clamp_min(1e-30) / 127.0)).clamp_min(-30)), 2.0 ** -30)
        if before:
            want = torch.maximum(want, scale[b])
            codes[b] = codes[b].clone()
            codes[b][:, :before] = torch.round(codes[b][:, :before] * (scale[b] / want)[:, None, None])
        else:
            codes[b] = torch.zeros_like(codes[b])
        at = max(first, start) - first
        codes[b][:, at:at + part.shape[0]] = torch.round(part.transpose(0, 1) / want[:, None, None]).clamp(-127, 127)
        scale[b] = want
    return codes, scale


def exact(case, seed):
    """What run() returns, from the definitions in 64 bits (whole numbers as they are)."""
    s = _data(case, seed)
    if case["kind"] == "prefill":
        outs, at_q, at_k = [], 0, 0
        for b, (n, m) in enumerate(zip(s["lq"], s["lk"])):
            p, j = torch.arange(m - n, m, device="cuda")[:, None], torch.arange(m, device="cuda")[None, :]
            mask = torch.ones((n, m), dtype=torch.bool, device="cuda")
            if case["causal"]:
                mask &= (j <= p) | (j < (s["pre"][b] if s["pre"] else 0))
            if s["docs"]:
                ids = torch.from_numpy(s["docs"][b]).cuda()
                mask &= (ids[p] == ids[j]) & (ids[j] >= 0)
            outs.append(_heads64(s["q"][at_q:at_q + n], s["k"][at_k:at_k + m], s["v"][at_k:at_k + m], mask, (p - j).abs().double(),
                                 s["slopes"], case["cap"]))
            at_q, at_k = at_q + n, at_k + m
        return torch.cat(outs)
    page, n = case["page"], s["n"]
    table = s["table"].tolist()
    ids = [table[s["rows"][b]][:(m + page - 1) // page] for b, m in enumerate(n)]
    if case["kind"] == "decode":
        outs = []
        for b, m in enumerate(n):
            k, v = (_values64(p, ids[b], m) for p in s["layers"][0])
            away = torch.arange(m - 1, -1, -1, device="cuda").double()[None, :]
            outs.append(_heads64(s["q"][b:b + 1], k, v, torch.ones((1, m), dtype=torch.bool, device="cuda"), away, s["slopes"], case["cap"]))
        return torch.cat(outs)
    if case["kind"] == "append":
        if sum(s["new"]) > 6000:                     # (block by block on the host's side: too long beyond)
            return None
        outs = ([], [])
        at = 0
        for b, (m, new) in enumerate(zip(n, s["new"])):
            for which, x in enumerate((s["k"], s["v"])):
                codes, scale = s["layers"][0][which]
                old = [codes[i, blk].double() for i in ids[b] for blk in range(page // BLOCK)]
                sc = [scale[i, blk].double() for i in ids[b] for blk in range(page // BLOCK)]
                c, z = _exact_blocks(old, sc, x[at:at + new].double(), m - new)
                outs[which].append(torch.cat([(a * f[:, None, None]).transpose(0, 1) for a, f in zip(c, z)])[:m])
            at += new
        return tuple(torch.cat(o) for o in outs)
    keep = [i for i in range(len(n)) if case["kind"] == "fork" or i % 3 != 1]
    times = case.get("copies", 1)
    read = [tuple(torch.cat([_values64(p, ids[i], n[i]) for i in keep for _ in range(times)]) for p in pools) for pools in s["layers"]]
    return [None] * 6 + [read]
