"""Performance cases of the operators for several sequences that continue one prompt (the beams of a beam search, parallel
samples, candidate blocks): appending their keys and values to a paged cache, attention that reads the prompt's pages once
for all of them, the choice of the beams' next tokens, and the reordering of their page tables.

A case is a dict of plain values; `prepare` makes what a program holds before the call, `run` makes one pass and returns its
outputs (plain torch operations, or with `own` the library's calls), `work` states the bytes and operations that the pass
cannot do without, `exact` gives the outputs in 64 bits.

Heads are those of the models that the repository works with (12 x 64, 40 x 128 with keys and values of their own, 48 x 128
on one key / value head) and a generic grouped layout, 32 on 8.  A page of one layer holds a block for the keys of each
key / value head, [token][channel], and one for the values, [channel][token], in bf16."""
import math

import torch

own = False

HEADS = {"12x64": (12, 12, 64), "40x128": (40, 40, 128), "48on1x128": (48, 1, 128), "32on8x128": (32, 8, 128), "16on2x64": (16, 2, 64)}
DTYPE = {"fp32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-6


# ---- the cases -------------------------------------------------------------------------------------------------------

def listed():
    return [
        # one decoding step of four beams of the 68M-class draft model: the smallest call, made once a layer and token
        {"name": "append-beams-4", "kind": "append", "heads": "12x64", "dtype": "fp32", "seqs": 4, "tok": 1, "rows": 0, "prefix": 523,
         "own": 37, "page": 16, "rope": True, "gains": False},
        # a decoding step of a serving batch whose heads are normalised before the rotation
        {"name": "append-decode-192", "kind": "append", "heads": "32on8x128", "dtype": "bf16", "seqs": 192, "tok": 1, "rows": 0,
         "prefix": 2048, "own": 300, "page": 64, "rope": True, "gains": True},
        # ragged continuations (turns of a chat) of three sequences of the 13B-class target in one pass, padding rows between them
        {"name": "append-turns-5999", "kind": "append", "heads": "40x128", "dtype": "bf16", "seqs": 3, "tok": 0, "rows": 5999,
         "prefix": 211, "own": 2400, "page": 16, "rope": True, "gains": False},
        # attention of four beams of the draft model: the smallest call
        {"name": "attn-beams-4", "kind": "attn", "heads": "12x64", "dtype": "fp32", "seqs": 4, "tok": 1, "prefix": 523, "own": 37, "page": 16},
        # eight beams of the 13B-class target in the precision of the decode path: every query head has keys of its own
        {"name": "attn-13b-beams-8", "kind": "attn", "heads": "40x128", "dtype": "fp32", "seqs": 8, "tok": 1, "prefix": 2048, "own": 130,
         "page": 16},
        # sixteen candidate blocks of six tokens verified behind one code prompt by the multi-query target
        {"name": "attn-mqa-blocks-16x6", "kind": "attn", "heads": "48on1x128", "dtype": "bf16", "seqs": 16, "tok": 6, "prefix": 3001,
         "own": 77, "page": 16},
        # a serving batch behind a long shared document: the largest
        {"name": "attn-gqa-96-long", "kind": "attn", "heads": "32on8x128", "dtype": "bf16", "seqs": 96, "tok": 1, "prefix": 65537,
         "own": 700, "page": 64},
        # four beams over the vocabulary of the 13B-class pair
        {"name": "select-4x32000", "kind": "select", "groups": 1, "beams": 4, "vocab": 32000, "k": 4, "dtype": "fp32", "done": False},
        # eight prompts of eight beams, twice as many candidates as beams (those that end are taken out by the caller)
        {"name": "select-8x8x49152", "kind": "select", "groups": 8, "beams": 8, "vocab": 49152, "k": 16, "dtype": "fp32", "done": True},
        # a batch of 64 prompts of sixteen beams over a large vocabulary, logits in bf16
        {"name": "select-64x16x128001", "kind": "select", "groups": 64, "beams": 16, "vocab": 128001, "k": 16, "dtype": "bf16", "done": True},
        # four beams of the 13B-class target: forty layers of the page that is being filled
        {"name": "reorder-4-13b", "kind": "reorder", "groups": 1, "beams": 4, "heads": "40x128", "layers": 40, "page": 16, "cols": 4, "len": 37},
        # sixteen prompts of eight beams
        {"name": "reorder-16x8-gqa", "kind": "reorder", "groups": 16, "beams": 8, "heads": "32on8x128", "layers": 16, "page": 16, "cols": 6,
         "len": 71},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges; costs no more than the largest listed one of its kind."""
    kind = rng.choice(["append", "attn", "attn", "select", "reorder"])
    heads = rng.choice(sorted(HEADS))
    nq, nkv, dh = HEADS[heads]
    page, dtype = rng.choice([4, 12, 16, 16, 32, 64]), rng.choice(["fp32", "bf16"])
    if kind == "append":
        rope, gains = rng.random() < 0.8, rng.random() < 0.3
        if rng.random() < 0.5:
            seqs, tok = _log(rng, 1, 200), rng.choice([1, 1, 1, 2, 5, 16])
            return {"kind": kind, "heads": heads, "dtype": dtype, "seqs": seqs, "tok": tok, "rows": 0, "prefix": _log(rng, 1, 9000),
                    "own": tok + _log(rng, 1, 300), "page": page, "rope": rope, "gains": gains}
        rows = min(_log(rng, 17, 8000), 5999 * 120 * 128 * 2 // ((nq + 2 * nkv) * dh * (4 if dtype == "fp32" else 2)))
        seqs = rng.randint(1, 6)
        return {"kind": kind, "heads": heads, "dtype": dtype, "seqs": seqs, "tok": 0, "rows": rows, "prefix": _log(rng, 1, 4000),
                "own": rows // seqs + rng.randint(rows // seqs // 2 + seqs + 2, rows + 5), "page": page, "rope": rope, "gains": gains}
    if kind == "attn":
        prefix = 0 if rng.random() < 0.1 else _log(rng, 1, 66000)
        tok = rng.choice([1, 1, 1, 2, 5, 8])
        seqs = min(_log(rng, 1, 100), max(1, int(1.0e11 / (4.0 * nq * dh * tok * (prefix + 1000)))), max(1, int(8.0e8 / (nq * tok * (prefix + 1000)))))
        return {"kind": kind, "heads": heads, "dtype": dtype, "seqs": seqs, "tok": tok, "prefix": prefix, "own": tok + _log(rng, 1, 900), "page": page}
    if kind == "select":
        beams, vocab = rng.choice([1, 2, 4, 5, 8, 16, 32]), _log(rng, 500, 130000)
        groups = _log(rng, 1, max(1, min(64, 64 * 16 * 128001 // (beams * vocab * (2 if dtype == "fp32" else 1)))))
        return {"kind": kind, "groups": groups, "beams": beams, "vocab": vocab, "k": min(64, beams * rng.choice([1, 2])), "dtype": dtype,
                "done": rng.random() < 0.5}
    beams, layers, cols = rng.choice([2, 3, 4, 8, 16]), _log(rng, 2, 40), rng.randint(2, 12)
    groups = _log(rng, 1, max(1, min(16, int(2.0e9 / (beams * layers * cols * 4 * nkv * page * dh)))))
    return {"kind": kind, "groups": groups, "beams": beams, "heads": heads, "layers": layers, "page": page, "cols": cols,
            "len": rng.randint(1, cols * page)}


# ---- inputs ----------------------------------------------------------------------------------------------------------

def _lens(c):
    """Own lengths of the sequences: all up to c["own"], ragged, none shorter than the call's tokens."""
    low = max(1, c["tok"])
    return [low + (c["own"] - low) * (97 - (61 * b) % 97) // 97 for b in range(c["seqs"])]


def _turns(c):
    """Ragged rows: (sequence, own position) of every row, -1 for the padding behind each sequence's rows."""
    n, s = c["rows"], c["seqs"]
    share, seq, pos = n // s, [], []
    for b in range(s):
        m = share if b + 1 < s else n - share * (s - 1)
        live = m - (m // 40 if m > 40 else 0)
        first = (c["own"] - m) * (b + 1) // (s + 1) if c["own"] > m else 0
        seq += [b] * live + [-1] * (m - live)
        pos += list(range(first, first + live)) + [-1] * (m - live)
    return seq, pos


def _pages_per_seq(c):
    return -(-c["own"] // c["page"])


def _copies(beams):
    """Beams of a group that the reorder cases let end."""
    return max(1, beams * 3 // 8)


def prepare(case, seed):
    c, dev = case, torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(seed)

    def ints(v):
        return torch.tensor(v, dtype=torch.int32, device=dev)

    if c["kind"] == "select":
        rows = c["groups"] * c["beams"]
        st = {"case": c, "logits": (2.5 * torch.randn(rows, c["vocab"], generator=g, device=dev)).to(DTYPE[c["dtype"]]),
              "scores": -20.0 * torch.rand(rows, generator=g, device=dev), "done": None}
        if c["done"]:
            st["done"] = (torch.rand(rows, generator=g, device=dev) < 0.1).to(torch.int32)
            st["done"][:: c["beams"]] = 0            # a group with every beam done is not searched on
        return st
    nq, nkv, dh = HEADS[c["heads"]]
    if c["kind"] == "reorder":
        n, nb = c["groups"] * c["beams"], c["beams"]
        order = torch.randperm(n * c["cols"], generator=g, device=dev).to(torch.int32).reshape(n, c["cols"])
        pool = torch.randn(c["layers"], n * c["cols"], 2, nkv, c["page"] * dh, generator=g, device=dev, dtype=torch.float32).to(torch.bfloat16) \
            if c["layers"] * n * c["cols"] * nkv * c["page"] * dh < 1 << 27 else \
            torch.randint(0, 1 << 14, (c["layers"], n * c["cols"], 2, nkv, c["page"] * dh), generator=g, device=dev, dtype=torch.int16).view(torch.bfloat16)
        # some beams end, as many of the others go on twice; the order of the children is random
        rank = torch.rand(c["groups"], nb, generator=g, device=dev).argsort(1)
        dead = _copies(nb)
        kids = torch.cat([rank[:, dead:], rank[:, dead:dead + 1].expand(-1, max(0, 2 * dead - nb)), rank[:, dead:2 * dead]], 1)[:, :nb]
        parents = kids.gather(1, torch.rand(c["groups"], nb, generator=g, device=dev).argsort(1)).to(torch.int32).contiguous()
        return {"case": c, "pool": pool, "tables": order, "parents": parents, "tables_out": torch.empty_like(order)}
    cols = _pages_per_seq(c)
    n = c["seqs"] * cols
    st = {"case": c, "tables": torch.randperm(n, generator=g, device=dev).to(torch.int32).reshape(c["seqs"], cols),
          "pages": torch.randn(n, 2, nkv, c["page"] * dh, generator=g, device=dev).to(torch.bfloat16), "dims": (nq, nkv, dh)}
    if c["kind"] == "append":
        if c["rows"]:
            seq, pos = _turns(c)
            st["seq"], st["pos"], st["lens"], rows = ints(seq), ints(pos), None, c["rows"]
        else:
            st["seq"], st["pos"], st["lens"], rows = None, None, ints(_lens(c)), c["seqs"] * c["tok"]
        st["qkv"] = torch.randn(rows, (nq + 2 * nkv) * dh, generator=g, device=dev).to(DTYPE[c["dtype"]])
        st["q"] = torch.zeros(rows, nq * dh, dtype=DTYPE[c["dtype"]], device=dev)
        st["gains"] = tuple(1.0 + 0.2 * torch.randn(2, dh, generator=g, device=dev)) if c["gains"] else (None, None)
        st["rope"] = None
        if c["rope"]:                                # (cos, sin) of every position and channel pair: a program keeps one table
            at = torch.arange(c["prefix"] + cols * c["page"], device=dev, dtype=torch.float64)[:, None]
            at = at * torch.pow(torch.tensor(10000.0, device=dev, dtype=torch.float64), -torch.arange(dh // 2, device=dev, dtype=torch.float64) * 2 / dh)
            st["rope"] = torch.stack([at.cos(), at.sin()], -1).to(torch.float32).contiguous()
        return st
    np_ = -(-c["prefix"] // c["page"])
    st["prefix_table"] = torch.randperm(max(1, np_), generator=g, device=dev).to(torch.int32)
    st["prefix_pages"] = torch.randn(max(1, np_), 2, nkv, c["page"] * dh, generator=g, device=dev).to(torch.bfloat16)
    st["lens"] = ints(_lens(c))
    # queries a little longer than a unit normal: some positions carry weight, as trained heads have it
    st["q"] = (1.5 * torch.randn(c["seqs"] * c["tok"], nq * dh, generator=g, device=dev)).to(DTYPE[c["dtype"]])
    st["out"], st["lse"] = torch.empty_like(st["q"]), torch.empty(c["seqs"] * c["tok"], nq, dtype=torch.float32, device=dev)
    return st


# ---- one pass --------------------------------------------------------------------------------------------------------

def _plain_append(c, st):
    nq, nkv, dh = st["dims"]
    x = st["qkv"].float().reshape(-1, nq + 2 * nkv, dh)
    rows, cols, pt = x.shape[0], st["tables"].shape[1], c["page"]
    if c["rows"]:
        seq, pos = st["seq"].long(), st["pos"].long()
        live = seq >= 0
    else:
        i = torch.arange(rows, device=x.device)
        seq = i // c["tok"]
        pos = st["lens"].long()[seq] - c["tok"] + i % c["tok"]
        live = torch.ones_like(seq, dtype=torch.bool)
    at = torch.where(live, pos, torch.zeros_like(pos))
    x, v = x[:, :nq + nkv], x[:, nq + nkv:]
    if c["gains"]:
        gain = torch.cat([st["gains"][0].expand(nq, dh), st["gains"][1].expand(nkv, dh)])
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * gain
    if c["rope"]:
        cs, sn = st["rope"][c["prefix"] + at][:, None].unbind(-1)
        a, b = x[..., :dh // 2], x[..., dh // 2:]
        x = torch.cat([a * cs - b * sn, b * cs + a * sn], -1)
    st["q"].copy_(torch.where(live[:, None], x[:, :nq].reshape(rows, -1).to(st["q"].dtype), st["q"]))
    slot = st["tables"].long()[torch.where(live, seq, torch.zeros_like(seq)), at // pt] * pt + at % pt
    keys, vals = x[:, nq:].to(torch.bfloat16), v.to(torch.bfloat16)
    slot, keys, vals = slot[live], keys[live], vals[live]
    pages = st["pages"]
    pages[:, 0].view(-1, nkv, pt, dh)[slot // pt, :, slot % pt] = keys
    pages[:, 1].view(-1, nkv, dh, pt)[slot // pt, :, :, slot % pt] = vals
    return {"q": st["q"], "pages": pages}


def _plain_attn(c, st):
    nq, nkv, dh = st["dims"]
    s, t, g, pt, p = c["seqs"], c["tok"], nq // nkv, c["page"], c["prefix"]
    # queries of a key / value head: [head][sequence][token and query head][channel]
    q = st["q"].float().reshape(s, t, nkv, g, dh).permute(2, 0, 1, 3, 4).reshape(nkv, s, t * g, dh) * (dh ** -0.5)
    own_pages = st["pages"][st["tables"].long()].float()                           # [sequence][page][K | V][head][...]
    n = own_pages.shape[1] * pt
    k = own_pages[:, :, 0].reshape(s, -1, nkv, pt, dh).permute(2, 0, 4, 1, 3).reshape(nkv, s, dh, n)
    v = own_pages[:, :, 1].reshape(s, -1, nkv, dh, pt).permute(2, 0, 1, 4, 3).reshape(nkv, s, n, dh)
    see = st["lens"].long()[:, None] - t + 1 + torch.arange(t, device=q.device)    # own positions that a token sees
    see = torch.arange(n, device=q.device) < see[:, :, None]                       # [sequence][token][position]
    see = see[:, :, None].expand(s, t, g, n).reshape(s, t * g, n)
    a = torch.matmul(q, k).masked_fill(~see, -math.inf)
    m = a.amax(-1, keepdim=True)
    if p:
        pre = st["prefix_pages"][st["prefix_table"].long()].float()
        pk = pre[:, 0].reshape(-1, nkv, pt, dh).permute(1, 3, 0, 2).reshape(nkv, dh, -1)[:, :, :p].contiguous()
        pv = pre[:, 1].reshape(-1, nkv, dh, pt).permute(1, 0, 3, 2).reshape(nkv, -1, dh)[:, :p].contiguous()
        b = torch.matmul(q.reshape(nkv, -1, dh), pk).reshape(nkv, s, t * g, p)
        m = torch.maximum(m, b.amax(-1, keepdim=True))
        b = (b - m).exp_()
    a = (a - m).exp_()
    l, o = a.sum(-1, keepdim=True), torch.matmul(a, v)
    if p:
        l = l + b.sum(-1, keepdim=True)
        o = o + torch.matmul(b.reshape(nkv, -1, p), pv).reshape(nkv, s, t * g, dh)
    out = (o / l).reshape(nkv, s, t, g, dh).permute(1, 2, 0, 3, 4).reshape(s * t, nq * dh)
    lse = (m + l.log()).reshape(nkv, s, t, g).permute(1, 2, 0, 3).reshape(s * t, nq)
    return {"out": out.to(st["q"].dtype), "lse": lse}


def _plain_select(c, st):
    ng, nb, v, k = c["groups"], c["beams"], c["vocab"], c["k"]
    x = st["logits"].double()                        # candidates of different beams can be closer than 32 bits tell
    m = x.amax(-1, keepdim=True)
    lse = m + (x - m).exp_().sum(-1, keepdim=True).log()
    score = st["scores"].double()[:, None]
    key = x - lse + score
    if c["done"]:                                    # a finished beam goes on with the end token (id 2) and its score
        end = torch.arange(v, device=x.device) == 2
        key = torch.where(st["done"][:, None] != 0, torch.where(end, score, torch.full_like(score, -math.inf)), key)
    key = key.reshape(ng, nb * v)
    border = key.topk(k, 1).values[:, -1:]
    above, at_border = key > border, key == border
    need = k - above.sum(1, keepdim=True)
    take = above | (at_border & (at_border.cumsum(1, dtype=torch.int32) <= need))
    # the k taken places in ascending order, then by key: equal keys keep their order
    place = torch.arange(nb * v, 0, -1, device=x.device, dtype=torch.int32)
    place = nb * v - torch.where(take, place, torch.zeros_like(place)).topk(k, 1).values.long()
    best, order = key.gather(1, place).sort(dim=1, descending=True, stable=True)
    place = place.gather(1, order)
    parent, token = (place // v).to(torch.int32), (place % v).to(torch.int32)
    done = token == 2
    if c["done"]:
        done = done | (st["done"].reshape(ng, nb).gather(1, parent.long()) != 0)
    return {"tokens": token, "parents": parent, "scores": best.float(), "done": done.to(torch.int32)}


def _plain_reorder(c, st):
    ng, nb, pt = c["groups"], c["beams"], c["page"]
    full, live = c["len"] // pt, c["len"] % pt
    old, par = st["tables"].reshape(ng, nb, -1), st["parents"].long()
    new = st["tables_out"].copy_(st["tables"]).view(ng, nb, -1)
    new[:, :, :full] = old.gather(1, par[:, :, None].expand(-1, -1, full))
    if live:
        b = torch.arange(nb, device=old.device)
        same = par[:, :, None] == par[:, None, :]                                  # [group][child][other child]
        further = (same & (b[None, :] < b[:, None])).any(2)                        # not its parent's first child
        ended = ~(par[:, :, None] == b).any(1)
        free = torch.where(ended, b, b + nb).argsort(1)                            # beams without a child, in order
        page = old[:, :, full].long()
        src = page.gather(1, par)
        dst = torch.where(further, page.gather(1, free.gather(1, (further.cumsum(1) - 1).clamp(min=0))), src)
        new[:, :, full] = dst.to(torch.int32)
        st["pool"][:, dst.reshape(-1)] = st["pool"][:, src.reshape(-1)]
    return {"tables": st["tables_out"], "pool": st["pool"]}


def _own(c, st):
    from paper_2405_04304_amd import binding as B

    kind = c["kind"]
    if kind == "select":
        if "ws" not in st:
            n, dev = (c["groups"], c["k"]), st["logits"].device
            st["ws"] = torch.empty(B.disco_beam_select_bytes(c["groups"], c["beams"], c["vocab"], c["k"]), dtype=torch.uint8, device=dev)
            st["res"] = {"tokens": torch.empty(n, dtype=torch.int32, device=dev), "parents": torch.empty(n, dtype=torch.int32, device=dev),
                         "scores": torch.empty(n, dtype=torch.float32, device=dev), "done": torch.empty(n, dtype=torch.int32, device=dev)}
        r = st["res"]
        B.disco_beam_select(st["logits"], st["scores"], c["groups"], c["beams"], c["k"], r["tokens"], r["parents"], r["scores"], st["ws"],
                            done=st["done"], done_out=r["done"], end_token=2)
        return r
    if kind == "reorder":
        nq, nkv, dh = HEADS[c["heads"]]
        B.disco_beam_reorder(st["pool"], st["tables"], st["parents"], st["tables_out"], c["groups"], c["beams"], c["len"], c["page"])
        return {"tables": st["tables_out"], "pool": st["pool"]}
    nq, nkv, dh = st["dims"]
    if kind == "append":
        if "kv" not in st:
            st["kv"] = B.SharedKV(st["pages"], st["tables"], st["lens"], c["page"], nkv, dh, prefix_len=c["prefix"])
        B.disco_append(st["kv"], st["qkv"], nq, st["q"], seq=st["seq"], pos=st["pos"], rope=st["rope"], q_gain=st["gains"][0],
                       k_gain=st["gains"][1], eps=EPS)
        return {"q": st["q"], "pages": st["pages"]}
    if "kv" not in st:
        st["kv"] = B.SharedKV(st["pages"], st["tables"], st["lens"], c["page"], nkv, dh, prefix_pages=st["prefix_pages"],
                              prefix_len=c["prefix"], prefix_table=st["prefix_table"])
        st["ws"] = torch.empty(B.disco_attn_shared_bytes(st["kv"], c["tok"], nq, max_len=c["own"]), dtype=torch.uint8, device=st["q"].device)
    B.disco_attn_shared(st["kv"], st["q"], c["tok"], nq, st["out"], st["ws"], lse=st["lse"], max_len=c["own"])
    return {"out": st["out"], "lse": st["lse"]}


def run(state):
    c = state["case"]
    if own:
        return _own(c, state)
    return {"append": _plain_append, "attn": _plain_attn, "select": _plain_select, "reorder": _plain_reorder}[c["kind"]](c, state)


# ---- what a pass cannot do without -----------------------------------------------------------------------------------

def work(case):
    c = case
    if c["kind"] == "select":
        rows = c["groups"] * c["beams"]
        return {"bytes": rows * c["vocab"] * (4 if c["dtype"] == "fp32" else 2) + 4 * rows + 16 * c["groups"] * c["k"], "flops": 4 * rows * c["vocab"]}
    nq, nkv, dh = HEADS[c["heads"]]
    if c["kind"] == "reorder":
        n = c["groups"] * c["beams"]
        copied = c["groups"] * _copies(c["beams"]) if c["len"] % c["page"] else 0
        return {"bytes": 8 * n * c["cols"] + 4 * n + 2 * copied * c["layers"] * 4 * nkv * c["page"] * dh, "flops": 0}
    es = 4 if c["dtype"] == "fp32" else 2
    if c["kind"] == "append":
        rows = c["rows"] or c["seqs"] * c["tok"]
        return {"bytes": rows * (((nq + 2 * nkv) + nq) * dh * es + 4 * nkv * dh + (4 * dh if c["rope"] else 0)), "flops": rows * (nq + nkv) * dh * 8}
    own_len = sum(_lens(c))
    rows = c["seqs"] * c["tok"] * nq
    pairs = nq * c["tok"] * (c["seqs"] * (c["prefix"] - (c["tok"] - 1) / 2) + own_len)
    return {"bytes": rows * (2 * dh * es + 4) + 4 * nkv * dh * (c["prefix"] + own_len), "flops": 4 * dh * pairs}


# ---- the outputs in 64 bits ------------------------------------------------------------------------------------------

def _exact_append(c, st):
    nq, nkv, dh = st["dims"]
    pt, half = c["page"], dh // 2
    x = st["qkv"].double().reshape(-1, nq + 2 * nkv, dh)
    tables, lens = st["tables"].tolist(), st["lens"].tolist() if st["lens"] is not None else None
    where = list(zip(*_turns(c))) if c["rows"] else [(b, lens[b] - c["tok"] + t) for b in range(c["seqs"]) for t in range(c["tok"])]
    rows = [i for i, (b, _) in enumerate(where) if b >= 0]
    idx = torch.tensor(rows, device=x.device)
    pos = torch.tensor([where[i][1] for i in rows], device=x.device)
    page = torch.tensor([tables[where[i][0]][where[i][1] // pt] for i in rows], device=x.device)
    y = x[idx].clone()
    if c["gains"]:
        for lo, hi, gain in ((0, nq, st["gains"][0]), (nq, nq + nkv, st["gains"][1])):
            part = y[:, lo:hi]
            y[:, lo:hi] = part / (part.pow(2).sum(-1, keepdim=True) / dh + EPS).sqrt() * gain.double()
    if c["rope"]:
        z = torch.complex(y[:, :nq + nkv, :half].contiguous(), y[:, :nq + nkv, half:].contiguous())
        z = z * torch.view_as_complex(st["rope"].double()[c["prefix"] + pos])[:, None]
        y[:, :nq + nkv, :half], y[:, :nq + nkv, half:] = z.real, z.imag
    q = st["q"].double()
    q[idx] = y[:, :nq].reshape(len(rows), -1)
    pages = st["pages"].double()
    flat = pages.view(-1)
    chan = torch.arange(dh, device=x.device)
    head = torch.arange(nkv, device=x.device)[:, None]
    base = (page * 2 * nkv * pt * dh)[:, None, None]
    off = (pos % pt)[:, None, None]
    flat[base + head * pt * dh + off * dh + chan] = y[:, nq:nq + nkv]
    flat[base + (nkv + head) * pt * dh + chan * pt + off] = y[:, nq + nkv:]
    return {"q": q, "pages": pages}


def _exact_attn(c, st):
    nq, nkv, dh = st["dims"]
    pt, t, g = c["page"], c["tok"], nq // nkv
    q = st["q"].double().reshape(c["seqs"], t, nq, dh)
    out, lse = torch.empty_like(q), torch.empty(c["seqs"], t, nq, dtype=torch.float64, device=q.device)
    tables, lens = st["tables"].long(), _lens(c)
    for h in range(nkv):
        pre = st["prefix_pages"][st["prefix_table"].long(), :, h].double()
        pk, pv = pre[:, 0].reshape(-1, dh)[:c["prefix"]], pre[:, 1].reshape(-1, dh, pt).transpose(1, 2).reshape(-1, dh)[:c["prefix"]]
        qh = q[:, :, h * g:(h + 1) * g].contiguous()
        a = (qh.reshape(-1, dh) @ pk.T).reshape(c["seqs"], t * g, -1) / math.sqrt(dh)
        for b in range(c["seqs"]):
            ow = st["pages"][tables[b], :, h].double()
            k, v = ow[:, 0].reshape(-1, dh)[:lens[b]], ow[:, 1].reshape(-1, dh, pt).transpose(1, 2).reshape(-1, dh)[:lens[b]]
            w = (qh[b].reshape(-1, dh) @ k.T).reshape(t, g, -1) / math.sqrt(dh)
            for j in range(t - 1):
                w[j, :, lens[b] - t + 1 + j:] = -math.inf
            w = torch.cat([a[b], w.reshape(t * g, -1)], 1)
            z = torch.logsumexp(w, 1)
            w = (w - z[:, None]).exp()
            o = w[:, :c["prefix"]] @ pv + w[:, c["prefix"]:] @ v
            out[b, :, h * g:(h + 1) * g] = o.reshape(t, g, dh)
            lse[b, :, h * g:(h + 1) * g] = z.reshape(t, g)
    return {"out": out.reshape(-1, nq * dh), "lse": lse.reshape(-1, nq)}


def _exact_select(c, st):
    """The scores alone: tokens and parents are whole numbers."""
    got = []
    for gr in range(c["groups"]):
        parts = []
        for b in range(gr * c["beams"], (gr + 1) * c["beams"]):
            if c["done"] and int(st["done"][b]):
                parts.append(st["scores"][b:b + 1].double())
            else:
                parts.append((torch.log_softmax(st["logits"][b].double(), 0) + st["scores"][b].double()).topk(min(c["k"], c["vocab"])).values)
        got.append(torch.cat(parts).topk(c["k"]).values)
    return {"tokens": None, "parents": None, "scores": torch.stack(got), "done": None}


def exact(case, seed):
    if case["kind"] == "reorder":
        return None                                  # page ids and moved bits
    st = prepare(case, seed)
    return {"append": _exact_append, "attn": _exact_attn, "select": _exact_select}[case["kind"]](case, st)
