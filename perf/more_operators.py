"""Drafting and eviction on a paged key/value cache held in 4 bits, as a program that serves tokens calls them.

The cache keeps, for every token and every key/value head, a row of `d` keys and a row of `d` values as 4-bit ids of 16 levels that the
head has learned, times the row's largest magnitude:

  codes   [pages, heads, page, d/2] uint8, channel 2b in the low and 2b+1 in the high half of byte b
  scale   [pages, heads, page]      of the cache's type, the largest magnitude of the row
  levels  [heads, 16]               of the cache's type, ascending

and beside it, where tokens are to be evicted, one float32 a token and head (the same layout as the scales): the attention weight that the
token has been given so far.

Four kinds of call:

  tree     softmax(q.K) V for a tree of drafted tokens, the last ones of their sequence: a query sees what lies before the tree, and
           of the tree the tokens whose bits its row of the mask has set
  weigh    the attention weights of some queries, from the logarithms of their softmax sums, added up for every token that they see
  choose   the places of a sequence that stay: its first ones, its last ones, and those with the largest weights
  compact  the rows of the places that stay, moved to the front: in place or into other pages; then read back

The sizes are generic ones around the rows of 64 and 128 features that this library's workloads have, with odd and ragged lengths among
them.
"""
import math
import random

import numpy as np
import torch

own = False

_TYPES = {"fp16": torch.float16, "bf16": torch.bfloat16}


def _tree(name, dtype, B, n, S, H, G, d, page, wide=4, ragged=True, window=0):
    return {"name": name, "kind": "tree", "dtype": dtype, "B": B, "n": n, "S": S, "H": H, "G": G, "d": d, "page": page, "wide": wide,
            "ragged": ragged, "window": window}


def _weigh(name, dtype, B, n, S, H, G, d, page, held="old", decay=1.0, ragged=True, window=0):
    """held: which tokens have weights already: "old" the ones before the queries, "none", "all"."""
    return {"name": name, "kind": "weigh", "dtype": dtype, "B": B, "n": n, "S": S, "H": H, "G": G, "d": d, "page": page, "held": held,
            "decay": decay, "ragged": ragged, "window": window}


def _choose(name, B, S, H, page, keep, first, last, ragged=True):
    return {"name": name, "kind": "choose", "dtype": "bf16", "B": B, "S": S, "H": H, "d": 32, "page": page, "keep": keep, "first": first,
            "last": last, "ragged": ragged}


def _compact(name, dtype, B, S, H, d, page, keep, way, ragged=True):
    """way: "branch" an accepted branch of a tree of S tokens, in place behind a prefix; "ends" the first tokens and the last ones, in
    place; "heavy" another choice for each head, into other pages."""
    return {"name": name, "kind": "compact", "dtype": dtype, "B": B, "S": S, "H": H, "d": d, "page": page, "keep": keep, "way": way,
            "ragged": ragged}


def listed():
    return [
        # one short sequence, a small tree: latency
        _tree("tree_1x13x700", "bf16", 1, 13, 700, 8, 4, 128, 16),
        # a ragged batch, medium trees, a window of 2048 tokens
        _tree("tree_16x40x4000_window_d64", "fp16", 16, 40, 4000, 4, 7, 64, 32, wide=6, window=2048),
        # long sequences, large trees
        _tree("tree_8x121x20000", "bf16", 8, 121, 20000, 8, 4, 128, 64, wide=8),
        # one short sequence decodes: latency
        _weigh("weigh_1x1x700", "bf16", 1, 1, 700, 8, 4, 128, 16),
        # a large batch decodes, weights fade
        _weigh("weigh_64x1x8192", "bf16", 64, 1, 8192, 8, 4, 128, 64, decay=0.98),
        # the last queries of long prompts say which of their tokens matter
        _weigh("weigh_6x32x15000_d64", "fp16", 6, 32, 15000, 4, 6, 64, 32, held="none"),
        # every query of a chunk of a long prompt
        _weigh("weigh_2x4096x9000", "bf16", 2, 4096, 9000, 8, 4, 128, 64),
        # one short sequence: latency
        _choose("choose_1x1100", 1, 1100, 8, 16, 512, 4, 64),
        # a batch at its bound
        _choose("choose_64x8192", 64, 8192, 8, 64, 2048, 4, 256),
        # one very long sequence
        _choose("choose_1x131072", 1, 131072, 8, 64, 16384, 16, 1024, ragged=False),
        # accepted branches of a batch of drafted trees
        _compact("compact_48x40_branch", "fp16", 48, 40, 4, 64, 32, 5, "branch"),
        # a batch of long prompts is cut down
        _compact("compact_32x8192_heavy", "bf16", 32, 8192, 8, 128, 64, 2048, "heavy"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    dtype = rng.choice(["bf16", "fp16"])
    kind = rng.choice(["tree", "tree", "weigh", "weigh", "weigh", "choose", "choose", "compact", "compact"])
    d = rng.choice([64, 96, 128, 128, 160, 192, 256])
    page = rng.choice([16, 32, 64, 128, 256])
    H = rng.randint(1, 12)
    G = rng.choice([1, 2, 3, 4, 6, 8, 12, 16])
    most = 64 * 8192 * 8 * 128 // (H * d)                        # tokens in all, by the largest listed batch
    if kind == "tree":
        n = _log_int(rng, 2, 128)
        S = max(n, _log_int(rng, n, min(32768, most, 8 * 121 * 20000 * 32 * 128 // (n * H * G * d))))
        B = rng.randint(1, max(1, min(16, 8 * 121 * 20000 * 32 * 128 // (n * H * G * d * S), most // S)))
        return _tree("", dtype, B, n, S, H, G, d, page, rng.randint(1, 10), rng.random() < 0.7, rng.choice([0, 0, _log_int(rng, 1, S)]))
    if kind == "weigh":
        n = rng.choice([1, 1, rng.randint(2, 64), _log_int(rng, 64, 4096)])
        work = 2 * 4096 * 9000 * 32 * 128 // (n * H * G * d)
        S = max(n, _log_int(rng, n, max(n, min(131072 if n == 1 else 32768, most, work))))
        B = _log_int(rng, 1, max(1, min(64, most // S, work // S)))
        return _weigh("", dtype, B, n, S, H, G, d, page, rng.choice(["old", "none", "all"]), rng.choice([1.0, 0.9]), rng.random() < 0.7,
                      rng.choice([0, 0, _log_int(rng, 1, S)]))
    if kind == "choose":
        S = _log_int(rng, 30, 131072)
        B = _log_int(rng, 1, max(1, min(64, 64 * 8192 * 8 // (S * H))))
        keep = max(4, int(S * rng.uniform(0.05, 0.9)))
        return _choose("", B, S, H, page, keep, rng.randint(0, min(16, keep // 4)), rng.randint(0, keep // 2), rng.random() < 0.7)
    way = rng.choice(["branch", "ends", "heavy"])
    if way == "branch":
        n = rng.randint(8, 128)
        return _compact("", dtype, _log_int(rng, 1, 64), n, H, d, page, rng.randint(2, max(2, n // 6)), way, rng.random() < 0.7)
    S = _log_int(rng, 30, 65536)
    keep = max(2, int(S * rng.uniform(0.05, 0.45 if way == "ends" else 0.9)))
    return _compact("", dtype, _log_int(rng, 1, max(1, min(64, 32 * 2048 * 8 * 128 // (keep * H * d)))), S, H, d, page, keep, way,
                    rng.random() < 0.7)


def _lengths(case):
    """(tokens of each sequence, queries of each): made from the case alone."""
    B, n, S = case["B"], case.get("n", 0), case["S"]
    lens, queries = [], []
    for b in range(B):
        less = (b * 7919 + 13) % (S * 3 // 4 + 1) if case["ragged"] and b else 0
        few = (b * 31) % (n // 2 + 1) if case["ragged"] and b else 0
        lens.append(max(S - less, n - few))
        queries.append(n - few)
    return lens, queries


def _kept(case):
    """Rows that each sequence keeps."""
    if case["way"] == "branch":
        return [max(1, min(case["keep"] - (b * 5 % case["keep"] if case["ragged"] else 0), L // 2)) for b, L in enumerate(_lengths(case)[0])]
    return [min(case["keep"], L) if case["way"] == "heavy" else min(case["keep"], L // 2) for L in _lengths(case)[0]]


def _before(case, b):
    """Tokens before the tree of an accepted branch, 0 otherwise."""
    return 37 + (b * 41) % 150 if case["way"] == "branch" else 0


def work(case):
    H, d, B = case["H"], case["d"], case["B"]
    lens, queries = _lengths(case)
    tokens = sum(lens)
    if case["kind"] == "choose":
        return {"bytes": H * (4 * tokens + 4 * sum(min(L, case["keep"]) for L in lens)), "flops": tokens * H}
    row = d + 4                                                   # codes and scales of keys and values
    if case["kind"] == "compact":
        rows = sum(_kept(case)) * H
        places = rows if case["way"] == "heavy" else rows // H
        # read and write the rows and their weights, read the places; read the rows back
        return {"bytes": rows * (2 * (row + 4) + row + 4 * d) + 4 * places, "flops": 2 * rows * d}
    w, rows = case["window"], sum(queries) * H * case["G"]
    pairs = seen = 0
    for L, n in zip(lens, queries):
        if case["kind"] == "tree":                                # at least what lies before the tree, and itself
            pairs += n * min(L - n + 1, w or L)
        else:
            pairs += sum(min(p + 1, w or L) for p in range(L - n, L))
        seen += min(L, w + n) if w else L
    pairs *= H * case["G"] * d
    if case["kind"] == "tree":
        return {"bytes": seen * H * row + 4 * rows * d + 8 * sum(queries) * (-(-case["n"] // 64)), "flops": 4 * pairs}
    old = tokens if case["held"] == "all" else 0 if case["held"] == "none" else tokens - sum(queries)
    return {"bytes": seen * H * (d // 2 + 2) + 4 * H * (tokens + old) + rows * (2 * d + 4), "flops": 2 * pairs}


def _levels(H, t, g, device):
    """16 ascending levels a head, closer together in the middle, as clusters of bell-shaped values have them."""
    x = torch.linspace(-1, 1, 16, device=device)
    x = (x * (0.6 + 0.4 * x * x)).expand(H, 16) + 0.01 * torch.randn(H, 16, generator=g, device=device)
    return x.sort(dim=1).values.to(t).contiguous()


def _codes(pages, H, page, d, g, device):
    """Ids of bell-shaped values, two to a byte."""
    edges = torch.linspace(-0.8, 0.8, 15, device=device)
    edges = edges * (0.6 + 0.4 * edges * edges)
    out = torch.empty(pages, H, page, d // 2, dtype=torch.uint8, device=device)
    step = max(1, (1 << 26) // (H * page * d))
    for at in range(0, pages, step):
        part = out[at:at + step]
        ids = torch.bucketize(torch.randn(*part.shape, 2, generator=g, device=device) * 0.37, edges, out_int32=True)
        part.copy_(ids[..., 0] | (ids[..., 1] << 4))
    return out


def _masks(queries, words, wide, seed):
    """A random tree for each sequence, `wide` roots, every other token below one of the `3 * wide` before it: its rows of bits."""
    r = random.Random(seed)
    rows = []
    for n in queries:
        sees = []
        for i in range(n):
            parent = r.randint(max(0, i - 3 * wide), i - 1) if i >= wide else -1
            sees.append((sees[parent] if parent >= 0 else 0) | 1 << i)
        rows += sees
    words64 = [[(x >> 64 * w) & (1 << 64) - 1 for w in range(words)] for x in rows]
    return torch.from_numpy(np.array(words64, dtype=np.uint64).reshape(len(rows), words).view(np.int64)).cuda()


def _table(held, order, dev):
    """Page tables of sequences that hold so many pages each, from `order`."""
    table = torch.zeros(len(held), max(held), dtype=torch.int32, device=dev)
    at = 0
    for b, n in enumerate(held):
        table[b, :n] = order[at:at + n]
        at += n
    return table


def prepare(case, seed):
    dev = "cuda"
    g = torch.Generator(device=dev).manual_seed(seed)
    t, B, H, d, P, kind = _TYPES[case["dtype"]], case["B"], case["H"], case["d"], case["page"], case["kind"]
    lens, queries = _lengths(case)
    before = [_before(case, b) for b in range(B)] if kind == "compact" else [0] * B
    held = [-(-(L + c) // P) for L, c in zip(lens, before)]
    more = [-(-c // P) for c in _kept(case)] if kind == "compact" and case["way"] == "heavy" else []
    pages = sum(held) + sum(more) + 3
    order = torch.randperm(pages, generator=g, device=dev).to(torch.int32)
    s = {"case": case, "pages": _table(held, order, dev), "lens": torch.tensor(lens, dtype=torch.int32, device=dev)}
    s["k_levels"], s["v_levels"] = _levels(H, t, g, dev), _levels(H, t, g, dev)
    s["k_codes"], s["v_codes"] = _codes(pages, H, P, d, g, dev), _codes(pages, H, P, d, g, dev)
    s["k_scale"] = (2.7 * (0.8 + 0.4 * torch.rand(pages, H, P, generator=g, device=dev))).to(t)
    s["v_scale"] = (2.7 * (0.8 + 0.4 * torch.rand(pages, H, P, generator=g, device=dev))).to(t)
    if kind != "tree":                                            # a few tokens have most of the weight
        s["mass"] = torch.randn(pages, H, P, generator=g, device=dev).mul_(1.5).exp_().mul_(1e-3)
    if kind in ("tree", "weigh"):
        starts = [sum(queries[:b]) for b in range(B + 1)]
        s["q"] = (1.5 * torch.randn(starts[-1], H * case["G"], d, generator=g, device=dev)).to(t)
        s["q_start"] = torch.tensor(starts, dtype=torch.int32, device=dev)
        s["max_q"], s["max_len"] = max(queries), max(lens)
    if kind == "tree":
        s["tree"] = _masks(queries, -(-case["n"] // 64), case["wide"], seed)
    if kind == "weigh":
        s["out"] = torch.zeros_like(s["mass"])
        s["known"] = {"old": s["lens"] - torch.tensor(queries, dtype=torch.int32, device=dev), "none": torch.zeros_like(s["lens"]),
                      "all": s["lens"].clone()}[case["held"]]
        s["lse"] = _logs(s)                                       # what attention to the same tokens has left
    if kind == "choose":
        s["max_len"] = max(lens)
    if kind == "compact":
        keep = _kept(case)
        longest, where = max(keep), torch.zeros(B, H if case["way"] == "heavy" else 1, max(keep), dtype=torch.int32, device=dev)
        for b, (L, n) in enumerate(zip(lens, keep)):
            if case["way"] == "heavy":
                where[b, :, :n] = torch.rand(H, L, generator=g, device=dev).argsort(dim=1)[:, :n].sort(dim=1).values.int()
            elif case["way"] == "ends":                           # the first four and the last ones, none of which lies where rows go
                where[b, 0, :n] = torch.cat([torch.arange(min(4, n), device=dev), torch.arange(L - n + min(4, n), L, device=dev)]).int()
            else:                                                 # a root of a wide tree, then tokens behind all that are kept
                deep = (torch.rand(L - n, generator=g, device=dev).argsort()[:n - 1] + n).sort().values
                where[b, 0, :n] = torch.cat([torch.zeros(1, device=dev, dtype=torch.long), deep]).int()
        s["where"], s["counts"] = where, torch.tensor(keep, dtype=torch.int32, device=dev)
        s["start"] = torch.tensor(before, dtype=torch.int32, device=dev)
        s["to"] = _table(more, order[sum(held):], dev) if more else s["pages"]
        b = torch.repeat_interleave(torch.arange(B, device=dev), s["counts"].long())
        place = torch.cat([torch.arange(c, c + n, device=dev) for c, n in zip(before, keep)])
        s["slots"] = s["to"][b, place // P].long() * P + place % P
    if own:
        from paper_2603_09229_amd import binding as fk
        s["cache"] = fk.KVCache(s["k_codes"], s["v_codes"], s["k_scale"], s["v_scale"], s["k_levels"], s["v_levels"])
        if kind == "tree":
            s["ws"] = fk.make_kv_workspace(s["cache"], B, case["G"] * H, s["q"].shape[0], s["max_q"], s["max_len"])
    return s


def _own(s):
    from paper_2603_09229_amd import binding as fk
    case = s["case"]
    if case["kind"] == "tree":
        return fk.fk_kv_attend_tree(s["cache"], s["q"], s["pages"], s["lens"], s["tree"], q_start=s["q_start"], max_q=s["max_q"],
                                    max_len=s["max_len"], window=case["window"], ws=s["ws"])
    if case["kind"] == "weigh":
        return fk.fk_kv_weigh(s["cache"], s["q"], s["lse"], s["pages"], s["lens"], s["mass"], q_start=s["q_start"], max_q=s["max_q"],
                              max_len=s["max_len"], window=case["window"], known=s["known"], decay=case["decay"], out=s["out"])
    if case["kind"] == "choose":
        return fk.fk_kv_choose(s["cache"], s["mass"], s["pages"], s["lens"], case["keep"], first=case["first"], last=case["last"],
                               max_len=s["max_len"])
    fk.fk_kv_compact(s["cache"], s["pages"], s["where"], s["counts"], start=s["start"], to_pages=s["to"], mass=s["mass"])
    return (*fk.fk_kv_read(s["cache"], s["slots"]), s["mass"])


def _values(codes, scale, levels):
    """codes [N, H, ..., d/2] -> values in 32 bits."""
    ids = torch.stack([codes & 15, codes >> 4], dim=-1).flatten(-2).int()
    head = torch.arange(levels.shape[0], device=codes.device, dtype=torch.int32) * 16
    ids += head.view(1, -1, *[1] * (ids.dim() - 2))
    return levels.float().flatten()[ids] * scale.float()[..., None]


def _rows(s, which):
    """Keys or values of all sequences, [B, H, longest, d] in 32 bits."""
    page = s["pages"].long()
    return _values(s[which + "_codes"][page].transpose(1, 2).flatten(2, 3), s[which + "_scale"][page].transpose(1, 2).flatten(2, 3),
                   s[which + "_levels"])


def _scores(s):
    """Scores [B, H, G, n, longest] in 32 bits, -inf where a query does not see the token; sequence and number of every query."""
    case = s["case"]
    B, H, G, d, n = case["B"], case["H"], case["G"], case["d"], s["max_q"]
    dev = s["q"].device
    counts = s["q_start"][1:] - s["q_start"][:-1]
    rows = torch.arange(s["q"].shape[0], device=dev)
    seq = torch.searchsorted(s["q_start"][1:].contiguous(), rows, right=True)
    at = rows - s["q_start"][seq]
    q = torch.zeros(B, n, H * G, d, device=dev)
    q[seq, at] = s["q"].float()
    q = q.view(B, n, H, G, d).permute(0, 2, 3, 1, 4).reshape(B, H, G * n, d)
    x = torch.matmul(q, _rows(s, "k").transpose(-1, -2)).mul_(1 / math.sqrt(d)).view(B, H, G, n, -1)
    tokens = torch.arange(x.shape[-1], device=dev)
    base = (s["lens"] - counts)[:, None]
    live = torch.arange(n, device=dev) < counts[:, None]
    if case["kind"] == "weigh":
        pos = (base + torch.arange(n, device=dev))[..., None]                          # positions of the queries
        sees = tokens <= pos
        if case["window"]:
            sees &= tokens > pos - case["window"]
    else:
        bits = torch.zeros(B, n, s["tree"].shape[1], dtype=torch.int64, device=dev)
        bits[seq, at] = s["tree"]
        j = tokens - base                                                              # [B, longest] numbers in the tree
        word = (j.clamp(0, 64 * bits.shape[2] - 1) // 64)[:, None].expand(B, n, -1)
        set_ = (bits.gather(2, word) >> (j.clamp_min(0) % 64)[:, None]) & 1 == 1
        sees = (j < 0)[:, None] | (set_ & (j < counts[:, None])[:, None])
        if case["window"]:                                                             # the last ones of what is seen
            after = sees.flip(-1).cumsum(-1).flip(-1)
            sees &= after <= case["window"]
    sees &= (tokens < s["lens"][:, None])[:, None] & live[..., None]
    return x.masked_fill_(~sees[:, None, None], -math.inf), seq, at


def _exps(x):
    """exp(x - largest of its row), in place; the largest."""
    top = x.amax(dim=-1, keepdim=True)
    top = torch.where(top > -math.inf, top, 0.0)
    return x.sub_(top).exp_(), top


def _logs(s):
    """Logarithms of the softmax sums, [Tq, H * G]."""
    x, seq, at = _scores(s)
    x, top = _exps(x)
    lse = x.sum(dim=-1).log_() + top[..., 0]
    return lse.permute(0, 3, 1, 2).flatten(2)[seq, at].contiguous()


def run(s):
    if own:
        return _own(s)
    case, P = s["case"], s["case"]["page"]
    B, H, dev = case["B"], case["H"], s["lens"].device
    if case["kind"] == "tree":
        x, seq, at = _scores(s)
        x, _ = _exps(x)
        total = x.sum(dim=-1, keepdim=True)
        G, n, d = case["G"], s["max_q"], case["d"]
        out = torch.matmul(x.view(B, H, G * n, -1), _rows(s, "v")).view(B, H, G, n, d) / torch.where(total > 0, total, 1.0)
        return out.permute(0, 3, 1, 2, 4).reshape(B, n, H * G, d)[seq, at].to(s["q"].dtype)
    tokens = torch.arange(s["pages"].shape[1] * P, device=dev)
    inside = tokens < s["lens"][:, None]
    page = s["pages"].long().repeat_interleave(P, dim=1)
    if case["kind"] == "weigh":
        x, seq, at = _scores(s)
        lse = torch.full((B, s["max_q"], H * case["G"]), math.inf, device=dev)
        lse[seq, at] = s["lse"]
        x.sub_(lse.view(B, -1, H, case["G"]).permute(0, 2, 3, 1)[..., None]).exp_()
        new = x.sum(dim=(2, 3)).transpose(1, 2)                                        # [B, longest, H]
        b, tok = inside.nonzero(as_tuple=True)
        old = s["mass"][page[b, tok], :, tok % P] * case["decay"]
        old[tok >= s["known"][b]] = 0.0
        s["out"][page[b, tok], :, tok % P] = old + new[b, tok]
        return s["out"]
    if case["kind"] == "choose":
        keep, first, last = case["keep"], case["first"], case["last"]
        w = s["mass"][page, :, (tokens % P).expand_as(page)].transpose(1, 2)           # [B, H, longest]
        L = s["lens"][:, None, None]
        ends = (tokens < first) | (tokens >= L - last)
        order = w.masked_fill(ends | (tokens >= L), -math.inf).sort(dim=-1, descending=True, stable=True).indices
        stays = torch.zeros_like(w, dtype=torch.bool).scatter_(2, order[..., :keep - first - last], True)
        stays = ((stays | ends) & (tokens < L)) | ((L <= keep) & (tokens < L))
        kept = torch.full((B, H, keep), -1, dtype=torch.int32, device=dev)
        b, h, tok = stays.nonzero(as_tuple=True)
        kept[b, h, (stays.cumsum(-1) - 1)[b, h, tok]] = tok.int()
        return kept, s["lens"].clamp(max=keep)
    j = torch.arange(s["where"].shape[2], device=dev)
    b, j = (j < s["counts"][:, None]).nonzero(as_tuple=True)
    head = torch.arange(H, device=dev)
    place = s["start"][b, None] + s["where"].expand(B, H, -1)[b, :, j]                 # [rows, H]
    src = s["pages"][b[:, None], place // P].long()
    to = s["start"][b] + j
    dst = s["to"][b, to // P].long()
    for name in ("k_codes", "v_codes", "k_scale", "v_scale", "mass"):
        s[name][dst, :, to % P] = s[name][src, head, place % P]
    read = lambda x: _values(s[x + "_codes"][dst, :, to % P], s[x + "_scale"][dst, :, to % P], s[x + "_levels"]).to(s["k_scale"].dtype)  # noqa: E731
    return read("k"), read("v"), s["mass"]


def _exact_values(codes, scale, levels):
    """One head's rows [N, d/2] in 64 bits."""
    x = torch.empty(*codes.shape[:-1], 2 * codes.shape[-1], dtype=torch.float64, device=codes.device)
    table = levels.double()
    x[..., 0::2] = table[(codes % 16).long()]
    x[..., 1::2] = table[(codes // 16).long()]
    return x * scale.double()[..., None]


def _exact_sees(s, b, L, n, at):
    """[n, L]: which tokens each query of sequence b sees."""
    w, dev = s["case"]["window"], s["q"].device
    if s["case"]["kind"] == "weigh":
        gap = (L - n + torch.arange(n, device=dev))[:, None] - torch.arange(L, device=dev)[None]
        return (gap >= 0) & (gap < (w or L))
    sees = np.zeros((n, L), dtype=bool)
    for i, row in enumerate(s["tree"][at:at + n].cpu().numpy().view(np.uint64).tolist()):
        seen = np.concatenate([np.arange(L - n), [L - n + j for j in range(n) if row[j // 64] >> (j % 64) & 1]]).astype(np.int64)
        sees[i, seen[-w:]] = True
    return torch.from_numpy(sees).to(dev)


def exact(case, seed):
    s = prepare(case, seed)
    H, P, lens, kind = case["H"], case["page"], _lengths(case)[0], case["kind"]
    if kind == "choose":
        kept = torch.full((case["B"], H, case["keep"]), -1, dtype=torch.int32)
        for b, L in enumerate(lens):
            places = [s["pages"][b, :-(-L // P)].long()]
            for h in range(H):
                w = s["mass"][places[0], h].reshape(-1)[:L].double().cpu().numpy()
                if L <= case["keep"]:
                    stays = np.arange(L)
                else:
                    middle = np.arange(case["first"], L - case["last"])
                    best = np.lexsort((middle, -w[middle]))[:case["keep"] - case["first"] - case["last"]]
                    stays = np.sort(np.concatenate([np.arange(case["first"]), middle[best], np.arange(L - case["last"], L)]))
                kept[b, h, :len(stays)] = torch.from_numpy(stays.astype(np.int32))
        return kept, torch.tensor([min(L, case["keep"]) for L in lens], dtype=torch.int32)
    if kind == "compact":
        keys, vals, mass = [], [], s["mass"].clone()
        for b, n in enumerate(_kept(case)):
            start = _before(case, b)
            to = torch.arange(start, start + n, device=mass.device)
            k, v = [], []
            for h in range(H):
                at = start + s["where"][b, h % s["where"].shape[1], :n].long()
                page = s["pages"][b].long()[at // P]
                k.append(_exact_values(s["k_codes"][page, h, at % P], s["k_scale"][page, h, at % P], s["k_levels"][h]))
                v.append(_exact_values(s["v_codes"][page, h, at % P], s["v_scale"][page, h, at % P], s["v_levels"][h]))
                mass[s["to"][b].long()[to // P], h, to % P] = s["mass"][page, h, at % P]
            keys.append(torch.stack(k, 1))
            vals.append(torch.stack(v, 1))
        return torch.cat(keys), torch.cat(vals), mass.double()
    G, d = case["G"], case["d"]
    out = s["out"].double().clone() if kind == "weigh" else torch.zeros(*s["q"].shape, dtype=torch.float64, device=s["q"].device)
    at = 0
    for b, (L, n) in enumerate(zip(*_lengths(case))):
        held = s["pages"][b, :-(-L // P)].long()
        sees = _exact_sees(s, b, L, n, at).repeat_interleave(G, dim=0)
        tok = torch.arange(L, device=sees.device)
        for h in range(H):
            k = _exact_values(s["k_codes"][held, h], s["k_scale"][held, h], s["k_levels"][h]).reshape(-1, d)[:L]
            x = s["q"][at:at + n, h * G:(h + 1) * G].double().reshape(n * G, d) @ k.T / math.sqrt(d)
            if kind == "weigh":
                e = torch.exp(x - s["lse"][at:at + n, h * G:(h + 1) * G].double().reshape(n * G, 1)).masked_fill(~sees, 0.0).sum(0)
                old = s["mass"][held[tok // P], h, tok % P].double()
                out[held[tok // P], h, tok % P] = e + torch.where(tok < s["known"][b], case["decay"] * old, 0.0)
                continue
            v = _exact_values(s["v_codes"][held, h], s["v_scale"][held, h], s["v_levels"][h]).reshape(-1, d)[:L]
            x = x.masked_fill(~sees, -math.inf)
            e = torch.exp(x - x.amax(-1, keepdim=True).clamp_min(-1e300))
            out[at:at + n, h * G:(h + 1) * G] = ((e @ v) / e.sum(-1, keepdim=True).clamp_min(1e-300)).reshape(n, G, d)
        at += n
    return out
