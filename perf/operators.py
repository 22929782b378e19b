"""The operators on a paged key/value cache held in 4 bits, as a program that serves tokens calls them.

A cache keeps, for every token and every key/value head, a row of `d` keys and a row of `d` values as 4-bit ids of 16
levels that the head has learned (the centroids of one-dimensional clusters), times the row's largest magnitude:

  codes   [pages, heads, page, d/2] uint8, channel 2b in the low and 2b+1 in the high half of byte b
  scale   [pages, heads, page]      of the cache's type, the largest magnitude of the row
  levels  [heads, 16]               of the cache's type, ascending

Three kinds of call:

  append  new keys (turned by the angles of their positions) and values go into the cache, the new queries are turned
          too; the rows just written are then read back as the values they stand for
  read    rows of the cache, as the values they stand for
  attend  softmax(q.K) V over the cache, for one query token a sequence (a decoding step) or several (tokens
          drafted ahead, chunks of a prompt, whole prompts)

The sizes are generic ones around the rows of 64 and 128 features that this library's workloads have, with odd and ragged
lengths among them.
"""
import math

import torch

own = False

_TYPES = {"fp16": torch.float16, "bf16": torch.bfloat16}


def _append(name, dtype, T, H, G, d, page, rot, interleaved=False, fused=True):
    return {"name": name, "kind": "append", "dtype": dtype, "T": T, "H": H, "G": G, "d": d, "page": page, "rot": rot,
            "interleaved": interleaved, "fused": fused}


def _read(name, dtype, T, H, d, page):
    return {"name": name, "kind": "read", "dtype": dtype, "T": T, "H": H, "d": d, "page": page}


def _attend(name, dtype, B, n, S, H, G, d, page, ragged=True, idle=0, window=0):
    return {"name": name, "kind": "attend", "dtype": dtype, "B": B, "n": n, "S": S, "H": H, "G": G, "d": d, "page": page,
            "ragged": ragged, "idle": idle, "window": window}


def listed():
    return [
        # one sequence decodes: the smallest call, bound by its launches
        _append("append_1", "bf16", 1, 8, 4, 128, 64, 128),
        # a decoding step of 113 sequences
        _append("append_113", "fp16", 113, 8, 4, 128, 16, 128),
        # a ragged batch of prompts, half of each row turned, pairs side by side
        _append("append_4099_d64", "fp16", 4099, 4, 6, 64, 32, 32, interleaved=True, fused=False),
        # a long prompt
        _append("append_16384", "bf16", 16384, 8, 4, 128, 64, 128),
        # a shared prefix is copied out
        _read("read_777_d64", "fp16", 777, 5, 64, 16),
        _read("read_20000", "bf16", 20000, 8, 128, 64),
        # one short sequence decodes: latency
        _attend("decode_1x700", "bf16", 1, 1, 700, 8, 4, 128, 16),
        # a decoding step of a batch of ragged sequences, two of its places idle, a window of 2048 tokens
        _attend("decode_24x5000_window_d64", "fp16", 24, 1, 5000, 4, 7, 64, 32, idle=2, window=2048),
        # one very long sequence decodes
        _attend("decode_1x131072", "bf16", 1, 1, 131072, 8, 8, 128, 64, ragged=False),
        # a large batch decodes
        _attend("decode_64x8192", "bf16", 64, 1, 8192, 8, 4, 128, 64),
        # drafted tokens are checked, wide rows
        _attend("draft_8x5x4000_d256", "fp16", 8, 5, 4000, 2, 8, 256, 16),
        # a chunk of a long prompt
        _attend("chunk_2x4096x9000", "bf16", 2, 4096, 9000, 8, 4, 128, 64),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    dtype = rng.choice(["bf16", "fp16"])
    kind = rng.choice(["append", "read", "decode", "decode", "draft", "chunk"])
    d = rng.choice([64, 96, 128, 128, 160, 192, 256])
    page = rng.choice([16, 32, 64, 128, 256])
    H = rng.randint(1, 12)
    G = rng.choice([1, 2, 3, 4, 6, 8, 12, 16])
    if kind == "append":
        T = _log_int(rng, 1, max(2, min(16384, 16384 * 8 * 128 * 6 // (H * d * (G + 2)))))
        rot = rng.choice([0, d // 2, d, d])
        return _append("", dtype, T, H, G, d, page, rot, rng.random() < 0.5, rng.random() < 0.5)
    if kind == "read":
        return _read("", dtype, _log_int(rng, 1, max(2, 20000 * 8 * 128 // (H * d))), H, d, page)
    if kind == "decode":
        most = 64 * 8192 * 8 * 128 // (H * d)                    # tokens in all, by the largest listed case
        S = _log_int(rng, 1, min(131072, most))
        B = _log_int(rng, 1, max(1, min(128, most // S)))
        window = rng.choice([0, 0, _log_int(rng, 1, S)])
        return _attend("", dtype, B, 1, S, H, G, d, page, rng.random() < 0.7, min(rng.choice([0, 0, 1]), B - 1), window)
    n = rng.randint(2, 9) if kind == "draft" else _log_int(rng, 10, 4096)
    most = min(32768, 2 * 4096 * 9000 * 32 * 128 // (n * H * G * d), 64 * 8192 * 8 * 128 // (H * d))
    S = max(n, _log_int(rng, 1, max(n + 1, most)))
    B = rng.randint(1, max(1, min(16, most // S)))
    return _attend("", dtype, B, n, S, H, G, d, page, rng.random() < 0.7, 0, rng.choice([0, 0, _log_int(rng, 1, S)]))


def _lengths(case):
    """(tokens of each sequence in the cache, queries of each): made from the case alone."""
    B, n, S = case["B"], case["n"], case["S"]
    lens, queries = [], []
    for b in range(B):
        idle = b >= B - case["idle"]
        less = (b * 7919 + 13) % (S * 3 // 4 + 1) if case["ragged"] and b else 0
        few = (b * 31) % (n // 2 + 1) if case["ragged"] and b else 0
        lens.append(0 if idle else S - less)
        queries.append(n - few)
    return lens, queries


def _seen(case):
    """(pairs of a query token and a token that it sees, cache tokens that some query sees)."""
    pairs, tokens = 0, 0
    w = case["window"]
    for L, n in zip(*_lengths(case)):
        lo, hi = max(1, L - n + 1), L                             # tokens up to the first and the last query that sees any
        if w and lo < w:
            cut = min(hi, w)
            pairs += (lo + cut) * (cut - lo + 1) // 2 + (hi - cut) * w
        elif w:
            pairs += (hi - lo + 1) * w
        elif hi >= lo:
            pairs += (lo + hi) * (hi - lo + 1) // 2
        tokens += min(L, w + n - 1) if w else L
    return pairs, tokens


def work(case):
    H, d = case["H"], case["d"]
    row = 2 * (d // 2 + 2)                                        # keys and values of a token in a head: codes and scales
    if case["kind"] == "read":
        T = case["T"]
        return {"bytes": T * H * (row + 4 * d) + 8 * T, "flops": 2 * T * H * d}
    if case["kind"] == "append":
        T, Q = case["T"], H * case["G"]
        # read keys, values, queries, the angles' row and two numbers a token; write the cache and the queries; read the rows back
        moved = T * (4 * H * d + 4 * Q * d + 4 * case["rot"] + 12) + 2 * T * H * row + T * H * 4 * d
        return {"bytes": moved, "flops": T * (8 * H * d + 3 * (H + Q) * case["rot"])}
    pairs, tokens = _seen(case)
    queries = sum(_lengths(case)[1])
    return {"bytes": tokens * H * row + 4 * queries * H * case["G"] * d, "flops": 4 * pairs * H * case["G"] * d}


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


def prepare(case, seed):
    dev = "cuda"
    g = torch.Generator(device=dev).manual_seed(seed)
    t, H, d, P = _TYPES[case["dtype"]], case["H"], case["d"], case["page"]
    if case["kind"] == "attend":
        lens, queries = _lengths(case)
        held = [-(-max(L, 1) // P) for L in lens]
        pages = sum(held) + 3
        order = torch.randperm(pages, generator=g, device=dev).to(torch.int32)
        table = torch.zeros(case["B"], max(held), dtype=torch.int32, device=dev)
        at = 0
        for b, n in enumerate(held):
            table[b, :n] = order[at:at + n]
            at += n
    else:
        pages = -(-case["T"] // P) + 5
    s = {"case": case, "k_codes": _codes(pages, H, P, d, g, dev), "v_codes": _codes(pages, H, P, d, g, dev),
         "k_levels": _levels(H, t, g, dev), "v_levels": _levels(H, t, g, dev)}
    s["k_scale"] = (2.7 * (0.8 + 0.4 * torch.rand(pages, H, P, generator=g, device=dev))).to(t)
    s["v_scale"] = (2.7 * (0.8 + 0.4 * torch.rand(pages, H, P, generator=g, device=dev))).to(t)
    if case["kind"] == "attend":
        Q = H * case["G"]
        starts = [sum(queries[:b]) for b in range(case["B"] + 1)]
        s["q"] = (1.5 * torch.randn(starts[-1], Q, d, generator=g, device=dev)).to(t)
        s["pages"] = table
        s["lens"] = torch.tensor(lens, dtype=torch.int32, device=dev)
        s["q_start"] = torch.tensor(starts, dtype=torch.int32, device=dev)
        s["max_q"], s["max_len"] = max(queries), max(lens)
    else:
        T = case["T"]
        order = torch.randperm(pages, generator=g, device=dev)
        s["slots"] = (order[torch.arange(T, device=dev) // P] * P + torch.arange(T, device=dev) % P).contiguous()
        if T < 256:                                               # one token to each sequence: places with nothing in common
            s["slots"] = torch.randperm(pages * P, generator=g, device=dev)[:T].contiguous()
    if case["kind"] == "append":
        T, Q, R = case["T"], H * case["G"], case["rot"]
        s["spread"] = 0.5 + torch.rand(H, d, generator=g, device=dev)          # some channels are larger than others
        qkv = torch.randn(T, Q + 2 * H, d, generator=g, device=dev)
        qkv[:, Q:Q + H] *= s["spread"]
        qkv = qkv.to(t)
        s["q"], s["k"], s["v"] = qkv[:, :Q], qkv[:, Q:Q + H], qkv[:, Q + H:]   # one projection's output
        if not case["fused"]:
            s["q"], s["k"], s["v"] = s["q"].contiguous(), s["k"].contiguous(), s["v"].contiguous()
        most = max(4096, T)
        angle = torch.arange(most, device=dev, dtype=torch.float32)[:, None] * 10000.0 ** (
            -torch.arange(R // 2, device=dev, dtype=torch.float32) / max(1, R // 2))
        s["cos_sin"] = torch.cat([angle.cos(), angle.sin()], dim=1).contiguous()
        s["positions"] = (torch.arange(T, device=dev, dtype=torch.int32) if T >= 256 else
                          torch.randint(0, most, (T,), generator=g, device=dev, dtype=torch.int32))
    if own:
        from paper_2603_09229_amd import binding as fk
        s["cache"] = fk.KVCache(s["k_codes"], s["v_codes"], s["k_scale"], s["v_scale"], s["k_levels"], s["v_levels"])
        if case["kind"] == "attend":
            s["ws"] = fk.make_kv_workspace(s["cache"], case["B"], case["G"] * H, s["q"].shape[0], s["max_q"], s["max_len"])
    return s


def _own(s):
    from paper_2603_09229_amd import binding as fk
    case = s["case"]
    if case["kind"] == "read":
        return fk.fk_kv_read(s["cache"], s["slots"])
    if case["kind"] == "append":
        q = fk.fk_kv_append(s["cache"], s["k"], s["v"], s["slots"], positions=s["positions"], cos_sin=s["cos_sin"],
                             interleaved=case["interleaved"], q=s["q"])
        return (q, *fk.fk_kv_read(s["cache"], s["slots"]))
    return fk.fk_kv_attend(s["cache"], s["q"], s["pages"], s["lens"], q_start=s["q_start"], max_q=s["max_q"],
                            max_len=s["max_len"], causal=True, window=case["window"], ws=s["ws"])


def _turn(x, s):
    """x [T, heads, d] turned by the angles of its positions, in its own type."""
    R = s["cos_sin"].shape[1]
    cs = s["cos_sin"][s["positions"].long()][:, None]
    c, sn = cs[..., :R // 2], cs[..., R // 2:]
    y = x.float()
    if s["case"]["interleaved"]:
        a, b = y[..., 0:R:2], y[..., 1:R:2]
        turned = torch.stack([a * c - b * sn, b * c + a * sn], dim=-1).flatten(-2)
    else:
        a, b = y[..., :R // 2], y[..., R // 2:R]
        turned = torch.cat([a * c - b * sn, b * c + a * sn], dim=-1)
    return torch.cat([turned, y[..., R:]], dim=-1).to(x.dtype)


def _put(x, levels, codes, scale, page, place):
    """Rows x [T, H, d] into the cache."""
    y = x.float()
    s = y.abs().amax(dim=-1)
    u = y / torch.where(s > 0, s, 1.0)[..., None]
    ids = (u[..., None] - levels.float()[None, :, None, :]).abs().argmin(dim=-1)
    codes[page, :, place] = (ids[..., 0::2] | (ids[..., 1::2] << 4)).to(torch.uint8)
    scale[page, :, place] = s.to(scale.dtype)


def _values(codes, scale, levels):
    """codes [N, H, ..., d/2] -> values in 32 bits."""
    ids = torch.stack([codes & 15, codes >> 4], dim=-1).flatten(-2).int()
    head = torch.arange(levels.shape[0], device=codes.device, dtype=torch.int32) * 16
    ids += head.view(1, -1, *[1] * (ids.dim() - 2))
    return levels.float().flatten()[ids] * scale.float()[..., None]


def _get(s, page, place, t):
    return (_values(s["k_codes"][page, :, place], s["k_scale"][page, :, place], s["k_levels"]).to(t),
            _values(s["v_codes"][page, :, place], s["v_scale"][page, :, place], s["v_levels"]).to(t))


def _rows(s, which):
    """Keys or values of all sequences, [B, H, longest, d] in 32 bits."""
    page = s["pages"].long()
    x = _values(s[which + "_codes"][page].transpose(1, 2).flatten(2, 3),
                s[which + "_scale"][page].transpose(1, 2).flatten(2, 3), s[which + "_levels"])
    return x


def run(s):
    if own:
        return _own(s)
    case, P = s["case"], s["case"]["page"]
    if case["kind"] != "attend":
        page, place = s["slots"] // P, s["slots"] % P
        if case["kind"] == "read":
            return _get(s, page, place, s["k_scale"].dtype)
        _put(_turn(s["k"], s), s["k_levels"], s["k_codes"], s["k_scale"], page, place)
        _put(s["v"], s["v_levels"], s["v_codes"], s["v_scale"], page, place)
        return (_turn(s["q"], s), *_get(s, page, place, s["k"].dtype))
    B, H, G, d, n = case["B"], case["H"], case["G"], case["d"], s["max_q"]
    dev, t = s["q"].device, s["q"].dtype
    counts = s["q_start"][1:] - s["q_start"][:-1]
    rows = torch.arange(s["q"].shape[0], device=dev)
    seq = torch.searchsorted(s["q_start"][1:].contiguous(), rows, right=True)
    at = rows - s["q_start"][seq]
    q = torch.zeros(B, n, H * G, d, device=dev)
    q[seq, at] = s["q"].float()
    q = q.view(B, n, H, G, d).permute(0, 2, 3, 1, 4).reshape(B, H, G * n, d)
    x = torch.matmul(q, _rows(s, "k").transpose(-1, -2)).mul_(1 / math.sqrt(d))
    tokens = torch.arange(x.shape[-1], device=dev)
    last = (s["lens"] - counts)[:, None] + torch.arange(n, device=dev)                 # [B, n] positions of the queries
    sees = (tokens <= last[..., None]) & (tokens < s["lens"][:, None, None])
    if case["window"]:
        sees &= tokens > last[..., None] - case["window"]
    x = x.view(B, H, G, n, -1).masked_fill_(~sees[:, None, None], -math.inf)
    top = x.amax(dim=-1, keepdim=True)
    x = x.sub_(torch.where(top > -math.inf, top, 0.0)).exp_()
    total = x.sum(dim=-1, keepdim=True)
    out = torch.matmul(x.view(B, H, G * n, -1), _rows(s, "v")).view(B, H, G, n, d) / torch.where(total > 0, total, 1.0)
    return out.permute(0, 3, 1, 2, 4).reshape(B, n, H * G, d)[seq, at].to(t)


def _exact_values(codes, scale, levels):
    """One head's rows [N, d/2] in 64 bits."""
    x = torch.empty(*codes.shape[:-1], 2 * codes.shape[-1], dtype=torch.float64, device=codes.device)
    table = levels.double()
    x[..., 0::2] = table[(codes % 16).long()]
    x[..., 1::2] = table[(codes // 16).long()]
    return x * scale.double()[..., None]


def _exact_stored(x, levels):
    """What rows [T, d] of one head read back as, in 64 bits."""
    y, table = x.double(), levels.double()
    s = y.abs().max(dim=-1, keepdim=True).values
    best, off = torch.zeros_like(y), torch.full_like(y, math.inf)
    for level in table:                                           # ascending: the first of two equally near ones stays
        far = (y - s * level).abs()
        best, off = torch.where(far < off, s * level, best), torch.minimum(far, off)
    return best


def _exact_turn(x, s):
    y, R = x.double().clone(), s["cos_sin"].shape[1]
    cs = s["cos_sin"].double()[s["positions"].long()]
    for p in range(R // 2):
        i, j = (2 * p, 2 * p + 1) if s["case"]["interleaved"] else (p, p + R // 2)
        c, sn = cs[:, p, None], cs[:, R // 2 + p, None]
        a, b = x[..., i].double(), x[..., j].double()
        y[..., i], y[..., j] = a * c - b * sn, a * sn + b * c
    return y


def exact(case, seed):
    s = prepare(case, seed)
    H, P, d = case["H"], case["page"], case["d"]
    if case["kind"] != "attend":
        page, place = s["slots"] // P, s["slots"] % P
        if case["kind"] == "read":
            k = [_exact_values(s["k_codes"][page, h, place], s["k_scale"][page, h, place], s["k_levels"][h]) for h in range(H)]
            v = [_exact_values(s["v_codes"][page, h, place], s["v_scale"][page, h, place], s["v_levels"][h]) for h in range(H)]
            return torch.stack(k, 1), torch.stack(v, 1)
        turned = _exact_turn(s["k"], s).to(s["k"].dtype)          # a key is rounded to its type before it is coded
        k = torch.stack([_exact_stored(turned[:, h], s["k_levels"][h]) for h in range(H)], 1)
        v = torch.stack([_exact_stored(s["v"][:, h], s["v_levels"][h]) for h in range(H)], 1)
        return _exact_turn(s["q"], s), k, v
    lens, queries = _lengths(case)
    G, w = case["G"], case["window"]
    out = torch.zeros(*s["q"].shape, dtype=torch.float64, device=s["q"].device)
    at = 0
    for b, (L, n) in enumerate(zip(lens, queries)):
        first = max(0, L - n + 1 - w) if w else 0                 # tokens that some query sees
        held = s["pages"][b, first // P:-(-L // P)].long()
        first = first // P * P
        for h in range(H if L else 0):
            k = _exact_values(s["k_codes"][held, h], s["k_scale"][held, h], s["k_levels"][h]).reshape(-1, d)[:L - first]
            v = _exact_values(s["v_codes"][held, h], s["v_scale"][held, h], s["v_levels"][h]).reshape(-1, d)[:L - first]
            x = s["q"][at:at + n, h * G:(h + 1) * G].double().reshape(n * G, d) @ k.T / math.sqrt(d)
            pos = (L - n + torch.arange(n, device=x.device)).repeat_interleave(G)[:, None]
            tok = first + torch.arange(L - first, device=x.device)[None]
            hide = tok > pos
            if w:
                hide |= tok + w <= pos
            e = torch.exp(x.masked_fill(hide, -math.inf) - x.masked_fill(hide, -1e300).amax(-1, keepdim=True))
            e = e.masked_fill(hide, 0.0)
            out[at:at + n, h * G:(h + 1) * G] = ((e @ v) / e.sum(-1, keepdim=True).clamp_min(1e-300)).reshape(n, G, d)
        at += n
    return out
