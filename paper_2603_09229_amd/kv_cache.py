"""Serving from a key/value cache whose 4-bit levels are learned by k-means: the calls in the order a program makes them.

    levels   16 centroids of single numbers a head, from a sample of rows divided by their largest magnitudes (fk_lloyd_iter)
    append   new tokens go into their slots, keys and queries turned by the angles of their positions (fk_kv_append)
    attend   the queries read the cache: a prompt's own tokens first, then one token a sequence and step (fk_kv_attend)
    draft    a tree of drafted tokens a sequence is appended and attended to, each token over its branch (fk_kv_attend_tree); the branch that is
             accepted moves to the front of the tree's places (fk_kv_compact)
    evict    sequences are cut down to the tokens with the largest attention weights, which every step adds up (fk_kv_weigh, fk_kv_choose,
             fk_kv_compact)

``python -m paper_2603_09229_amd.kv_cache`` runs a small batch of ragged prompts and some decoding steps, compares every result with
attention over the uncoded keys and values, and prints what the coding costs with learned levels and with evenly spaced ones; then drafts and
evictions, and how much of the attention weight the tokens that stay have.
"""
from __future__ import annotations

import math

import torch

from paper_2603_09229_amd import binding as fk


def even_levels(heads: int, dtype: torch.dtype, device) -> torch.Tensor:
    """16 evenly spaced levels from -1 to 1 for each head."""
    return torch.linspace(-1, 1, 16, device=device).to(dtype).expand(heads, 16).contiguous()


def learn_levels(rows: torch.Tensor, iters: int = 12) -> torch.Tensor:
    """rows [N, heads, d] (keys as they are cached, so after turning, or values) -> levels [heads, 16], ascending.

    One k-means instance a head over all its numbers, each divided by the largest magnitude of its row: N * d points of one feature,
    16 clusters, which is the shape of the few-cluster pass.  It starts from the 16 even quantiles, so that levels stay in order.
    Rows that are not finite are refused: one of them would make all levels of its head NaN.  No gradient goes through a fit."""
    rows = rows.detach()
    N, H, d = rows.shape
    if not N:
        raise ValueError("levels are learned from at least one row")
    if not rows.isfinite().all():
        raise ValueError("rows must be finite")
    top = rows.float().abs().amax(dim=-1, keepdim=True)
    x = (rows.float() / torch.where(top > 0, top, 1.0)).to(rows.dtype).transpose(0, 1).reshape(H, N * d, 1).contiguous()
    at = ((torch.arange(16, device=x.device) + 0.5) / 16 * (N * d)).long()
    C = x[:, :, 0].float().sort(dim=1).values[:, at].unsqueeze(-1).contiguous()
    fk.fk_lloyd_iter(x, C, iters)
    return C[..., 0].clamp(-1, 1).sort(dim=1).values.to(rows.dtype).contiguous()


def angles(max_pos: int, rot: int, device, base: float = 10000.0) -> torch.Tensor:
    """cos | sin of every position, [max_pos, rot] float32."""
    a = torch.arange(max_pos, device=device, dtype=torch.float32)[:, None] * base ** (
        -torch.arange(rot // 2, device=device, dtype=torch.float32) / max(1, rot // 2))
    return torch.cat([a.cos(), a.sin()], dim=1).contiguous()


def tree_masks(parents: list[list[int]], device=None) -> tuple[torch.Tensor, list[int]]:
    """The masks of drafted trees for fk_kv_attend_tree, and how deep their tokens lie.

    parents[b][i]: the token of sequence b's tree that token i follows, -1: none of them, so the sequence's last token.  Parents come before
    their children.  -> masks [tokens of all trees, words] int64, bit j of a row: the token itself (j = i) and its ancestors; depths, 0 for roots"""
    words = max(1, -(-max((len(tree) for tree in parents), default=0) // 64))
    rows, depths = [], []
    for tree in parents:
        masks, deep = [], []
        for i, p in enumerate(tree):
            if not -1 <= p < i:
                raise ValueError(f"token {i} of a tree follows token {p}, which does not come before it")
            masks.append((masks[p] if p >= 0 else 0) | 1 << i)
            deep.append(deep[p] + 1 if p >= 0 else 0)
        rows += masks
        depths += deep
    low = (1 << 64) - 1
    signed = [[(x >> 64 * w & low) - ((x >> 64 * w & low) >> 63 << 64) for w in range(words)] for x in rows]
    return torch.tensor(signed, dtype=torch.int64).reshape(len(rows), words).to(device), depths


class Server:
    """A batch of sequences over one cache: slots are given out page by page, prompts and steps go through the three calls.

    max_len: tokens that a sequence holds at a time; max_pos: positions that it may take in all, where some tokens are evicted (max_len if not
    given: an eviction then frees places, but no positions); weights: every step adds its attention weights up, so that `evict` knows what to keep."""

    max_pos = None
    mass = None                                                       # attention weights of the cached tokens, with `weights`
    _draft = None                                                     # the drafted trees that wait for `accept`
    _empty = False                                                    # the last call was a draft without any: nothing waits

    def __init__(self, k_levels, v_levels, d: int, batch: int, max_len: int, page_size: int = 64, max_pos: int | None = None,
                 weights: bool = False):
        if batch < 1 or max_len < 1:
            raise ValueError(f"batch and max_len must be positive, got {batch}, {max_len}")
        if max_pos is not None and max_pos < max_len:
            raise ValueError(f"max_pos={max_pos} is less than max_len={max_len}")
        dev = k_levels.device
        self.max_pages = -(-max_len // page_size)
        self.cache = fk.KVCache.empty(batch * self.max_pages, page_size, k_levels, v_levels, d)
        # pages in any order: a page table need not be contiguous
        self.pages = torch.randperm(batch * self.max_pages, device=dev).view(batch, self.max_pages).to(torch.int32).contiguous()
        self.lens = torch.zeros(batch, dtype=torch.int32, device=dev)
        self.gone = torch.zeros(batch, dtype=torch.int32, device=dev)     # tokens that were evicted: positions run on
        self.max_len, self.max_pos = max_len, max_pos or max_len
        self.cos_sin = angles(self.max_pos, d, dev)
        if weights:
            self.mass = torch.zeros(self.cache.k_scale.shape, dtype=torch.float32, device=dev)

    def _check(self, q, k, v, counts: list[int], levels: list[int] | None = None):
        """Refused before anything changes: counts that are not one for each sequence or not those of the rows, and a sequence that would hold
        more than max_len tokens or pass position max_pos (they would have no page, or no angle).  levels: how many positions a sequence's
        tokens take, where that is not one each."""
        if len(counts) != len(self.lens) or any(c < 0 for c in counts) or not sum(counts) == len(q) == len(k) == len(v):
            raise ValueError(f"counts {counts} for {len(self.lens)} sequences and rows of {len(q)}, {len(k)}, {len(v)} tokens")
        limited = self.max_pos is not None
        held, *gone = torch.stack((self.lens, self.gone)).tolist() if limited else [self.lens.tolist()]
        over = [b for b, (h, c) in enumerate(zip(held, counts)) if h + c > self.max_len]
        if over:
            raise ValueError(f"sequences {over} would hold more than {self.max_len} tokens")
        if self._draft is not None:
            raise ValueError("drafted tokens wait for accept()")
        if limited:
            over = [b for b, (h, g, c) in enumerate(zip(held, *gone, levels or counts)) if h + g + c > self.max_pos]
            if over:
                raise ValueError(f"sequences {over} would pass position {self.max_pos}")
        self._empty = False

    def _append(self, q, k, v, counts: list[int], depths: list[int] | None = None):
        """New rows into the cache behind what the sequences hold -> (turned queries, starts); lens is left as it is.  depths: the
        positions of drafted tokens behind the sequence's, which otherwise follow each other."""
        dev, P = q.device, self.cache.page_size
        n = torch.tensor(counts, device=dev)
        start = torch.zeros(len(counts) + 1, dtype=torch.int32, device=dev)
        start[1:] = n.cumsum(0)
        seq = torch.repeat_interleave(torch.arange(len(counts), device=dev), n, output_size=len(q))
        place = self.lens[seq] + torch.arange(len(q), device=dev, dtype=torch.int32) - start[seq]
        slots = self.pages[seq, (place // P).long()].long() * P + place % P
        positions = place
        if depths is not None:
            positions = (self.lens + self.gone)[seq] + torch.tensor(depths, dtype=torch.int32, device=dev)
        elif self.mass is not None:                                   # (otherwise nothing is ever evicted)
            positions = place + self.gone[seq]
        return fk.fk_kv_append(self.cache, k, v, slots, positions=positions, cos_sin=self.cos_sin, q=q), start

    def _weigh(self, q, lse, start, most: int, before):
        fk.fk_kv_weigh(self.cache, q, lse, self.pages, self.lens, self.mass, q_start=start, max_q=most, max_len=self.max_len, known=before)

    def step(self, q, k, v, counts: list[int]) -> torch.Tensor:
        """counts[b] new tokens of sequence b, one after the other in q [T, q_heads, d], k, v [T, heads, d] -> attention [T, q_heads, d]."""
        self._check(q, k, v, counts)
        if not sum(counts):
            return torch.empty_like(q)
        q, start = self._append(q, k, v, counts)
        before = self.lens.clone() if self.mass is not None else None
        self.lens += start.diff()
        out = fk.fk_kv_attend(self.cache, q, self.pages, self.lens, q_start=start, max_q=max(counts), max_len=self.max_len,
                              lse=self.mass is not None)
        if self.mass is None:
            return out
        out, lse = out
        self._weigh(q, lse, start, max(counts), before)
        return out

    def draft(self, q, k, v, parents: list[list[int]]) -> torch.Tensor:
        """A tree of drafted tokens for each sequence (parents as in tree_masks, rows as in `step`, trees may be empty) -> attention of each
        token over what the sequence holds and its branch [T, q_heads, d].  `accept` says which of them stay."""
        counts = [len(tree) for tree in parents]
        masks, depths = tree_masks(parents, q.device)
        left = iter(depths)
        self._check(q, k, v, counts, [max((next(left) + 1 for _ in tree), default=0) for tree in parents])   # (tokens of a level share a position)
        if not sum(counts):
            self._empty = True
            return torch.empty_like(q)
        q, start = self._append(q, k, v, counts, depths)
        held = self.lens + start.diff()
        out = fk.fk_kv_attend_tree(self.cache, q, self.pages, held, masks, q_start=start, max_q=max(counts), max_len=self.max_len,
                                   lse=self.mass is not None)
        out, lse = out if self.mass is not None else (out, None)
        self._draft = ([list(tree) for tree in parents], q, lse)
        return out

    def accept(self, branches: list[list[int]]):
        """The drafted tokens that each sequence keeps, a branch from a root down, or none of them; the others are forgotten."""
        if self._draft is None and not self._empty:
            raise ValueError("there is no draft")
        parents, q, lse = self._draft or ([[]] * len(self.lens), None, None)
        if len(branches) != len(parents):
            raise ValueError(f"{len(branches)} branches for {len(parents)} sequences")
        for tree, branch in zip(parents, branches):
            if any(not 0 <= i < len(tree) or tree[i] != p for p, i in zip([-1] + branch, branch)):
                raise ValueError(f"{branch} is no branch from a root of the tree {tree}")
        self._draft, self._empty = None, False
        counts, most = [len(branch) for branch in branches], max(map(len, branches))
        if not most:
            return
        dev = self.lens.device
        kept = torch.tensor([branch + [-1] * (most - len(branch)) for branch in branches], dtype=torch.int32).to(dev)[:, None]
        before, n = self.lens.clone(), torch.tensor(counts, dtype=torch.int32).to(dev)
        fk.fk_kv_compact(self.cache, self.pages, kept, n, start=before)
        self.lens += n
        if self.mass is None:
            return
        # the accepted tokens are the last ones of their sequences now, and see what they saw in the tree
        firsts = [sum(len(tree) for tree in parents[:b]) for b in range(len(parents))]
        rows = torch.tensor([f + i for f, branch in zip(firsts, branches) for i in branch]).to(dev)
        start = torch.tensor([sum(counts[:b]) for b in range(len(counts) + 1)], dtype=torch.int32).to(dev)
        self._weigh(q[rows], lse[rows], start, most, before)

    def evict(self, keep: int, first: int = 4, last: int = 32):
        """Cuts every sequence of more than `keep` tokens down to that many: its first ones, its last ones, and for each head those of the others
        that were given the most attention.  Positions of later tokens run on."""
        if self.mass is None:
            raise ValueError("evict() goes by attention weights: Server(..., weights=True) adds them up")
        if self._draft is not None:
            raise ValueError("drafted tokens wait for accept()")
        kept, counts = fk.fk_kv_choose(self.cache, self.mass, self.pages, self.lens, keep, first=first, last=last, max_len=self.max_len)
        fk.fk_kv_compact(self.cache, self.pages, kept, counts, mass=self.mass)
        self.gone += self.lens - counts
        self.lens = counts


def turned(x, cos_sin, pos):
    """Rows [T, heads, d] turned by the angles of their positions, in 32 bits."""
    c, s = cos_sin[pos][:, None].chunk(2, dim=-1)
    a, b = x.float().chunk(2, dim=-1)
    return torch.cat([a * c - b * s, b * c + a * s], dim=-1)


def uncoded(q, k, v, cos_sin) -> torch.Tensor:
    """Attention of one sequence's last len(q) tokens over its keys and values as they are, in 32 bits."""
    n, L, G = len(q), len(k), q.shape[1] // k.shape[1]
    pos = torch.arange(L, device=q.device)
    Q = turned(q, cos_sin, pos[L - n:]).transpose(0, 1)
    K = turned(k, cos_sin, pos).transpose(0, 1).repeat_interleave(G, dim=0)
    V = v.float().transpose(0, 1).repeat_interleave(G, dim=0)
    x = (Q @ K.transpose(1, 2)) / math.sqrt(q.shape[2])
    x = x.masked_fill(pos > pos[L - n:, None], -math.inf)
    return (torch.softmax(x, dim=-1) @ V).transpose(0, 1)


def demo(batch: int = 4, heads: int = 4, group: int = 4, d: int = 128, prompt: int = 300, steps: int = 8,
         dtype: torch.dtype = torch.bfloat16, device="cuda") -> dict:
    """Ragged prompts, then `steps` tokens each; -> root mean square error relative to the result, learned and even levels."""
    g = torch.Generator(device=device).manual_seed(3)
    counts = [max(1, prompt - 37 * b) for b in range(batch)]
    draw = lambda n, h: torch.randn(n, h, d, generator=g, device=device).to(dtype)
    parts = [counts] + [[1] * batch] * steps
    data = [(draw(sum(c), heads * group), draw(sum(c), heads), draw(sum(c), heads)) for c in parts]
    cos_sin = angles(prompt + steps, d, device)
    first = torch.cat([torch.arange(c, device=device) for c in counts])
    learned = [learn_levels(turned(data[0][1], cos_sin, first).to(dtype)), learn_levels(data[0][2])]
    even = [even_levels(heads, dtype, device)] * 2
    result = {}
    for name, (kl, vl) in (("learned", learned), ("even", even)):
        server = Server(kl, vl, d, batch, prompt + steps)
        off = norm = 0.0
        keys, values = [[] for _ in counts], [[] for _ in counts]
        for c, (q, k, v) in zip(parts, data):
            out = server.step(q, k, v, c).float()
            for b, (qb, kb, vb, ob) in enumerate(zip(q.split(c), k.split(c), v.split(c), out.split(c))):
                keys[b].append(kb)
                values[b].append(vb)
                want = uncoded(qb, torch.cat(keys[b]), torch.cat(values[b]), cos_sin)
                off += (ob - want).square().sum().item()
                norm += want.square().sum().item()
        result[name] = math.sqrt(off / norm)
    return result


def demo_eviction(batch: int = 3, heads: int = 2, group: int = 4, d: int = 64, prompt: int = 400, steps: int = 24, keep: int = 128,
                  dtype: torch.dtype = torch.bfloat16, device="cuda") -> dict:
    """Prompts, then steps of a drafted tree each, of which a branch is accepted, cut down to `keep` tokens whenever a sequence holds half as many
    more -> the share of all attention weight that the tokens which stayed had, and the most tokens held."""
    g = torch.Generator(device=device).manual_seed(4)
    draw = lambda n, h: torch.randn(n, h, d, generator=g, device=device).to(dtype)
    topic = 1.5 * torch.randn(heads, 8, d, generator=g, device=device)    # keys and queries of a few kinds, so that some tokens matter
    about = lambda n, h: (topic[torch.arange(h, device=device) * heads // h, torch.randint(0, 8, (n, 1), generator=g, device=device)]
                          + draw(n, h).float()).to(dtype)
    counts = [prompt - 29 * b for b in range(batch)]
    k, v = about(sum(counts), heads), draw(sum(counts), heads)
    server = Server(learn_levels(k), learn_levels(v), d, batch, prompt + 16, max_pos=prompt + 4 * steps, weights=True)
    server.step(about(sum(counts), heads * group), k, v, counts)
    tree, branches = [-1, -1, 0, 0, 1, 2], [[0, 2, 5], [1], [0, 3]]
    share, most = [], 0
    for i in range(steps):
        n = len(tree) * batch
        server.draft(about(n, heads * group), about(n, heads), draw(n, heads), [tree] * batch)
        server.accept([branches[(i + b) % 3] for b in range(batch)])
        if max(server.lens.tolist()) > keep * 3 // 2:
            before = [server.mass[server.pages[b].long()].transpose(0, 1).flatten(1)[:, :L].sum().item() for b, L in enumerate(server.lens.tolist())]
            server.evict(keep)
            after = [server.mass[server.pages[b].long()].transpose(0, 1).flatten(1)[:, :L].sum().item() for b, L in enumerate(server.lens.tolist())]
            share.append(sum(after) / sum(before))
        most = max(most, *server.lens.tolist())
    return {"share": min(share), "held": most}


if __name__ == "__main__":
    for name, error in demo().items():
        print(f"{name} levels: attention off by {100 * error:.2f} % of its size")
    kept = demo_eviction()
    print(f"evictions kept {100 * kept['share']:.0f} % of the attention weight and {kept['held']} tokens at most")
