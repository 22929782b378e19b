"""Serving from a key/value cache whose 4-bit levels are learned by k-means: the calls in the order a program makes them.

    levels   16 centroids of single numbers a head, from a sample of rows divided by their largest magnitudes (fk_lloyd_iter)
    append   new tokens go into their slots, keys and queries turned by the angles of their positions (fk_kv_append)
    attend   the queries read the cache: a prompt's own tokens first, then one token a sequence and step (fk_kv_attend)

``python -m paper_2603_09229_amd.kv_cache`` runs a small batch of ragged prompts and some decoding steps, compares every result with
attention over the uncoded keys and values, and prints what the coding costs with learned levels and with evenly spaced ones.
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


class Server:
    """A batch of sequences over one cache: slots are given out page by page, prompts and steps go through the three calls."""

    def __init__(self, k_levels, v_levels, d: int, batch: int, max_len: int, page_size: int = 64):
        if batch < 1 or max_len < 1:
            raise ValueError(f"batch and max_len must be positive, got {batch}, {max_len}")
        dev = k_levels.device
        self.max_pages = -(-max_len // page_size)
        self.cache = fk.KVCache.empty(batch * self.max_pages, page_size, k_levels, v_levels, d)
        # pages in any order: a page table need not be contiguous
        self.pages = torch.randperm(batch * self.max_pages, device=dev).view(batch, self.max_pages).to(torch.int32).contiguous()
        self.lens = torch.zeros(batch, dtype=torch.int32, device=dev)
        self.cos_sin = angles(max_len, d, dev)
        self.max_len = max_len

    def step(self, q, k, v, counts: list[int]) -> torch.Tensor:
        """counts[b] new tokens of sequence b, one after the other in q [T, q_heads, d], k, v [T, heads, d] -> attention [T, q_heads, d].

        Refused before anything changes: counts that are not one for each sequence or not those of the rows, and a sequence that would hold more
        than max_len tokens (they would have no page, and no angle)."""
        if len(counts) != len(self.lens) or any(c < 0 for c in counts) or not sum(counts) == len(q) == len(k) == len(v):
            raise ValueError(f"counts {counts} for {len(self.lens)} sequences and rows of {len(q)}, {len(k)}, {len(v)} tokens")
        over = [b for b, (held, c) in enumerate(zip(self.lens.tolist(), counts)) if held + c > self.max_len]
        if over:
            raise ValueError(f"sequences {over} would hold more than {self.max_len} tokens")
        if not sum(counts):
            return torch.empty_like(q)
        dev, P = q.device, self.cache.page_size
        n = torch.tensor(counts, device=dev)
        start = torch.zeros(len(counts) + 1, dtype=torch.int32, device=dev)
        start[1:] = n.cumsum(0)
        seq = torch.repeat_interleave(torch.arange(len(counts), device=dev), n, output_size=len(q))
        pos = self.lens[seq] + torch.arange(len(q), device=dev, dtype=torch.int32) - start[seq]
        slots = self.pages[seq, (pos // P).long()].long() * P + pos % P
        q = fk.fk_kv_append(self.cache, k, v, slots, positions=pos, cos_sin=self.cos_sin, q=q)
        self.lens += n.to(torch.int32)
        return fk.fk_kv_attend(self.cache, q, self.pages, self.lens, q_start=start, max_q=max(counts), max_len=self.max_len)


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


if __name__ == "__main__":
    for name, error in demo().items():
        print(f"{name} levels: attention off by {100 * error:.2f} % of its size")
