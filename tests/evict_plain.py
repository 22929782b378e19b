"""Trees of drafted tokens, attention weights, the choice of places and compaction in 64 bits and plain loops: what the kernels are compared
with."""
import math

import torch


def tree_sees(masks, L, n, window):
    """masks: n integers, bit j: token j of the tree.  -> [n, L], of what each row sees the last `window`."""
    sees = torch.zeros(n, L, dtype=torch.bool)
    for i in range(n):
        seen = [t for t in range(L) if t < L - n or masks[i] >> (t - L + n) & 1]
        sees[i, seen[-window:] if window else seen] = True
    return sees


def row_sees(L, n, causal, window):
    """The same for queries in a row."""
    pos, tok = torch.arange(L - n, L)[:, None], torch.arange(L)[None]
    sees = torch.ones(n, L, dtype=torch.bool)
    if causal:
        sees &= tok <= pos
    if window:
        sees &= tok > pos - window
    return sees


def words_of(masks, words):
    """Integers as rows of 64-bit words, int64."""
    cut = [[(x >> 64 * w) & (1 << 64) - 1 for w in range(words)] for x in masks]
    return torch.tensor([[x - (1 << 64) if x >> 63 else x for x in row] for row in cut], dtype=torch.int64).reshape(len(masks), words)


def scores(k, q, held, h, L, G, scale):
    """Scores [n, G, L] of one sequence and cache head in 64 bits, and a bound of their rounding error in 32 bits."""
    K = k[held, h].reshape(-1, k.shape[-1])[:L].nan_to_num()
    x = q[:, h * G:(h + 1) * G].double()
    worst = (x.abs() @ K.abs().T) * abs(scale)
    return x @ K.T * scale, (k.shape[-1] + 16) * 2.0 ** -24 * worst


def attend(k, v, q, table, lens, starts, scale, sees):
    """k, v [pages, H, P, d] in 64 bits, sees: [n, L] of each sequence -> as kv_plain.attend."""
    H, P, d = k.shape[1:]
    G = q.shape[1] // H
    out = torch.zeros(q.shape, dtype=torch.float64, device=q.device)
    mag, lse = torch.zeros_like(out), torch.full(q.shape[:2], -math.inf, dtype=torch.float64, device=q.device)
    err = torch.zeros_like(lse)
    for b, L in enumerate(lens):
        s0, n = starts[b], starts[b + 1] - starts[b]
        if not n or not L:
            continue
        held, hide = table[b, :-(-L // P)].long(), ~sees[b].to(q.device)[:, None]
        for h in range(H):
            x, off = scores(k, q[s0:s0 + n], held, h, L, G, scale)
            V = v[held, h].reshape(-1, d)[:L].nan_to_num()
            x = x.masked_fill(hide, -math.inf)
            top = x.amax(-1, keepdim=True).clamp_min(-1e300)
            e = torch.exp(x - top)
            tot = e.sum(-1, keepdim=True)
            at = (slice(s0, s0 + n), slice(h * G, (h + 1) * G))
            out[at] = torch.where(tot > 0, e @ V / tot, 0.0)
            mag[at] = torch.where(tot > 0, e @ V.abs() / tot, 0.0)
            lse[at] = torch.where(tot > 0, top + torch.log(tot), -math.inf)[..., 0]
            err[at] = off.masked_fill(hide, 0.0).amax(-1)
    return out, lse, mag, err


def weigh(k, q, lse, table, lens, starts, scale, sees, known, decay, mass, out):
    """-> (weights, bound of their error): `out` in 64 bits with the sequences' places filled, the bound 0 elsewhere.

    A weight's exponent in 32 bits is off by the score's rounding, by the logarithm's product with log2 e and by the difference's rounding,
    2^-24 of each; the exponential by 2^-23 of itself.  Sums of N positive numbers are off by N 2^-24 of the sum, the old weight's
    product and the last sum by 2^-24 each."""
    H, P = k.shape[1:3]
    G = q.shape[1] // H
    out = out.double().clone()
    bound = torch.zeros_like(out)
    for b, L in enumerate(lens):
        s0, n = starts[b], starts[b + 1] - starts[b]
        if not L:
            continue
        tok = torch.arange(L, device=q.device)
        page, place = table[b, tok // P].long(), tok % P
        for h in range(H):
            new, off = torch.zeros(2, L, dtype=torch.float64, device=q.device)
            if n:
                x, err = scores(k, q[s0:s0 + n], table[b, :-(-L // P)].long(), h, L, G, scale)
                ls = lse[s0:s0 + n, h * G:(h + 1) * G].double()[..., None]
                w = torch.where(sees[b].to(q.device)[:, None] & (ls > -math.inf), torch.exp(x - ls), 0.0)
                e = err + 2.0 ** -24 * (2 * x.abs() + 2 * ls.abs().nan_to_num(posinf=0.0) + (x - ls).abs().nan_to_num(posinf=0.0)) * 1.5 + 2.0 ** -22
                new = w.sum((0, 1))
                off = (w * torch.expm1(e)).sum((0, 1)) + (n * G + 16) * 2.0 ** -24 * new + n * G * 2.0 ** -126
            old = torch.where(tok < known[b], decay * mass[page, h, place].double().nan_to_num(), 0.0)
            out[page, h, place] = old + new
            bound[page, h, place] = off + 2.0 ** -23 * (old.abs() + new)
    return out, bound


def choose(mass, table, lens, P, keep, first, last):
    """-> kept [B, H, keep], counts [B] on the host."""
    H = mass.shape[1]
    kept = torch.full((len(lens), H, keep), -1, dtype=torch.int32)
    for b, L in enumerate(lens):
        for h in range(H):
            w = [mass[table[b, t // P], h, t % P].item() for t in range(L)]
            stays = list(range(L))
            if L > keep:
                middle = sorted(range(first, L - last), key=lambda t: (w[t] != w[t], -w[t] if w[t] == w[t] else 0.0, t))
                stays = sorted(list(range(first)) + middle[:keep - first - last] + list(range(L - last, L)))
            kept[b, h, :len(stays)] = torch.tensor(stays, dtype=torch.int32)
    return kept, torch.tensor([min(L, keep) for L in lens], dtype=torch.int32)


def compact(tensors, table, kept, counts, start, to):
    """tensors [pages, H, P, ...] on the host -> copies with the rows moved."""
    H, P = tensors[0].shape[1:3]
    new = [x.clone() for x in tensors]
    for b, n in enumerate(counts):
        for h in range(H):
            for j in range(n):
                place = int(kept[b, h if kept.shape[1] > 1 else 0, j])
                if place < 0:
                    continue
                src, dst = start[b] + place, start[b] + j
                for x, y in zip(tensors, new):
                    y[to[b, dst // P], h, dst % P] = x[table[b, src // P], h, src % P]
    return new
