"""The 4-bit key/value cache in 64 bits and plain loops over sequences and heads: what the kernels are compared with."""
import math

import torch


def levels(H, t, seed, device="cpu"):
    g = torch.Generator().manual_seed(seed)
    x = torch.linspace(-1, 1, 16) * torch.rand(H, 1, generator=g).mul(0.4).add(0.6) + 0.04 * torch.rand(H, 16, generator=g)
    return x.clamp(-1, 1).sort(dim=1).values.to(t).to(device)


def values(codes, scale, lv):
    """codes [pages, H, P, d/2] uint8, scale [pages, H, P], lv [H, 16] -> [pages, H, P, d] in 64 bits."""
    ids = torch.stack([codes & 15, codes >> 4], dim=-1).flatten(-2).long()
    table = lv.double()[None, :, None, :].expand(*codes.shape[:3], 16)
    return table.gather(-1, ids) * scale.double()[..., None]


def turned(x, cos_sin, positions, interleaved):
    """Rows x [T, heads, d] turned in 32 bits, every product and sum rounded by itself, as the header defines it; of x's type."""
    R = cos_sin.shape[1]
    cs = cos_sin[positions.long().clamp(0, cos_sin.shape[0] - 1)][:, None]
    c, s = cs[..., :R // 2], cs[..., R // 2:]
    y = x.float().clone()
    i, j = (slice(0, R, 2), slice(1, R, 2)) if interleaved else (slice(0, R // 2), slice(R // 2, R))
    a, b = x[..., i].float(), x[..., j].float()
    y[..., i], y[..., j] = a * c - b * s, b * c + a * s
    return y.to(x.dtype)


def attend(k, v, q, table, lens, starts, scale, causal, window):
    """k, v [pages, H, P, d] in 64 bits; -> (out, lse, mean of |weight * value|, bound of a score's rounding error in 32 bits)."""
    H, P, d = k.shape[1:]
    G = q.shape[1] // H
    out = torch.zeros(q.shape, dtype=torch.float64, device=q.device)
    mag = torch.zeros_like(out)
    lse = torch.full(q.shape[:2], -math.inf, dtype=torch.float64, device=q.device)
    err = torch.zeros_like(lse)
    for b, L in enumerate(lens):
        s0, n = starts[b], starts[b + 1] - starts[b]
        pos = L - n + torch.arange(n, device=q.device)
        tok = torch.arange(L, device=q.device)
        sees = torch.ones(n, L, dtype=torch.bool, device=q.device)
        if causal:
            sees &= tok <= pos[:, None]
        if window:
            sees &= tok > pos[:, None] - window
        if not n or not L:
            continue
        held = table[b, :-(-L // P)].long()
        for h in range(H):
            K = k[held, h].reshape(-1, d)[:L].nan_to_num()
            V = v[held, h].reshape(-1, d)[:L].nan_to_num()
            for g in range(h * G, (h + 1) * G):
                x = q[s0:s0 + n, g].double()
                sc = (x @ K.T * scale).masked_fill(~sees, -math.inf)
                top = sc.amax(-1, keepdim=True).clamp_min(-1e300)
                e = torch.exp(sc - top)
                tot = e.sum(-1, keepdim=True)
                live = tot[:, 0] > 0
                out[s0:s0 + n, g] = torch.where(tot > 0, e @ V / tot, 0.0)
                mag[s0:s0 + n, g] = torch.where(tot > 0, e @ V.abs() / tot, 0.0)
                lse[s0:s0 + n, g] = torch.where(live, top[:, 0] + torch.log(tot[:, 0]), -math.inf)
                worst = ((x.abs() @ K.abs().T) * abs(scale)).masked_fill(~sees, 0.0).amax(-1)
                err[s0:s0 + n, g] = (d + 16) * 2.0 ** -24 * worst
    return out, lse, mag, err
