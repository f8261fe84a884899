"""64-bit references for the 4-bit cache, the accumulated weights and the
eviction, written from the definitions in include/gva.h."""

from __future__ import annotations

import math

import torch

LEVELS = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)


def quantize(x: torch.Tensor):
    """Rows [..., d] -> (codes, one per element; scale bytes [..., d/32])."""
    b = x.double().unflatten(-1, (-1, 32))
    amax = b.abs().amax(-1)
    byte = torch.full(amax.shape, 252, dtype=torch.int64)
    for e in range(125, -120, -1):                       # the smallest scale that reaches amax
        byte = torch.where(amax <= 7.0 * 2.0 ** e, torch.full_like(byte, e + 127), byte)
    y = b.abs() / torch.exp2(byte.double() - 127).unsqueeze(-1)
    dist = (y.unsqueeze(-1) - LEVELS).abs()
    near = dist.amin(-1, keepdim=True)
    tied = dist == near
    even = tied & (torch.arange(8) % 2 == 0)             # of two levels as near, the even code
    code = torch.where(even.any(-1), even.int().argmax(-1), tied.int().argmax(-1))
    code = code + 8 * torch.signbit(b)
    bad = ~torch.isfinite(b).all(-1)
    code = torch.where(bad.unsqueeze(-1), torch.zeros_like(code), code)
    return code.flatten(-2).to(torch.uint8), torch.where(bad, torch.full_like(byte, 255), byte).to(torch.uint8)


def values(code: torch.Tensor, byte: torch.Tensor) -> torch.Tensor:
    """fp64 rows that codes and scale bytes stand for."""
    v = LEVELS[(code & 7).long()] * torch.where(code >= 8, -1.0, 1.0)
    s = torch.exp2(byte.double() - 127)
    s = torch.where(byte == 255, torch.full_like(s, math.nan), s)
    return (v.unflatten(-1, (-1, 32)) * s.unsqueeze(-1)).flatten(-2)


def _code_at(T, d):
    """[T, d]: byte of a stream that holds element (t, i)."""
    t, i = torch.arange(T).unsqueeze(1), torch.arange(d).unsqueeze(0)
    R, P = 2048 // d, d // 4
    return t // R * 1024 + (i // P * 16 + t % 16) * 16 + t % R // 16 * 8 + i % P // 2


def _scale_at(T, d):
    t, c = torch.arange(T).unsqueeze(1), torch.arange(d // 32).unsqueeze(0)
    return t // 32 * d + (c * 16 + t % 16) * 2 + t % 32 // 16


def pack(code: torch.Tensor, byte: torch.Tensor):
    """Codes [..., T, d] and scale bytes [..., T, d/32] in the library's layouts."""
    *lead, T, d = code.shape
    c = code.reshape(-1, T * d).int()
    at = _code_at(T, d).reshape(-1)
    out = torch.zeros(c.shape[0], T * d // 2, dtype=torch.int32)
    shift = (4 * (torch.arange(d, dtype=torch.int32) % 2)).repeat(T)
    out.index_add_(1, at, c << shift)
    s = torch.zeros(c.shape[0], T * d // 32, dtype=torch.uint8)
    s[:, _scale_at(T, d).reshape(-1)] = byte.reshape(c.shape[0], -1)
    return out.to(torch.uint8).reshape(*lead, T, d // 2), s.reshape(*lead, T, d // 32)


def unpack(codes: torch.Tensor, scales: torch.Tensor):
    """Inverse of pack."""
    *lead, T, h = codes.shape
    d = 2 * h
    flat = codes.reshape(-1, T * h)
    c = flat[:, _code_at(T, d).reshape(-1)].int() >> (4 * (torch.arange(d) % 2)).repeat(T) & 15
    s = scales.reshape(flat.shape[0], -1)[:, _scale_at(T, d).reshape(-1)]
    return c.to(torch.uint8).reshape(*lead, T, d), s.reshape(*lead, T, d // 32)


def rotate(x: torch.Tensor, pos, base=10000.0) -> torch.Tensor:
    D = x.shape[-1]
    if D == 0:
        return x.double()
    th = base ** (-torch.arange(0, D, 2, dtype=torch.float64) / D)
    a = torch.as_tensor(pos).double().unsqueeze(-1) * th
    x0, x1 = x[..., 0::2].double(), x[..., 1::2].double()
    return torch.stack((x0 * a.cos() - x1 * a.sin(), x0 * a.sin() + x1 * a.cos()), -1).flatten(-2)


def scores(q, m, v, kr, lens, seen, n_groups):
    """Scaled scores [B, N, H, T] of the last N queries over explicit keys
    (rows a query does not see -inf), and a bound on each one's sum of
    magnitudes.  q [B, N, H, dc+dr], v [B, G, T, dv] and kr [B, T, dr] fp64."""
    B, N, H, W = q.shape
    T, dr, hpg = v.shape[2], kr.shape[-1], H // n_groups
    dc = W - dr
    x = torch.full((B, N, H, T), -math.inf, dtype=torch.float64)
    size = torch.zeros(B, N, H, T, dtype=torch.float64)
    for b in range(B):
        L = min(max(int(lens[b]), 0), T)
        at = int(seen[b]) - N + torch.arange(N)
        hidden = torch.arange(L).unsqueeze(0) > (L - N + torch.arange(N)).unsqueeze(1)
        for h in range(H):
            vb = v[b, h // hpg, :L]
            qr = rotate(q[b, :, h, dc:], at.clamp(min=0))
            qa = q[b, :, h, :dc].double() @ m[h].double().t()
            s = ((qa @ vb.t()) + (qr @ kr[b, :L].t())) / math.sqrt(W)
            x[b, :, h, :L] = s.masked_fill(hidden, -math.inf)
            size[b, :, h, :L] = (qa.abs() @ vb.abs().t() + qr.abs() @ kr[b, :L].abs().t()) / math.sqrt(W)
    return x, size


def attend(x, v, n_groups):
    """(o [B, N, H, dv], lse) of scores x."""
    B, N, H, T = x.shape
    lse = torch.logsumexp(x, -1)
    p = torch.where(torch.isneginf(lse).unsqueeze(-1), torch.zeros_like(x),
                    torch.exp(x - torch.where(torch.isneginf(lse), torch.zeros_like(lse), lse).unsqueeze(-1)))
    vv = v.repeat_interleave(H // n_groups, 1)
    o = torch.stack([p[:, i].unsqueeze(2).matmul(torch.nan_to_num(vv)).squeeze(2) for i in range(N)], 1)
    return o, lse


def evict(weights, lens, row_pos, seen, keep, first, recent):
    """Per sequence: (new length, [(to, from)] of the rows that move, and the
    source row of every row kept, by its new place)."""
    out = []
    for b in range(len(lens)):
        L = int(lens[b])
        if L <= keep:
            out.append((L, [], {t: t for t in range(L)}))
            continue
        w, pos = weights[b].tolist(), row_pos[b].tolist()

        def rank(t):
            if pos[t] < first or pos[t] >= int(seen[b]) - recent:
                return (0, 0.0, t)
            return (2, 0.0, t) if math.isnan(w[t]) else (1, -w[t], t)
        best = set(sorted(range(L), key=rank)[:keep])
        holes = [t for t in range(keep) if t not in best]
        movers = sorted(t for t in best if t >= keep)
        src = {t: t for t in best if t < keep}
        src.update(zip(holes, movers))
        out.append((keep, list(zip(holes, movers)), src))
    return out
