"""64-bit references for the calls that serve many requests on one cache (page
tables, slots, packed and tree attention, tree commit), written from the
definitions in include/gva.h."""

from __future__ import annotations

import math

import torch

BASE = 10000.0


def page_tables(lens, n_new, table, free, n_free, n_rows, T, R, n_pages):
    """Lists in, lists out; table and free are changed in place."""
    pages = lambda x: -(-x // R)                               # noqa: E731
    lens = [min(max(x, 0), T) for x in lens]
    n = [min(max(x, -L), T) for x, L in zip(n_new, lens)]
    top = min(max(n_free, 0), n_pages)
    for b, L in enumerate(lens):
        if n[b] < 0:
            for page in range(pages(L + n[b]), pages(L)):
                if top < n_pages:
                    free[top] = table[b][page]
                    top += 1
    asked, start, new_lens, cu, seq, row, slot = 0, top, [], [0], [], [], []
    for b, L in enumerate(lens):
        want = L + n[b]
        ok = want <= T
        if ok and n[b] > 0:
            need = pages(want) - pages(L)
            asked += need
            ok = need == 0 or asked <= start
            if ok:
                for page in range(pages(L), pages(want)):
                    top -= 1
                    table[b][page] = free[top]
        new_lens.append(L if n[b] > 0 and not ok else want)
        cu.append(cu[-1] + max(n[b], 0))
        for i in range(max(n[b], 0)):
            if len(seq) >= n_rows:
                break
            t = L + i if ok else -1
            page = table[b][t // R] if ok else -1
            seq.append(b)
            row.append(t)
            slot.append(page * R + t % R if 0 <= page < n_pages else -1)
    pad = [-1] * (n_rows - len(seq))
    return {"lens": new_lens, "n_free": top, "cu": [min(c, n_rows) for c in cu], "seq": seq + pad, "row": row + pad,
            "slot": slot + pad}


def rotate(x, pos):
    """fp64 rows [..., D] rotated in interleaved pairs at pos [...]."""
    D = x.shape[-1]
    if D == 0:
        return x.double()
    a = torch.as_tensor(pos).double().unsqueeze(-1) * BASE ** (-torch.arange(0, D, 2, dtype=torch.float64) / D)
    x0, x1 = x[..., 0::2].double(), x[..., 1::2].double()
    return torch.stack((x0 * a.cos() - x1 * a.sin(), x0 * a.sin() + x1 * a.cos()), -1).flatten(-2)


def parents(parent):
    """What a list of parents is read as."""
    return [a if 0 <= a < i else -1 for i, a in enumerate(parent)]


def ancestors(parent, i):
    """The path from the root to node i."""
    path = []
    while i >= 0:
        path.append(i)
        i = parent[i]
    return path[::-1]


def window(L, n, parent=None):
    """(visible [n, L], positions [n]) of a sequence's last n of L rows; rows of the window below 0 see nothing."""
    P = L - n
    see = torch.zeros(n, max(L, 0), dtype=torch.bool)
    pos = []
    for i in range(n):
        if parent is None:
            see[i, :max(0, P + i + 1)] = True
            pos.append(P + i)
            continue
        path = ancestors(parent, i)
        pos.append(P + len(path) - 1)
        if P + i < 0:
            continue
        see[i, :max(P, 0)] = True
        for a in path:
            if P + a >= 0:
                see[i, P + a] = True
    return see, torch.tensor(pos, dtype=torch.float64).clamp(min=0)


def attend(q, m, v, kr, see, pos, G, dtype):
    """One sequence: q [n, H, dc + dr], m [H, dv, dc], v [G, L, dv], kr [L, dr].
    Returns fp64 (o, lse) and bounds (do, dlse) on the kernel's error, from its
    roundings, each at most eps / 2 of its value (2^-24 fp32, 2^-8 bf16):
     - q~: d_c products summed in fp32; bf16: entered as two bf16 parts, off by
       at most 2^-17 (the remainder of the first is below 2^-8, its own
       rounding at most 2^-9 of that);
     - a score: d_v + d_r products, twice for two parts, summed in fp32; the
       rotation's sine and cosine, the scale, the difference from the maximum
       and the exponential: 8 more of the largest score's size;
     - a weight: that of its score, as a factor; bf16: its own rounding in the
       numerator;
     - the sums over L rows, and the output's rounding.
    Errors of higher order add a tenth."""
    n, H, W = q.shape
    dv, dr = v.shape[-1], kr.shape[-1]
    dc, L, hpg = W - dr, v.shape[1], H // G
    u, bf = 2.0 ** -24, dtype == torch.bfloat16
    q, m, v, kr = q.double(), m.double(), v.double(), kr.double()
    qr = rotate(q[..., dc:], pos.unsqueeze(-1)) if n else q[..., dc:]
    o, lse = torch.zeros(n, H, dv, dtype=torch.float64), torch.full((n, H), -math.inf, dtype=torch.float64)
    do, dlse = torch.zeros_like(o), torch.zeros_like(lse)
    for h in range(H):
        vh = torch.nan_to_num(v[h // hpg], 0, 0, 0)
        kk = torch.nan_to_num(kr, 0, 0, 0)
        qa = q[:, h, :dc] @ m[h].t()
        size0 = q[:, h, :dc].abs() @ m[h].abs().t() @ vh.abs().t() + qr[:, h].abs() @ kk.abs().t() * 2
        size = qa.abs() @ vh.abs().t() + qr[:, h].abs() @ kk.abs().t() * 2
        x = ((qa @ vh.t()) + qr[:, h] @ kk.t()) / math.sqrt(W)
        size, size0 = size / math.sqrt(W), size0 / math.sqrt(W)
        dx = size * ((2.0 ** -17 if bf else 0) + (2 * (dv + dr) + 4) * u) + size0 * (dc + 4) * u
        top = (size * see).amax(-1, keepdim=True) if L else torch.zeros(n, 1)
        dx = 1.1 * (dx + 8 * u * (1 + top))
        x = x.masked_fill(~see, -math.inf)
        some = see.any(-1)
        lse[:, h] = torch.logsumexp(x, -1) if L else lse[:, h]
        w = torch.where(some.unsqueeze(-1), torch.exp(x - torch.where(some, lse[:, h], torch.zeros(n)).unsqueeze(-1)),
                        torch.zeros(n, L)) if L else torch.zeros(n, 0)
        w = w.double()
        rel = torch.expm1(dx) * see
        o[:, h] = w @ vh
        part = (w * rel).sum(-1, keepdim=True) + (L + 8) * u
        do[:, h] = (w * (rel + (2.0 ** -8 if bf else 0) + (L + 8) * u)) @ vh.abs() + part * o[:, h].abs()
        do[:, h] = 1.1 * do[:, h] + (2.0 ** -8 if bf else 2.0 ** -24) * (o[:, h].abs() + do[:, h]) + 1e-30
        dlse[:, h] = 1.1 * part.squeeze(-1) + 4 * u * (1 + lse[:, h].abs().nan_to_num(0, 0, 0))
    return o, lse, do, dlse
