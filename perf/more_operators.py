"""Timed cases of the operators that serve many requests at once on one cache:
block tables and slot maps built from the requests' lengths, rows appended at
slots, attention of packed prompts of different lengths, attention of drafted
token trees, and the commit of a tree's accepted path.

Each case has a plain form in elementary torch operations and, where ``own`` is
set, the calls of the library.  Both take the same state: caches in the
library's storage layout, queries, maps, lengths and tables as a serving
program holds them.

Caches.  ``page_rows`` 0: contiguous, values [B][G][T][d_v] and positional keys
[B][T][d_r].  Else pools of pages, [pages][G][page_rows][d_v] and
[pages][page_rows][d_r], and a block table [B][T / page_rows]; row t of a
sequence is row t % page_rows of page table[t / page_rows], and slot page *
page_rows + t % page_rows.  A stream or page is stored in tiles of 16 rows, the
16-byte pieces of the rows piece-major.

Packed rows.  The new rows (or queries) of all sequences lie one behind the
other, sequence b's at cu[b] .. cu[b + 1] - 1.  With L_b cached rows, the new
ones included, and n_b of them new, the first L_b - n_b are the prefix.  A
prompt's row i stands at position L_b - n_b + i and sees the rows up to its own.
A tree's node i (parent[i] < i, -1: it hangs on the prefix) stands at position
L_b - n_b + its depth and sees the prefix, its ancestors and itself.
"""

import math

import torch

own = False

_DT = {"bf16": torch.bfloat16, "f32": torch.float32}
_BASE = 10000.0


def _case(name, kind, dtype="bf16", *, batch, t_max, groups=8, heads=32, d_v=128, d_c=None, d_r=16, page_rows=64, new_min=1,
          new_max=1, prefix_min=0, prefix_max=0, plan="step", spare=1.0):
    c = {"kind": kind, "dtype": dtype, "batch": batch, "t_max": t_max, "heads": heads, "groups": groups, "d_v": d_v,
         "d_c": d_v if d_c is None else d_c, "d_r": d_r, "page_rows": page_rows, "new_min": new_min, "new_max": new_max,
         "prefix_min": prefix_min, "prefix_max": prefix_max, "plan": plan, "spare": spare}
    return dict(c, name=name) if name else c


def listed():
    return [
        # A decode step's bookkeeping for 64 chats: a row each, now and then a new page.
        _case("tables_step_b64", "tables", batch=64, t_max=8192, prefix_min=128, prefix_max=8000),
        # A scheduler's busy tick: of 512 requests some end and give their pages back, some drop rejected drafts, some
        # begin with prompts of up to 4096 tokens, the rest go on by a token.
        _case("tables_mixed_b512", "tables", batch=512, t_max=8192, prefix_min=64, prefix_max=8000, new_min=16, new_max=4096,
              plan="mixed"),
        # The drafted trees of 32 requests, 16 nodes each: few rows, scattered over pages, positions by depth.
        _case("append_trees_b32", "append", batch=32, t_max=1024, new_min=16, new_max=16, prefix_min=100, prefix_max=1000),
        # The rows of 12 prompts packed behind each other, 17 K in all.
        _case("append_prompts_b12", "append", batch=12, t_max=4096, new_min=256, new_max=4096),
        # Four short prompts at the 350M head shapes: the smallest prompt call.
        _case("prompt_short_b4", "prompt", batch=4, t_max=256, groups=4, heads=16, d_v=64, page_rows=32, new_min=17, new_max=200),
        # A batch of new prompts of 700 to 4000 tokens, 15 K in all.
        _case("prompt_packed_b8", "prompt", batch=8, t_max=4096, new_min=700, new_max=4000),
        # Chunks of two long prompts behind 12 K and 30 K cached rows (contiguous caches, the wider positional slice).
        _case("prompt_chunk_b2_t32k", "prompt", batch=2, t_max=32768, d_r=32, page_rows=0, new_min=300, new_max=600,
              prefix_min=8000, prefix_max=32000),
        # A prompt's few new tokens and single decode steps in one packed call, eight heads a group.
        _case("prompt_tail_b24", "prompt", batch=24, t_max=16384, groups=2, heads=16, page_rows=256, new_min=1, new_max=40,
              prefix_min=200, prefix_max=16000),
        # One request's tree of eight drafts at the 350M head shapes: the smallest tree.
        _case("tree_b1_n8", "tree", batch=1, t_max=512, groups=4, heads=16, d_v=64, page_rows=0, new_min=8, new_max=8,
              prefix_min=400, prefix_max=400),
        # A serving batch that verifies 16 drafts each behind 8 K rows: bound by the cache's bytes.
        _case("tree_b32_n16_t8k", "tree", batch=32, t_max=8192, new_min=16, new_max=16, prefix_min=8000, prefix_max=8176),
        # Large trees of a few requests with 2 K to 32 K rows.
        _case("tree_b8_n64_t32k", "tree", batch=8, t_max=32768, new_min=48, new_max=64, prefix_min=2000, prefix_max=32000),
        # What is left of 32 trees of 64 drafts once their paths are accepted.
        _case("commit_b32_n64", "commit", batch=32, t_max=1024, new_min=64, new_max=64, prefix_min=60, prefix_max=900),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    kind = rng.choice(["tables", "tables", "append", "append", "prompt", "prompt", "prompt", "prompt", "tree", "tree", "tree",
                       "tree", "commit"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    groups = rng.choice([1, 2, 4, 8])
    hpg = rng.choice([1, 2, 4, 4, 8])
    d_v = rng.choice([64, 128])
    R = rng.choice([0, 32, 64, 96, 256])
    s = dict(groups=groups, heads=groups * hpg, d_v=d_v, d_c=rng.choice([d_v, d_v, 64, 128]), d_r=rng.choice([0, 8, 16, 16, 24, 32, 64]))

    def capacity(rows, page):
        step = page if page else 32
        return max(step, (rows + step - 1) // step * step)

    if kind == "tables":
        R = R or 128
        batch, most = _log_int(rng, 1, 1024), _log_int(rng, 64, 16384)
        plan = rng.choice(["step", "mixed", "mixed"])
        hi = rng.randint(1, 512) if plan == "mixed" else rng.choice([1, 1, rng.randint(2, 64)])
        return _case(None, kind, batch=batch, t_max=capacity(most + hi, R), page_rows=R, new_min=1, new_max=hi, prefix_min=1,
                     prefix_max=most, plan=plan, spare=rng.choice([1.0, 1.0, rng.uniform(0.0, 0.9)]), **s)
    if kind in ("append", "commit"):
        R = R or (128 if kind == "append" else 0)
        batch = _log_int(rng, 1, 64)
        hi = rng.randint(1, 64) if kind == "commit" else _log_int(rng, 1, max(1, 16384 // batch))
        pre = _log_int(rng, 1, 1024)
        return _case(None, kind, dtype, batch=batch, t_max=capacity(pre + hi, R), page_rows=R, new_min=rng.randint(0, hi), new_max=hi,
                     prefix_min=0, prefix_max=pre, **s)
    if kind == "tree":
        batch, hi = _log_int(rng, 1, 32), rng.choice([rng.randint(1, 64), rng.randint(1, 24), rng.randint(1, 256)])
        pairs = (1 << 28) if dtype == "bf16" else (1 << 26)      # (query, head, cached row), padded
        cells = (1 << 27) if dtype == "bf16" else (1 << 25)      # cached values
    else:
        batch = _log_int(rng, 1, 32)
        hi = rng.choice([_log_int(rng, 1, 32768 // batch), _log_int(rng, 1, 64)])
        pairs = (1 << 31) if dtype == "bf16" else (1 << 28)
        cells = (1 << 27) if dtype == "bf16" else (1 << 26)
    room = min(pairs // (batch * hi * groups * hpg), cells // (batch * groups * d_v), 65536)
    hi = max(1, min(hi, room))
    pre = rng.choice([0, _log_int(rng, 1, max(1, room - hi)), _log_int(rng, 1, max(1, room - hi))])
    if kind == "tree":
        pre = max(pre, 1)
    return _case(None, kind, dtype, batch=batch, t_max=capacity(pre + hi, R), page_rows=R, new_min=rng.randint(0, hi) if batch > 1 else hi,
                 new_max=hi, prefix_min=rng.randint(0, pre), prefix_max=pre, **s)


# ----------------------------------------------------------------- inputs
def _spread(lo, hi, n):
    """n quantiles of the log-uniform distribution over lo .. hi (lo 0: from 1 on, the first of them 0)."""
    a, b = math.log(max(1, lo)), math.log(max(1, hi))
    out = [round(math.exp(a + (i + 0.5) / n * (b - a))) for i in range(n)]
    if lo == 0:
        out[0] = 0 if n > 1 or hi == 0 else out[0]
    return [0 if hi == 0 else x for x in out]


def _counts(c):
    """[(cached rows before, rows that come or go)] of the case's sequences."""
    B, T = c["batch"], c["t_max"]
    pre = _spread(c["prefix_min"], c["prefix_max"], B)
    new = _spread(c["new_min"], c["new_max"], B)
    step = next(k for k in range(B // 2 + 1, 2 * B + 2) if math.gcd(k, B) == 1)      # no short one only beside a short one
    pairs = [(pre[i], new[i * step % B]) for i in range(B)]
    if c["kind"] == "tables" and c["plan"] == "mixed":
        kinds = ["go", "end", "go", "begin", "drop", "go", "go", "go"]
        out = []
        for i, (p, n) in enumerate(pairs):
            k = kinds[i * 5 % 8]
            out.append((p, -p) if k == "end" else (0, n) if k == "begin" else (p, -min(p, 1 + n % 40)) if k == "drop" else (p, 1))
        pairs = out
    return [(min(p, T - max(n, 0)), n) for p, n in pairs]


def _n_rows(c):
    return sum(max(n, 0) for _, n in _counts(c))


def _tile(x):
    """Row-major [..., T, D] in the 16-row tiled layout (same shape)."""
    *lead, T, D = x.shape
    P = 16 // x.element_size()
    if D == 0:
        return x
    return x.reshape(*lead, T // 16, 16, D // P, P).transpose(-3, -2).contiguous().reshape(*lead, T, D)


def _untile(y):
    *lead, T, D = y.shape
    P = 16 // y.element_size()
    if D == 0:
        return y
    return y.reshape(*lead, T // 16, D // P, 16, P).transpose(-3, -2).reshape(*lead, T, D)


def _rotate(x, pos):
    """x [..., D] rotated in interleaved pairs at positions pos [...], angles and products in 64 bits."""
    D = x.shape[-1]
    if D == 0:
        return x.double()
    theta = _BASE ** (-torch.arange(0, D, 2, dtype=torch.float64, device=x.device) / D)
    a = pos.double().unsqueeze(-1) * theta
    x0, x1 = x[..., 0::2].double(), x[..., 1::2].double()
    return torch.stack((x0 * a.cos() - x1 * a.sin(), x0 * a.sin() + x1 * a.cos()), -1).flatten(-2)


def _inputs(c, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    host = torch.Generator()
    host.manual_seed(int(seed))
    dt = _DT[c["dtype"]]
    B, T, H, G, R = c["batch"], c["t_max"], c["heads"], c["groups"], c["page_rows"]
    dv, dc, dr = c["d_v"], c["d_c"], c["d_r"]

    def normal(*shape, std=1.0):
        return torch.randn(shape, generator=g, dtype=torch.float32, device="cuda").mul_(std).to(dt)

    counts = _counts(c)
    counts = [counts[i] for i in torch.randperm(B, generator=host).tolist()]
    pre, new = (torch.tensor(v, dtype=torch.int32) for v in zip(*counts))
    n = int(new.clamp(min=0).sum())
    x = {"n_rows": n, "pre": pre.cuda(), "new": new.cuda()}
    cu = torch.zeros(B + 1, dtype=torch.int32)
    cu[1:] = new.clamp(min=0).cumsum(0)
    x["cu"] = cu.cuda()
    x["lens"] = (pre + new).to(torch.int32).cuda()
    if R:
        # pages in random order: those that the sequences hold, then the free ones
        held = [-(-(p if c["kind"] == "tables" else p + m) // R) for p, m in zip(pre.tolist(), new.tolist())]
        wish = sum(max(0, -(-(p + m) // R) + (-p // R)) for p, m in zip(pre.tolist(), new.tolist()))
        pages = sum(held) + max(1, round(c["spare"] * wish) if c["kind"] == "tables" else 3)
        order = torch.randperm(pages, generator=host).to(torch.int32)
        table = torch.full((B, T // R), -1, dtype=torch.int32)
        at = torch.arange(T // R).unsqueeze(0) < torch.tensor(held).unsqueeze(1)
        table[at] = order[:sum(held)]
        x["table"], x["pages"] = table.cuda(), pages
        free = torch.full((pages,), -1, dtype=torch.int32)
        free[:pages - sum(held)] = order[sum(held):]
        x["free"], x["n_free"] = free.cuda(), torch.tensor([pages - sum(held)], dtype=torch.int32).cuda()
    if c["kind"] == "tables":
        return x
    rows = (x["pages"], G, R) if R else (B, G, T)
    x["v_rows"], x["kr_rows"] = normal(*rows, dv), normal(rows[0], rows[2], dr)
    seq = torch.arange(B).repeat_interleave(new.long())
    node = torch.arange(n) - cu.long()[seq]
    if c["kind"] in ("tree", "commit", "append"):
        # node i hangs on one of the few nodes before it, or on the prefix
        back = 1 + (torch.rand(n, generator=host) ** 2 * 6).long()
        parent = torch.where(torch.rand(n, generator=host) < 0.1, torch.full_like(node, -1), node - back).clamp(min=-1)
        x["parent"] = parent.to(torch.int32).cuda()
    if c["kind"] == "append":
        at = pre[seq].long() + node
        x["slot"] = (x["table"].cpu()[seq, at // R].long() * R + at % R).to(torch.int32).cuda()
        x["pos"] = (pre[seq].long() + node // 3).to(torch.int32).cuda()
        x["v_new"], x["kr_new"] = normal(n, G, dv), normal(n, dr)
    if c["kind"] == "commit":
        leaf = (torch.rand(B, generator=host) * (new + 1)).long() - 1
        x["leaf"] = torch.minimum(leaf, new.long() - 1).to(torch.int32).cuda()
    if c["kind"] in ("prompt", "tree"):
        x["m"] = normal(H, dv, dc, std=1.0 / math.sqrt(dv))
        x["q"] = normal(n, H, dc + dr)
    return x


def prepare(case, seed):
    c, x = case, _inputs(case, seed)
    s = {"case": c, **{k: v for k, v in x.items() if k not in ("v_rows", "kr_rows")}}
    if "v_rows" in x:
        s["v"], s["kr"] = _tile(x["v_rows"]), _tile(x["kr_rows"])
    counts = _counts(c)
    s["most_new"] = max(max(n, 0) for _, n in counts)
    s["most_rows"] = max(p + max(n, 0) for p, n in counts)
    if own:
        s.update(_handle(s))
    return s


# ------------------------------------------------------------- plain forms
def _plain_tables(s):
    c = s["case"]
    B, T, R, pages, n_rows = c["batch"], c["t_max"], c["page_rows"], s["pages"], s["n_rows"]
    lens = s["pre"].long().clamp(0, T)
    n = torch.minimum(torch.maximum(s["new"].long(), -lens), torch.full_like(lens, T))
    want, have = lens + n, (lens + R - 1) // R
    held = (want + R - 1) // R
    fits = want <= T
    zero = torch.zeros_like(n)
    need = torch.where(fits & (n > 0), held - have, zero)
    back = torch.where(n < 0, have - held, zero)
    n_free = s["n_free"].long().clamp(0, pages)
    top = (n_free + back.sum()).clamp(max=pages)
    cum = need.cumsum(0)
    ok = fits & ((need == 0) | (cum <= top))
    got = torch.where(ok, need, zero)
    page = torch.arange(T // R, device="cuda")
    # pages that come back, onto the stack in order of sequence and page
    goes = (page >= held.unsqueeze(1)) & (page < have.unsqueeze(1)) & (n < 0).unsqueeze(1)
    to = n_free + (back.cumsum(0) - back).unsqueeze(1) + page - held.unsqueeze(1)
    goes &= to < pages
    s["free"][to[goes]] = s["table"][goes]
    # pages from its top
    comes = (page >= have.unsqueeze(1)) & (page < (have + got).unsqueeze(1))
    of = top - 1 - ((cum - need).unsqueeze(1) + page - have.unsqueeze(1))
    s["table"][comes] = s["free"][of[comes]]
    new_lens = torch.where((n > 0) & ~ok, lens, want)
    cu = torch.zeros(B + 1, dtype=torch.long, device="cuda")
    cu[1:] = n.clamp(min=0).cumsum(0)
    cu = cu.clamp(max=n_rows)
    r = torch.arange(n_rows, device="cuda")
    seq = torch.searchsorted(cu[1:].contiguous(), r, right=True)
    live = seq < B
    seq = seq.clamp(max=B - 1)
    row = lens[seq] + r - cu[seq]
    live &= ok[seq]
    row = torch.where(live, row, torch.full_like(row, -1))
    owner = torch.where(r < cu[B], seq, torch.full_like(seq, -1))
    of = s["table"].long()[seq, row.clamp(min=0) // R]
    live &= (of >= 0) & (of < pages)
    slot = torch.where(live, of * R + row % R, torch.full_like(row, -1))
    out = {"table": s["table"], "free": s["free"], "n_free": top - got.sum(), "lens": new_lens, "cu": cu, "seq": owner, "row": row,
           "slot": slot}
    return {k: v.to(torch.int32) for k, v in out.items()}


def _plain_append(s):
    c = s["case"]
    R, G, dv, dr, n = c["page_rows"], c["groups"], c["d_v"], c["d_r"], s["n_rows"]
    P = 16 // s["v"].element_size()
    slot = s["slot"].long()
    page, t = slot // R, slot % R
    s["v"].view(-1, G, R // 16, dv // P, 16, P)[page, :, t // 16, :, t % 16] = s["v_new"].view(n, G, dv // P, P)
    if dr:
        k = _rotate(s["kr_new"], s["pos"]).to(s["kr"].dtype)
        s["kr"].view(-1, R // 16, dr // P, 16, P)[page, t // 16, :, t % 16] = k.view(n, dr // P, P)
    return {"v": s["v"], "kr": s["kr"]}


def _above(s):
    """[B, N, N]: whether node j is node i or one of its ancestors."""
    B, N = s["case"]["batch"], s["most_new"]
    i = torch.arange(N, device="cuda")
    at = (s["cu"][:-1].long().unsqueeze(1) + i).clamp(max=max(0, s["n_rows"] - 1))
    parent = torch.where(i < s["new"].unsqueeze(1), s["parent"].long()[at], torch.full_like(at, -1))
    up = (parent.unsqueeze(-1) == i) | (i.unsqueeze(-1) == i)
    for _ in range(max(1, (N - 1).bit_length())):      # paths of up to 1, 2, 4, .. edges
        up = torch.matmul(up.float(), up.float()) > 0
    return up


def _cached(s, pool, rows):
    """The first `rows` cached rows of every sequence, fp32: [B, G, rows, D] of a value cache, [B, rows, D] of positional keys."""
    R = s["case"]["page_rows"]
    x = _untile(pool)
    if not R:
        return x[..., :rows, :].float()
    x = x[s["table"][:, :-(-rows // R)].long().clamp(min=0)]
    x = x.transpose(1, 2) if x.dim() == 5 else x
    return x.flatten(-3, -2)[..., :rows, :].float()


def _plain_attend(s):
    c = s["case"]
    B, H, G, dv, dc, dr = (c[k] for k in ("batch", "heads", "groups", "d_v", "d_c", "d_r"))
    hpg, N, T, n = H // G, s["most_new"], s["most_rows"], s["n_rows"]
    v = _cached(s, s["v"], T)
    i, t = torch.arange(N, device="cuda"), torch.arange(T, device="cuda")
    start = (s["lens"] - s["new"]).long()
    is_row = i < s["new"].unsqueeze(1)
    at = (s["cu"][:-1].long().unsqueeze(1) + i).clamp(max=max(0, n - 1))
    q = s["q"][at].float()                             # padded: [B, N, H, dc + dr]
    if c["kind"] == "tree":
        up = _above(s)
        node = (t - start.unsqueeze(1)).clamp(0, N - 1)                      # [B, T]
        sees = up.gather(2, node.unsqueeze(1).expand(B, N, T)) & (t < s["lens"].unsqueeze(1)).unsqueeze(1)
        sees = sees | (t < start.unsqueeze(1)).unsqueeze(1)
        pos = start.unsqueeze(1) + up.sum(-1) - 1
    else:
        pos = start.unsqueeze(1) + i
        sees = t <= pos.unsqueeze(-1)
    qa = torch.bmm(q[..., :dc].permute(2, 0, 1, 3).reshape(H, B * N, dc), s["m"].float().transpose(1, 2).contiguous())
    qa = qa.reshape(G, hpg, B, N, dv).permute(2, 0, 3, 1, 4).reshape(B, G, N * hpg, dv)
    x = torch.matmul(qa, v.transpose(-1, -2).contiguous()).view(B, G, N, hpg, T)
    if dr:
        qr = _rotate(q[..., dc:], pos.unsqueeze(-1)).float()
        qr = qr.view(B, N, G, hpg, dr).transpose(1, 2).reshape(B, G * N * hpg, dr)
        x += torch.matmul(qr, _cached(s, s["kr"], T).transpose(-1, -2).contiguous()).view(B, G, N, hpg, T)
    x *= 1.0 / math.sqrt(dc + dr)
    x.masked_fill_(~sees[:, None, :, None, :], -math.inf)
    top = x.amax(-1, keepdim=True)
    top = torch.where(torch.isneginf(top), torch.zeros_like(top), top)
    x = torch.exp_(x.sub_(top))
    z = x.sum(-1, keepdim=True)
    o = torch.matmul(x.view(B, G, N * hpg, T), v).view(B, G, N, hpg, dv) / torch.where(z == 0, torch.ones_like(z), z)
    lse = (top + torch.log(z)).squeeze(-1)
    o = o.transpose(1, 2).reshape(B, N, H, dv)[is_row]
    return {"o": o.to(_DT[c["dtype"]]), "lse": lse.transpose(1, 2).reshape(B, N, H)[is_row]}


def _plain_commit(s):
    c = s["case"]
    B, R, G, dv, dr, N, n = c["batch"], c["page_rows"], c["groups"], c["d_v"], c["d_r"], s["most_new"], s["n_rows"]
    leaf = s["leaf"].long()
    on = _above(s)[torch.arange(B, device="cuda"), leaf.clamp(min=0)] & (leaf >= 0).unsqueeze(1)
    k = on.cumsum(1) - 1
    start = (s["lens"] - s["new"]).long()
    b, i = on.nonzero(as_tuple=True)
    k = k[b, i]
    src, dst = start[b] + i, start[b] + k

    def place(t):                                      # the page or sequence of row t, and the row inside
        return (s["table"].long()[b, t // R], t % R) if R else (b, t)

    P = 16 // s["v"].element_size()
    rows = R if R else c["t_max"]
    v = s["v"].view(-1, G, rows // 16, dv // P, 16, P)
    (p0, t0), (p1, t1) = place(src), place(dst)
    v[p1, :, t1 // 16, :, t1 % 16] = v[p0, :, t0 // 16, :, t0 % 16]
    if dr:
        kr = s["kr"].view(-1, rows // 16, dr // P, 16, P)
        kr[p1, t1 // 16, :, t1 % 16] = kr[p0, t0 // 16, :, t0 % 16]
    accepted = torch.full((n,), -1, dtype=torch.int32, device="cuda")
    accepted[s["cu"].long()[b] + k] = i.to(torch.int32)
    return {"v": s["v"], "kr": s["kr"], "lens": (start + on.sum(1)).to(torch.int32), "accepted": accepted}


# ------------------------------------------------------ the library's calls
def _handle(s):
    """What a program keeps beside its caches: dims, paging, the split plan, workspaces, outputs and the marshalled calls."""
    from paper_2609_13285_amd import gva
    c = s["case"]
    B, T, H, G, R, dv, dr, n = (*(c[k] for k in ("batch", "t_max", "heads", "groups", "page_rows", "d_v", "d_r")), s["n_rows"])
    d = gva.make_dims(B, H, G, dv, c["d_c"], dr, T, _DT[c["dtype"]])
    pg = gva.GvaPaging(R, T // R, s["pages"]) if R else None
    kr = s.get("kr") if dr else None
    table = s["table"] if R else None

    def ints(*shape):
        return torch.empty(*shape, dtype=torch.int32, device="cuda")

    if c["kind"] == "tables":
        out = {"table": s["table"], "free": s["free"], "n_free": ints(1), "lens": ints(B), "cu": ints(B + 1), "seq": ints(n),
               "row": ints(n), "slot": ints(n)}
        call = gva.prepare(gva.gva_page_tables, d, pg, s["pre"], s["new"], s["table"], s["free"], s["n_free"], out["lens"],
                           out["n_free"], out["cu"], out["seq"], out["row"], out["slot"])
        return {"call": call, "out": out}
    if c["kind"] == "append":
        call = gva.prepare(gva.gva_append_slots, d, pg, s["v"], kr, s["v_new"], s["kr_new"] if dr else None, s["slot"], s["pos"])
        return {"call": call, "out": {"v": s["v"], "kr": s["kr"]}}
    if c["kind"] == "commit":
        lens, accepted = ints(B), ints(n)
        call = gva.prepare(gva.gva_tree_commit, d, s["v"], kr, s["lens"], s["cu"], s["parent"], s["leaf"], lens, accepted,
                           paging=pg, block_table=table)
        return {"call": call, "out": {"v": s["v"], "kr": s["kr"], "lens": lens, "accepted": accepted}}
    S, rows = gva.packed_plan_for(d, s["lens"], s["new"], n)
    ws = gva.packed_workspace_for(d, n, S)
    o, lse = torch.empty(n, H, dv, dtype=_DT[c["dtype"]], device="cuda"), torch.empty(n, H, device="cuda")
    more = dict(lse=lse, paging=pg, block_table=table, num_splits=S, split_rows=rows, workspace=ws)
    if c["kind"] == "tree":
        call = gva.prepare(gva.gva_tree_attention, d, s["q"], s["m"], s["v"], kr, s["lens"], s["cu"], s["parent"], o, **more)
    else:
        call = gva.prepare(gva.gva_packed_prefill, d, s["q"], s["m"], s["v"], kr, s["lens"], s["cu"], o, **more)
    return {"call": call, "out": {"o": o, "lse": lse}, "hold": ws}


def run(state):
    s = state
    if own:
        s["call"]()
        return s["out"]
    kind = s["case"]["kind"]
    if kind == "tables":
        return _plain_tables(s)
    if kind == "append":
        return _plain_append(s)
    if kind == "commit":
        return _plain_commit(s)
    return _plain_attend(s)


# -------------------------------------------------------------------- work
def work(case):
    c = case
    B, T, H, G, R, dv, dc, dr = (c[k] for k in ("batch", "t_max", "heads", "groups", "page_rows", "d_v", "d_c", "d_r"))
    e = 4 if c["dtype"] == "f32" else 2
    counts, n = _counts(c), _n_rows(c)
    row = (G * dv + dr) * e
    if c["kind"] == "tables":
        moved = sum(abs(-(-(p + m) // R) + (-p // R)) for p, m in counts)       # pages
        return {"bytes": 16 * B + 8 * moved + 12 * n, "flops": 0}
    if c["kind"] == "append":
        return {"bytes": n * (2 * row + 8), "flops": 0}
    if c["kind"] == "commit":
        # a path of about a third of its tree's nodes at the most
        return {"bytes": sum(2 * row * m // 4 for _, m in counts) + 8 * n + 8 * B, "flops": 0}
    cached = sum(p + m for p, m in counts if m > 0)
    pairs = H * sum(m * p + (m * (m + 1) // 2 if c["kind"] == "prompt" else m) for p, m in counts)
    return {"bytes": cached * row + H * dv * dc * e + n * H * ((dc + dr) * e + dv * e + 4),
            "flops": 2 * (2 * dv + dr) * pairs + 2 * n * H * dv * dc}


# ------------------------------------------------- the definition in 64 bits
def _exact_place(c, x, b, t):
    return (int(x["table"][b, t // c["page_rows"]]), t % c["page_rows"]) if c["page_rows"] else (b, t)


def _exact_tiled(y):
    """fp64 rows in the storage order of their type."""
    rows, e = y
    *lead, T, D = rows.shape
    return rows if D == 0 else rows.reshape(*lead, T // 16, 16, D * e // 16, 16 // e).transpose(-3, -2).reshape(*lead, T, D)


def exact(case, seed):
    c, x = case, _inputs(case, seed)
    B, H, G, R, dv, dc, dr = (c[k] for k in ("batch", "heads", "groups", "page_rows", "d_v", "d_c", "d_r"))
    e = 4 if c["dtype"] == "f32" else 2
    if c["kind"] == "tables":
        return None
    if c["kind"] == "append":
        v, kr = x["v_rows"].double(), x["kr_rows"].double()
        page, t = x["slot"].long() // R, x["slot"].long() % R
        v[page, :, t], kr[page, t] = x["v_new"].double(), _rotate(x["kr_new"], x["pos"])
        return {"v": _exact_tiled((v, e)), "kr": _exact_tiled((kr, e)) if dr else None}
    lens, new, cu = x["lens"].tolist(), x["new"].tolist(), x["cu"].tolist()
    parent = x["parent"].tolist() if "parent" in x else None
    if c["kind"] == "commit":
        v, kr = x["v_rows"].double(), x["kr_rows"].double()
        for b in range(B):
            path, i = [], int(x["leaf"][b])
            while i >= 0:
                path.append(i)
                i = parent[cu[b] + i]
            for k, i in enumerate(reversed(path)):
                (p0, t0), (p1, t1) = (_exact_place(c, x, b, lens[b] - new[b] + j) for j in (i, k))
                v[p1, :, t1], kr[p1, t1] = v[p0, :, t0].clone(), kr[p0, t0].clone()
        return {"v": _exact_tiled((v, e)), "kr": _exact_tiled((kr, e)) if dr else None, "lens": None, "accepted": None}
    n = x["n_rows"]
    o = torch.zeros(n, H, dv, dtype=torch.float64, device="cuda")
    lse = torch.zeros(n, H, dtype=torch.float64, device="cuda")
    for b, (L, m) in enumerate(zip(lens, new)):
        if m == 0:
            continue
        P = L - m
        depth, hidden = list(range(m)), torch.ones(m, L, dtype=torch.bool)
        if c["kind"] == "tree":
            hidden[:, :P] = False
            for i in range(m):
                j, k = i, -1
                while j >= 0:
                    hidden[i, P + j] = False
                    j, k = parent[cu[b] + j], k + 1
                depth[i] = k
        else:
            hidden = torch.arange(L).unsqueeze(0) > torch.arange(P, L).unsqueeze(1)
        hidden = hidden.cuda()
        at = P + torch.tensor(depth, device="cuda")
        if R:
            table = x["table"][b, :-(-L // R)].long()
            vb, kb = x["v_rows"][table].transpose(0, 1).flatten(1, 2)[:, :L], x["kr_rows"][table].flatten(0, 1)[:L]
        else:
            vb, kb = x["v_rows"][b, :, :L], x["kr_rows"][b, :L]
        for h in range(H):
            vh = vb[h // (H // G)].double()
            keys = torch.cat((vh @ x["m"][h].double(), kb.double()), -1)
            q = x["q"][cu[b]:cu[b] + m, h].double()
            q = torch.cat((q[:, :dc], _rotate(q[:, dc:], at)), -1)
            sc = ((q @ keys.t().contiguous()) / math.sqrt(dc + dr)).masked_fill_(hidden, -math.inf)
            lse[cu[b]:cu[b] + m, h] = torch.logsumexp(sc, -1)
            o[cu[b]:cu[b] + m, h] = torch.softmax(sc, -1) @ vh
    return {"o": o, "lse": lse}
