"""The 4-bit step, the accumulated weights and the eviction at the sizes that
serving runs them at (many tiles a wave, absorption outside the launch, several
tiles a workgroup, selection over blocks), and what their plans and sizes refuse."""

import ctypes
import math

import pytest
import torch

import q4_ref as ref
from gpu_helpers import note
from paper_2609_13285_amd import gva
from test_q4_evict import A, check_step, dims, evict_case, problem, step, step_status, weights_status

gpu = pytest.mark.gpu


# ---------------------------------------------------------------- refusals
@pytest.mark.parametrize("kw", [dict(n_heads=24), dict(n_heads=128), dict(d_c=48), dict(d_c=544), dict(d_c=0), dict(dtype="f32")])
def test_plan_and_size_refuse_what_the_step_refuses(kw):
    d = dims(**{**dict(batch=1, n_heads=32, n_groups=8, t_max=131072), **kw})
    assert step_status(d) == gva.GVA_ERR_UNSUPPORTED
    assert gva.gva_q4_pick_splits(d, None, 256) == (1, 0)
    n = ctypes.c_size_t(7)
    assert gva.lib().gva_q4_decode_workspace_size(ctypes.byref(d), 4, 0, ctypes.byref(n)) == gva.GVA_ERR_UNSUPPORTED
    assert n.value == 7


def test_every_call_refuses_null_dims():
    L, d = gva.lib(), ctypes.POINTER(gva.GvaDims)()
    n = ctypes.byref(ctypes.c_size_t())
    big = 1 << 40
    for status in (L.gva_q4_append_kv(d, A, A, A, A, A, A, A, None, 4, None, None),
                   L.gva_append_rows(d, A, A, A, A, A, A, None, 4, None, None),
                   L.gva_q4_unpack_kv(d, A, A, A, A, None),
                   L.gva_q4_decode_workspace_size(d, 1, 0, n),
                   L.gva_q4_decode_step(d, A, A, A, A, A, A, None, 2, 0, A, big, A, A, None),
                   L.gva_weights_workspace_size(d, 1, n),
                   L.gva_accumulate_weights(d, 1, A, A, A, None, A, A, None, A, 1.0, A, A, A, big, None),
                   L.gva_evict_workspace_size(d, n),
                   L.gva_evict_rows(d, 16, 0, 0, A, None, A, A, None, A, None, A + 256, A + 512, None, A, big, None)):
        assert status == gva.GVA_ERR_INVALID_ARG
    assert L.gva_q4_pick_splits(d, None, 256, None) == 1


def test_more_query_rows_than_the_absorption_takes_are_refused():
    d = dims(batch=1 << 10, t_max=1 << 12)
    assert weights_status(d, N=(1 << 10) + 1) == gva.GVA_ERR_UNSUPPORTED
    assert step_status(dims(batch=(1 << 20) + 1, t_max=32), S=1) == gva.GVA_ERR_UNSUPPORTED


# --------------------------------------------------------------- plans
@pytest.mark.parametrize("kw,lens", [
    (dict(batch=53, n_heads=4, n_groups=1, d_r=16, t_max=2144), [1072 + 1072 * i // 52 for i in range(53)]),
    (dict(batch=28, n_heads=8, n_groups=4, d_v=64, d_r=32, t_max=4352), [round(128 * 34 ** (i / 27)) for i in range(28)]),
    (dict(batch=74, n_heads=8, n_groups=1, d_r=16, t_max=3136), [1568 + 1568 * i // 73 for i in range(74)])])
def test_plans_count_the_absorption_that_they_cause(kw, lens):
    """Streams of a few thousand rows: splits past two workgroups per CU save less
    than the absorption's launch, which they make necessary, takes."""
    d = dims(**kw)
    S, rows = gva.gva_q4_pick_splits(d, torch.tensor(lens))
    assert not absorbs_outside(d, S, rows)


def test_plans_fit_the_registers_of_wide_positional_keys():
    """Two workgroups of four waves on a CU at d_r > 32, not three."""
    d = dims(batch=40, n_heads=32, n_groups=8, d_r=40, t_max=4096)
    lens = [2048 + 2048 * i // 39 for i in range(40)]
    S, rows = gva.gva_q4_pick_splits(d, torch.tensor(lens), 256)
    assert S == 1 or sum(-(-n // rows) if rows else S for n in lens) * 8 <= 2 * 256


# --------------------------------------------------------------- decode
def tiles_of_longest_split(T, S, rows):
    """32-row tiles of a full sequence's splits (include/gva.h's split rule)."""
    n = S if rows == 0 else min(S, max(1, -(-T // rows)))
    return -(-(-(-T // n)) // 32)


def absorbs_outside(d, S, rows):
    """Whether the workspace holds absorbed queries beside the splits' partials."""
    up = lambda n: -(-n // 256) * 256                    # noqa: E731
    BH = d.batch * d.n_heads
    parts = up(BH * S * d.d_v * 4) + up(BH * S * 4) if S > 1 else 0
    return gva.gva_q4_decode_workspace_size(d, S, rows) > parts


@gpu
@pytest.mark.parametrize("hpg", [1, 2, 4, 8])
@pytest.mark.parametrize("d_v,d_r", [(64, 16), (128, 40), (64, 40), (128, 16)])
@pytest.mark.parametrize("S,rows", [(1, 0), (2, 1504)])
def test_step_many_tiles_a_wave(hpg, d_v, d_r, S, rows):
    """Splits of over four tiles for each of eight waves: the weights in two
    parts, the tiles in registers taken round several times."""
    T = 2976
    x = problem(4, T, 2 * hpg, 2, d_v, 64, d_r, [T, 2081, 37, 1291], extra=77, seed=hpg + d_v + d_r)
    note(f"q4 step, long splits hpg={hpg} d={d_v}/{d_r} S={S} rows={rows}")
    assert tiles_of_longest_split(T, S, rows) > 4 * 8
    assert not absorbs_outside(x["d"], S, rows)
    check_step(x, *step(x, S, rows))


@gpu
@pytest.mark.parametrize("hpg,d_v,d_r", [(1, 64, 8), (2, 128, 24), (4, 64, 64), (4, 128, 40), (8, 64, 40), (8, 128, 16)])
@pytest.mark.parametrize("B,S,rows", [(300, 1, 0), (100, 3, 0), (100, 3, 32)])
def test_step_absorption_outside(hpg, d_v, d_r, B, S, rows):
    """More workgroups than two per CU: queries absorbed, and rotated at seen -
    1, by a launch before, with splits and bounded chunks."""
    T = 96
    lens = torch.randint(-2, T + 9, (B,), generator=torch.Generator().manual_seed(B + S + hpg)).tolist()
    lens[:5] = [T, 0, 1, 33, T - 1]
    x = problem(B, T, 2 * hpg, 2, d_v, 64, d_r, lens, extra=1000, seed=hpg * 10 + d_r)
    note(f"q4 step, absorption outside hpg={hpg} d={d_v}/{d_r} B={B} S={S} rows={rows}")
    assert absorbs_outside(x["d"], S, rows)
    check_step(x, *step(x, S, rows))


@gpu
@pytest.mark.parametrize("hpg", [4, 8])
def test_step_eight_waves_absorption_outside(hpg):
    """Long chunks of few streams, but more (sequence, split) slots than are
    resident, and wide maps."""
    B, T, S, rows = 65, 8256, 4, 4128
    lens = [T, 8192 - 31] + [1 + 97 * i % 400 for i in range(B - 2)]
    x = problem(B, T, 2 * hpg, 2, 64, 288, 16, lens, extra=5, seed=hpg)
    d = x["d"]
    note(f"q4 step, eight waves, absorption outside hpg={hpg}")
    assert absorbs_outside(d, S, rows) and B * 2 <= 256 <= gva.device_cu_count()
    check_step(x, *step(x, S, rows))


@gpu
@pytest.mark.parametrize("hpg", [1, 2, 4])
@pytest.mark.parametrize("B,d_v", [(3, 64), (64, 128), (600, 64)])
def test_step_weight_parts(hpg, B, d_v):
    """Two rows with scores 0 and x in (-2, 0) (log2), x = q~ v with one column:
    o = v e / (1 + e) there, e = 2^x.  In units of 2^-24: x is off by 4.2 |x| (the
    scale, its product, two sums of the parts, the parts), so e by 5.8 of itself, by
    2 more for the exponential and by 1/4 for its three parts (2^-26); the products'
    and waves' sums, the division and the stored result are 7.  Two parts alone
    would be off by up to 128."""
    G, H = 2, 2 * hpg
    d = dims(batch=B, n_heads=H, n_groups=G, d_v=d_v, d_c=32, d_r=0, t_max=32)
    q, m = torch.zeros(B, H, 32), torch.zeros(H, d_v, 32)
    q[..., 5] = -0.05 - 1.2 * torch.rand(B, H, generator=torch.Generator().manual_seed(B + hpg))
    m[:, 7, 5] = 1.0
    q, m = q.to(torch.bfloat16), m.to(torch.bfloat16)
    v = torch.zeros(B, 2, G, d_v, dtype=torch.bfloat16)
    v[:, 1, :, 7] = 6.0
    note(f"q4 step, weight parts hpg={hpg} B={B} d_v={d_v}")
    c, s = gva.q4_cache(d)
    seq, row = torch.arange(B, dtype=torch.int32).repeat_interleave(2).cuda(), torch.arange(2, dtype=torch.int32).repeat(B).cuda()
    gva.gva_q4_append_kv(d, c, s, None, v.view(2 * B, G, d_v).cuda(), None, seq, row)
    o, lse = gva.q4_decode(d, q.cuda(), m.cuda(), c, s, None, torch.full((B,), 2, dtype=torch.int32, device="cuda"))
    e = torch.exp(6.0 * q[..., 5].double() / math.sqrt(32))
    want = 6.0 * e / (1 + e)
    assert float((o[..., 7].cpu().double() / want - 1).abs().max()) <= 16 * 2.0 ** -24
    # the logarithm of a sum in (1, 2), in base 2, and the factor to the natural one
    assert float((lse.cpu().double() - torch.log1p(e)).abs().max()) <= 16 * 2.0 ** -24


@gpu
@pytest.mark.parametrize("hpg,bits", [(1, 21), (2, 21), (4, 21), (8, 16)])
@pytest.mark.parametrize("d_r,at", [(8, 6), (40, 38), (64, 32)])
@pytest.mark.parametrize("B", [3, 600])
def test_step_positional_query_parts(hpg, bits, d_r, at, B):
    """One row at position 0, one column of the positional key: lse is the score.
    In three parts (up to four heads a group) the query is off by 2^-26 of itself,
    and the scale, its product, the parts' sums and the factor at the end by 2^-24
    each, under 2^-21; in two parts by 2^-17 more."""
    G, H, d_v = 2, 2 * hpg, 64
    d = dims(batch=B, n_heads=H, n_groups=G, d_v=d_v, d_c=32, d_r=d_r, t_max=32)
    q, m = torch.zeros(B, H, 32 + d_r), torch.zeros(H, d_v, 32)
    q[..., 32 + at] = torch.randn(B, H, generator=torch.Generator().manual_seed(hpg + d_r))
    q = q.to(torch.bfloat16)
    v, k = torch.zeros(B, G, d_v, dtype=torch.bfloat16), torch.zeros(B, d_r, dtype=torch.bfloat16)
    k[:, at] = 24.0
    note(f"q4 step, positional query parts hpg={hpg} d_r={d_r} B={B}")
    c, s = gva.q4_cache(d)
    kr = torch.zeros(B, 32, d_r, dtype=torch.bfloat16, device="cuda")
    seq = torch.arange(B, dtype=torch.int32).cuda()
    gva.gva_q4_append_kv(d, c, s, kr, v.cuda(), k.cuda(), seq, torch.zeros_like(seq))
    o, lse = gva.q4_decode(d, q.cuda(), m.to(torch.bfloat16).cuda(), c, s, kr, torch.ones_like(seq))
    want = 24.0 * q[..., 32 + at].double() / math.sqrt(32 + d_r)
    assert bool(((lse.cpu().double() - want).abs() <= 2.0 ** -bits * want.abs()).all())


# -------------------------------------------------------------- weights
def rows_per_workgroup(d, N):
    """gva_accumulate_weights' rule: whole tiles, few enough for two workgroups per CU."""
    joined = d.dtype == gva.GVA_DTYPE_BF16 and not (N == 1 and d.n_heads // d.n_groups in (1, 2, 4, 8))
    streams, chunk = d.batch * (d.n_groups if joined else 1), 512
    while chunk > 32 and streams * -(-d.t_max // chunk) < 2 * gva.device_cu_count():
        chunk //= 2
    return chunk


def large_weights(cache, B, T, H, G, d_v, d_r, N, lens, least, seed, d_c=64):
    """gva_accumulate_weights against 64 bits on the GPU.  Values are 4-bit
    numbers (every block holds its largest, 6 * 2^-2), so that every cache holds
    them exactly.  Tolerances: a score of two bf16 parts is off by 2^-17 of its sum
    of magnitudes (fp32: 2^-24), its fp32 sums over at most 192 terms by 200 *
    2^-24, the absorbed query by (d_c + 2) 2^-24 of its terms' magnitudes, the
    log-sum-exp's difference by a few 2^-24 of both; the sum over queries and heads by
    2^-23 a term."""
    d = dims(batch=B, n_heads=H, n_groups=G, d_v=d_v, d_c=d_c, d_r=d_r, t_max=T, dtype="f32" if cache == "f32" else "bf16")
    assert rows_per_workgroup(d, N) >= least
    dt, hpg, W = d.torch_dtype, H // G, d_c + d_r
    g = torch.Generator(device="cuda").manual_seed(seed)
    rand = lambda *shape: torch.randn(*shape, generator=g, device="cuda")     # noqa: E731
    level = torch.cat((ref.LEVELS, -ref.LEVELS)).float().cuda() / 4
    rows = level[torch.randint(0, 16, (B, G, T, d_v), generator=g, device="cuda")]
    rows[..., ::32] = 1.5
    kr, q, m = rand(B, T, d_r).to(dt), rand(B, N, H, W).to(dt), (rand(H, d_v, d_c) / math.sqrt(d_c)).to(dt)
    ln = torch.tensor(lens, dtype=torch.int32, device="cuda")
    L = ln.clamp(0, T)
    dead = torch.arange(T, device="cuda") >= L.unsqueeze(1)
    kc = gva.tiled(kr.masked_fill(dead[..., None], math.nan)) if d_r else None
    if cache == "q4":
        vc, sc = gva.q4_cache(d)
        sc.fill_(255)                                    # rows never written read as NaN
        seq, row = (~dead).nonzero(as_tuple=True)
        spare = torch.zeros(B, T, d_r, dtype=dt, device="cuda") if d_r else None
        gva.gva_q4_append_kv(d, vc, sc, spare, rows.transpose(1, 2)[seq, row].to(dt).contiguous(), kr[seq, row].contiguous() if d_r else None,
                             seq.int(), row.int())
    else:
        vc, sc = gva.tiled(rows.to(dt).masked_fill(dead[:, None, :, None], math.nan)), None
    seen = L + 11
    # the definition, and what its terms allow
    x = torch.full((B, N, H, T), -math.inf, dtype=torch.float64, device="cuda")
    size, made = torch.zeros_like(x), torch.zeros_like(x)
    for b in range(B):
        n = int(L[b])
        if n == 0:
            continue
        qd = q[b].double()
        qa = torch.matmul(qd[..., :d_c].transpose(0, 1).contiguous(), m.double().transpose(1, 2).contiguous())      # [H, N, d_v]
        terms = torch.matmul(qd[..., :d_c].abs().transpose(0, 1).contiguous(), m.double().abs().transpose(1, 2).contiguous())
        qr = ref.rotate(qd[..., d_c:].cpu(), (int(seen[b]) - N + torch.arange(N)).clamp(min=0).unsqueeze(1)).cuda().transpose(0, 1).contiguous()
        vb = rows[b, :, :n].double().repeat_interleave(hpg, 0).transpose(1, 2).contiguous()
        kb = kr[b, :n].double().t().contiguous()
        hidden = torch.arange(n, device="cuda") > (n - N + torch.arange(N, device="cuda")).unsqueeze(1)
        s = (torch.matmul(qa, vb) + torch.matmul(qr, kb)) / math.sqrt(W)
        x[b, :, :, :n] = s.masked_fill(hidden, -math.inf).transpose(0, 1)
        size[b, :, :, :n] = ((torch.matmul(qa.abs(), vb.abs()) + torch.matmul(qr.abs(), kb.abs())) / math.sqrt(W)).transpose(0, 1)
        made[b, :, :, :n] = (torch.matmul(terms, vb.abs()) / math.sqrt(W)).transpose(0, 1)
    lse = torch.logsumexp(x, -1).float()
    w = torch.rand(B, T, generator=g, device="cuda").masked_fill(dead, math.nan)
    out = torch.full((B, T), 55.0, device="cuda")
    note(f"weights {cache} B={B} T={T} H={H} G={G} d={d_v}/{d_r} N={N}")
    ws = gva.weights_workspace_for(d, N)
    ws.fill_(0xFF)
    gva.gva_accumulate_weights(d, N, q, m, vc, sc, kc, ln, lse, w, out, workspace=ws, seen=seen, decay=0.75)
    some = torch.isfinite(lse).unsqueeze(-1)
    l64 = torch.where(some, lse.double().unsqueeze(-1), torch.zeros_like(x[..., :1]))
    p = torch.exp(x - l64) * some
    dx = size * ((2.0 ** -24 if cache == "f32" else 2.0 ** -17) + 200 * 2.0 ** -24) + made * (d_c + 2) * 2.0 ** -24 + 4 * 2.0 ** -24 * (1 + l64.abs() + size)
    want = p.sum((1, 2)) + 0.75 * w.double()
    tol = (p * torch.expm1(dx)).sum((1, 2)) + 2.0 ** -23 * (N * H + 4) * want
    err = (out.double() - want).abs()
    assert bool((err <= tol)[~dead].all()), float((err / tol)[~dead].max())
    assert bool((out[dead] == 55.0).all())


def ragged(B, T):
    """Lengths that end inside a tile, on one, in the first and the last chunk; full, none."""
    some = [T, T - 1, 0, 1, T // 2 + 3, 33, 512, 513, T - 31, T - 32, 3 * T // 4 + 17, 479]
    return [some[i % 12] for i in range(B)]


@gpu
@pytest.mark.parametrize("cache", ["q4", "bf16", "f32"])
@pytest.mark.parametrize("G,hpg,d_v,d_r,T,least", [(4, 4, 64, 16, 8160, 256), (8, 1, 64, 40, 4096, 128), (2, 8, 128, 0, 8192, 256),
                                                   (11, 2, 64, 8, 4064, 128)])
def test_weights_of_a_token_many_tiles(cache, G, hpg, d_v, d_r, T, least):
    """Several tiles a wave: the start tile of a stream's own, the ring of
    tiles in registers, groups in rounds."""
    large_weights(cache, 16, T, G * hpg, G, d_v, d_r, 1, ragged(16, T), least, seed=G)


@gpu
@pytest.mark.parametrize("cache", ["q4", "bf16", "f32"])
@pytest.mark.parametrize("G,hpg,d_v,d_r,N", [(4, 4, 64, 16, 3), (4, 4, 64, 40, 12), (4, 4, 128, 0, 40), (8, 3, 64, 24, 1),
                                             (4, 3, 64, 8, 17)])
def test_weights_of_a_window_many_tiles(cache, G, hpg, d_v, d_r, N):
    """One, two and over four column sets (tiles dealt over four, two waves and
    one), each over several tiles."""
    T = 4096 - 16 * (cache != "q4")
    large_weights(cache, 16, T, G * hpg, G, d_v, d_r, N, ragged(16, T), 128, seed=N)


@gpu
@pytest.mark.parametrize("cache", ["q4", "bf16", "f32"])
@pytest.mark.parametrize("G,hpg,d_v,d_c,d_r,N", [(2, 16, 64, 1024, 56, 1), (1, 40, 128, 96, 64, 2), (3, 5, 128, 32, 0, 1),
                                                 (1, 1, 64, 256, 8, 33)])
def test_weights_any_heads_per_group_wide_maps(cache, G, hpg, d_v, d_c, d_r, N):
    T = 224
    large_weights(cache, 5, T, G * hpg, G, d_v, d_r, N, [T, 0, 97, 33, T + 3], 32, seed=hpg, d_c=d_c)


@gpu
@pytest.mark.parametrize("cache,N", [("q4", 1), ("q4", 3), ("bf16", 1), ("bf16", 3), ("f32", 1), ("f32", 3)])
@pytest.mark.parametrize("low,q_at", [(-1e9, 1.0), (float(torch.finfo(torch.bfloat16).min), 0.01),
                                      (float(torch.finfo(torch.bfloat16).min), 6.0)])
def test_weights_where_finite_values_hide_every_row(cache, N, low, q_at):
    """A sequence with nothing but rows hidden by a large finite value: scores and
    log-sum-exp are as large, and their difference is rounding.  Hidden rows draw no
    weight; the other sequence's weights are its own."""
    H, T = 8, 96
    x = problem(2, T, H, 2, 64, 64, 16, [T, 70], N=N, cache=cache, seed=3)
    d = x["d"]
    x["q"][..., -2:] = torch.tensor([q_at, 0.0])         # the slowest pair: hardly turned at these positions
    x["kr"][0, :, 14] = low
    x["kr"] = x["kr"].to(d.torch_dtype).double()
    x["kc"] = gva.tiled(x["kr"].to(d.torch_dtype)).cuda()
    s, _ = ref.scores(x["q"], x["m"], x["v"], x["kr"], x["lens"], x["seen"], 2)
    lse = torch.logsumexp(s, -1).float().cuda()
    note(f"weights, every row hidden by {low}, {cache} N={N}")
    w = torch.zeros(2, T, device="cuda")
    gva.accumulate_weights(d, x["q"].cuda(), x["m"].cuda(), x["vc"], x["kc"], x["lens"].cuda(), lse, w, v4_scale=x["sc"],
                           seen=x["seen"].cuda(), decay=0.0)
    assert bool((w[0] == 0).all())
    p = torch.exp(s[1] - lse[1].cpu().double().unsqueeze(-1)).sum((0, 1))
    assert float((w[1, :70].cpu().double() - p[:70]).abs().max()) <= 1e-3 * N * H


@gpu
@pytest.mark.parametrize("cache,N", [("q4", 1), ("q4", 3), ("bf16", 1), ("bf16", 3), ("f32", 1), ("f32", 3)])
def test_weights_of_a_nan_row_are_nan(cache, N):
    """A NaN in a value row reaches that row's weight, and no other's."""
    H, T = 8, 96
    x = problem(2, T, H, 2, 64, 64, 16, [T, 70], N=N, cache=cache, seed=4)
    d = x["d"]
    s, _ = ref.scores(x["q"], x["m"], x["v"], x["kr"], x["lens"], x["seen"], 2)
    lse = torch.logsumexp(s, -1).float().cuda()
    if cache == "q4":
        code, byte = ref.unpack(x["vc"].cpu(), x["sc"].cpu())
        byte[0, 1, 37, 1] = 255
        x["sc"] = ref.pack(code, byte)[1].cuda()
    else:
        v = gva.untiled(x["vc"].cpu())
        v[0, 1, 37, 40] = math.nan
        x["vc"] = gva.tiled(v).cuda()
    note(f"weights, a NaN row, {cache} N={N}")
    w = torch.zeros(2, T, device="cuda")
    gva.accumulate_weights(d, x["q"].cuda(), x["m"].cuda(), x["vc"], x["kc"], x["lens"].cuda(), lse, w, v4_scale=x["sc"],
                           seen=x["seen"].cuda(), decay=0.0)
    nan = torch.zeros(2, T, dtype=torch.bool)
    nan[0, 37] = True
    assert torch.equal(torch.isnan(w).cpu(), nan)


@gpu
def test_two_streams_at_once():
    """A step, its weights and an eviction on each of two streams, with buffers
    of their own, give what they give one after the other."""
    def work(x, stream):
        d = x["d"]
        with torch.cuda.stream(stream):
            o, lse = gva.q4_decode(d, x["q1"], x["m1"], x["vc"], x["sc"], x["kc"], x["l1"], seen=x["s1"])
            w = gva.accumulate_weights(d, x["q1"], x["m1"], x["vc"], x["kc"], x["l1"], lse, x["w0"].clone(), v4_scale=x["sc"], seen=x["s1"])
            out = gva.evict(d, 5000, x["vc"].clone(), x["kc"].clone(), x["l1"], w, n_first=2, n_recent=40, v4_scale=x["sc"].clone(),
                            seen=x["s1"], row_pos=x["rp"])
        return o, lse, w, *out

    xs = []
    for k in range(2):
        x = problem(3, 8640, 8, 2, 64, 64, 16, [8640, 5001, 7000 + k], extra=3, seed=50 + k)
        x.update(q1=x["q"][:, 0].contiguous().cuda(), m1=x["m"].cuda(), l1=x["lens"].cuda(), s1=x["seen"].cuda(),
                 w0=torch.rand(3, 8640, generator=torch.Generator().manual_seed(k)).cuda(),
                 rp=torch.arange(8640, dtype=torch.int32, device="cuda").expand(3, 8640).contiguous())
        xs.append(x)
    note("two streams at once")
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    want = [work(x, streams[0]) for x in xs]
    torch.cuda.synchronize()
    for _ in range(3):
        got = [work(x, s) for x, s in zip(xs, streams)]
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert all(torch.equal(u.view(torch.uint8), v.view(torch.uint8)) for u, v in zip(a, b))


# ------------------------------------------------------------- eviction
def order_weights(kind, B, T):
    g = torch.Generator().manual_seed(T)
    if kind == "equal":
        return torch.full((B, T), 0.5)
    if kind == "special":
        few = torch.tensor([0.0, -0.0, math.nan, math.inf, -math.inf, -1.0, 1e-40, -1e-40, 3.0, 3.4e38])
        return few[torch.randint(0, 10, (B, T), generator=g)]
    if kind == "close":                                  # neighbouring floats: the border's last digit decides
        return 1.0 + torch.randint(0, 300, (B, T), generator=g) * 2.0 ** -23
    up = torch.arange(T).float().div(3).floor().expand(B, T).contiguous()      # threes alike
    return -up if kind == "decreasing" else up


@gpu
@pytest.mark.parametrize("kind", ["equal", "special", "close", "increasing", "decreasing"])
@pytest.mark.parametrize("T,keep", [(6016, 2500), (8192, 5000), (13024, 6500), (20000, 9001), (8224, 8200)])
def test_evict_orders_over_blocks(kind, T, keep):
    """Ties on the border over several blocks on both sides of the budget (past
    8192 rows) or eight rows a thread, sequences that keep every row beside others."""
    lens = [T, 0, keep - 1, keep, keep + 1, T - 7]
    w = order_weights(kind, len(lens), T)
    note(f"evict order {kind} T={T} keep={keep}")
    evict_case(len(lens), T, 1, 64, 0, "q4", lens, keep, 2, 30, weights=w, seed=1)
    evict_case(len(lens), T, 1, 64, 0, "q4", lens, keep, 0, 0, with_pos=False, weights=w, seed=2, runs=1)


@gpu
@pytest.mark.parametrize("cache,G,d_v,d_r", [("bf16", 2, 64, 24), ("f32", 1, 20, 8), ("q4", 2, 128, 16)])
@pytest.mark.parametrize("T,keep,first,recent", [(12320, 5000, 4, 700), (9280, 1, 0, 0), (16400, 12288, 5000, 4200), (9296, 20000, 0, 0)])
def test_evict_over_blocks(cache, G, d_v, d_r, T, keep, first, recent):
    """The rows themselves, at sizes of the selection over blocks: few weights
    that many rows share, protected ranges longer than a block."""
    T = (T + 31) // 32 * 32
    lens = [T - 5, min(keep, T), T, 17]
    note(f"evict over blocks {cache} T={T} keep={keep}")
    evict_case(len(lens), T, G, d_v, d_r, cache, lens, keep, first, recent, seed=keep, runs=1)
    evict_case(len(lens), T, G, d_v, d_r, cache, lens, keep, first, recent, with_pos=False, seed=keep + 1, runs=1)
