"""Many requests on one cache: page tables, appends at slots, attention of packed
prompts and of drafted trees, the commit of a tree.  Against 64-bit references
on the GPU, and their refusals on the CPU."""

import ctypes
import math
import random

import pytest
import torch

import packed_ref as ref
from gpu_helpers import note
from paper_2609_13285_amd import gva

A = 0x100000     # an aligned address that a refused call never reads
gpu = pytest.mark.gpu
BAD, UNSUP = gva.GVA_ERR_INVALID_ARG, gva.GVA_ERR_UNSUPPORTED


def dims(**kw):
    base = dict(batch=2, n_heads=8, n_groups=2, d_v=128, d_c=128, d_r=16, t_max=128, dtype="bf16")
    base.update(kw)
    return gva.make_dims(**base)


def paging(R=64, pages=2, n=5):
    return gva.GvaPaging(R, pages, n)


# ---------------------------------------------------------------- refusals
def pg_ref(pg):
    return None if pg is None else ctypes.byref(pg)


def tables_status(d, pg=paging(), lens=A, n_new=A + 4096, table=A, free=A, n_free=A + 8192, n=4, new=A + 12288,
                  new_free=A + 16384, cu=A + 20480, seq=A, row=A, slot=A):
    return gva.lib().gva_page_tables(ctypes.byref(d), pg_ref(pg), lens, n_new, table, free, n_free, n, new, new_free, cu, seq,
                                     row, slot, None)


def slots_status(d, pg=paging(), v=A, k=A, vn=A, kn=A, slot=A, pos=A, n=4):
    return gva.lib().gva_append_slots(ctypes.byref(d), pg_ref(pg), v, k, vn, kn, slot, pos, n, None)


def prompt_status(d, pg=None, q=A, m=A, v=A, k=A, table=None, lens=A, cu=A, n=4, S=1, rows=0, ws=A, nb=1 << 40, o=A, lse=A):
    return gva.lib().gva_packed_prefill(ctypes.byref(d), pg_ref(pg), q, m, v, k, table, lens, cu, n, S, rows, ws, nb, o, lse,
                                        None)


def tree_status(d, pg=None, q=A, m=A, v=A, k=A, table=None, lens=A, cu=A, parent=A, n=4, S=1, rows=0, ws=A, nb=1 << 40, o=A,
                lse=A):
    return gva.lib().gva_tree_attention(ctypes.byref(d), pg_ref(pg), q, m, v, k, table, lens, cu, parent, n, S, rows, ws, nb, o,
                                        lse, None)


def commit_status(d, pg=None, v=A, k=A, table=None, lens=A, cu=A, parent=A, leaf=A, n=4, new=A + 4096, acc=A):
    return gva.lib().gva_tree_commit(ctypes.byref(d), pg_ref(pg), v, k, table, lens, cu, parent, leaf, n, new, acc, None)


CALLS = [tables_status, slots_status, prompt_status, tree_status, commit_status]


@pytest.mark.parametrize("call", CALLS)
@pytest.mark.parametrize("kw", [dict(batch=0), dict(n_groups=3), dict(d_r=-2), dict(d_v=0), dict(dtype=5), dict(t_max=0)])
def test_bad_dims_refused(call, kw):
    assert call(dims(**kw)) == BAD


@pytest.mark.parametrize("call", CALLS)
def test_bad_paging_refused(call):
    more = {} if call in (tables_status, slots_status) else dict(table=A)
    for pg in (paging(48), paging(0), paging(64, 3), paging(64, 2, 0), paging(128, 2)):
        assert call(dims(), pg=pg, **more) == BAD
    assert call(dims(t_max=32 * 4097), pg=paging(32, 4097), **more) == UNSUP
    if not more:
        assert call(dims(), pg=None) == BAD
        assert call(dims(), pg=paging(64, 2, 1 << 25)) == UNSUP       # slots past 2^31
        return
    assert call(dims(), pg=paging()) == BAD and call(dims(), table=A) == BAD      # one without the other


@pytest.mark.parametrize("call,names", [
    (tables_status, "lens n_new table free n_free new new_free cu"), (slots_status, "v k vn kn slot pos"),
    (prompt_status, "q m v k lens cu o"), (tree_status, "q m v k lens cu parent o"),
    (commit_status, "v k lens cu parent leaf new")])
def test_missing_and_misaligned_pointers_refused(call, names):
    for name in names.split():
        assert call(dims(), **{name: None}) == BAD, name
        assert call(dims(), **{name: A + 1}) == BAD, name
    assert call(dims(), n=-1) == BAD


def test_tables_refuse_overlaps():
    for to in ("new", "new_free", "cu"):
        for of in ("lens", "n_new", "n_free"):
            at = {"lens": A, "n_new": A + 4096, "n_free": A + 8192}[of]
            assert tables_status(dims(), **{to: at}) == BAD, (to, of)
    far = {k: A * (i + 2) for i, k in enumerate(("lens", "n_new", "n_free", "new", "new_free", "cu"))}
    assert tables_status(dims(batch=65536), **far) == UNSUP
    assert commit_status(dims(), new=A + 4) == BAD


@pytest.mark.parametrize("call", [prompt_status, tree_status])
def test_attention_refusals(call):
    for kw in (dict(d_v=96), dict(d_c=48), dict(d_c=544), dict(d_c=0), dict(d_r=12), dict(d_r=72), dict(n_heads=6, n_groups=2),
               dict(n_heads=32, n_groups=2), dict(t_max=120), dict(d_v=256)):
        for dtype in ("bf16", "f32"):
            assert call(dims(**{**kw, "dtype": dtype})) == UNSUP, kw
    assert call(dims(), S=0) == BAD and call(dims(), S=257) == BAD
    assert call(dims(), rows=16) == BAD and call(dims(), rows=-32) == BAD
    assert call(dims(), n=(1 << 20) + 1) == UNSUP
    assert call(dims(t_max=(1 << 30) + 32), pg=paging((1 << 30) + 32, 1, 1), table=A) == UNSUP
    need = gva.gva_packed_workspace_size(dims(), 4, 3)
    assert need >= 4 * 8 * 3 * 129 * 4
    assert call(dims(), S=3, ws=None) == BAD and call(dims(), S=3, nb=need - 1) == BAD and call(dims(), S=3, ws=A + 16) == BAD
    assert call(dims(), n=0, q=None, m=None, v=None, o=None) == gva.GVA_OK          # nothing to do
    assert gva.gva_packed_workspace_size(dims(), 0, 3) == 0
    with pytest.raises(gva.GvaError):
        gva.gva_packed_workspace_size(dims(), 4, 0)


def test_maps_refuse_overlaps():
    apart = dict(seq=2 * A, row=3 * A, slot=4 * A, table=5 * A, free=6 * A)
    reads = (A, A + 4096, A + 8192)                    # lens, n_new, n_free
    for name in ("seq", "row", "slot"):
        for at in reads + (5 * A, 6 * A):
            assert tables_status(dims(), **{**apart, name: at}) == BAD, name
    for name in ("table", "free"):
        for at in reads + (A + 12288, A + 16384, A + 20480):
            assert tables_status(dims(), **{**apart, name: at}) == BAD, name
    assert tables_status(dims(), **{**apart, "free": 5 * A + 8}) == BAD
    apart = dict(lens=A, cu=2 * A, parent=3 * A, leaf=4 * A, new=5 * A, acc=6 * A)
    for name in ("new", "acc"):
        for at in range(1, 5):
            assert commit_status(dims(), **{**apart, name: at * A}) == BAD, (name, at)


def test_commit_and_slots_shapes():
    assert commit_status(dims(t_max=120)) == UNSUP and commit_status(dims(d_v=12)) == UNSUP
    assert slots_status(dims(d_v=12)) == UNSUP
    assert slots_status(dims(), n=0, v=None, slot=None) == gva.GVA_OK


def test_plans_are_host_only():
    d = dims(batch=4, n_heads=32, n_groups=8, t_max=32768)
    lens = torch.tensor([100, 32768, 5000, 70000], dtype=torch.int32)
    for new in ([1, 1, 1, 1], [0, 16, 16, -5], [512, 1, 0, 700]):
        n = sum(max(x, 0) for x in new)
        S, rows = gva.packed_plan_for(d, lens, torch.tensor(new, dtype=torch.int32))
        assert 1 <= S <= gva.GVA_MAX_SPLITS and rows >= 0 and rows % 32 == 0
        assert gva.gva_packed_pick_splits(d, lens, torch.tensor(new, dtype=torch.int32), n_cu=256, chunked=False)[1] == 0
    assert gva.gva_packed_pick_splits(d, None, None, 64)[0] > 1          # few queries, long caches
    assert gva.gva_packed_pick_splits(dims(d_v=96), None, None, 64) == (1, 0)
    assert gva.gva_packed_pick_splits(d, lens, torch.tensor([(1 << 31) - 1] * 4, dtype=torch.int32), 64)[0] >= 1
    with pytest.raises(ValueError):
        gva.packed_plan_for(d, lens[:3], lens)


def test_binding_refuses_cpu_tensors_and_wrong_shapes():
    d, pg = dims(), paging()
    i = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError):
        gva.gva_page_tables(d, pg, i, i, torch.zeros(2, 2, dtype=torch.int32), i, i, i, i, i, i)
    q = torch.zeros(3, 8, 144, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        gva.gva_packed_prefill(d, q, q, q, q, i, i, q)
    with pytest.raises(ValueError):
        gva.gva_packed_prefill(d, q[0], q, q, q, i, i, q)
    with pytest.raises(ValueError):
        gva.gva_tree_commit(d, q, q, i, i, i, i, i, block_table=i)
    with pytest.raises(ValueError):
        gva.gva_page_tables(d, pg, i, i, i, i, i, i, i, i)


def test_reference_window_of_a_chain_is_causal():
    for L, n in ((9, 4), (3, 5), (4, 4), (0, 2)):
        chain = ref.window(L, n, [i - 1 for i in range(n)])
        plain = ref.window(L, n)
        assert torch.equal(chain[0], plain[0]) and torch.equal(chain[1], plain[1])


# ------------------------------------------------------------------ tables
def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def run_tables(d, pg, lens, new, table, free, n_free, n_rows, maps=True):
    B = d.batch
    out = {"table": ints(table), "free": ints(free), "lens": ints([7] * B), "n_free": ints([7]), "cu": ints([7] * (B + 1)),
           "seq": ints([7] * n_rows), "row": ints([7] * n_rows), "slot": ints([7] * n_rows)}
    args = (d, pg, ints(lens), ints(new), out["table"], out["free"], ints([n_free]), out["lens"], out["n_free"], out["cu"])
    for again in range(2):                             # a repeated call gives the same
        if maps:
            gva.gva_page_tables(*args, out["seq"], out["row"], out["slot"])
        else:
            gva.gva_page_tables(*args, n_rows=n_rows)
    return {k: v.tolist() for k, v in out.items()}


def tables_case(B, R, most, seed, spare, n_rows=None, maps=True, wild=False):
    rng = random.Random(seed)
    T = R * most
    lens = [min(T, rng.choice([0, 1, R - 1, R, R + 1, T, rng.randint(0, T)])) for _ in range(B)]
    new = [rng.choice([0, 1, 1, 1, -1, -min(5, L), -L, R, rng.randint(0, 3 * R), T - L]) for L in lens]
    held = [-(-L // R) for L in lens]
    n_pages = sum(held) + spare
    order = list(range(n_pages))
    rng.shuffle(order)
    table = [[-7] * most for _ in range(B)]
    it = iter(order)
    for b in range(B):
        table[b][:held[b]] = [next(it) for _ in range(held[b])]
    rest = list(it)
    n_free = len(rest)
    free = rest + [-9] * (n_pages - n_free)
    if wild:                                           # values that no caller should pass
        lens = [rng.choice([L, -3, T + 100]) for L in lens]
        new = [rng.choice([x, -(1 << 31), (1 << 31) - 1]) for x in new]
        n_free = rng.choice([-5, n_free, n_pages + 50])
        table[0][0] = 1 << 30
    if n_rows is None:
        n_rows = sum(min(max(x, 0), T) for x in new) + 3
    d = dims(batch=B, t_max=T)
    note(f"tables B={B} R={R} pages {most} seed {seed} spare {spare} rows {n_rows} wild {wild}")
    got = run_tables(d, gva.GvaPaging(R, most, max(1, n_pages)), lens, new, table, free or [0], n_free, n_rows, maps)
    want = ref.page_tables(lens, new, table, free, n_free, n_rows, T, R, max(1, n_pages))
    want.update(table=table, free=free or [0])
    if not maps:
        want.update(seq=[7] * n_rows, row=[7] * n_rows, slot=[7] * n_rows)
    for k in want:
        assert got[k] == (want[k] if k != "n_free" else [want[k]]), k


@gpu
@pytest.mark.parametrize("B,R,most", [(1, 32, 4), (2, 64, 1), (5, 32, 70), (64, 96, 5), (255, 32, 6), (256, 64, 3), (257, 32, 9),
                                      (700, 32, 4), (3000, 32, 2)])
@pytest.mark.parametrize("spare", [0, 3, 4000])
def test_tables(B, R, most, spare):
    tables_case(B, R, most, 100 * B + spare, spare)


@gpu
def test_tables_rows_cut_off_padded_and_not_asked_for():
    tables_case(9, 32, 8, 1, 100, n_rows=5)
    tables_case(9, 32, 8, 2, 100, n_rows=0)
    tables_case(9, 32, 8, 3, 100, n_rows=2000)
    tables_case(9, 32, 8, 4, 100, n_rows=77, maps=False)


@gpu
@pytest.mark.parametrize("seed", range(6))
def test_tables_clamp_what_they_read(seed):
    tables_case(40, 32, 3, seed, 10, n_rows=5000, wild=True)


# ------------------------------------------------------------------- slots
@gpu
@pytest.mark.parametrize("dtype,G,d_v,d_r", [("bf16", 2, 128, 16), ("bf16", 1, 64, 0), ("f32", 4, 64, 24), ("f32", 1, 20, 4)])
@pytest.mark.parametrize("n", [1, 17, 700])
def test_append_slots(dtype, G, d_v, d_r, n):
    R, pages = 96, 11
    d, pg = dims(batch=3, n_heads=G, n_groups=G, d_v=d_v, d_r=d_r, t_max=5 * R, dtype=dtype), gva.GvaPaging(R, 5, pages)
    dt = d.torch_dtype
    g = torch.Generator().manual_seed(n)
    v = torch.full((pages, G, R, d_v), 3.0, dtype=dt)
    kr = torch.full((pages, R, d_r), 5.0, dtype=dt)
    vn, kn = torch.randn(n, G, d_v, generator=g).to(dt), torch.randn(n, d_r, generator=g).to(dt)
    slot = torch.randperm(R * pages, generator=g)[:n].to(torch.int32)
    pos = torch.randint(0, 200000, (n,), generator=g, dtype=torch.int32)
    slot[::5] = torch.tensor([-1, R * pages, -(1 << 31), (1 << 31) - 1])[torch.arange(0, n, 5) % 4].to(torch.int32)
    note(f"slots {dtype} G={G} {d_v}/{d_r} n={n}")
    dev = [gva.tiled(v).cuda(), gva.tiled(kr).cuda() if d_r else kr.cuda()]
    gva.gva_append_slots(d, pg, dev[0], dev[1] if d_r else None, vn.cuda(), kn.cuda() if d_r else None, slot.cuda(), pos.cuda())
    rot = ref.rotate(kn, pos)
    for r in range(n):
        s = int(slot[r])
        if 0 <= s < R * pages:
            v[s // R, :, s % R] = vn[r]
            kr[s // R, s % R] = rot[r].to(dt)
    assert torch.equal(gva.untiled(dev[0].cpu()), v)
    if d_r:
        got = gva.untiled(dev[1].cpu())
        # a rotation in 64 bits, rounded once: a neighbour only where the two 64-bit results straddle a border
        step = 2.0 ** -24 if dtype == "f32" else 2.0 ** -8
        off = (got.double() - kr.double()).abs()
        assert bool((off <= 2 * step * kr.double().abs() + 1e-30).all())
        assert float((got != kr).double().mean()) <= 1e-3


# --------------------------------------------------------------- attention
def problem(lens, new, H, G, d_v, d_c, d_r, T, R=0, dtype="bf16", seed=0, sharp=1.0, parent=None, spare=2):
    """A cache with rows for `lens`, NaN in every other row and page; packed queries."""
    B = len(lens)
    g = torch.Generator().manual_seed(seed)
    d = gva.make_dims(B, H, G, d_v, d_c, d_r, T, dtype)
    dt = d.torch_dtype
    n = sum(new)
    cu = [sum(new[:b]) for b in range(B + 1)]
    x = {"d": d, "lens": lens, "new": new, "cu": cu, "n": n, "parent": parent, "R": R, "pg": None, "table": None}
    x["v"] = torch.randn(B, G, T, d_v, generator=g).to(dt)
    x["kr"] = torch.randn(B, T, d_r, generator=g).to(dt)
    x["m"] = (torch.randn(H, d_v, d_c, generator=g) / math.sqrt(d_v)).to(dt)
    x["q"] = (torch.randn(n, H, d_c + d_r, generator=g) * sharp).to(dt)
    for b, L in enumerate(lens):
        x["v"][b, :, min(max(L, 0), T):] = math.nan
        x["kr"][b, min(max(L, 0), T):] = math.nan
    if R:
        held = [-(-min(max(L, 0), T) // R) for L in lens]
        pages = sum(held) + spare
        order = torch.randperm(pages, generator=g)
        table = torch.full((B, T // R), (1 << 30), dtype=torch.int32)       # entries of no page, past the lengths
        k = 0
        for b in range(B):
            table[b, :held[b]] = order[k:k + held[b]].to(torch.int32)
            k += held[b]
        x["table"], x["pg"] = table, gva.GvaPaging(R, T // R, pages)
    return x


def upload(x):
    """The caches as the library stores them."""
    v, kr, R = x["v"], x["kr"], x["R"]
    if R:
        pages, (B, G, T, dv), dr = x["pg"].n_pages, v.shape, kr.shape[-1]
        pv, pk = torch.full((pages, G, R, dv), math.nan, dtype=v.dtype), torch.full((pages, R, dr), math.nan, dtype=v.dtype)
        for b in range(B):
            for j in range(T // R):
                p = int(x["table"][b, j])
                if p < pages:
                    pv[p], pk[p] = v[b, :, j * R:(j + 1) * R], kr[b, j * R:(j + 1) * R]
        v, kr = pv, pk
    return gva.tiled(v).cuda(), gva.tiled(kr).cuda() if kr.shape[-1] else None


def call(x, S=1, rows=0, dev=None, o=None, lse=None, ws=None, stream=None, n=None):
    d = x["d"]
    n = x["n"] if n is None else n
    v, kr = upload(x) if dev is None else dev
    o = torch.full((n, d.n_heads, d.d_v), 77.0, dtype=d.torch_dtype, device="cuda") if o is None else o
    lse = torch.full((n, d.n_heads), 77.0, device="cuda") if lse is None else lse
    if ws is None:
        ws = gva.packed_workspace_for(d, n, S)
        if ws is not None:
            ws.fill_(0xFF)                             # NaN wherever it is read unwritten
    q = x["q"]
    if n > x["n"]:
        q = torch.cat((q, torch.full((n - x["n"], *q.shape[1:]), math.nan, dtype=q.dtype)))
    args = [d, q.cuda(), x["m"].cuda(), v, kr, ints(x["lens"]), ints(x["cu"])]
    more = dict(lse=lse, paging=x["pg"], block_table=None if x["table"] is None else x["table"].cuda(), num_splits=S,
                split_rows=rows, workspace=ws, stream=stream)
    if x["parent"] is None:
        gva.gva_packed_prefill(*args, o, **more)
    else:
        flat = [a for p in x["parent"] for a in p] + [0] * (n - x["n"])
        gva.gva_tree_attention(*args, ints(flat), o, **more)
    return o, lse


def check(x, o, lse, only=None, skip=None):
    """Outputs against the reference's; `only` these sequences, and not the rows that `skip` [n_rows] names."""
    d, T = x["d"], x["d"].t_max
    o, lse = o.cpu().double(), lse.cpu().double()
    worst = 0.0
    for b, (L, n) in enumerate(zip(x["lens"], x["new"])):
        if n == 0 or (only is not None and b not in only):
            continue
        L = min(max(L, 0), T)
        at = slice(x["cu"][b], x["cu"][b] + n)
        parent = None if x["parent"] is None else ref.parents(x["parent"][b])
        if parent is not None and n > gva.GVA_MAX_TREE:
            assert bool((o[at] == 0).all()) and bool(torch.isneginf(lse[at]).all())
            continue
        see, pos = ref.window(L, n, parent)
        wo, wl, do, dl = ref.attend(x["q"][at], x["m"], x["v"][b, :, :L], x["kr"][b, :L], see, pos, d.n_groups, d.torch_dtype)
        none = torch.isneginf(wl)
        assert torch.equal(torch.isneginf(lse[at]), none), f"sequence {b}: empty rows"
        assert bool((o[at][none] == 0).all())
        if skip is not None:
            none = none | skip[at].unsqueeze(1)
        e = ((o[at] - wo).abs() / do)[~none]
        f = ((lse[at] - wl).abs() / dl)[~none]
        if e.numel():
            assert not bool(torch.isnan(e).any()) and not bool(torch.isnan(f).any()), f"sequence {b}: NaN"
            assert float(e.max()) <= 1, f"sequence {b}: o {float(e.max())} of its bound"
            assert float(f.max()) <= 1, f"sequence {b}: lse {float(f.max())} of its bound"
            worst = max(worst, float(e.max()), float(f.max()))
    return worst


def random_tree(rng, n, kind="mixed"):
    if kind == "chain":
        return [i - 1 for i in range(n)]
    if kind == "star":
        return [-1] * n
    return [-1 if rng.random() < 0.15 else rng.randint(max(-1, i - 6), i - 1) for i in range(n)]


def trees(new, seed=0, kind="mixed"):
    rng = random.Random(seed)
    return [random_tree(rng, n, kind) for n in new]


# heads, groups, d_v, d_c, d_r: every number of heads per group, widths and positional chunks
SHAPES = [(4, 4, 64, 64, 16), (4, 2, 128, 128, 16), (8, 2, 64, 32, 0), (8, 2, 128, 96, 32), (16, 2, 128, 128, 8),
          (8, 1, 64, 128, 64), (4, 1, 128, 64, 64), (2, 2, 128, 512, 24)]


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("R", [0, 32, 96])
@pytest.mark.parametrize("H,G,d_v,d_c,d_r", SHAPES)
def test_prompts(H, G, d_v, d_c, d_r, R, dtype):
    # nothing new, one token, a whole prompt, one behind a prefix, more queries than rows, an empty cache, over capacity
    lens, new = [200, 1, 70, 288, 20, 0, 400, 33], [0, 1, 70, 45, 30, 4, 40, 33]
    x = problem(lens, new, H, G, d_v, d_c, d_r, 288, R, dtype, seed=d_v + d_r)
    note(f"prompts H={H} G={G} {d_v}/{d_c}/{d_r} R={R} {dtype}")
    dev = upload(x)
    for S, rows in ((1, 0), (3, 0), (5, 64)):
        check(x, *call(x, S, rows, dev))


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("R", [0, 64])
@pytest.mark.parametrize("H,G,d_v,d_c,d_r", SHAPES)
def test_trees(H, G, d_v, d_c, d_r, R, dtype):
    lens, new = [150, 1, 40, 256, 20, 0, 300, 97], [0, 1, 40, 33, 30, 4, 70, 5]
    x = problem(lens, new, H, G, d_v, d_c, d_r, 256, R, dtype, seed=d_v + d_r + 1, parent=trees(new, H))
    note(f"trees H={H} G={G} {d_v}/{d_c}/{d_r} R={R} {dtype}")
    dev = upload(x)
    for S, rows in ((1, 0), (4, 0), (3, 96)):
        check(x, *call(x, S, rows, dev))


# queries per sequence that take 32, 64 and 128 columns a workgroup, one set of waves and several
@gpu
@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("H,G,d_v,n", [(8, 1, 128, 1), (8, 1, 64, 4), (8, 1, 128, 5), (8, 2, 128, 8), (8, 2, 64, 9), (8, 2, 128, 16),
                                       (4, 4, 64, 17), (4, 4, 128, 33), (2, 1, 128, 40), (8, 1, 128, 130), (16, 16, 64, 129)])
def test_columns_of_a_workgroup(H, G, d_v, n, tree):
    lens, new = [n + 300, 257, n, 640], [n, max(1, n - 1), n, min(n + 2, 200)]
    x = problem(lens, new, H, G, d_v, 64, 16, 640, 32, seed=n, parent=trees(new, n) if tree else None)
    note(f"columns H={H} G={G} {d_v} n={n} tree={tree}")
    dev = upload(x)
    for S, rows in ((1, 0), (6, 128)):
        check(x, *call(x, S, rows, dev))


# few queries per sequence with wide positional keys: three or four sets of waves
@gpu
@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("n", [3, 8])
@pytest.mark.parametrize("d_v,d_c,d_r", [(128, 64, 24), (128, 128, 32), (128, 32, 40), (128, 256, 64), (64, 64, 32), (64, 96, 64)])
def test_sets_of_waves(d_v, d_c, d_r, n, tree):
    lens, new = [n + 290, 257, n, 640, 30], [n, n - 1, n, n, 0]
    for R in (0, 32, 160):
        x = problem(lens, new, 8, 1, d_v, d_c, d_r, 640, R, seed=n + d_r, parent=trees(new, n) if tree else None)
        note(f"sets {d_v}/{d_c}/{d_r} n={n} R={R} tree={tree}")
        dev = upload(x)
        for S, rows in ((1, 0), (3, 128)):
            check(x, *call(x, S, rows, dev))


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_bases_below_one(dtype, monkeypatch):
    """Angles of thousands of millions of quarter turns.  The fastest pair's is 7e9 at the last
    position, whose roundings (2^-53 of it, three of them) are 2e-6; scores are off by less than
    4e-5 for it (entries of normal numbers stay below 4), which the bound holds: 2^-17 (bf16) or
    164 x 2^-24 (fp32) of the sizes of the scores' products, of about 40."""
    base = 4e-9
    monkeypatch.setattr(ref, "BASE", base)
    x = problem([300, 77], [40, 3], 4, 2, 64, 64, 16, 320, seed=5, dtype=dtype)
    x["d"] = gva.make_dims(2, 4, 2, 64, 64, 16, 320, dtype, rope_base=base)
    note(f"base {base} {dtype}")
    for S in (1, 3):
        check(x, *call(x, S))


@gpu
@pytest.mark.parametrize("d_v", [64, 128])
@pytest.mark.parametrize("B", [70, 260, 600])
def test_many_sequences(B, d_v):
    """Items found over one, five and ten sequences a lane; some sequences without queries."""
    rng = random.Random(B)
    lens = [rng.randint(0, 192) for _ in range(B)]
    new = [rng.choice([0, 1, 2, 40, L]) for L in lens]
    x = problem(lens, new, 4, 2, d_v, 32, 8, 192, 32, seed=B)
    note(f"many sequences {B} {d_v}")
    dev = upload(x)
    for S, rows in ((1, 0), (2, 64)):
        check(x, *call(x, S, rows, dev))


@gpu
@pytest.mark.parametrize("kind", ["chain", "star", "mixed"])
@pytest.mark.parametrize("n", [31, 32, 33, 64, 255, 256, 257])
def test_tree_sizes(kind, n):
    x = problem([n + 45, n], [n, n], 4, 2, 64, 32, 16, 320, 0, seed=n, parent=trees([n, n], n, kind))
    note(f"tree of {n}, {kind}")
    dev = upload(x)
    for S, rows in ((1, 0), (3, 96)):
        check(x, *call(x, S, rows, dev))


@gpu
def test_tree_parents_that_are_none():
    """A parent that is the node itself, behind it, or below -1 is read as -1."""
    bad = [0, 5, -7, 1 << 30, -(1 << 31), 3, 6, 2]
    x = problem([60], [8], 4, 1, 64, 32, 16, 64, 0, seed=3, parent=[bad])
    note("bad parents")
    check(x, *call(x))


@gpu
@pytest.mark.parametrize("sharp", [2.5, 6.0])
@pytest.mark.parametrize("tree", [False, True])
def test_sharp_scores(sharp, tree):
    lens, new = [700, 64], [50, 64]
    x = problem(lens, new, 8, 2, 128, 128, 32, 704, 0, seed=11, sharp=sharp, parent=trees(new) if tree else None)
    note(f"sharp {sharp} tree {tree}")
    dev = upload(x)
    for S, rows in ((1, 0), (4, 192)):
        check(x, *call(x, S, rows, dev))


@gpu
def test_far_positions():
    T = 140000
    lens, new = [139999], [3]
    x = problem(lens, new, 2, 1, 64, 32, 64, T // 32 * 32, 0, seed=12)
    note("far positions")
    dev = upload(x)
    check(x, *call(x, 16, 0, dev))
    check(x, *call(x, 1, 0, dev))


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_what_is_hidden_does_not_reach_a_query(bad, dtype):
    """A bad value or key row of the window reaches the queries that see it (as NaN) and no other."""
    lens, new = [100, 90, 40], [60, 90, 33]
    for tree in (False, True):
        x = problem(lens, new, 8, 2, 128, 64, 16, 128, 32, dtype, seed=13, parent=trees(new, 5) if tree else None)
        where = [(0, 70), (1, 31), (1, 64), (2, 39)]
        for b, t in where:
            x["v"][b, 1, t, 5:9] = bad
        clean = problem(lens, new, 8, 2, 128, 64, 16, 128, 32, dtype, seed=13, parent=x["parent"])
        note(f"hidden {bad} {dtype} tree {tree}")
        for S, rows in ((1, 0), (3, 32)):
            o, lse = (u.cpu() for u in call(x, S, rows))
            o0, lse0 = (u.cpu() for u in call(clean, S, rows))
            hits = torch.zeros(x["n"], dtype=torch.bool)
            for b in range(3):
                par = ref.parents(x["parent"][b]) if tree else None
                see, _ = ref.window(lens[b], new[b], par)
                hit = torch.zeros(new[b], dtype=torch.bool)
                for bb, t in where:
                    if bb == b:
                        hit |= see[:, t]
                at = slice(x["cu"][b], x["cu"][b] + new[b])
                assert torch.equal(o[at, :4], o0[at, :4]) and torch.equal(lse[at, :4], lse0[at, :4])   # the other group
                hits[at] = hit
                if math.isnan(bad):
                    assert bool(torch.isnan(o[at, 4:][hit]).all())
            check(clean, o, lse, skip=hits)


@gpu
def test_a_nan_key_and_a_hiding_one():
    """A NaN positional key is seen as NaN; one at the type's lowest value takes its row out of the sum, or puts all weight on it."""
    x = problem([50], [20], 4, 2, 64, 32, 16, 64, 0, seed=14)
    x["kr"][0, 40, 3] = math.nan
    note("nan key")
    o, lse = (u.cpu() for u in call(x))
    assert bool(torch.isnan(o[10:]).all()) and not bool(torch.isnan(o[:10]).any())
    assert not bool(torch.isnan(lse[:10]).any())


@gpu
@pytest.mark.parametrize("tree", [False, True])
def test_rows_of_no_sequence_are_left_and_lse_may_be_none(tree):
    """A batch padded past its last sequence, and one that begins behind row 0."""
    lens, new = [64, 90], [20, 9]
    x = problem(lens, new, 8, 2, 64, 64, 16, 96, 32, seed=15, parent=trees(new) if tree else None)
    note("padding")
    dev = upload(x)
    for S, rows in ((1, 0), (3, 32)):
        o, lse = call(x, S, rows, dev, n=61)
        check(x, o, lse)
        assert bool((o[29:] == 77.0).all()) and bool((lse[29:] == 77.0).all())
        late = dict(x, cu=[20, 20, 29], new=[0, 9])
        o, lse = call(late, S, rows, dev)
        check(late, o, lse)
        assert bool((o[:20] == 77.0).all()) and bool((lse[:20] == 77.0).all())
        d, args = x["d"], [x["d"], x["q"].cuda(), x["m"].cuda(), *dev, ints(lens), ints(x["cu"])]
        more = dict(paging=x["pg"], block_table=x["table"].cuda(), num_splits=S, split_rows=rows,
                    workspace=gva.packed_workspace_for(d, 29, S))
        o2 = torch.empty(29, 8, 64, dtype=torch.bfloat16, device="cuda")
        if tree:
            gva.gva_tree_attention(*args, ints(sum(x["parent"], [])), o2, **more)
        else:
            gva.gva_packed_prefill(*args, o2, **more)
        assert torch.equal(o2, call(x, S, rows, dev)[0])


@gpu
def test_offsets_that_are_out_of_range_or_not_in_order():
    """cu_rows is clamped: nothing outside the outputs is written, whatever it says."""
    x = problem([64, 90, 80], [20, 9, 10], 8, 2, 64, 64, 16, 96, 32, seed=16)
    dev = upload(x)
    pad = 4096
    note("wild offsets")
    for cu in ([0, 1 << 30, -5, 39], [30, 10, 39, 1 << 31 - 1], [-(1 << 31), 5, 3, 50], [0, 0, 0, 0]):
        for S in (1, 3):
            raw = torch.full((pad + 39 * 8 * 64 + pad,), 77.0, dtype=torch.bfloat16, device="cuda")
            rawl = torch.full((pad + 39 * 8 + pad,), 77.0, device="cuda")
            call(dict(x, cu=cu), S, 0, dev, o=raw[pad:-pad].view(39, 8, 64), lse=rawl[pad:-pad].view(39, 8))
            for r in (raw, rawl):
                assert bool((r[:pad] == 77.0).all()) and bool((r[-pad:] == 77.0).all())


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_prompt_is_the_equal_length_prompt(dtype, orc):
    """Equal lengths on a contiguous cache: what gva_prefill, or a decode step of each row, gives."""
    import gva_inputs
    B, N, T, H, G = 2, 40, 96, 8, 2
    x = problem([96, 70], [N, N], H, G, 64, 64, 16, T, 0, dtype, seed=17)
    note(f"against the equal-length prompt {dtype}")
    o, lse = (u.cpu().double() for u in call(x))
    v, kr = torch.nan_to_num(x["v"]), torch.nan_to_num(x["kr"])
    wo, wl = orc.prefill(x["q"].view(B, N, H, -1), x["m"], v, kr, torch.tensor(x["lens"], dtype=torch.int32), rope_base=10000.0)
    # a weight and an output off by 2^-8 each, of values below 4; what else attend() counts is below 2^-10 here
    assert float((o.view(B, N, H, -1) - wo).abs().max()) <= (2.0 ** -5 if dtype == "bf16" else 2.0 ** -10)
    assert float((lse.view(B, N, H) - wl).abs().max()) <= 2.0 ** -10


# ---------------------------------------------------------- streams, graphs
@gpu
@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("S", [1, 3])
def test_streams_graph_and_guards(S, tree):
    """On a side stream beside the same call on another; captured, replayed with
    eager work between; nothing written outside the outputs."""
    lens, new = [256, 17, 130], [30, 17, 2]
    x = problem(lens, new, 16, 4, 128, 128, 16, 256, 64, seed=8, parent=trees(new) if tree else None)
    d, n = x["d"], x["n"]
    note(f"streams, graph, guards S={S} tree={tree}")
    dev = upload(x)
    base = call(x, S, 0, dev)
    pad = 4096
    raw = torch.full((pad + n * 16 * 128 + pad,), 123.0, dtype=torch.bfloat16, device="cuda")
    rawl = torch.full((pad + n * 16 + pad,), 123.0, device="cuda")
    size = gva.gva_packed_workspace_size(d, n, S)
    raww = torch.full((size + 8192,), 0x77, dtype=torch.uint8, device="cuda")
    o, lse, ws = raw[pad:-pad].view(n, 16, 128), rawl[pad:-pad].view(n, 16), raww[4096:4096 + size]
    q, m, le, cu = x["q"].cuda(), x["m"].cuda(), ints(lens), ints(x["cu"])
    par, table = ints(sum(x["parent"], [])) if tree else None, x["table"].cuda()

    def go(o, lse, ws, stream=None):
        more = dict(lse=lse, paging=x["pg"], block_table=table, num_splits=S, workspace=ws if size else None, stream=stream)
        if tree:
            gva.gva_tree_attention(d, q, m, *dev, le, cu, par, o, **more)
        else:
            gva.gva_packed_prefill(d, q, m, *dev, le, cu, o, **more)

    sides = [torch.cuda.Stream(), torch.cuda.Stream()]
    outs = [(torch.empty_like(o), torch.empty_like(lse), torch.empty_like(ws)) for _ in sides]
    torch.cuda.synchronize()
    for _ in range(3):
        for s, out in zip(sides, outs):
            go(*out, stream=s)
    torch.cuda.synchronize()
    for out in outs:
        assert torch.equal(out[0], base[0]) and torch.equal(out[1], base[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        go(o, lse, ws)
    for _ in range(4):
        o.fill_(math.nan)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, base[0]) and torch.equal(lse, base[1])
        go(*outs[0])
        torch.cuda.synchronize()
    for r in (raw, rawl):
        assert bool((r[:pad] == 123.0).all()) and bool((r[-pad:] == 123.0).all())
    assert bool((raww[:4096] == 0x77).all()) and bool((raww[4096 + size:] == 0x77).all())


@gpu
def test_pools_past_two_gigabytes():
    """Pages whose offsets pass 2^31 and 2^32 bytes, appended, attended and committed."""
    R, G, dv, dr = 64, 4, 128, 16
    pages = 70000                                      # 4.6 GB of values
    d, pg = gva.make_dims(1, 8, G, dv, 128, dr, 4 * R, "bf16"), gva.GvaPaging(R, 4, pages)
    table = torch.tensor([[pages - 1, 3, 40000, 69000]], dtype=torch.int32)
    note("pools past 4 GB")
    v = torch.empty(pages, G, R, dv, dtype=torch.bfloat16, device="cuda")
    kr = torch.empty(pages, R, dr, dtype=torch.bfloat16, device="cuda")
    n, P = 200, 180
    x = problem([n], [n - P], 8, G, dv, 128, dr, 4 * R, 0, seed=21, parent=trees([n - P], 1))
    rows = x["v"][0, :, :n].transpose(0, 1).contiguous()
    t = torch.arange(n)
    slot = (table[0].long()[t // R] * R + t % R).to(torch.int32)
    raw = ref.rotate(x["kr"][0, :n], -t)               # so that the append's rotation gives x["kr"] back, but for a rounding
    gva.gva_append_slots(d, pg, v, kr, rows.cuda(), raw.to(torch.bfloat16).cuda(), slot.cuda(), t.to(torch.int32).cuda())
    idx = table[0].long().cuda()
    kept = gva.untiled(kr[idx].cpu()).reshape(1, 4 * R, dr)
    assert torch.equal(gva.untiled(v[idx].cpu()).transpose(0, 1).reshape(G, 4 * R, dv)[:, :n], x["v"][0, :, :n])
    x.update(pg=pg, table=table, kr=kept)
    for S in (1, 4):
        check(x, *call(x, S, 0, (v, kr)))
    leaf = n - P - 1
    path = ref.ancestors(ref.parents(x["parent"][0]), leaf)
    new, acc = ints([0]), ints([0] * (n - P))
    gva.gva_tree_commit(d, v, kr, ints([n]), ints(x["cu"]), ints(x["parent"][0]), ints([leaf]), new, acc, paging=pg,
                        block_table=table.cuda())
    assert new.tolist() == [P + len(path)] and acc.tolist()[:len(path)] == path
    got = gva.untiled(v[idx].cpu()).transpose(0, 1).reshape(G, 4 * R, dv)
    for k, a in enumerate(path):
        assert torch.equal(got[:, P + k], x["v"][0, :, P + a])


# ------------------------------------------------------------------ commit
@gpu
@pytest.mark.parametrize("dtype,G,d_v,d_r", [("bf16", 2, 128, 16), ("bf16", 1, 24, 0), ("f32", 3, 64, 8), ("f32", 1, 260, 64)])
@pytest.mark.parametrize("R", [0, 32])
def test_commit(dtype, G, d_v, d_r, R):
    rng = random.Random(d_v)
    T = 320
    lens = [100, 40, 33, 320, 7, 0, 300, 290, 64, 120]
    new = [30, 40, 5, 256, 9, 3, 257, 100, 0, 64]
    leaf = [29, 20, -1, 255, 2, 0, 3, 100, 0, -(1 << 31)]       # 100 of 100 nodes: none
    par = [random_tree(rng, n, "chain" if n in (40, 256) else "mixed") for n in new]
    par[0] = [-1, 0, 0, 1, 7, 3, -9, 5] + par[0][8:]
    x = problem(lens, new, G, G, d_v, 32, d_r, T, R, dtype, seed=d_v, parent=par)
    x["v"], x["kr"] = torch.nan_to_num(x["v"], 9.0), torch.nan_to_num(x["kr"], 9.0)
    note(f"commit {dtype} G={G} {d_v}/{d_r} R={R}")
    v, kr = upload(x)
    B, n = len(lens), x["n"]
    want_v, want_k, want_l, want_a = x["v"].clone(), x["kr"].clone(), [], [-1] * n
    for b in range(B):
        P = lens[b] - new[b]
        path = ref.ancestors(ref.parents(par[b]), leaf[b]) if new[b] <= 256 and P >= 0 and 0 <= leaf[b] < new[b] else []
        for k, a in enumerate(path):
            want_v[b, :, P + k], want_k[b, P + k] = x["v"][b, :, P + a], x["kr"][b, P + a]
            want_a[x["cu"][b] + k] = a
        want_l.append(max(P, 0) + len(path))
    new_l, acc = ints([7] * B), ints([7] * n)
    gva.gva_tree_commit(x["d"], v, kr, ints(lens), ints(x["cu"]), ints(sum(par, [])), ints(leaf), new_l, acc, paging=x["pg"],
                        block_table=None if not R else x["table"].cuda())
    assert new_l.tolist() == want_l and acc.tolist() == want_a
    x.update(v=want_v, kr=want_k)
    ev, ek = upload(x)
    for got, want in ((v, ev), (kr, ek)):
        if got is not None:
            assert torch.equal(torch.nan_to_num(got, 9.0), torch.nan_to_num(want, 9.0))


# ------------------------------------------------------------- all together
@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_serving_many_requests(dtype):
    """Requests that begin, draft trees, keep a path and end, on a pool that is at
    times too small, against a plain simulation of the pages and rows."""
    rng, g = random.Random(7), torch.Generator().manual_seed(7)
    B, R, most, n_pages, H, G, dv, dc, dr = 6, 32, 6, 9, 8, 2, 64, 64, 16
    T = R * most
    d, pg = gva.make_dims(B, H, G, dv, dc, dr, T, dtype), gva.GvaPaging(R, most, n_pages)
    dt = d.torch_dtype
    m = (torch.randn(H, dv, dc, generator=g) / math.sqrt(dv)).to(dt)
    v = torch.full((n_pages, G, R, dv), math.nan, dtype=dt, device="cuda")
    kr = torch.full((n_pages, R, dr), math.nan, dtype=dt, device="cuda")
    table, free, n_free = ints([[-1] * most] * B), ints(list(range(n_pages))), ints([n_pages])
    lens = ints([0] * B)
    sim_table, sim_free, sim_n, sim_lens = [[-1] * most for _ in range(B)], list(range(n_pages)), n_pages, [0] * B
    sim_v, sim_k = torch.zeros(B, G, T, dv, dtype=dt), torch.zeros(B, T, dr, dtype=dt)
    refused = 0

    def tables(new, n_rows):
        nonlocal lens, n_free, sim_n, sim_lens
        out = {k: ints([7] * s) for k, s in (("lens", B), ("n_free", 1), ("cu", B + 1), ("seq", n_rows), ("row", n_rows),
                                            ("slot", n_rows))}
        gva.gva_page_tables(d, pg, lens, ints(new), table, free, n_free, out["lens"], out["n_free"], out["cu"], out["seq"],
                            out["row"], out["slot"])
        want = ref.page_tables(sim_lens, new, sim_table, sim_free, sim_n, n_rows, T, R, n_pages)
        for k in want:
            assert out[k].tolist() == (want[k] if k != "n_free" else [want[k]]), k
        assert table.tolist() == sim_table
        held = sorted(sim_table[b][j] for b in range(B) for j in range(-(-want["lens"][b] // R)))
        assert len(set(held)) == len(held) == n_pages - want["n_free"]        # no page twice, none lost
        lens, n_free, sim_n, sim_lens = out["lens"], out["n_free"], want["n_free"], want["lens"]
        return out, want

    for step in range(12):
        note(f"serving {dtype} step {step}")
        tree = step % 2 == 1
        before = list(sim_lens)
        new = []
        for b in range(B):
            if before[b] == 0:
                new.append(rng.choice([0, 5, 40, 90]) if not tree else 0)
            elif tree:
                new.append(rng.choice([1, 8, 20]))
            else:
                new.append(rng.choice([1, 1, 33, -before[b]]))
        parent = trees([max(n, 0) for n in new], step)
        n_rows = sum(max(n, 0) for n in new)
        out, want = tables(new, n_rows + 2)
        ok = [new[b] > 0 and want["lens"][b] == before[b] + new[b] for b in range(B)]
        refused += sum(new[b] > 0 and not ok[b] for b in range(B))
        pos = []
        for b in range(B):
            for i in range(max(new[b], 0)):
                pos.append(before[b] + (len(ref.ancestors(parent[b], i)) - 1 if tree else i))
        vn = torch.randn(n_rows + 2, G, dv, generator=g).to(dt)
        kn = torch.randn(n_rows + 2, dr, generator=g).to(dt)
        gva.gva_append_slots(d, pg, v, kr, vn.cuda(), kn.cuda(), out["slot"], ints(pos + [0, 0]))
        rot = ref.rotate(kn[:n_rows], torch.tensor(pos)).to(dt) if n_rows else kn[:0]
        r = 0
        for b in range(B):
            for i in range(max(new[b], 0)):
                if ok[b]:
                    sim_v[b, :, before[b] + i], sim_k[b, before[b] + i] = vn[r], rot[r]
                r += 1
        q = torch.randn(n_rows + 2, H, dc + dr, generator=g).to(dt)
        o = torch.zeros(n_rows + 2, H, dv, dtype=dt, device="cuda")
        lse = torch.zeros(n_rows + 2, H, device="cuda")
        S, rows = [(1, 0), (3, 0), (4, 32)][step % 3]
        more = dict(lse=lse, paging=pg, block_table=table, num_splits=S, split_rows=rows,
                    workspace=gva.packed_workspace_for(d, n_rows + 2, S))
        if tree:
            flat = ints(sum(parent, []) + [0, 0])
            gva.gva_tree_attention(d, q.cuda(), m.cuda(), v, kr, lens, out["cu"], flat, o, **more)
        else:
            gva.gva_packed_prefill(d, q.cuda(), m.cuda(), v, kr, lens, out["cu"], o, **more)
        x = {"d": d, "lens": sim_lens, "new": [max(n, 0) for n in new], "cu": want["cu"], "parent": parent if tree else None,
             "v": sim_v, "kr": sim_k, "q": q, "m": m}
        check(x, o, lse, only=[b for b in range(B) if ok[b]])
        if not tree:
            continue
        # keep a path of every tree that got its rows, and give the rest back
        new = [n if o_ else 0 for n, o_ in zip(new, ok)]
        leaf = [rng.randint(-1, n - 1) if n else -1 for n in new]
        sub = [p if o_ else [] for p, o_ in zip(parent, ok)]
        cu = [sum(new[:b]) for b in range(B + 1)]
        kept, acc = ints([7] * B), ints([7] * cu[-1])
        gva.gva_tree_commit(d, v, kr, lens, ints(cu), ints(sum(sub, [])), ints(leaf), kept, acc if cu[-1] else None, paging=pg,
                            block_table=table)
        final = []
        for b in range(B):
            path = ref.ancestors(ref.parents(sub[b]), leaf[b]) if leaf[b] >= 0 else []
            old_v, old_k = sim_v[b].clone(), sim_k[b].clone()
            for k, a in enumerate(path):
                sim_v[b, :, before[b] + k], sim_k[b, before[b] + k] = old_v[:, before[b] + a], old_k[before[b] + a]
            final.append(sim_lens[b] - new[b] + len(path))
        assert kept.tolist() == final
        tables([a - b for a, b in zip(final, sim_lens)], 0)
        assert sim_lens == final
    assert refused > 0
