"""The packed calls where they could go wrong without an ordinary test showing it:
the order of reads and copies in LDS, offsets past 32 bits, the largest sizes,
plans for other devices, many splits and sequences, values at the ends of their
types, captured bookkeeping."""

import os
import re
import shutil
import subprocess

import pytest
import torch

import packed_ref as ref
from gpu_helpers import note
from paper_2609_13285_amd import gva
from test_packed import A, BAD, UNSUP, call, check, dims, ints, problem, prompt_status, tree_status, trees, upload

gpu = pytest.mark.gpu
LLVM = "/opt/rocm/llvm/bin"


# ------------------------------------------- sets of one wave share their queries
def listings(tmp_path, pattern):
    """{symbol: instructions} of the library's own kernels whose name matches."""
    lib = shutil.copy(gva.LIB_PATH, tmp_path)
    subprocess.run([f"{LLVM}/llvm-objdump", "--offloading", lib], check=True, capture_output=True, cwd=tmp_path)
    out = {}
    for name in sorted(os.listdir(tmp_path)):
        if not name.endswith("gfx950"):
            continue
        path = os.path.join(tmp_path, name)
        syms = subprocess.run([f"{LLVM}/llvm-readelf", "-sW", path], check=True, capture_output=True, text=True).stdout
        for sym in sorted({w for w in syms.split() if re.search(pattern, w) and "." not in w}):
            text = subprocess.run([f"{LLVM}/llvm-objdump", "-d", f"--disassemble-symbols={sym}", path], check=True,
                                  capture_output=True, text=True).stdout
            out[sym] = [x.split("//")[0].strip() for x in text.splitlines() if x.startswith("\t")]
    return out


@pytest.mark.skipif(not os.path.exists(f"{LLVM}/llvm-objdump"), reason="no disassembler")
def test_shared_queries_are_read_before_copies_overwrite_them(tmp_path):
    """Sets of one wave pass their queries' parts on through tile buffers: behind the barrier
    after which they are read, and ahead of the first copy into LDS, there has to be another one
    that waits for those reads."""
    found = 0
    for sym, code in listings(tmp_path, r"window_kernelILi\d+ELi\d+ELi1ELi[34]E").items():
        d_v = int(re.search(r"window_kernelILi(\d+)E", sym).group(1))
        parts = 3 * d_v // 16
        starts = [i for i, x in enumerate(code) if x.startswith("s_barrier")]
        shared = [i for i in starts if sum(x.startswith("ds_read_b128") for x in code[i + 1:i + 1 + 2 * parts]) >= parts]
        assert len(shared) == 1, sym
        rest = code[shared[0] + 1:]
        end = next(i for i, x in enumerate(rest) if x.startswith("s_barrier") or re.match(r"buffer_load.* lds", x))
        assert rest[end].startswith("s_barrier"), f"{sym}: {rest[end]}"
        reads = [i for i, x in enumerate(rest[:end]) if x.startswith("ds_read_b128")]
        assert len(reads) == parts, sym
        assert any(x.startswith("s_waitcnt") and "lgkmcnt(0)" in x for x in rest[reads[-1]:end]), sym
        found += 1
    assert found == 6                                  # d_v 64 and 128 at three widths of the positional key


@gpu
@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("d_v,d_r", [(64, 16), (64, 64), (128, 16), (128, 64)])
def test_sets_of_one_wave_repeat_themselves(d_v, d_r, tree):
    """Sequences whose sets start a tile apart, or have none, many workgroups at once: bit for bit the same each time."""
    B = 96
    lens, new = [(37 * b) % 640 + 1 for b in range(B)], [1 + b % 4 for b in range(B)]
    x = problem(lens, new, 8, 1, d_v, 64, d_r, 1024, 32, seed=d_v + d_r, parent=trees(new, 3) if tree else None)
    note(f"sets of one wave {d_v}/{d_r} tree={tree}")
    dev = upload(x)
    first = call(x, 1, 0, dev)
    check(x, *first)
    for _ in range(20):
        o, lse = call(x, 1, 0, dev)
        assert torch.equal(o, first[0]) and torch.equal(lse, first[1])


# ------------------------------------------------------------- places and sizes
@gpu
@pytest.mark.parametrize("tree", [False, True])
def test_sequences_past_sixty_four_gigabytes(tree):
    """34 streams of almost 2 GiB each: their offsets in 16-byte pieces pass 2^32 within a sequence and
    between the two.  Only the rows that the lengths cover are written, or read."""
    H = G = 34
    d_v, d_c, d_r, T = 128, 32, 16, (((1 << 31) - (1 << 24)) // 256 - 1) // 32 * 32
    assert (G - 1) * T * d_v * 2 // 16 > 1 << 32
    size = 2 * G * T * d_v * 2
    if torch.cuda.mem_get_info()[0] < size + (4 << 30):
        pytest.skip("too little memory on this GPU")
    note(f"sequences of {size >> 31} GiB tree={tree}")
    v = torch.empty(2, G, T, d_v, dtype=torch.bfloat16, device="cuda")
    kr = torch.empty(2, T, d_r, dtype=torch.bfloat16, device="cuda")
    try:
        for new in ([3, 2], [40, 70]):                 # sets of one wave, and one set of four
            lens, rows = [new[0] + 30, new[1] + 90], 160
            x = problem(lens, new, H, G, d_v, d_c, d_r, rows, 0, seed=30 + new[0], parent=trees(new, 2) if tree else None)
            v[:, :, :rows], kr[:, :rows] = (t.cuda() for t in (gva.tiled(x["v"]), gva.tiled(x["kr"])))
            x["d"] = gva.make_dims(2, H, G, d_v, d_c, d_r, T, "bf16")
            for S, split in ((1, 0), (3, 64)):
                check(x, *call(x, S, split, (v, kr)))
    finally:
        del v, kr
        torch.cuda.empty_cache()


@gpu
def test_maps_of_all_rows_that_an_int_counts():
    """n_rows = 2^31 - 1: the last rows are written, and nothing around them."""
    n, pad, R = (1 << 31) - 1, 4097, 32
    d, pg = dims(batch=3, t_max=4 * R), gva.GvaPaging(R, 4, 12)
    if torch.cuda.mem_get_info()[0] < 5 * n + (4 << 30):
        pytest.skip("too little memory on this GPU")
    note("maps of 2^31 - 1 rows")
    raw = torch.full((n + 2 * pad,), 7, dtype=torch.int32, device="cuda")
    lens, new, table, free = [5, 0, 40], [2, 33, -10], [[3, -7, -7, -7], [-7] * 4, [9, 1, -7, -7]], list(range(12))
    try:
        out = {k: ints([7] * s) for k, s in (("lens", 3), ("n_free", 1), ("cu", 4))}
        gva.gva_page_tables(d, pg, ints(lens), ints(new), ints(table), ints(free), ints([6]), out["lens"], out["n_free"], out["cu"],
                            slot=raw[pad:pad + n])
        want = ref.page_tables(lens, new, table, free, 6, 64, 4 * R, R, 12)
        assert all(out[k].tolist() == (want[k] if k != "n_free" else [want[k]]) for k in out)
        assert raw[pad:pad + 64].tolist() == want["slot"]
        for part in raw[pad + 64:pad + n].split(1 << 28):
            assert bool((part == -1).all())
        assert bool((raw[:pad] == 7).all()) and bool((raw[pad + n:] == 7).all())
    finally:
        del raw
        torch.cuda.empty_cache()


# ---------------------------------------------------------------------- plans
@pytest.mark.parametrize("H,G,T,L,n", [(16, 2, 512, 330, 2), (16, 2, 512, 312, 8), (16, 4, 2048, 1705, 64), (32, 4, 4096, 2235, 32)])
def test_plans_are_for_the_device_that_they_are_asked_for(H, G, T, L, n):
    """Four times the sequences on four times the compute units: as many workgroups a unit, so the same kernel and splits.
    The times that do not scale with the units (partials through memory) are small at these sizes."""
    plans = []
    for k in (1, 4):
        d = dims(batch=16 * k, n_heads=H, n_groups=G, t_max=T)
        lens, new = (torch.full((16 * k,), x, dtype=torch.int32) for x in (L, n))
        plans.append(gva.gva_packed_pick_splits(d, lens, new, n_cu=64 * k))
    assert plans[0] == plans[1]


@pytest.mark.parametrize("attend", [prompt_status, tree_status])
def test_calls_of_more_threads_than_a_launch_has_are_refused(attend):
    """2^32 threads: of the merge (a wave per row and head) and of the attention (a workgroup per block, split and group)."""
    n = 1 << 20
    merge = dims(batch=1, n_heads=64, n_groups=64, d_v=64, d_c=32)
    assert attend(merge, n=n, S=2, lens=None) == UNSUP
    assert attend(merge, n=n - 1, S=2, lens=None) == BAD           # (a missing pointer, looked for later)
    blocks = dims(batch=1, n_heads=32, n_groups=32, d_v=64, d_c=32)
    assert attend(blocks, n=n, S=63, lens=None) == BAD             # 2^13 blocks, 63 splits, 2^5 groups, 2^8 threads
    for d, S in ((blocks, 64), (dims(batch=1 << 18, n_heads=64, n_groups=64, d_v=64, d_c=32), 1)):
        assert attend(d, n=n, S=S, lens=None) == UNSUP
        with pytest.raises(gva.GvaError):
            gva.gva_packed_workspace_size(d, n, S)
    assert gva.gva_packed_pick_splits(merge, None, None, n) == (1, 0)


@pytest.mark.parametrize("attend", [prompt_status, tree_status])
@pytest.mark.parametrize("d_v,dtype,size", [(64, "bf16", 2), (128, "bf16", 2), (64, "f32", 4), (128, "f32", 4)])
def test_the_longest_capacity(attend, d_v, dtype, size):
    """T rows of values below 2^31 - 2^24 bytes; paged, with pages of a 32nd of it."""
    most = ((1 << 31) - (1 << 24)) // (d_v * size)
    R = most // 32 // 32 * 32
    for T, pg, want in ((most - 16, None, BAD), (most, None, UNSUP), (32 * (R - 32), gva.GvaPaging(R - 32, 32, 4), BAD),
                        (32 * (R + 32), gva.GvaPaging(R + 32, 32, 4), UNSUP)):
        assert attend(dims(d_v=d_v, dtype=dtype, t_max=T), pg=pg, table=A if pg else None, lens=None) == want, (T, pg)


# ------------------------------------------------- many splits, sequences, odd tiles
@gpu
@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("S,rows", [(64, 0), (65, 0), (130, 64), (200, 0), (256, 32), (256, 0)])
def test_many_splits(S, rows, tree):
    """Up to 256 splits, most of which have rows, some sequences with few of them."""
    lens, new = [8000, 9, 6500, 4097], [3, 9, 40, 1]
    for dtype in ("bf16", "f32"):
        x = problem(lens, new, 4, 2, 64, 32, 16, 8192, 64, dtype, seed=S, parent=trees(new, 4) if tree else None)
        note(f"{S} splits of {rows} {dtype} tree={tree}")
        check(x, *call(x, S, rows))


@gpu
@pytest.mark.parametrize("S", [1, 2])
def test_thousands_of_sequences(S):
    """More than 64 sequences a lane of the search for a workgroup's item; some without queries."""
    B = 5000
    lens, new = [(11 * b) % 65 for b in range(B)], [(b * b) % 4 for b in range(B)]
    x = problem(lens, new, 2, 2, 64, 32, 8, 64, 32, seed=S)
    note(f"{B} sequences, {S} splits")
    o, lse = call(x, S, 0)
    check(x, o, lse, only=set(range(0, B, 23)) | set(range(4090, 4105)) | set(range(B - 9, B)))
    assert not bool((lse == 77.0).any())               # and every row was written


@gpu
@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("T", [16, 48, 80, 272, 1040])
def test_capacities_that_end_inside_a_tile(T, tree):
    """Contiguous caches of 16 rows past a multiple of 32: the next sequence's rows begin within the last tile."""
    lens = [T, T - 15, T - 16, T, max(1, T - 17)]
    for n in (3, 40):
        new = [min(n, L) for L in lens]
        for dtype in ("bf16", "f32"):
            x = problem(lens, new, 8, 2, 128, 64, 24, T, 0, dtype, seed=T + n, parent=trees(new, n) if tree else None)
            note(f"capacity {T}, {n} queries {dtype} tree={tree}")
            dev = upload(x)
            for S, rows in ((1, 0), (3, 0), (4, 32)):
                check(x, *call(x, S, rows, dev))


@gpu
@pytest.mark.parametrize("cu", [[30, 10, 39, (1 << 31) - 1], [(1 << 31) - 1] * 4, [0, (1 << 31) - 1, 39, 39], [-1, -1, -1, 39]])
def test_the_largest_offsets(cu):
    """Offsets at the ends of their type: nothing outside the outputs is written."""
    x = problem([64, 90, 80], [20, 9, 10], 8, 2, 64, 64, 16, 96, 32, seed=16)
    dev, pad = upload(x), 4096
    note(f"offsets {cu}")
    for S in (1, 3):
        raw = torch.full((pad + 39 * 8 * 64 + pad,), 77.0, dtype=torch.bfloat16, device="cuda")
        rawl = torch.full((pad + 39 * 8 + pad,), 77.0, device="cuda")
        call(dict(x, cu=cu), S, 0, dev, o=raw[pad:-pad].view(39, 8, 64), lse=rawl[pad:-pad].view(39, 8))
        for r in (raw, rawl):
            assert bool((r[:pad] == 77.0).all()) and bool((r[-pad:] == 77.0).all())


# -------------------------------------------------- values at the ends of their types
def scores(x, h, t, b=0):
    """Head h's scores of row t of sequence b, one for every query, in 64 bits."""
    d, n = x["d"], x["new"][b]
    par = None if x["parent"] is None else ref.parents(x["parent"][b])
    see, pos = ref.window(x["lens"][b], n, par)
    q = x["q"][x["cu"][b]:x["cu"][b] + n, h].double()
    row = x["v"][b, h // (d.n_heads // d.n_groups), t].double()
    s = (q[:, :d.d_c] @ x["m"][h].double().t()) * row
    k = ref.rotate(q[:, d.d_c:], pos) * x["kr"][b, t].double()
    return (s.sum(-1) + k.sum(-1)) / (d.d_c + d.d_r) ** 0.5, see


def without(x, t, b=0):
    """What the queries of sequence b get from the rows but t: (o, lse, bounds)."""
    d, n, L = x["d"], x["new"][b], x["lens"][b]
    par = None if x["parent"] is None else ref.parents(x["parent"][b])
    see, pos = ref.window(L, n, par)
    see[:, t] = False
    v, kr = x["v"][b, :, :L].clone(), x["kr"][b, :L].clone()
    v[:, t], kr[t] = 0, 0
    return ref.attend(x["q"][x["cu"][b]:x["cu"][b] + n], x["m"], v, kr, see, pos, d.n_groups, d.torch_dtype)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("t", [10, 107])
@pytest.mark.parametrize("where", ["key", "value"])
def test_a_row_at_the_lowest_value(where, t, tree, dtype):
    """A key or value entry at the type's lowest value, in a row that all queries see or some: with a
    score near the lowest number the row is out of the sum, with one near the largest it has all the
    weight, and o is its values.  (Scores stay within fp32: the entry's factor is below 1.)"""
    lens, new = [120], [20]
    x = problem(lens, new, 4, 2, 64, 32, 16, 128, 0, dtype, seed=t, parent=[[-1] + [i // 2 for i in range(19)]] if tree else None)
    low = torch.finfo(x["d"].torch_dtype).min
    if where == "key":
        x["kr"][0, t, 3] = low
    else:
        x["v"][0, :, t, 5] = low
    note(f"lowest {where} in row {t} {dtype} tree={tree}")
    wo, wl, do, dl = without(x, t)
    seen = {True: 0, False: 0}
    for S, rows in ((1, 0), (3, 32)):
        o, lse = (u.cpu().double() for u in call(x, S, rows))
        for h in range(4):
            s, see = scores(x, h, t)
            assert float(s.abs().max()) * 1.4427 < 0.99 * float(torch.finfo(torch.float32).max)
            for i in range(20):
                if bool(see[i, t]) and float(s[i]) > 0:
                    seen[True] += 1
                    assert torch.equal(o[i, h], x["v"][0, h // 2, t].double()), (h, i)
                    # the query's parts (2^-17), products and sums of 80 entries, the scale, two logarithms' factors
                    assert abs(float(lse[i, h] / s[i]) - 1) <= 2.0 ** -15, (h, i)
                else:
                    seen[False] += bool(see[i, t])
                    assert bool(((o[i, h] - wo[i, h]).abs() <= do[i, h]).all()), (h, i)
                    assert float((lse[i, h] - wl[i, h]).abs()) <= float(dl[i, h]), (h, i)
    assert seen[True] > 4 and seen[False] > 4


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("t", [10, 107])
@pytest.mark.parametrize("bad", [float("inf"), float("-inf")])
def test_an_infinite_value_that_a_query_sees(bad, t, tree, dtype):
    """With a score of +inf, o and lse are NaN.  With one of -inf the row draws no weight, or the parts of
    the query make a NaN of it; nothing else is put in its place."""
    x = problem([120], [20], 4, 2, 64, 32, 16, 128, 0, dtype, seed=t, parent=[[-1] + [i // 2 for i in range(19)]] if tree else None)
    x["v"][0, :, t, 5] = bad
    note(f"{bad} in row {t} {dtype} tree={tree}")
    wo, wl, do, dl = without(x, t)
    some = 0
    for S, rows in ((1, 0), (3, 32)):
        o, lse = (u.cpu().double() for u in call(x, S, rows))
        for h in range(4):
            s, see = scores(x, h, t)
            for i in range(20):
                if bool(see[i, t]) and not float(s[i]) < 0:
                    some += 1
                    assert bool(torch.isnan(o[i, h]).all()) and bool(torch.isnan(lse[i, h])), (h, i)
                else:
                    ok = (o[i, h] - wo[i, h]).abs() <= do[i, h]
                    okl = (lse[i, h] - wl[i, h]).abs() <= dl[i, h]
                    if bool(see[i, t]):
                        ok |= torch.isnan(o[i, h])
                        okl |= torch.isnan(lse[i, h])
                    assert bool(ok.all()) and bool(okl), (h, i)
    assert some > 4


# ----------------------------------------------------------- captured bookkeeping
def step_state(seed):
    """A step's inputs: tables to build, rows to append, a tree to attend and commit, bf16, six sequences."""
    R, most, B, H, G, dv, dc, dr = 32, 6, 6, 8, 2, 64, 64, 16
    g = torch.Generator().manual_seed(seed)
    d, pg = gva.make_dims(B, H, G, dv, dc, dr, R * most, "bf16"), gva.GvaPaging(R, most, 30)
    lens, new = [40, 0, 64, 100, 5, 33], [12, 5, 1, 40, 0, -33]
    held = [-(-L // R) for L in lens]
    order = torch.randperm(30, generator=g).tolist()
    table, at = torch.full((B, most), -1, dtype=torch.int32), 0
    for b in range(B):
        table[b, :held[b]] = torch.tensor(order[at:at + held[b]], dtype=torch.int32)
        at += held[b]
    free = order[at:] + [-1] * at
    n = sum(max(k, 0) for k in new)
    par = trees([max(k, 0) for k in new], seed)
    pos = [L + len(ref.ancestors(p, i)) - 1 for L, p in zip(lens, par) for i in range(len(p))]
    leaf = [len(p) - 1 for p in par]
    dt = torch.bfloat16
    host = {"v0": torch.randn(30, G, R, dv, generator=g).to(dt), "k0": torch.randn(30, R, dr, generator=g).to(dt),
            "vn": torch.randn(n, G, dv, generator=g).to(dt), "kn": torch.randn(n, dr, generator=g).to(dt),
            "q": torch.randn(n, H, dc + dr, generator=g).to(dt), "m": (torch.randn(H, dv, dc, generator=g) / 8).to(dt)}
    s = {k: v.cuda() for k, v in host.items()}
    s.update(d=d, pg=pg, n=n, lens0=ints(lens), new=ints(new), table0=table.cuda(), free0=ints(free), n_free0=ints([30 - at]),
             parent=ints(sum(par, [])), pos=ints(pos), leaf=ints(leaf))
    return s


def step_buffers(s):
    B, n, H, dv = s["d"].batch, s["n"], s["d"].n_heads, s["d"].d_v
    size = {"lens": B, "n_free": 1, "cu": B + 1, "seq": n, "row": n, "slot": n, "kept": B, "acc": n}
    out = {k: torch.full((v,), 7, dtype=torch.int32, device="cuda") for k, v in size.items()}
    out.update(table=torch.empty_like(s["table0"]), free=torch.empty_like(s["free0"]), v=torch.empty_like(s["v0"]),
               kr=torch.empty_like(s["k0"]), o=torch.zeros(n, H, dv, dtype=torch.bfloat16, device="cuda"),
               lse=torch.zeros(n, H, device="cuda"))
    return out


def step(s, out, stream=None):
    """The whole step, from the same start each time."""
    for k, k0 in (("table", "table0"), ("free", "free0"), ("v", "v0"), ("kr", "k0")):
        out[k].copy_(s[k0])
    more = dict(paging=s["pg"], block_table=out["table"], stream=stream)
    gva.gva_page_tables(s["d"], s["pg"], s["lens0"], s["new"], out["table"], out["free"], s["n_free0"], out["lens"], out["n_free"],
                        out["cu"], out["seq"], out["row"], out["slot"], stream=stream)
    gva.gva_append_slots(s["d"], s["pg"], out["v"], out["kr"], s["vn"], s["kn"], out["slot"], s["pos"], stream=stream)
    gva.gva_tree_attention(s["d"], s["q"], s["m"], out["v"], out["kr"], out["lens"], out["cu"], s["parent"], out["o"], out["lse"],
                           **more)
    gva.gva_tree_commit(s["d"], out["v"], out["kr"], out["lens"], out["cu"], s["parent"], s["leaf"], out["kept"], out["acc"],
                        **more)


def same(a, b):
    return [k for k in a if not torch.equal(a[k], b[k])]


@gpu
def test_a_step_on_two_streams_and_in_a_graph():
    """Tables, slots, a tree and its commit: on two streams at once, each with buffers of its own, and
    captured, replayed several times with eager steps between."""
    s = step_state(5)
    note("a whole step, eager")
    base = step_buffers(s)
    step(s, base)
    want = ref.page_tables([40, 0, 64, 100, 5, 33], [12, 5, 1, 40, 0, -33], s["table0"].tolist(), s["free0"].tolist(),
                           int(s["n_free0"]), s["n"], 192, 32, 30)
    assert {k: base[k].tolist() for k in want} == {k: v if k != "n_free" else [v] for k, v in want.items()}
    note("two streams")
    sides = [torch.cuda.Stream(), torch.cuda.Stream()]
    outs = [step_buffers(s) for _ in sides]
    torch.cuda.synchronize()
    for _ in range(3):
        for side, out in zip(sides, outs):
            with torch.cuda.stream(side):
                step(s, out, side)
    torch.cuda.synchronize()
    for out in outs:
        assert same(base, out) == []
    note("a graph")
    out = step_buffers(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(s, out)
    for again in range(4):
        for t in out.values():
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert same(base, out) == [], again
        step(s, outs[0])
        torch.cuda.synchronize()
        assert same(base, outs[0]) == [], again


# --------------------------------------------------------- requests past the capacity
@gpu
def test_requests_past_the_capacity():
    """More rows than T are read as T: an empty sequence gets them, the packed offsets count T; another gets none."""
    R, T = 32, 128
    d, pg = dims(batch=3, t_max=T), gva.GvaPaging(R, 4, 20)
    note("requests past the capacity")
    table, free, out = ints([[-1] * 4] * 3), ints(list(range(20))), {k: ints([7] * s) for k, s in (("lens", 3), ("n", 1), ("cu", 4))}
    slot = ints([7] * 300)
    gva.gva_page_tables(d, pg, ints([0, 10, 0]), ints([T + 5, T - 9, 2]), table, free, ints([19]), out["lens"], out["n"], out["cu"],
                        slot=slot)
    assert out["lens"].tolist() == [T, 10, 2] and out["cu"].tolist() == [0, T, 2 * T - 9, 2 * T - 7] and out["n"].tolist() == [14]
    assert table.tolist() == [[18, 17, 16, 15], [-1] * 4, [14, -1, -1, -1]]
    assert slot[T:2 * T - 9].tolist() == [-1] * (T - 9) and slot[2 * T - 9:].tolist() == [14 * R, 14 * R + 1] + [-1] * (300 - 2 * T + 7)
