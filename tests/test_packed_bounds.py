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
