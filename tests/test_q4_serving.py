"""The 4-bit step, the accumulated weights and the eviction at the sizes that
serving runs them at (many tiles a wave, absorption outside the launch, several
tiles a workgroup, selection over blocks), and what their plans and sizes refuse."""

import ctypes

import pytest

from paper_2609_13285_amd import gva
from test_q4_evict import A, dims, step_status, weights_status

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
