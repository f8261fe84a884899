"""The 4-bit step, the accumulated weights and the eviction at the sizes that
serving runs them at (many tiles a wave, absorption outside the launch, several
tiles a workgroup, selection over blocks), and what their plans and sizes refuse."""

import ctypes

import pytest
import torch

from paper_2609_13285_amd import gva
from test_q4_evict import A, dims, step_status

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
