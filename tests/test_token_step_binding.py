"""CPU-side checks of the rotation's and the trees' part of the C ABI and of what the binding refuses: layouts, calls without
a handle, arrays that do not fit."""
import ctypes

import numpy as np
import pytest

from test_library_abi import _c_layout, libpath  # noqa: F401

from paper_2607_18582_gb300 import mure


def test_rotary_struct_layout_matches_header(tmp_path):
    names = [f for f, _ in mure._RotaryDesc._fields_]
    size, offs = _c_layout(tmp_path, "mure_rotary_desc", names)
    assert ctypes.sizeof(mure._RotaryDesc) == size
    assert [getattr(mure._RotaryDesc, f).offset for f in names] == offs


def test_null_handles_are_refused(libpath):  # noqa: F811
    L, out = mure.lib(), ctypes.c_void_p()
    b = mure._TokensBatch()
    assert L.mure_rotary_create(None, ctypes.byref(mure._RotaryDesc()), ctypes.byref(out)) == 1
    assert L.mure_tokens_plan_create_tree(None, ctypes.byref(b), None, ctypes.byref(out)) == 1
    assert L.mure_tokens_plan_set_tree(None, ctypes.byref(b), None) == 1
    assert L.mure_tokens_rotate(None, None, None, None, 0, None, None, None, None) == 1
    assert L.mure_tokens_append_rotated(None, None, None, None, 0, None, None, None, None) == 1
    assert L.mure_tokens_copy_pages(None, None, 0, None, None) == 1
    assert L.mure_tokens_keep(None, None, None, None) == 1
    L.mure_rotary_free(None)


@pytest.mark.parametrize("bad", [dict(freq=[1.0] * 3), dict(axis=[0] * 5), dict(axis=[0, 0, 0, -1]), dict(axis=[0, 0, 0, 256]),
                                 dict(axis=[0, 0, 0, 0.5]), dict(q_weight=np.ones(7)), dict(k_weight=np.ones(9)),
                                 dict(head_dim=2 ** 32 + 8), dict(n_axes=2 ** 32 + 1)])
def test_rotary_arrays(bad):
    """(Looked at before the context is.)"""
    with pytest.raises(ValueError):
        mure.mure_rotary_create(None, **{**dict(head_dim=8, rot_dim=8), **bad})


class _Plan:
    n_heads, n_new, n_seqs = 2, 3, 2


def test_kept_lists_and_pages():
    for bad in ([[0]], [[0], [1], []], [[0.5], []], [[2 ** 31], []]):
        with pytest.raises(ValueError):
            mure.mure_tokens_keep(None, _Plan, bad)
    for a, b in (([0], [1, 2]), ([0.5], [1]), ([0], [2 ** 31])):
        with pytest.raises(ValueError):
            mure.mure_tokens_copy_pages(None, a, b)
