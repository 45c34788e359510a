"""CPU-side checks of the token caches' part of the C ABI: the binding's structures have the header's
layout, and calls without a context or a handle are refused."""
import ctypes

from test_library_abi import _c_layout, libpath  # noqa: F401


def test_token_struct_layouts_match_header(tmp_path):
    from paper_2607_18582_gb300 import mure
    for struct, cls in (("mure_tokens_desc", mure._TokensDesc), ("mure_tokens_batch", mure._TokensBatch),
                        ("mure_tokens_rows", mure._TokensRows)):
        names = [f for f, _ in cls._fields_]
        size, offs = _c_layout(tmp_path, struct, names)
        assert ctypes.sizeof(cls) == size, struct
        assert [getattr(cls, f).offset for f in names] == offs, struct


def test_null_handles_are_refused(libpath):  # noqa: F811
    from paper_2607_18582_gb300 import mure
    L, out = mure.lib(), ctypes.c_void_p()
    assert L.mure_tokens_create(None, ctypes.byref(mure._TokensDesc()), ctypes.byref(out)) == 1
    assert L.mure_tokens_plan_create(None, ctypes.byref(mure._TokensBatch()), ctypes.byref(out)) == 1
    assert L.mure_tokens_plan_set(None, ctypes.byref(mure._TokensBatch())) == 1
    assert L.mure_tokens_buffers(None, ctypes.byref(mure._TokensDesc())) == 1
    assert L.mure_tokens_append(None, None, None, None) == 1
    assert L.mure_tokens_read(None, None, 0, None, None) == 1
    assert L.mure_tokens_attend(None, None, None, None, None) == 1
    assert L.mure_synchronize(None) == 1
    L.mure_tokens_free(None)
    L.mure_tokens_plan_free(None)
