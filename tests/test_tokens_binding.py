"""What the Python binding of the token caches makes of a batch's arrays, on the CPU."""
import numpy as np
import pytest

from paper_2607_18582_gb300 import mure


def batch(new=(2,), pos=(14,), kv=(16,), table=((0,),)):
    b, keep = mure._tokens_batch(4, new, pos, kv, table, 0, 0, 0.0)
    return [np.asarray(a) for a in keep]


@pytest.mark.parametrize("kind", [list, np.int32, np.int64, np.uint8, np.float64])
def test_whole_numbers_of_any_type(kind):
    make = (lambda x: list(x)) if kind is list else (lambda x: np.array(x, kind))
    got = batch(make([1, 0, 3]), make([5, 6, 7]), make([6, 6, 10]), np.array([[1, 2], [3, 4], [5, 6]], None if kind is list else kind))
    assert [g.tolist() for g in got] == [[1, 0, 3], [5, 6, 7], [6, 6, 10], [[1, 2], [3, 4], [5, 6]]]
    assert all(g.dtype == np.int32 and g.flags.c_contiguous for g in got)


def test_empty_batches():
    assert [g.size for g in batch([], [], [], np.zeros((0, 1), np.int32))] == [0, 0, 0, 0]


@pytest.mark.parametrize("name", ["new", "pos", "kv"])
@pytest.mark.parametrize("value", [2 ** 32 + 2, 2 ** 31, -2 ** 33 + 1, np.uint64(2 ** 63), 1e12, float("nan"), float("inf")])
@pytest.mark.parametrize("kind", [list, np.array])
def test_lengths_do_not_wrap(name, value, kind):
    with pytest.raises((ValueError, OverflowError)):
        batch(**{name: kind([value])})


def test_page_ids_do_not_wrap():
    """A page id past 32 bits stays one that the library refuses where it reads it, and is let be where it does not."""
    assert batch(table=np.array([[3, 2 ** 32]], np.int64))[3].tolist() == [[3, -1]]
    assert batch(table=np.array([[0xFFFFFFFF, 7]], np.uint32))[3].tolist() == [[-1, 7]]


@pytest.mark.parametrize("bad", [dict(new=(1.5,)), dict(kv=(16.25,)), dict(table=((0.5,),)), dict(new=("a",)), dict(pos=(None,))])
def test_what_is_no_whole_number_is_refused(bad):
    with pytest.raises((ValueError, TypeError)):
        batch(**bad)


def test_shapes():
    for bad in (dict(new=(1, 2)), dict(kv=()), dict(table=(0, 1)), dict(table=np.zeros((0, 4), np.int32))):
        with pytest.raises(ValueError):
            batch(**bad)


@pytest.mark.parametrize("bad", [dict(n_heads=2 ** 32 + 4), dict(window=2 ** 32 + 16), dict(window=2 ** 31), dict(sinks=-2 ** 32 + 4)])
def test_single_numbers_do_not_wrap(bad):
    args = dict(n_heads=4, new_len=(2,), pos=(14,), kv_len=(16,), page_table=((0,),), window=0, sinks=0, scale=0.0)
    with pytest.raises(ValueError):
        mure._tokens_batch(**{**args, **bad})


@pytest.mark.parametrize("bad", [dict(n_kv_heads=2 ** 32 + 2), dict(head_dim=2 ** 32 + 64), dict(page_size=2 ** 32 + 16),
                                 dict(n_pages=2 ** 64 + 4)])
def test_a_cache_s_sizes_do_not_wrap(bad):
    """(They are looked at before the context is.)"""
    with pytest.raises(ValueError):
        mure.mure_tokens_create(None, **{**dict(n_kv_heads=2, head_dim=64, page_size=16, n_pages=4), **bad})
