"""Token caches where calls go wrong first: work without cells beside work with some, scales and values at the
ends of their range, long sums, rows computed again by the definition, arguments that do not fit.  Attention
against the 64-bit form of test_gpu_tokens.py, with its tolerances."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

from test_gpu_tokens import M, Batch, ctx  # noqa: E402,F401


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("window,pos", [(0, 0), (32, 900)])
def test_chunks_without_cells_after_short_ones(M, ctx, d, window, pos):  # noqa: F811
    """Blocks that go from one short piece with cells to several of twice the rows without any (no cells held,
    or a window past them): zeros there, no wait that runs out."""
    new = [128] * 200 + [256] * 300
    at = [70] * 200 + [pos] * 300
    kv = [198] * 200 + [0 if window == 0 else 60] * 300
    t = Batch(M, ctx, new, at, kv, 2, 2, d, 16, "bf16", "same", window=window)
    for _ in range(2):
        out, lse = t.check()
        assert not bool(out[200 * 128:].any()) and bool((lse[200 * 128:] == -math.inf).all())
