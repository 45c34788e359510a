"""The example of trees runs, and its texts do not depend on the guesses (fp32 cells; choices are compared, not losses)."""
import os
import sys

import numpy as np
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

from conftest import ROOT  # noqa: E402


@pytest.fixture(scope="module")
def example():
    from paper_2607_18582_gb300 import build
    build.build()
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    import token_trees
    return token_trees


@pytest.mark.parametrize("mutants,depth", [(6, 2), (1, 3), (12, 1)])
def test_texts_are_the_original_s(example, mutants, depth):
    r = example.run(prompts=8, mutants=mutants, steps=5, depth=depth)
    assert r["by_tree"] == r["alone"]
    kept = np.array(r["kept"])
    assert kept.shape == (5, 8) and kept.min() >= 1 and kept.max() <= depth + 1 and kept.max() > 1


def test_e4m3_cells_run(example):
    r = example.run(prompts=4, steps=3, form="e4m3")
    assert all(len(t) >= 3 for t in r["by_tree"])
