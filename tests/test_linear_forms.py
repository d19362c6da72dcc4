"""How products are cut: the sizes that the GPU tests compare are those of every kernel, tile and way of laying out.  No GPU is needed."""
import ctypes

import pytest

from paper_2207_10741_amd import layers as L
from tests.linear_forms import FORMS, desc_of, described


@pytest.mark.parametrize("size,form", FORMS, ids=lambda v: "x".join(str(p) for p in v))
def test_sizes_are_cut_as_the_table_says(size, form):
    assert described(L.linear_cut(desc_of(*size))) == form


def test_the_table_has_every_form():
    """Every form that a grid of sizes is cut into."""
    forms = {form for _, form in FORMS}
    for rows in (1, 16, 17, 33, 50, 65, 128, 300, 700, 1024, 2048, 4100, 8192, 16000):
        for n in (16, 100, 260, 1000, 1500, 3000, 5000, 8192, 16384):
            for k in (1, 40, 64, 200, 400, 512, 1000, 2048, 4096, 8192):
                for odd in ("", "x", "w", "xw"):
                    form = described(L.linear_cut(desc_of(rows, k, n, odd)))
                    assert form in forms, (rows, k, n, odd, form)


def test_refusals():
    cut = L.LinearCut()
    assert L.lib().fc_linear_cut_of(None, ctypes.byref(cut)) == -1 and L.lib().fc_linear_cut_of(ctypes.byref(desc_of(1, 8, 8, "")), None) == -1
    assert L.lib().fc_linear_cut_of(ctypes.byref(desc_of(1, 0, 8, "")), ctypes.byref(cut)) == -2
