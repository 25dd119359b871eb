"""Rows of doubles with more than 65536 tiles of 32 columns: more than a grid's second index counts.  Tolerances: those of test_gpu_entropy."""
import pytest
import torch

from tests.test_gpu_entropy import check, make, run

pytestmark = pytest.mark.gpu


def test_more_columns_of_doubles_than_a_grids_second_index_has_tiles():
    T, V, D = 5, 17, 32 * 65536 + 33
    print("entropy T=%d V=%d D=%d double" % (T, V, D), flush=True)
    h, w, targets = make(1, T, V, D, torch.float64, outside=0.0)
    for reduction in ("mean", "none"):
        check(h, w, targets, reduction, *run(h, w, targets, reduction))
