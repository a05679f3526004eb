"""Collected weights where sequences' chains of rows are long enough for groups of
waves, against the definition in 64 bits: every head size and type of cache, sequences
of few rows and none beside long ones, the last rows of a tile, wide tables."""
import pytest
import torch

from tests import cache8_ref as c8
from tests.test_gpu_attention import BF, HF, Problem, _check
from tests.test_gpu_attention8 import Problem8

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


LENS, NEW = [300, 40, 0, 705, 129], [300, 3, 0, 421, 129]


@pytest.mark.parametrize("dim", [64, 80, 128, 192, 256])
@pytest.mark.parametrize("cache", [BF, HF, c8.E4M3, c8.I8])
def test_heads_and_caches(dim, cache):
    if cache in (BF, HF):
        _check(Problem(LENS, NEW, 8, 2, dim, dtype=cache))
    else:
        _check(Problem8(cache, LENS, NEW, 8, 2, dim))


@pytest.mark.parametrize("heads", [1, 3, 7])
@pytest.mark.parametrize("cache", [BF, c8.E4M3])
def test_last_rows(heads, cache):
    """Rows that end within a tile, at its end and one behind it."""
    for c in (255, 256, 257, 289):
        pr = (Problem(*([c + 70], [c], heads, 1, 64)) if cache == BF else Problem8(cache, [c + 70], [c], heads, 1, 64))
        _check(pr)


@pytest.mark.parametrize("dim", [128, 256])
def test_wide_table(dim):
    pr = Problem(LENS, NEW, 8, 2, dim)
    pr.table = torch.cat([pr.table, torch.full((len(LENS), 5 * pr.table.shape[1]), -7, dtype=torch.int32)], 1)
    pr.cap = pr.table.shape[1] * 16
    _check(pr)
