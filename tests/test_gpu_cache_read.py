"""mvk_cache_read on a given stream, where the call allocates its rows."""
import pytest
import torch

from tests import cache8_ref as c8
from tests.test_gpu_cache8 import BF, Append

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


@pytest.mark.parametrize("cache", [c8.E4M3, c8.I8, BF])
def test_rows_that_the_call_allocates_are_zeroed_before_they_are_written(cache):
    """The zeros of rows without an entry are of the stream that writes the others: filled by the
    current stream, which is late here, they would come after them."""
    import paper_2609_10264_amd as mvk
    a = Append([40, 17, 2], [23, 5, 4], 2, 64, cache)
    a.call()
    torch.cuda.synchronize()
    want = mvk.cache_read(a.cache, a.seqs, tokens=40)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    junk = [torch.full((40, 2, 64), 7.0, dtype=BF, device="cuda") for _ in range(4)]
    del junk  # (the memory that the call is given holds something)
    torch.cuda.synchronize()
    torch.cuda._sleep(200_000_000)  # about 0.1 s
    got = mvk.cache_read(a.cache, a.seqs, tokens=40, stream=side)
    torch.cuda.synchronize()
    for x, y in zip(got, want):
        assert bool((y != 0).any()) and torch.equal(x, y)
        assert bool((x[28:30] == 0).all()) and bool((x[32:] == 0).all())  # without an entry, of no sequence
