"""More token rows than 32 bits hold are refused by the attention calls, not cut to
their last 32 bits."""
import pytest
import torch

pytestmark = pytest.mark.gpu

MANY = 2**32 + 3


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.int8])
def test_rows(dtype):
    import paper_2609_10264_amd as mvk
    cache = mvk.KVCache.allocate(2, 1, 16, 8, dtype=dtype)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    seqs = mvk.Sequences(i32([[0]]), i32([5]), i32([0, 3]))
    rows = lambda: torch.zeros((1, 1, 8), dtype=torch.bfloat16, device="cuda").expand(MANY, 1, 8)  # noqa: E731
    for call in (lambda: mvk.paged_attention(rows(), cache, seqs, out=rows()),
                 lambda: mvk.cache_read(cache, seqs, k_out=rows(), v_out=rows())):
        with pytest.raises(mvk.MvkError) as e:
            call()
        assert e.value.status == mvk._lib.MVK_ERANGE
