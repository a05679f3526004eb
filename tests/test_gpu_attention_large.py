"""Attention calls of more rows, entries and tiles than fit smaller counts."""
import pytest
import torch

from tests import attention_ref as ref
from tests.test_gpu_attention import _within

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def test_more_rows_than_one_launch_has_threads():
    """2^26 rows and some on the general path; the last tokens see entries, the others none."""
    import paper_2609_10264_amd as mvk
    T, H, n, page = 2**20 + 3, 64, 5, 8
    print(f"attention of {T} x {H} rows", flush=True)
    g = torch.Generator().manual_seed(2)
    K, V = (torch.randn((2, 1, page, 1), generator=g) for _ in range(2))
    tail = torch.randn((8, H, 1), generator=g)
    q = torch.zeros((T, H, 1), device="cuda")
    q[-8:] = tail.cuda()
    table, lens = torch.tensor([[0], [1]], dtype=torch.int32), torch.tensor([3, n], dtype=torch.int32)
    starts = torch.tensor([0, T - 4, T], dtype=torch.int32)
    out = torch.full_like(q, 9.0)
    mvk.paged_attention(q, mvk.KVCache(K.cuda(), V.cuda()), mvk.Sequences(table.cuda(), lens.cuda(), starts.cuda()), out=out)
    torch.cuda.synchronize()
    r = ref.Attention(tail, K, V, table, torch.tensor([3, n]), torch.tensor([0, 4, 8]))
    _within(out[-8:], r.o, r.o_err, "the last rows")
    assert r.covered.all() and bool((out[:-8] == 0).all())
