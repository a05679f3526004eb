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


def test_more_kept_entries_than_one_launch_has_threads():
    """2^26 entries and some, rows of 512 that are not aligned; pages of one row each, and
    a destination of which the pool holds the first and the last pages."""
    import paper_2609_10264_amd as mvk
    page, dim, n, dpage = 2**20, 512, 2**26 + 100, 64
    print(f"eviction of {n} entries", flush=True)
    pages = -(-n // page)
    one = torch.randn((2, pages * dim + 1), device="cuda").to(torch.bfloat16)[:, 1:]
    K, V = (x.view(pages, 1, 1, dim) for x in one)
    src = mvk.KVCache(K.expand(pages, 1, page, dim), V.expand(pages, 1, page, dim))
    dst = mvk.KVCache.allocate(3, 1, dpage, dim)
    width = -(-n // dpage)
    dtable = torch.full((1, width), -1, dtype=torch.int32, device="cuda")
    dtable[0, 0], dtable[0, -2], dtable[0, -1] = 0, 1, 2
    w = torch.zeros((1, 1, pages * page), device="cuda")
    lens = torch.tensor([n], dtype=torch.int32, device="cuda")
    table = torch.arange(pages, dtype=torch.int32, device="cuda").view(1, pages)
    kept, m = mvk.cache_evict(src, mvk.Sequences(table, lens), w, dst, dtable, n)
    torch.cuda.synchronize()
    assert m.tolist() == [n] and torch.equal(kept[0, 0], torch.arange(n, dtype=torch.int32, device="cuda"))
    for got, pool in ((dst.K, K), (dst.V, V)):
        assert torch.equal(got[0, 0], pool[0, 0].expand(dpage, dim))
        assert torch.equal(got[1, 0], pool[-1, 0].expand(dpage, dim))
        last = n - (width - 1) * dpage
        assert torch.equal(got[2, 0, :last], pool[-1, 0].expand(last, dim)) and not bool(got[2, 0, last:].any())
