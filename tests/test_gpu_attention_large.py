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


def test_a_large_batch_of_prompts():
    """More token rows than the tile kernels once took: 96 prompts of up to 4096."""
    import paper_2609_10264_amd as mvk
    S, H, hk, dim, page = 96, 64, 8, 16, 64
    print(f"attention of {S} prompts", flush=True)
    g = torch.Generator(device="cuda").manual_seed(3)
    new = [4096 - 7 * (s % 11) for s in range(S)]
    T, width = sum(new), 64
    q = torch.randn((T, H, dim), generator=g, device="cuda").to(torch.bfloat16)
    K, V = (torch.randn((S * width, hk, page, dim), generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    table = torch.randperm(S * width, generator=g, device="cuda").to(torch.int32).view(S, width)
    starts, lens = ref.starts(new), torch.tensor(new, dtype=torch.int32)
    w = torch.full((S, hk, width * page), -5.0, device="cuda")
    out = mvk.paged_attention(q, mvk.KVCache(K, V), mvk.Sequences(table, lens.cuda(), starts.cuda(), max_new=4096), weights_out=w)
    torch.cuda.synchronize()
    hK, hV, htable = K.cpu(), V.cpu(), table.cpu()
    for s in (0, 1, 50, S - 1):
        # some rows of the sequence, from the definition: each as the last token of a shorter one
        a, n = int(starts[s]), new[s]
        for i in (0, 1, 63, 64, 2047, n - 1):
            r = ref.Attention(q[a + i:a + i + 1].cpu(), hK, hV, htable[s:s + 1], torch.tensor([i + 1]),
                              torch.tensor([0, 1]))
            _within(out[a + i:a + i + 1], r.o, r.o_err, (s, i))
        total = w[s, :, :n].double().sum(1)
        # each token's weights of a head sum to one, up to 4 dx + 2^-18, dx = (dim + 8) 2^-24 |scale| |q| . |k| < 2^-16
        assert bool(((total - n * H // hk).abs() <= n * H // hk * 2.0**-13).all()) and bool((w[s, :, n:] == -5.0).all())


# many more new tokens than entries, over several tiles, in both forms
@pytest.mark.parametrize("hint", [1, 3000])
@pytest.mark.parametrize("heads", [2, 16])
def test_more_new_tokens_than_entries(hint, heads):
    import paper_2609_10264_amd as mvk
    new, lens = [3000, 1, 700, 300, 40], [5, 1, 130, 0, 200]
    g = torch.Generator().manual_seed(6)
    table, pages = ref.lay_out(lens, 16, 1)
    K, V = (torch.randn((pages, 2, 16, 64), generator=g).to(torch.bfloat16) for _ in range(2))
    q = torch.randn((sum(new), heads, 64), generator=g).to(torch.bfloat16)
    lens, starts = torch.tensor(lens, dtype=torch.int32), ref.starts(new)
    out, lse = torch.full_like(q, 9.0).cuda(), torch.zeros((sum(new), heads), device="cuda")
    mvk.paged_attention(q.cuda(), mvk.KVCache(K.cuda(), V.cuda()),
                        mvk.Sequences(table.cuda(), lens.cuda(), starts.cuda(), max_new=hint), out=out, lse=lse)
    torch.cuda.synchronize()
    r = ref.Attention(q, K, V, table, lens, starts)
    _within(out, r.o, r.o_err, "o")
    _within(lse, r.lse, r.lse_err, "lse")
