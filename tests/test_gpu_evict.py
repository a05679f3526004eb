"""Eviction from a paged cache by collected weight (mvk_cache_evict) against its
definition: whole numbers and copies, so every comparison is exact."""
import math

import pytest
import torch

from tests import attention_ref as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


BF, HF, F32, I32 = torch.bfloat16, torch.float16, torch.float32, torch.int32


def _run(lens, hk, dim, budget, recent, sinks, w=None, page=16, dpage=None, dtype=BF, seed=1, view=None):
    import paper_2609_10264_amd as mvk
    dpage = dpage or page
    g = torch.Generator().manual_seed(seed)
    table, pages = ref.lay_out(lens, page, seed)
    K, V = (torch.randn((pages, hk, page, dim), generator=g).to(dtype) for _ in range(2))
    cap = table.shape[1] * page
    if w is None:
        w = torch.rand((len(lens), hk, cap), generator=g)
    most = min(budget, cap)
    kept_n = [min(n, budget) for n in lens]
    dtable, dpages = ref.lay_out(kept_n, dpage, seed + 1)
    dtable = torch.cat([dtable, torch.full((len(lens), -(-most // dpage)), -1, dtype=I32)], 1)  # wide enough
    dst = mvk.KVCache(*(torch.full((dpages, hk, dpage, dim), 3.0, dtype=dtype, device="cuda") for _ in range(2)))
    src = mvk.KVCache(K.cuda(), V.cuda())
    if view:
        src, dst = view(src), view(dst)
    wo = torch.full((len(lens), hk, most + 3), -9.0, device="cuda")
    print(f"evict lens={lens[:6]} heads={hk} dim={dim} budget={budget} recent={recent} sinks={sinks}", flush=True)
    kept, n_out = mvk.cache_evict(src, mvk.Sequences(table.cuda(), torch.tensor(lens, dtype=I32).cuda()), w.cuda(), dst,
                                  dtable.cuda(), budget, recent=recent, sinks=sinks, weights_out=wo)
    torch.cuda.synchronize()
    assert n_out.tolist() == kept_n
    kept, wo, dK, dV = kept.cpu(), wo.cpu(), dst.K.cpu(), dst.V.cpu()
    touched = torch.zeros(dK.shape[:3], dtype=torch.bool)
    for s, n in enumerate(lens):
        m = kept_n[s]
        k_src, v_src = ref.entries(K, table[s], n), ref.entries(V, table[s], n)
        k_dst, v_dst = ref.entries(dK, dtable[s], m), ref.entries(dV, dtable[s], m)
        r = torch.arange(m)
        touched[dtable[s].long()[r // dpage], :, r % dpage] = True
        for h in range(hk):
            want = ref.evict(w[s, h, :n].tolist(), n, budget, recent, sinks)
            got = kept[s, h].tolist()
            assert got[:m] == want and all(x == -1 for x in got[m:]), (s, h)
            assert torch.equal(k_dst[h], k_src[h, want]) and torch.equal(v_dst[h], v_src[h, want])
            a, b = wo[s, h, :m], w[s, h, want]
            assert torch.equal(a.view(torch.int32), b.view(torch.int32))
            assert bool((wo[s, h, m:] == -9.0).all())
    assert bool((dK[~touched] == 3.0).all()) and bool((dV[~touched] == 3.0).all())


@pytest.mark.parametrize("budget,recent,sinks", [(1, 0, 0), (1, 1, 0), (1, 0, 1), (16, 4, 4), (64, 32, 32), (100, 17, 0),
                                                 (100, 0, 5), (63, 1, 1), (1000, 10, 10)])
def test_lengths_and_budgets(budget, recent, sinks):
    _run([0, 1, 2, 15, 63, 64, 65, 100, 101, 300], 3, 64, budget, recent, sinks)


@pytest.mark.parametrize("n", [1023, 1024, 1025, 4096, 5000, 20001])
@pytest.mark.parametrize("budget", [7, 512, 3333])
def test_long_rows(n, budget):
    _run([n, n // 2], 2, 16, budget, 3, 2, page=64)


def test_very_long_row():
    _run([150001, 9], 1, 8, 70000, 1000, 4, page=256)


@pytest.mark.parametrize("dim,dtype", [(1, BF), (7, HF), (80, BF), (128, HF), (512, BF), (64, F32), (33, F32)])
@pytest.mark.parametrize("page,dpage", [(16, 16), (1, 64), (64, 8)])
def test_dims_types_and_pages(dim, dtype, page, dpage):
    _run([40, 130, 3], 2, dim, 37, 8, 2, page=page, dpage=dpage, dtype=dtype)


# ties go to the lowest index, whatever else the row holds
@pytest.mark.parametrize("values", [[0.0], [0.0, -0.0], [1.0, 2.0], [0.0, 1e-45, 1e-38], [math.inf, 1.0],
                                    [math.nan, 0.0, -1.0], [-math.inf, math.nan], [-1.0, -2.0, 3.0], [math.nan]])
def test_ties_and_special_weights(values):
    g = torch.Generator().manual_seed(len(values))
    lens = [2500, 300, 64]
    w = torch.tensor(values)[torch.randint(0, len(values), (3, 2, 2560), generator=g)]
    for budget in (5, 200, 1200):
        _run(lens, 2, 8, budget, 2, 1, w=w, page=64)


def test_close_weights():
    """Weights that differ in their last bits only."""
    g = torch.Generator().manual_seed(9)
    w = (torch.randint(0, 300, (2, 2, 1024), generator=g) + 0x3F800000).to(torch.int32).view(torch.float32)
    _run([1000, 700], 2, 16, 333, 10, 1, w=w)


def test_strides():
    import paper_2609_10264_amd as mvk

    def entries_first(c):
        return mvk.KVCache(*(t.transpose(1, 2).contiguous().transpose(1, 2) for t in (c.K, c.V)))

    def odd(c):
        def shift(t):
            b = torch.zeros(t.numel() + 3, dtype=t.dtype, device="cuda")[3:].view(t.shape)
            return b.copy_(t)
        return mvk.KVCache(shift(c.K), shift(c.V))

    for view in (entries_first, odd):
        _run([130, 20, 77], 2, 64, 50, 8, 2, view=view)


def test_same_bits_every_time_and_in_a_graph():
    import paper_2609_10264_amd as mvk
    n, hk, page = 3000, 4, 64
    table = torch.randperm(48, device="cuda")[:47].to(I32).view(1, 47)
    cache = mvk.KVCache(*(torch.randn((48, hk, page, 64), device="cuda").to(BF) for _ in range(2)))
    lens = torch.tensor([n], dtype=I32, device="cuda")
    w = torch.rand((1, hk, 47 * page), device="cuda").round(decimals=2)
    dtable = torch.arange(16, dtype=I32, device="cuda").view(1, 16)

    def call(dst, wo):
        return mvk.cache_evict(cache, mvk.Sequences(table, lens), w, dst, dtable, 1000, recent=50, sinks=4, weights_out=wo)

    fresh = lambda: (mvk.KVCache.allocate(16, hk, page, 64), torch.zeros((1, hk, 1024), device="cuda"))  # noqa: E731
    dst, wo = fresh()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call(dst, wo)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        kept, m = call(dst, wo)
    for n2 in (3000, 1001, 900, 2999):
        lens.fill_(n2)
        w.copy_(w.flip(2))
        graph.replay()
        torch.cuda.synchronize()
        d2, wo2 = fresh()
        k2, m2 = call(d2, wo2)
        c = int(m2[0])
        assert c == min(n2, 1000) == int(m[0]) and torch.equal(kept, k2)
        assert torch.equal(wo[..., :c], wo2[..., :c])
        flat = lambda t: t.transpose(1, 2).reshape(-1, hk, 64)[:c]  # noqa: E731
        assert torch.equal(flat(dst.K), flat(d2.K)) and torch.equal(flat(dst.V), flat(d2.V))


def test_refusals():
    import paper_2609_10264_amd as mvk
    cache = mvk.KVCache.allocate(4, 2, 16, 64)
    dst = mvk.KVCache.allocate(4, 2, 16, 64)
    seqs = mvk.Sequences(torch.zeros((1, 4), dtype=I32, device="cuda"), torch.tensor([60], dtype=I32, device="cuda"))
    w = torch.zeros((1, 2, 64), device="cuda")
    dt = torch.zeros((1, 2), dtype=I32, device="cuda")
    with pytest.raises(mvk.MvkError):  # more protected than kept
        mvk.cache_evict(cache, seqs, w, dst, dt, 16, recent=10, sinks=7)
    with pytest.raises(mvk.MvkError):
        mvk.cache_evict(cache, seqs, w, dst, dt, 0)
    with pytest.raises(mvk.MvkError):  # a table too narrow for the budget
        mvk.cache_evict(cache, seqs, w, dst, dt, 33)
    with pytest.raises(mvk.MvkError):  # caches of other shapes
        mvk.cache_evict(cache, seqs, w, mvk.KVCache.allocate(4, 2, 16, 32), dt, 16)
    with pytest.raises(ValueError):  # weights shorter than the entries
        mvk.cache_evict(cache, seqs, w[..., :32], dst, dt, 16)
    with pytest.raises(ValueError):
        mvk.cache_evict(cache, seqs, w, dst, dt, 16, weights_out=torch.zeros((1, 2, 8), device="cuda"))
