"""A cache held in 8 bits: the append to it and reading it back against the
definition, code for code, and eviction from it; attention over it is in
test_gpu_attention8.py."""
import math

import pytest
import torch

from tests import attention_ref as ref
from tests import cache8_ref as c8

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


BF, HF, F32, FIELD = torch.bfloat16, torch.float16, torch.float32, torch.int32
P, BB = 2**31 - 1, 15 * 2**27 + 1


def _inputs(shape, dtype, seed, p=P):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(shape, generator=g)
    # rows of very different sizes, and rows whose largest value is far from the others
    x = x * 2.0 ** torch.randint(-12, 9, shape[:-1], generator=g)[..., None]
    x[::3, ..., :1] *= 40
    if dtype == FIELD:
        return ref.embed((x * 2**16).round().long().clamp(-(p // 2), p // 2), p)
    return x.to(dtype)


class Append:
    """An append and what the cache then holds, from the definition."""

    def __init__(self, lens, new, kv_heads, dim, cache, rot=None, layout="half", dtype=BF, heads=4, page=16, seed=1, p=P):
        import paper_2609_10264_amd as mvk
        self.lens, self.new, self.cache_type, self.p = lens, new, cache, p
        rot = dim if rot is None else rot
        T = sum(new)
        self.table, pages = ref.lay_out(lens, page, seed)
        self.q, self.k, self.v = (_inputs((T, h, dim), dtype, seed + i, p) for i, h in enumerate((heads, kv_heads, kv_heads)))
        g = torch.Generator().manual_seed(seed + 9)
        self.positions = torch.randint(0, 500, (T,), generator=g).to(torch.int32)
        self.rot_table = mvk.rotary_table(rot, 500) if rot else torch.zeros((1, 0), device="cuda")
        self.layout, self.page = layout, page
        self.cache = mvk.KVCache.allocate(pages, kv_heads, page, dim, dtype=cache)
        self.q_start = ref.starts(new)
        self.seqs = mvk.Sequences(self.table.cuda(), torch.tensor(lens, dtype=torch.int32).cuda(), self.q_start.cuda())
        self.scale = 2.0**-16 if dtype == FIELD else None

    def call(self, **kw):
        import paper_2609_10264_amd as mvk
        return mvk.rotary_append(self.q.cuda(), self.k.cuda(), self.v.cuda(), self.positions.cuda(), self.rot_table,
                                 self.cache, self.seqs, layout=self.layout, field_scale=self.scale, p=self.p, **kw)

    def rotated(self, x):
        x = ref.lift(x, self.scale or 1.0, self.p)
        rows = self.rot_table.cpu()[self.positions.long()] if self.rot_table.numel() else torch.zeros((len(x), 0))
        return ref.rotate(x, rows, self.layout)

    def places(self):
        """(token, page, place) of every token that has an entry."""
        for s, (n, c) in enumerate(zip(self.lens, self.new)):
            for i in range(c):
                if n - c + i >= 0:
                    yield int(self.q_start[s]) + i, int(self.table[s, (n - c + i) // self.page]), (n - c + i) % self.page

    def check(self):
        want = {"K": c8.hold(self.rotated(self.k), self.cache_type), "V": c8.hold(ref.lift(self.v, self.scale or 1.0, self.p), self.cache_type)}
        where = list(self.places())
        t, page, at = (torch.tensor(x, dtype=torch.long) for x in zip(*where))
        for name, ex in (("K", "k_exp"), ("V", "v_exp")):
            codes, e = getattr(self.cache, name).view(torch.int8).cpu(), getattr(self.cache, ex).cpu()
            assert torch.equal(e[page, :, at], want[name][1][t]), name
            assert c8.same_codes(codes[page, :, at], want[name][0][t], self.cache_type), name
            # nothing else was written
            codes[page, :, at], e[page, :, at] = 0, 0
            assert int(codes.view(torch.uint8).max()) == 0 and int(e.abs().max()) == 0
        return want, t


@pytest.mark.parametrize("cache", [c8.E4M3, c8.I8])
@pytest.mark.parametrize("dtype", [BF, HF, F32, FIELD])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_append_and_read_back(cache, dtype, layout):
    import paper_2609_10264_amd as mvk
    print(f"append {cache} {dtype} {layout}", flush=True)
    a = Append([40, 17, 3, 0, 5], [23, 1, 3, 0, 5], 2, 64, cache, rot=32, layout=layout, dtype=dtype)
    q = a.call()
    want, t = a.check()
    # the queries are as ever
    same = mvk.rotary(a.q.cuda(), a.positions.cuda(), a.rot_table, layout=layout, field_scale=a.scale)
    assert q.dtype == BF and torch.equal(q, same)
    for out in (BF, HF, F32):
        k, v = mvk.cache_read(a.cache, a.seqs, tokens=len(a.q), dtype=out)
        for got, name in ((k, "K"), (v, "V")):
            value = c8.worth(*want[name], cache)
            assert got.dtype == out and torch.equal(got.cpu(), value.to(out)), (name, out)
            if out == BF:
                assert torch.equal(got.double().cpu(), value)  # exact


# dims and rotated parts of every alignment; one and many heads
@pytest.mark.parametrize("cache", [c8.E4M3, c8.I8])
@pytest.mark.parametrize("dim,rot", [(1, 0), (2, 2), (7, 4), (16, 16), (20, 6), (33, 32), (64, 0), (80, 40), (96, 96), (100, 100),
                                     (128, 128), (128, 64), (192, 64), (256, 256), (512, 512), (509, 508)])
def test_dims(cache, dim, rot):
    print(f"append {cache} dim={dim} rot={rot}", flush=True)
    for i, (layout, dtype, heads) in enumerate((("half", BF, 1), ("interleaved", F32, 3), ("half", FIELD, 2))):
        a = Append([30, 1], [30, 1], heads, dim, cache, rot=rot, layout=layout, dtype=dtype, seed=i)
        a.call()
        a.check()


@pytest.mark.parametrize("cache", [c8.E4M3, c8.I8])
def test_many_tokens_and_heads(cache):
    a = Append([700, 300, 65], [300, 300, 1], 8, 128, cache, heads=16, page=64, dtype=FIELD)
    a.call()
    a.check()


@pytest.mark.parametrize("cache", [c8.E4M3, c8.I8])
def test_the_other_field(cache):
    a = Append([40, 5], [23, 5], 2, 32, cache, dtype=FIELD, p=BB)
    a.call()
    a.check()


# values on the borders between codes, for every code, at several exponents
@pytest.mark.parametrize("cache", [c8.E4M3, c8.I8])
@pytest.mark.parametrize("dtype", [F32, BF])
def test_ties_and_borders(cache, dtype):
    values, _ = c8.codes_of(cache)
    mid = (values[1:] + values[:-1]) / 2
    top = c8.LARGEST[cache]
    rows = []
    for shift in (-96, -20, 0, 9, 100):
        for i in range(0, len(mid), 60):
            x = torch.zeros(64, dtype=torch.float64)
            x[:len(mid[i:i + 60])] = mid[i:i + 60]
            x[60:] = torch.tensor([top, -top, top * 0.75, 1.0])
            rows.append(x * 2.0**shift)
            below, above = x * (1 - 2.0**-20), x * (1 + 2.0**-20)
            above[60:62] = x[60:62]
            rows += [below * 2.0**shift, above * 2.0**shift]
    # just above and below the largest value of an exponent
    for f in (1 - 2.0**-7, 1.0, 1 + 2.0**-7):
        rows.append(torch.full((64,), top * f, dtype=torch.float64))
    x = torch.stack(rows)[:, None].to(dtype)
    a = Append([len(x)], [len(x)], 1, 64, cache, rot=0, dtype=dtype)
    a.k, a.v, a.q = x, x.flip(0), x
    a.call()
    a.check()


@pytest.mark.parametrize("cache", [c8.E4M3, c8.I8])
def test_rows_of_zeros_tiny_huge_and_not_finite_values(cache):
    import paper_2609_10264_amd as mvk
    x = torch.randn((12, 2, 48), generator=torch.Generator().manual_seed(2))
    x[0] = 0
    x[1] *= 2.0**-126 * 2.0**-10
    x[2] *= 2.0**-100
    x[3] *= 2.0**124
    x[4] = torch.finfo(F32).max
    x[5, :, 3] = math.nan
    x[6, :, 4] = math.inf
    x[7, 1, 5] = -math.inf
    x[8] = math.nan
    x[9] = -0.0
    a = Append([12], [12], 2, 48, cache, rot=16, dtype=F32)
    a.k, a.v = x, x.flip(1).contiguous()
    a.call()
    want, _ = a.check()
    k, v = mvk.cache_read(a.cache, a.seqs, tokens=12, dtype=F32)
    for got, name in ((k, "K"), (v, "V")):
        value = c8.worth(*want[name], cache)
        assert torch.equal(got.cpu().isnan(), value.isnan()) and torch.equal(got.cpu().nan_to_num(0), value.nan_to_num(0).float())
    assert bool(k[8].isnan().all()) and bool(k[0].eq(0).all())


# pools, exponents and rows as views of other orders and of wider or unaligned buffers
@pytest.mark.parametrize("cache", [c8.E4M3, c8.I8])
@pytest.mark.parametrize("dim", [64, 40])
def test_strides(cache, dim):
    import paper_2609_10264_amd as mvk
    a = Append([40, 17], [23, 17], 3, dim, cache, rot=16)
    pages, hk, page, d = a.cache.K.shape
    both = torch.zeros((pages, page, hk, 2 * d + 3), dtype=torch.int8, device="cuda")
    exps = torch.zeros((page, hk, pages, 2), dtype=torch.int8, device="cuda")
    view = both.transpose(1, 2).view(cache)
    a.cache = mvk.KVCache(view[..., :d], view[..., d + 3:], exps[..., 0].permute(2, 1, 0), exps[..., 1].permute(2, 1, 0))
    T, H, _ = a.q.shape
    wide = torch.zeros((T, H * d + 2 * hk * d + 5), dtype=BF)
    parts = [wide[:, 5:5 + H * d].unflatten(1, (H, d)), wide[:, 5 + H * d:5 + (H + hk) * d].unflatten(1, (hk, d)),
             wide[:, 5 + (H + hk) * d:].unflatten(1, (hk, d))]
    for part, x in zip(parts, (a.q, a.k, a.v)):
        part.copy_(x)
    dw = wide.cuda()
    q, k, v = (dw[:, i:i + h * d].unflatten(1, (h, d)) for i, h in ((5, H), (5 + H * d, hk), (5 + (H + hk) * d, hk)))
    out = torch.zeros((H, T, d + 1), dtype=BF, device="cuda").transpose(0, 1)[..., 1:]
    mvk.rotary_append(q, k, v, a.positions.cuda(), a.rot_table, a.cache, a.seqs, layout=a.layout, out=out)
    assert torch.equal(out, mvk.rotary(a.q.cuda(), a.positions.cuda(), a.rot_table))
    want, t = a.check()
    assert int(both[..., d:d + 3].abs().max()) == 0  # between K and V
    back = torch.full((hk, T, d + 7), 9.0, dtype=F32, device="cuda").transpose(0, 1)[..., 2:2 + d]
    mvk.cache_read(a.cache, a.seqs, v_out=back)
    assert torch.equal(back.double().cpu(), c8.worth(*want["V"], cache))


@pytest.mark.parametrize("cache", [c8.E4M3, c8.I8])
def test_queries_in_place_and_keys_alone(cache):
    import paper_2609_10264_amd as mvk
    a = Append([40, 17], [23, 17], 2, 64, cache)
    q = a.q.cuda()
    same = mvk.rotary(q, a.positions.cuda(), a.rot_table)
    got = mvk.rotary_append(q, a.k.cuda(), a.v.cuda(), a.positions.cuda(), a.rot_table, a.cache, a.seqs, out=q)
    assert got is q and torch.equal(q, same)
    a.check()
    b = Append([40, 17], [23, 17], 2, 64, cache)
    assert mvk.rotary_append(None, b.k.cuda(), b.v.cuda(), b.positions.cuda(), b.rot_table, b.cache, b.seqs) is None
    b.check()


# tokens without an entry, pages outside the pool, rows behind the last sequence
@pytest.mark.parametrize("cache", [c8.E4M3, c8.I8, BF])
def test_rows_without_an_entry(cache):
    import paper_2609_10264_amd as mvk
    lens, new = [3, 20, 9], [5, 4, 2]
    a = Append(lens, new, 2, 32, cache)
    a.table[1, 1] = 10**6  # of entries 16 .. 19: all new ones of sequence 1
    a.table[2, 0] = -1
    a.seqs.table.copy_(a.table)
    T = sum(new) + 3  # three rows of no sequence
    g = torch.Generator().manual_seed(4)
    q, k, v = (torch.randn((T, h, 32), generator=g).to(BF).cuda() for h in (4, 2, 2))
    positions = torch.zeros(T, dtype=torch.int32, device="cuda")
    mvk.rotary_append(q, k, v, positions, a.rot_table, a.cache, a.seqs)
    used = {(int(a.table[0, 0]), i) for i in range(3)}
    written = (a.cache.K.view(torch.int8 if cache != BF else torch.int16) != 0).any(-1).any(1).nonzero().tolist()
    assert {tuple(x) for x in written} == used
    kb, vb = (torch.full((T, 2, 32), 5.0, device="cuda") for _ in range(2))
    mvk.cache_read(a.cache, a.seqs, k_out=kb, v_out=vb)
    for back in (kb, vb):
        assert bool((back[:2] == 5.0).all()) and bool((back[5:] == 5.0).all()) and not bool((back[2:5] == 5.0).any())


@pytest.mark.parametrize("dtype", [BF, HF, F32])
def test_read_back_of_other_caches(dtype):
    import paper_2609_10264_amd as mvk
    lens = [40, 17, 0, 33]
    table, pages = ref.lay_out(lens, 16, 3)
    g = torch.Generator().manual_seed(5)
    K, V = (torch.randn((pages, 3, 16, 24), generator=g).to(dtype) for _ in range(2))
    seqs = mvk.Sequences(table.cuda(), torch.tensor(lens, dtype=torch.int32).cuda(), ref.starts(lens).cuda())
    for out in (BF, F32):
        k, v = mvk.cache_read(mvk.KVCache(K.cuda(), V.cuda()), seqs, tokens=sum(lens), dtype=out)
        for got, pool in ((k, K), (v, V)):
            want = torch.cat([ref.entries(pool, table[s], n).transpose(0, 1) for s, n in enumerate(lens)])
            assert torch.equal(got.cpu(), want.to(out))


@pytest.mark.parametrize("cache", [c8.E4M3, c8.I8])
@pytest.mark.parametrize("dim", [64, 40])
def test_eviction_takes_codes_and_exponents(cache, dim):
    import paper_2609_10264_amd as mvk
    lens = [60, 5, 33]
    a = Append(lens, lens, 2, dim, cache)
    a.call()
    dst = mvk.KVCache.allocate(8, 2, 8, dim, dtype=cache)
    dtable = torch.randperm(8, generator=torch.Generator().manual_seed(1))[:6].view(3, 2).to(torch.int32)
    cap = a.table.shape[1] * 16
    w = torch.rand((3, 2, cap), generator=torch.Generator().manual_seed(2))
    kept, n = mvk.cache_evict(a.cache, a.seqs, w.cuda(), dst, dtable.cuda(), 13, recent=4, sinks=2)
    assert n.tolist() == [13, 5, 13]
    for s, m in enumerate(n.tolist()):
        for h in range(2):
            want = ref.evict(w[s, h, :lens[s]].tolist(), lens[s], 13, 4, 2)
            assert kept[s, h, :m].tolist() == want
            for r, j in enumerate(want):
                src, to = int(a.table[s, j // 16]), int(dtable[s, r // 8])
                for name in ("K", "V", "k_exp", "v_exp"):
                    x, y = (getattr(c, name)[i, h, at].view(torch.int8) for c, i, at in ((a.cache, src, j % 16), (dst, to, r % 8)))
                    assert torch.equal(x, y), (name, s, h, r)


@pytest.mark.parametrize("cache", [c8.E4M3, c8.I8])
def test_in_a_graph_and_on_another_stream(cache):
    import paper_2609_10264_amd as mvk
    a = Append([40, 17], [1, 1], 2, 64, cache)
    q, k, v, pos = a.q.cuda(), a.k.cuda(), a.v.cuda(), a.positions.cuda()
    out, kb, vb = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    side = torch.cuda.Stream()

    def step(stream=None):
        mvk.rotary_append(q, k, v, pos, a.rot_table, a.cache, a.seqs, out=out, stream=stream)
        mvk.cache_read(a.cache, a.seqs, k_out=kb, v_out=vb, stream=stream)

    torch.cuda.synchronize()
    step(side)
    torch.cuda.synchronize()
    a.check()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()
    for seed, lens in ((1, [39, 17]), (2, [12, 1]), (3, [40, 16])):
        for x in (a.cache.K, a.cache.V, a.cache.k_exp, a.cache.v_exp):
            x.view(torch.int8).zero_()
        a.lens = lens
        a.seqs.lens.copy_(torch.tensor(lens, dtype=torch.int32))
        a.k, a.v = _inputs(a.k.shape, BF, seed), _inputs(a.v.shape, BF, seed + 7)
        k.copy_(a.k), v.copy_(a.v)
        graph.replay()
        torch.cuda.synchronize()
        want, t = a.check()
        assert torch.equal(kb.double().cpu(), c8.worth(*want["K"], cache))
        assert torch.equal(vb.double().cpu(), c8.worth(*want["V"], cache))


def test_refusals():
    import paper_2609_10264_amd as mvk
    a = Append([40], [3], 2, 64, c8.E4M3)
    K, V, kx, vx = a.cache.K, a.cache.V, a.cache.k_exp, a.cache.v_exp
    for bad in (mvk.KVCache(K, V), mvk.KVCache(K, V, kx), mvk.KVCache(K, V, kx.float(), vx), mvk.KVCache(K, V, kx.cpu(), vx)):
        with pytest.raises(TypeError):
            mvk.cache_read(bad, a.seqs, tokens=3)
    with pytest.raises(ValueError):
        mvk.cache_read(mvk.KVCache(K, V, kx[:1], vx), a.seqs, tokens=3)
    with pytest.raises(ValueError):  # exponents of a cache that needs none
        mvk.cache_read(mvk.KVCache(K.to(BF), V.to(BF), kx, vx), a.seqs, tokens=3)
    with pytest.raises(TypeError):
        mvk.cache_read(mvk.KVCache(K, V.view(torch.int8), kx, vx), a.seqs, tokens=3)
    with pytest.raises(ValueError):
        mvk.cache_read(a.cache, a.seqs)
    with pytest.raises(ValueError):
        mvk.cache_read(a.cache, a.seqs, tokens=4, k_out=torch.zeros((3, 2, 64), device="cuda"))
    with pytest.raises(mvk.MvkError):  # field elements are not what a cache holds
        mvk.cache_read(a.cache, a.seqs, k_out=torch.zeros((3, 2, 64), dtype=torch.int32, device="cuda"))
    one = torch.zeros((3, 2, 64), device="cuda")
    with pytest.raises(mvk.MvkError):
        mvk.cache_read(a.cache, a.seqs, k_out=one, v_out=one)
    with pytest.raises(mvk.MvkError):  # queries are bfloat16
        a.call(out=torch.zeros((3, 4, 64), dtype=HF, device="cuda"))
    assert mvk.cache_read(a.cache, a.seqs, tokens=0)[0].shape == (0, 2, 64)
