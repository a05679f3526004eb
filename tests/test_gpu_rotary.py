"""Rotary positions and the append to the paged cache (mvk_rotary_table,
mvk_rotary_append) against their definitions in 64 bits."""
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
P, BB = 2**31 - 1, 15 * 2**27 + 1


@pytest.mark.parametrize("kw", [dict(), dict(base=500000.0), dict(scaling="linear", factor=4.0),
                                dict(scaling="base", factor=8.0),
                                dict(scaling="parts", factor=16.0, original_len=4096.0),
                                dict(scaling="parts", factor=4.0, original_len=2048.0, slow=0.5, fast=48.0)])
@pytest.mark.parametrize("rot,rows", [(128, 70001), (64, 1), (2, 300), (90, 1000)])
def test_table(rot, rows, kw):
    import paper_2609_10264_amd as mvk
    if kw.get("scaling") == "base" and rot < 4:
        pytest.skip("needs two frequencies")
    t = mvk.rotary_table(rot, rows, **kw).double().cpu()
    f, mag = ref.frequencies(rot, **kw)
    angle = torch.arange(rows, dtype=torch.float64)[:, None] * f
    want = torch.cat([angle.cos(), angle.sin()], 1) * mag
    # one rounding to 32 bits; frequencies by two pow functions, an ulp or so of 64 bits apart
    assert float((t - want).abs().max()) <= 2.0**-24 * mag * 1.01 + rows * 2.0**-50


def _inputs(T, H, D, dtype, g, p=P):
    x = torch.randn((T, H, D), generator=g)
    if dtype == I32:
        return ref.embed((x * 65536).round().long(), p)
    return x.to(dtype)


def _close(got, want, dtype, big):
    """One rounding to the type, and the 32-bit arithmetic before it (of values up to `big`)."""
    u = ref.ROUND[dtype]
    err = u * want.abs() * (1 + 2.0**-8) + 4 * 2.0**-24 * big + (2.0**-25 if dtype == HF else 0.0)
    d = (got.double().cpu() - want).abs()
    assert bool((d <= err).all()), (float((d - err).max()), int((d > err).sum()))


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("src,dst", [(I32, BF), (I32, HF), (BF, BF), (HF, HF), (F32, BF), (F32, HF), (BF, F32), (I32, F32)])
@pytest.mark.parametrize("T,H,D,rot", [(1, 1, 64, 64), (37, 5, 128, 128), (9, 3, 96, 48), (5, 2, 80, 16), (4, 3, 40, 10),
                                       (3, 2, 7, 4), (2, 1, 512, 512), (6, 2, 33, 0), (300, 8, 64, 32)])
def test_queries(layout, src, dst, T, H, D, rot):
    import paper_2609_10264_amd as mvk
    g = torch.Generator().manual_seed(T * D + rot)
    q = _inputs(T, H, D, src, g)
    pos = torch.randint(0, 5000, (T,), generator=g).to(I32)
    table = mvk.rotary_table(rot, 5000) if rot else torch.zeros((1, 0), device="cuda")
    scale = 2.0**-16 if src == I32 else None
    out = mvk.rotary(q.cuda(), pos.cuda(), table, layout=layout, field_scale=scale, out_dtype=dst)
    x = ref.lift(q, 2.0**-16)
    want = ref.rotate(x, table.cpu()[pos.long()], layout) if rot else x
    _close(out, want, dst, float(x.abs().max()))


class Append:
    def __init__(self, lens, new, H, hk, D, rot, page, src, dst, seed=1, p=P):
        g = torch.Generator().manual_seed(seed)
        self.lens, self.new, self.p = lens, new, p
        self.table, self.pages = ref.lay_out(lens, page, seed)
        T = sum(new)
        self.q, self.k, self.v = (_inputs(T, h, D, src, g, p) for h in (H, hk, hk))
        self.pos = torch.randint(0, 4000, (T,), generator=g).to(I32)  # (after evictions positions are not entry indices)
        self.K, self.V = (torch.randn((self.pages, hk, page, D), generator=g).to(dst) for _ in range(2))

    def run(self, layout="half", q=True, table=None):
        import paper_2609_10264_amd as mvk
        self.rot_table = mvk.rotary_table(table, 4000)
        self.cache = mvk.KVCache(self.K.cuda(), self.V.cuda())
        seqs = mvk.Sequences(self.table.cuda(), torch.tensor(self.lens, dtype=I32).cuda(), ref.starts(self.new).cuda())
        return mvk.rotary_append(self.q.cuda() if q else None, self.k.cuda(), self.v.cuda(), self.pos.cuda(),
                                 self.rot_table, self.cache, seqs, layout=layout,
                                 field_scale=2.0**-16 if self.q.dtype == I32 else None, p=self.p)

    def check(self, out, layout="half"):
        rows = self.rot_table.cpu()[self.pos.long()]
        x = {n: ref.lift(getattr(self, n), 2.0**-16, self.p) for n in "qkv"}
        big = max(float(t.abs().max()) for t in x.values())
        if out is not None:
            _close(out, ref.rotate(x["q"], rows, layout), self.K.dtype, big)
        k, v = ref.rotate(x["k"], rows, layout), x["v"]
        K, V = self.K.double(), self.V.double()
        page = self.K.shape[2]
        st = ref.starts(self.new).tolist()
        touched = torch.zeros(K.shape[:3], dtype=torch.bool)
        for s, (n, c) in enumerate(zip(self.lens, self.new)):
            for i in range(c):
                e = n - c + i
                if e < 0:
                    continue
                pg = int(self.table[s, e // page])
                K[pg, :, e % page], V[pg, :, e % page] = k[st[s] + i], v[st[s] + i]
                touched[pg, :, e % page] = True
        _close(self.cache.K, K, self.K.dtype, big)
        _close(self.cache.V, V, self.K.dtype, big)
        assert torch.equal(self.cache.K.cpu()[~touched], self.K[~touched])  # every other place is left alone
        assert torch.equal(self.cache.V.cpu()[~touched], self.V[~touched])


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("src,dst", [(I32, BF), (BF, BF), (HF, HF), (F32, BF), (F32, F32), (I32, HF)])
@pytest.mark.parametrize("H,hk,D,rot", [(4, 4, 128, 128), (6, 2, 96, 64), (7, 1, 64, 20), (5, 5, 20, 20)])
def test_append(layout, src, dst, H, hk, D, rot):
    a = Append([1, 40, 17, 70, 0, 33], [1, 7, 17, 0, 0, 1], H, hk, D, rot, 16, src, dst)
    a.check(a.run(layout, table=rot), layout)


@pytest.mark.parametrize("page", [1, 8, 64, 256])
def test_append_pages_and_many_sequences(page):
    g = torch.Generator().manual_seed(page)
    lens = torch.randint(0, 300, (90,), generator=g).tolist()
    new = [min(n, int(x)) for n, x in zip(lens, torch.randint(0, 12, (90,), generator=g))]
    a = Append(lens, new, 4, 2, 64, 64, page, BF, BF)
    a.check(a.run(table=64))


def test_append_long_prompt_and_keys_only():
    a = Append([2500, 3], [2400, 1], 8, 2, 128, 128, 64, I32, BF)
    a.check(a.run(table=128))
    assert a.run(q=False, table=128) is None
    a.check(None)


def test_more_new_tokens_than_entries_are_not_written():
    a = Append([3, 20], [5, 4], 2, 2, 64, 64, 8, BF, BF)
    a.check(a.run(table=64))


def test_babybear_elements():
    a = Append([40, 9], [30, 1], 4, 2, 128, 128, 16, I32, BF, p=BB)
    a.check(a.run(table=128))


def test_in_place_and_strides():
    import paper_2609_10264_amd as mvk
    g = torch.Generator().manual_seed(1)
    for D in (128, 40):
        q = _inputs(50, 6, D, BF, g).cuda()
        pos = torch.randint(0, 999, (50,), generator=g).to(I32).cuda()
        table = mvk.rotary_table(16, 999)
        want = mvk.rotary(q, pos, table)
        wide = torch.zeros((50, 6 * D + 3), dtype=BF, device="cuda")
        part = wide[:, 3:].unflatten(1, (6, D))  # rows at odd offsets
        part.copy_(q)
        assert torch.equal(mvk.rotary(part, pos, table), want)
        swapped = q.transpose(0, 1).contiguous().transpose(0, 1)
        out = torch.empty((6, 50, D + 8), dtype=BF, device="cuda").transpose(0, 1)[..., :D]
        assert torch.equal(mvk.rotary(swapped, pos, table, out=out), want)
        mvk.rotary(q, pos, table, out=q)
        assert torch.equal(q, want)


def test_positions_and_pages_out_of_range():
    import paper_2609_10264_amd as mvk
    q = torch.randn((4, 2, 64), device="cuda").to(BF)
    table = mvk.rotary_table(64, 100)
    got = mvk.rotary(q, torch.tensor([-5, 0, 99, 10**9], dtype=I32, device="cuda"), table)
    want = mvk.rotary(q, torch.tensor([0, 0, 99, 99], dtype=I32, device="cuda"), table)
    assert torch.equal(got, want)
    cache = mvk.KVCache.allocate(3, 2, 8, 64)
    seqs = mvk.Sequences(torch.tensor([[7, 1], [-1, 10**9]], dtype=I32, device="cuda"),
                         torch.tensor([9, 10**9], dtype=I32, device="cuda"), torch.tensor([0, 2, 4], dtype=I32, device="cuda"))
    mvk.rotary_append(q, q, q, torch.zeros(4, dtype=I32, device="cuda"), table, cache, seqs)
    torch.cuda.synchronize()
    # entry 7 of sequence 0 lies in page 7 (outside), entry 8 in page 1; sequence 1 has no page
    assert torch.equal(cache.V[1, :, 0], q[1]) and int((cache.V != 0).sum()) == int((q[1] != 0).sum())


def test_large_values_of_the_field():
    """Residues up to the half of the field keep 24 bits and their signs."""
    import paper_2609_10264_amd as mvk
    x = torch.tensor([0, 1, P - 1, (P - 1) // 2, (P + 1) // 2, 12345678, P - 12345678, 2**30 - 129], dtype=I32)
    out = mvk.rotary(x.view(1, 1, 8).cuda(), torch.zeros(1, dtype=I32, device="cuda"), mvk.rotary_table(8, 1),
                     field_scale=0.25, out_dtype=F32).cpu().view(-1).double()
    want = ref.lift(x, 0.25)
    assert bool(((out - want).abs() <= 2.0**-24 * want.abs()).all())
    assert math.copysign(1, float(out[4])) == -1.0


def test_refusals():
    import paper_2609_10264_amd as mvk
    q = torch.zeros((2, 2, 64), dtype=BF, device="cuda")
    pos = torch.zeros(2, dtype=I32, device="cuda")
    table = mvk.rotary_table(64, 10)
    with pytest.raises(ValueError):
        mvk.rotary(q, pos, table, layout="other")
    with pytest.raises(ValueError):
        mvk.rotary(q.to(I32), pos, table)  # field elements without their scale
    with pytest.raises(ValueError):
        mvk.rotary(q, pos[:1], table)
    with pytest.raises(TypeError):
        mvk.rotary(q.double(), pos, table)
    with pytest.raises(mvk.MvkError):  # wider than the head
        mvk.rotary(q, pos, mvk.rotary_table(128, 10))
    with pytest.raises(mvk.MvkError):  # odd
        mvk.rotary_table(7, 10)
    with pytest.raises(ValueError):
        mvk.rotary_table(8, 10, scaling="other")
    with pytest.raises(mvk.MvkError):
        mvk.rotary_table(8, 10, scaling="parts", factor=2.0)  # no original length
    cache = mvk.KVCache.allocate(3, 2, 8, 64, dtype=HF)
    seqs = mvk.Sequences(pos.view(1, 2), pos[:1], pos)
    with pytest.raises(mvk.MvkError):  # keys of another type than the queries
        mvk.rotary_append(q, q.half(), q.half(), pos, table, cache, seqs)
    with pytest.raises(ValueError):  # another head count than the cache's
        mvk.rotary_append(q, q[:, :1], q[:, :1], pos, table, cache, seqs)
