"""Attention over a paged cache (mvk_paged_attention) against its definition in
64 bits: head groups, dims, page sizes, ragged chunks, empty rows, unused and
masked places that hold anything, strides, streams, graphs, collected weights."""
import math

import pytest
import torch

from tests import attention_ref as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


BF, HF, F32 = torch.bfloat16, torch.float16, torch.float32


class Problem:
    def __init__(self, lens, new, heads, kv_heads, dim, page=16, dtype=BF, seed=1, sharp=1.0, fill=0.0):
        g = torch.Generator().manual_seed(seed)
        self.lens, self.new = list(lens), list(new)
        self.table, pages = ref.lay_out(lens, page, seed)
        rnd = lambda *s: torch.randn(s, generator=g).to(dtype)  # noqa: E731
        # places that no entry uses hold `fill`
        self.K, self.V = (torch.full((pages, kv_heads, page, dim), fill, dtype=dtype) for _ in range(2))
        for s, n in enumerate(lens):
            for j0 in range(0, n, page):
                m = min(page, n - j0)
                pg = int(self.table[s, j0 // page])
                self.K[pg, :, :m] = rnd(kv_heads, m, dim)
                self.V[pg, :, :m] = rnd(kv_heads, m, dim)
        T = sum(new)
        self.q = (rnd(T, heads, dim).float() * sharp).to(dtype)
        self.q_start = ref.starts(new)
        self.lens_t = torch.tensor(lens, dtype=torch.int32)
        self.cap = self.table.shape[1] * page

    def device(self):
        import paper_2609_10264_amd as mvk
        self.dq = self.q.cuda()
        self.cache = mvk.KVCache(self.K.cuda(), self.V.cuda())
        self.seqs = mvk.Sequences(self.table.cuda(), self.lens_t.cuda(), self.q_start.cuda(), max_new=max(self.new + [1]))
        return self

    def reference(self, **kw):
        return ref.Attention(self.q, self.K, self.V, self.table, self.lens_t, self.q_start, **kw)


def _within(got, want, err, what):
    got = got.double().cpu()
    assert torch.equal(torch.isnan(got), torch.isnan(want)), what
    ok = (got == want) | ((got - want).abs() <= err) | torch.isnan(want)
    assert bool(ok.all()), (what, float((got - want).abs().nan_to_num(0).max()), int((~ok).sum()))


def _check(pr, **kw):
    import paper_2609_10264_amd as mvk
    print(f"attention lens={pr.lens[:6]} new={pr.new[:6]} q={tuple(pr.q.shape)} pool={tuple(pr.K.shape)} {pr.q.dtype}",
          flush=True)
    pr.device()
    T, H, _ = pr.q.shape
    lse = torch.full((T, H), 123.0, device="cuda")
    w = torch.full((len(pr.lens), pr.K.shape[1], pr.cap), -5.0, device="cuda")
    out = mvk.paged_attention(pr.dq, pr.cache, pr.seqs, lse=lse, weights_out=w, **kw)
    alone = mvk.paged_attention(pr.dq, pr.cache, pr.seqs, **kw)
    torch.cuda.synchronize()
    r = pr.reference()
    _within(out, r.o, r.o_err, "o")
    _within(alone, r.o, r.o_err, "o without weights")
    _within(lse, r.lse, r.lse_err, "lse")
    for s, n in enumerate(pr.lens):
        _within(w[s, :, :n], r.w[s, :, :n], r.w_err[s, :, :n], f"w of sequence {s}")
        assert bool((w[s, :, n:] == -5.0).all())  # places beyond the entries are left alone
    return out


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (4, 4), (8, 1), (6, 2), (14, 2), (12, 1), (32, 1), (40, 1), (130, 1)])
def test_head_groups(heads, kv_heads, dtype):
    _check(Problem([5, 63, 64, 65, 130, 200], [1, 3, 64, 1, 17, 0], heads, kv_heads, 64, dtype=dtype))


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("dim", [8, 16, 24, 40, 64, 72, 80, 96, 112, 128, 136, 192, 256])
def test_head_dims(dim, dtype):
    _check(Problem([1, 31, 100, 129], [1, 5, 100, 33], 4, 2, dim, dtype=dtype))


# dims that are no multiple of 8, dims above 256, and 32-bit caches
@pytest.mark.parametrize("dim,dtype", [(1, BF), (7, HF), (100, BF), (264, BF), (300, HF), (512, BF), (64, F32), (128, F32),
                                       (33, F32)])
def test_dims_and_types_of_the_general_path(dim, dtype):
    _check(Problem([1, 30, 77], [1, 4, 20], 4, 2, dim, dtype=dtype))


@pytest.mark.parametrize("page", [1, 2, 8, 16, 32, 64, 128, 256, 1024])
def test_page_sizes(page):
    _check(Problem([1, 255, 256, 257, 40], [1, 1, 20, 130, 40], 8, 2, 128, page=page))


# single tokens: lengths around every boundary a tile may have, and long ones
@pytest.mark.parametrize("heads,kv_heads", [(4, 4), (8, 1), (16, 2)])
@pytest.mark.parametrize("dim", [64, 128])
def test_single_tokens(heads, kv_heads, dim):
    lens = [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257, 511, 513, 1000, 2049, 5000]
    _check(Problem(lens, [1] * len(lens), heads, kv_heads, dim, page=32))


def test_single_token_of_one_long_sequence():
    _check(Problem([40001], [1], 8, 2, 128, page=64))


def test_chunk_of_a_long_sequence():
    _check(Problem([5003], [77], 8, 2, 128, page=64))


@pytest.mark.parametrize("c", [1, 2, 31, 32, 33, 127, 128, 129, 300])
def test_whole_prompts(c):
    _check(Problem([c], [c], 4, 2, 64))


def test_many_sequences_of_many_lengths():
    g = torch.Generator().manual_seed(5)
    lens = torch.randint(0, 400, (150,), generator=g).tolist()
    new = [min(n, int(x)) for n, x in zip(lens, torch.randint(0, 9, (150,), generator=g))]
    _check(Problem(lens, new, 8, 4, 64))


# rows that see nothing: empty sequences, and sequences shorter than their new tokens
def test_rows_without_entries_are_zero():
    import paper_2609_10264_amd as mvk
    pr = Problem([0, 3, 0, 70, 2], [1, 5, 4, 140, 2], 8, 2, 128)
    out = _check(pr)
    assert bool((out[0] == 0).all()) and bool((out[1:3] == 0).all()) and not bool((out[3] == 0).all())
    lse = torch.zeros((sum(pr.new), 8), device="cuda")
    mvk.paged_attention(pr.dq, pr.cache, pr.seqs, lse=lse)
    assert bool(torch.isneginf(lse[:3]).all()) and bool(torch.isfinite(lse[3]).all())


@pytest.mark.parametrize("fill", [math.nan, math.inf, -math.inf, float(torch.finfo(BF).min)])
@pytest.mark.parametrize("dtype", [BF, HF])
def test_unused_places_hold_anything(fill, dtype):
    if dtype == HF and math.isfinite(fill):
        fill = float(torch.finfo(HF).min)
    _check(Problem([3, 17, 70, 129, 0], [1, 17, 5, 100, 1], 8, 2, 96, page=32, dtype=dtype, fill=fill))


# entries that some rows of a tile see and others do not
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("which", ["K", "V"])
@pytest.mark.parametrize("heads,kv_heads,dtype", [(4, 2, BF), (16, 2, HF), (1, 1, BF)])
def test_values_in_masked_places_do_not_reach_earlier_rows(bad, which, heads, kv_heads, dtype):
    pr = Problem([150, 70], [40, 70], heads, kv_heads, 128, page=16, dtype=dtype)
    for s, j in ((0, 130), (0, 149), (1, 3), (1, 40), (1, 69)):
        pool = getattr(pr, which)
        pool[int(pr.table[s, j // 16]), :, j % 16, 5:9] = bad
    r = pr.reference()
    assert bool(torch.isfinite(r.o[:20]).all()) and not bool(torch.isfinite(r.o[-1]).all())
    out = _check_o_only(pr, r)
    assert bool(torch.isfinite(out[:20]).all())


def _check_o_only(pr, r):
    import paper_2609_10264_amd as mvk
    pr.device()
    out = mvk.paged_attention(pr.dq, pr.cache, pr.seqs)
    torch.cuda.synchronize()
    got = out.double().cpu()
    same = torch.isfinite(got) == torch.isfinite(r.o)
    assert bool(same.all()), int((~same).sum())
    fin = torch.isfinite(r.o)
    assert bool(((got - r.o).abs() <= r.o_err)[fin].all())
    # infinities as the definition has them, where it has no not-a-number
    inf = torch.isinf(r.o)
    assert torch.equal(got[inf], r.o[inf])
    return out


# scores far apart (one entry takes all), far below zero, and all alike
@pytest.mark.parametrize("sharp", [0.0, 1e-3, 30.0])
def test_sharp_and_flat_scores(sharp):
    _check(Problem([3, 64, 200, 90], [3, 1, 70, 90], 8, 2, 64, sharp=sharp))


def test_very_negative_scores():
    pr = Problem([100, 64], [7, 64], 4, 2, 64)
    pr.K[:] = pr.K.abs()
    pr.q = (-pr.q.float().abs() * 20).to(BF)
    _check(pr)


@pytest.mark.parametrize("scale", [0.5, 1e-4, -0.1, 0.0])
def test_scale(scale):
    import paper_2609_10264_amd as mvk
    pr = Problem([70, 33], [20, 33], 4, 2, 64).device()
    out = mvk.paged_attention(pr.dq, pr.cache, pr.seqs, scale=scale)
    r = pr.reference(scale=scale)
    _within(out, r.o, r.o_err, scale)


@pytest.mark.parametrize("out_dtype", [BF, HF, F32])
def test_output_types(out_dtype):
    import paper_2609_10264_amd as mvk
    pr = Problem([70, 200, 1], [20, 1, 1], 8, 2, 128).device()
    out = mvk.paged_attention(pr.dq, pr.cache, pr.seqs, out_dtype=out_dtype)
    assert out.dtype == out_dtype
    r = pr.reference(out_dtype=out_dtype)
    _within(out, r.o, r.o_err, out_dtype)


@pytest.mark.parametrize("p", [2**31 - 1, 15 * 2**27 + 1])
@pytest.mark.parametrize("dim", [128, 33])
def test_field_output(p, dim):
    import paper_2609_10264_amd as mvk
    pr = Problem([70, 200, 1, 0], [20, 1, 1, 1], 8, 2, dim).device()
    scale = 2.0**-10
    out = mvk.paged_attention(pr.dq, pr.cache, pr.seqs, out_dtype=mvk.FIELD, field_scale=scale, p=p)
    assert out.dtype == torch.int32 and int(out.min()) >= 0 and int(out.max()) < p
    r = pr.reference(out_dtype=F32)
    got = ref.lift(out.cpu(), 1.0, p)
    assert bool(((got - r.o / scale).abs() <= 0.5 + r.o_err / scale + 2.0**-10).all())
    # magnitudes beyond the field's half are clamped
    big = mvk.paged_attention(pr.dq, pr.cache, pr.seqs, out_dtype=mvk.FIELD, field_scale=1e-20, p=p)
    assert set(ref.lift(big.cpu()[:21], 1.0, p).abs().unique().tolist()) <= {float((p - 1) // 2), 0.0}


# views with other strides and orders: entries before heads, a slice of a wider row, offset data
@pytest.mark.parametrize("dim", [128, 80, 20])
def test_strides(dim):
    import paper_2609_10264_amd as mvk
    pr = Problem([150, 70, 5], [20, 70, 1], 6, 2, dim).device()
    want = mvk.paged_attention(pr.dq, pr.cache, pr.seqs)
    other = lambda t: t.transpose(1, 2).contiguous().transpose(1, 2)  # noqa: E731
    pages, hk, page, d = pr.cache.K.shape
    both = torch.zeros((pages, hk, page, 2 * d), dtype=BF, device="cuda")  # K and V side by side
    both[..., :d], both[..., d:] = pr.cache.K, pr.cache.V
    odd = torch.zeros((pages * hk * page * d + 3,), dtype=BF, device="cuda")[3:].view(pages, hk, page, d)
    odd.copy_(pr.cache.K)
    T, H, _ = pr.q.shape
    wide = torch.zeros((T, H * d + 24), dtype=BF, device="cuda")
    wide[:, 8:8 + H * d] = pr.dq.reshape(T, H * d)
    q2 = wide[:, 8:8 + H * d].unflatten(1, (H, d))
    out2 = torch.zeros((H, T, d + 8), dtype=BF, device="cuda").transpose(0, 1)[..., :d]
    r = pr.reference()
    for cache in (mvk.KVCache(other(pr.cache.K), pr.cache.V), mvk.KVCache(both[..., :d], both[..., d:]),
                  mvk.KVCache(odd, pr.cache.V)):
        mvk.paged_attention(q2, cache, pr.seqs, out=out2)
        _within(out2, r.o, r.o_err, "strides")
    assert want.shape == out2.shape


def test_offsets_beyond_32_bits():
    """Pages whose elements lie above 2^32, in a pool of 2^33 bytes and more."""
    import paper_2609_10264_amd as mvk
    page, hk, d = 64, 8, 128
    per = page * hk * d
    pages = 2**32 // per + 40
    K, V = (torch.empty((pages, hk, page, d), dtype=BF, device="cuda") for _ in range(2))
    small = Problem([300, 1, 90], [33, 1, 1], 16, hk, d, page=page).device()
    used = small.table >= 0
    shift = pages - small.K.shape[0]
    table = torch.where(used, small.table + shift, small.table).cuda()
    K[shift:], V[shift:] = small.cache.K, small.cache.V
    out = mvk.paged_attention(small.dq, mvk.KVCache(K, V), mvk.Sequences(table, small.seqs.lens, small.seqs.q_start))
    r = small.reference()
    _within(out, r.o, r.o_err, "high pages")


def test_weights_add_up_and_new_entries_start_from_zero():
    import paper_2609_10264_amd as mvk
    for new in ([1, 1, 1], [5, 60, 1], [1, 200, 40]):
        pr = Problem([70, 260, 40], new, 8, 2, 128).device()
        w = torch.rand((3, 2, pr.cap + 5), generator=torch.Generator().manual_seed(3))
        dw = w.cuda()
        mvk.paged_attention(pr.dq, pr.cache, pr.seqs, weights=dw)
        r = pr.reference(w_in=w)
        for s, n in enumerate(pr.lens):
            _within(dw[s, :, :n], r.w[s, :, :n], r.w_err[s, :, :n], "w")
            assert torch.equal(dw[s, :, n:].cpu(), w[s, :, n:])
            total = r.w[s, :, :n].sum(-1) - w[s, :, :n - new[s]].double().sum(-1)
            assert torch.allclose(total, torch.full_like(total, 4.0 * new[s]))  # every row's weights sum to one


def test_same_bits_every_time_and_on_another_stream():
    import paper_2609_10264_amd as mvk
    pr = Problem([3000, 70, 260, 9], [1, 70, 3, 1], 8, 2, 128).device()

    def call():
        w = torch.zeros((4, 2, pr.cap), device="cuda")
        return mvk.paged_attention(pr.dq, pr.cache, pr.seqs, weights_out=w), w

    want = call()
    for _ in range(5):
        got = call()
        assert all(torch.equal(a, b) for a, b in zip(want, got))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = call()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))


def test_in_a_graph_with_changing_lengths():
    """One capture, replayed for other lengths and tables; each replay equals the eager call."""
    import paper_2609_10264_amd as mvk
    pr = Problem([900, 70, 260, 9], [1, 1, 1, 1], 8, 2, 128, page=64).device()
    w = torch.zeros((4, 2, pr.cap), device="cuda")
    out = torch.zeros_like(pr.dq)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        mvk.paged_attention(pr.dq, pr.cache, pr.seqs, out=out, weights_out=w)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        mvk.paged_attention(pr.dq, pr.cache, pr.seqs, out=out, weights_out=w)
    for lens in ([900, 70, 260, 9], [1, 70, 0, 5], [513, 2, 200, 9], [900, 70, 260, 9]):
        pr.seqs.lens.copy_(torch.tensor(lens, dtype=torch.int32))
        w.zero_()
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        w2 = torch.zeros_like(w)
        eager = mvk.paged_attention(pr.dq, pr.cache, pr.seqs, weights_out=w2)
        assert torch.equal(out, eager) and torch.equal(w, w2)


def test_metadata_out_of_range_is_clamped():
    """Lengths beyond the table, pages outside the pool and starts outside the
    rows: no read outside the buffers; rows of no sequence are left alone."""
    import paper_2609_10264_amd as mvk
    pr = Problem([64, 64], [2, 2], 4, 2, 64, page=16).device()
    pr.seqs.lens.copy_(torch.tensor([10**9, -5], dtype=torch.int32))
    pr.seqs.table[0, 0] = 10**9
    pr.seqs.table[0, 1] = -3
    out = torch.full_like(pr.dq, 9.0)
    mvk.paged_attention(pr.dq, pr.cache, pr.seqs, out=out)
    torch.cuda.synchronize()
    assert bool(torch.isfinite(out.float()).all()) and bool((out[2:] == 0).all())
    pr.seqs.q_start.copy_(torch.tensor([0, 1, 1], dtype=torch.int32))
    out.fill_(9.0)
    mvk.paged_attention(pr.dq, pr.cache, pr.seqs, out=out)
    assert bool((out[1:] == 9.0).all())
    pr.seqs.q_start.copy_(torch.tensor([3, 2, 10**9], dtype=torch.int32))
    mvk.paged_attention(pr.dq, pr.cache, pr.seqs, out=out)
    torch.cuda.synchronize()


def test_refusals():
    import paper_2609_10264_amd as mvk
    pr = Problem([64], [2], 4, 2, 64).device()
    with pytest.raises(mvk.MvkError):  # heads that do not divide
        mvk.paged_attention(pr.dq[:, :3].contiguous(), pr.cache, pr.seqs)
    with pytest.raises(mvk.MvkError):  # another type than the cache's
        mvk.paged_attention(pr.dq.half(), pr.cache, pr.seqs)
    with pytest.raises(mvk.MvkError):  # a page size that is no power of two
        mvk.paged_attention(pr.dq, mvk.KVCache(pr.cache.K[:, :, :15], pr.cache.V[:, :, :15]), pr.seqs)
    with pytest.raises(ValueError):  # another dim
        mvk.paged_attention(pr.dq[..., :32], pr.cache, pr.seqs)
    with pytest.raises(ValueError):  # no scale for field elements
        mvk.paged_attention(pr.dq, pr.cache, pr.seqs, out_dtype=mvk.FIELD)
    with pytest.raises(TypeError):
        mvk.paged_attention(pr.dq.cpu(), pr.cache, pr.seqs)
    with pytest.raises(ValueError):  # too short for the entries
        mvk.paged_attention(pr.dq, pr.cache, pr.seqs, weights_out=torch.zeros((1, 2, 8), device="cuda"))
    with pytest.raises(ValueError):
        mvk.paged_attention(pr.dq, pr.cache, mvk.Sequences(pr.seqs.table.long(), pr.seqs.lens, pr.seqs.q_start))


def test_starts_that_claim_the_same_rows_beyond_the_count_of_units():
    """Every second of 65535 sequences claims all 2048 rows over 2^20 entries: more units
    than are counted in 32 bits, so nothing is done, and the next call is as ever."""
    import paper_2609_10264_amd as mvk
    S, T, page = 65535, 2048, 1 << 20
    print(f"attention of {S} sequences with overlapping starts", flush=True)
    cache = mvk.KVCache.allocate(1, 1, page, 8)
    q = torch.ones((T, 1, 8), dtype=BF, device="cuda")
    starts = (torch.arange(S + 1, device="cuda") % 2 * T).to(torch.int32)
    seqs = mvk.Sequences(torch.zeros((S, 1), dtype=torch.int32, device="cuda"),
                         torch.full((S,), page, dtype=torch.int32, device="cuda"), starts, max_new=T)
    out = torch.full((T, 1, 8), 7.0, dtype=BF, device="cuda")
    mvk.paged_attention(q, cache, seqs, out=out)
    torch.cuda.synchronize()
    assert bool((out == 7.0).all())
    _check(Problem([70, 300], [5, 140], 4, 2, 64))
