"""Attention over a cache held in 8 bits against its definition in 64 bits over
the values that the codes stand for; they are exact in bfloat16, so the bounds
are those of a bfloat16 cache."""
import math

import pytest
import torch

from tests import cache8_ref as c8
from tests.test_gpu_attention import BF, F32, HF, Problem, _check, _check_o_only, _within

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


BOTH = pytest.mark.parametrize("kind", [c8.E4M3, c8.I8])


class Problem8(Problem):
    """K and V are what codes and exponents stand for; `spread` powers of two lie between rows."""

    def __init__(self, kind, *args, spread=2, edit=None, **kw):
        super().__init__(*args, **kw)
        g = torch.Generator().manual_seed(77)
        if edit is not None:
            edit(self)
        self.kind, self.held = kind, {}
        for name in ("K", "V"):
            x = getattr(self, name).double()
            if spread:
                x = x * 2.0 ** torch.randint(-spread, spread + 1, x.shape[:-1], generator=g)[..., None]
            self.held[name] = c8.hold(x, kind)
            value = c8.worth(*self.held[name], kind)
            setattr(self, name, value.to(BF))
            assert torch.equal(getattr(self, name).double().nan_to_num(7.0), value.nan_to_num(7.0))

    def reference(self, **kw):
        r = super().reference(**kw)
        # The weights are 32-bit floats: one below the least normal number, 2^-126, may be
        # lost, and with it at most 2^-126 |v|; n of them in a row.  (Codes of zero let such
        # a weight be a row's whole result: a weight of one times zero, and 1e-48 times 100.)
        r.o_err += max(self.lens) * 2.0**-126 * float(self.V.double().abs().nan_to_num(0, 0, 0).max())
        return r

    def device(self):
        import paper_2609_10264_amd as mvk
        super().device()
        (kc, ke), (vc, ve) = self.held["K"], self.held["V"]
        self.cache = mvk.KVCache(kc.view(self.kind).cuda(), vc.view(self.kind).cuda(), ke.cuda(), ve.cuda())
        return self


@BOTH
@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (4, 4), (8, 1), (6, 2), (14, 2), (32, 1), (40, 1), (130, 1)])
def test_head_groups(kind, heads, kv_heads):
    _check(Problem8(kind, [5, 63, 64, 65, 130, 200], [1, 3, 64, 1, 17, 0], heads, kv_heads, 64))


@BOTH
@pytest.mark.parametrize("dim", [8, 16, 24, 40, 64, 72, 80, 96, 112, 128, 136, 192, 256])
def test_head_dims(kind, dim):
    _check(Problem8(kind, [1, 31, 100, 129], [1, 5, 100, 33], 4, 2, dim))
    _check(Problem8(kind, [1, 31, 300], [1, 1, 1], 8, 2, dim))


@BOTH
@pytest.mark.parametrize("dim", [1, 7, 100, 264, 300, 512])
def test_dims_of_the_general_path(kind, dim):
    _check(Problem8(kind, [1, 30, 77], [1, 4, 20], 4, 2, dim))


@BOTH
@pytest.mark.parametrize("page", [1, 2, 8, 16, 32, 64, 128, 256, 1024])
def test_page_sizes(kind, page):
    _check(Problem8(kind, [1, 255, 256, 257, 40], [1, 1, 20, 130, 40], 8, 2, 128, page=page))
    _check(Problem8(kind, [1, 255, 256, 257, 40], [1] * 5, 8, 2, 128, page=page))


@BOTH
@pytest.mark.parametrize("heads,kv_heads", [(4, 4), (8, 1), (16, 2)])
@pytest.mark.parametrize("dim", [64, 128])
def test_single_tokens(kind, heads, kv_heads, dim):
    lens = [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257, 511, 513, 1000, 2049, 5000]
    _check(Problem8(kind, lens, [1] * len(lens), heads, kv_heads, dim, page=32))


@BOTH
def test_long_sequences(kind):
    _check(Problem8(kind, [40001], [1], 8, 2, 128, page=64))
    _check(Problem8(kind, [5003], [77], 8, 2, 128, page=64))


@BOTH
@pytest.mark.parametrize("c", [1, 2, 31, 32, 33, 127, 128, 129, 300])
def test_whole_prompts(kind, c):
    _check(Problem8(kind, [c], [c], 4, 2, 64))


@BOTH
def test_many_sequences_of_many_lengths(kind):
    g = torch.Generator().manual_seed(5)
    lens = torch.randint(0, 400, (150,), generator=g).tolist()
    new = [min(n, int(x)) for n, x in zip(lens, torch.randint(0, 9, (150,), generator=g))]
    _check(Problem8(kind, lens, new, 8, 4, 64))


@BOTH
def test_rows_without_entries_are_zero(kind):
    pr = Problem8(kind, [0, 3, 0, 70, 2], [1, 5, 4, 140, 2], 8, 2, 128)
    out = _check(pr)
    assert bool((out[0] == 0).all()) and bool((out[1:3] == 0).all()) and not bool((out[3] == 0).all())


@BOTH
@pytest.mark.parametrize("fill", [math.nan, math.inf, -math.inf, float(torch.finfo(BF).min)])
def test_unused_places_hold_anything(kind, fill):
    _check(Problem8(kind, [3, 17, 70, 129, 0], [1, 17, 5, 100, 1], 8, 2, 96, page=32, fill=fill, spread=0))
    _check(Problem8(kind, [3, 17, 70, 129, 0], [1] * 5, 8, 2, 128, page=32, fill=fill, spread=0))


# entries that some rows of a tile see and others do not: a not-a-number of one value (E4M3) or of the row (I8)
@BOTH
@pytest.mark.parametrize("which", ["K", "V"])
@pytest.mark.parametrize("heads,kv_heads", [(4, 2), (16, 2), (1, 1)])
@pytest.mark.parametrize("dim", [128, 40])
def test_values_in_masked_places_do_not_reach_earlier_rows(kind, which, heads, kv_heads, dim):
    def edit(pr):
        for s, j in ((0, 130), (0, 149), (1, 3), (1, 40), (1, 69)):
            getattr(pr, which)[int(pr.table[s, j // 16]), :, j % 16, 5:9] = math.inf

    pr = Problem8(kind, [150, 70], [40, 70], heads, kv_heads, dim, edit=edit)
    r = pr.reference()
    assert bool(torch.isfinite(r.o[:20]).all()) and not bool(torch.isfinite(r.o[-1]).all())
    out = _check_o_only(pr, r)
    assert bool(torch.isfinite(out[:20]).all())


@BOTH
@pytest.mark.parametrize("spread", [0, 12])
@pytest.mark.parametrize("sharp", [0.0, 1e-3, 4.0])
def test_exponents_far_apart_and_scores_sharp_and_flat(kind, spread, sharp):
    _check(Problem8(kind, [3, 64, 200, 90], [3, 1, 70, 90], 8, 2, 64, sharp=sharp, spread=spread))


@BOTH
@pytest.mark.parametrize("e", [c8.LEAST, -60, 100])
def test_exponents_at_the_ends_of_the_range(kind, e):
    """All of V near one end of the exponents: as exact as in the middle."""
    def edit(pr):
        pr.V = pr.V.double() * 2.0 ** (e + 4)

    pr = Problem8(kind, [70, 33], [20, 33], 4, 2, 64, edit=edit, spread=0)
    assert int(pr.held["V"][1].min()) <= e + 4
    _check_o_only(pr, pr.reference())


@BOTH
@pytest.mark.parametrize("out_dtype", [BF, HF, F32])
def test_output_types(kind, out_dtype):
    import paper_2609_10264_amd as mvk
    pr = Problem8(kind, [70, 200, 1], [20, 1, 1], 8, 2, 128, spread=1).device()
    out = mvk.paged_attention(pr.dq, pr.cache, pr.seqs, out_dtype=out_dtype)
    r = pr.reference(out_dtype=out_dtype)
    _within(out, r.o, r.o_err, out_dtype)


# views: entries before heads, codes beside other data, unaligned codes, exponents of any order
@BOTH
@pytest.mark.parametrize("dim", [128, 80, 20])
@pytest.mark.parametrize("new", [[20, 70, 1], [1, 1, 1]])
def test_strides(kind, dim, new):
    import paper_2609_10264_amd as mvk
    pr = Problem8(kind, [150, 70, 5], new, 6, 2, dim).device()
    K, V = pr.cache.K.view(torch.int8), pr.cache.V.view(torch.int8)
    other = lambda t: t.transpose(1, 2).contiguous().transpose(1, 2)  # noqa: E731
    pages, hk, page, d = K.shape
    both = torch.zeros((pages, hk, page, 2 * d), dtype=torch.int8, device="cuda")
    both[..., :d], both[..., d:] = K, V
    odd = torch.zeros((pages * hk * page * d + 3,), dtype=torch.int8, device="cuda")[3:].view(pages, hk, page, d)
    odd.copy_(K)
    exps = torch.stack((pr.cache.k_exp, pr.cache.v_exp)).permute(2, 3, 1, 0).contiguous()
    r = pr.reference()
    as8 = lambda t: t.view(kind)  # noqa: E731
    for k, v in ((other(K), V), (both[..., :d], both[..., d:]), (odd, V)):
        cache = mvk.KVCache(as8(k), as8(v), exps[..., 0].permute(2, 0, 1), exps[..., 1].permute(2, 0, 1))
        out = mvk.paged_attention(pr.dq, cache, pr.seqs)
        _within(out, r.o, r.o_err, "strides")


@BOTH
def test_offsets_beyond_32_bits(kind):
    import paper_2609_10264_amd as mvk
    page, hk, d = 64, 8, 128
    pages = 2**32 // (page * hk * d) + 40
    pr = Problem8(kind, [300, 1, 90], [33, 1, 1], 16, hk, d, page=page).device()
    shift = pages - pr.K.shape[0]
    K, V = (torch.zeros((pages, hk, page, d), dtype=torch.int8, device="cuda") for _ in range(2))
    ke, ve = (torch.zeros((pages, hk, page), dtype=torch.int8, device="cuda") for _ in range(2))
    for big, small in ((K, pr.cache.K.view(torch.int8)), (V, pr.cache.V.view(torch.int8)), (ke, pr.cache.k_exp), (ve, pr.cache.v_exp)):
        big[shift:] = small
    table = torch.where(pr.table >= 0, pr.table + shift, pr.table).cuda()
    for most in (33, 1):
        seqs = mvk.Sequences(table, pr.seqs.lens, pr.seqs.q_start, max_new=most)
        out = mvk.paged_attention(pr.dq, mvk.KVCache(K.view(kind), V.view(kind), ke, ve), seqs)
        r = pr.reference()
        _within(out, r.o, r.o_err, "high pages")


@BOTH
@pytest.mark.parametrize("new", [[1, 1, 1], [5, 60, 1], [1, 200, 40]])
def test_weights_add_up(kind, new):
    import paper_2609_10264_amd as mvk
    pr = Problem8(kind, [70, 260, 40], new, 8, 2, 128).device()
    w = torch.rand((3, 2, pr.cap + 5), generator=torch.Generator().manual_seed(3))
    dw = w.cuda()
    mvk.paged_attention(pr.dq, pr.cache, pr.seqs, weights=dw)
    r = pr.reference(w_in=w)
    for s, n in enumerate(pr.lens):
        _within(dw[s, :, :n], r.w[s, :, :n], r.w_err[s, :, :n], "w")
        assert torch.equal(dw[s, :, n:].cpu(), w[s, :, n:])


@BOTH
def test_same_bits_every_time_in_a_graph_and_on_another_stream(kind):
    import paper_2609_10264_amd as mvk
    pr = Problem8(kind, [3000, 70, 260, 9], [1, 70, 3, 1], 8, 2, 128).device()
    out, w = torch.zeros_like(pr.dq), torch.zeros((4, 2, pr.cap), device="cuda")

    def call(stream=None):
        mvk.paged_attention(pr.dq, pr.cache, pr.seqs, out=out, weights_out=w, stream=stream)

    call()
    want = out.clone(), w.clone()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for stream in (None, None, side, side):
        out.zero_(), w.zero_()
        torch.cuda.synchronize()
        call(stream)
        torch.cuda.synchronize()
        assert torch.equal(out, want[0]) and torch.equal(w, want[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        call()
    for lens in ([3000, 70, 260, 9], [1, 70, 0, 5], [513, 90, 200, 9]):
        pr.seqs.lens.copy_(torch.tensor(lens, dtype=torch.int32))
        out.zero_(), w.zero_()
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone(), w.clone()
        out.zero_(), w.zero_()
        call()
        assert torch.equal(got[0], out) and torch.equal(got[1], w)


@BOTH
def test_metadata_out_of_range_is_clamped(kind):
    import paper_2609_10264_amd as mvk
    pr = Problem8(kind, [64, 64], [2, 2], 4, 2, 64).device()
    pr.seqs.lens.copy_(torch.tensor([10**9, -5], dtype=torch.int32))
    pr.seqs.table[0, 0] = 10**9
    pr.seqs.table[0, 1] = -3
    for most in (1, 2, 100):
        seqs = mvk.Sequences(pr.seqs.table, pr.seqs.lens, pr.seqs.q_start, max_new=most)
        out = torch.full_like(pr.dq, 9.0)
        mvk.paged_attention(pr.dq, pr.cache, seqs, out=out)
        torch.cuda.synchronize()
        assert bool(torch.isfinite(out.float()).all()) and bool((out[2:] == 0).all())


@BOTH
def test_refusals(kind):
    import paper_2609_10264_amd as mvk
    pr = Problem8(kind, [64], [2], 4, 2, 64).device()
    for q in (pr.dq.half(), pr.dq.float()):
        with pytest.raises(mvk.MvkError):
            mvk.paged_attention(q, pr.cache, pr.seqs)
    with pytest.raises(TypeError):
        mvk.paged_attention(pr.dq, mvk.KVCache(pr.cache.K, pr.cache.V), pr.seqs)
