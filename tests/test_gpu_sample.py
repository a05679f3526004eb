"""mvk_sample_tokens against its definition, token for token."""
import math

import pytest
import torch

from tests import attention_ref as ref
from tests import steps_ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


BF, HF, F32, FIELD = torch.bfloat16, torch.float16, torch.float32, torch.int32
P, BB = 2**31 - 1, 15 * 2**27 + 1


def _logits(R, n, dtype, seed, p=P, banned=0.1):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((R, n), generator=g, dtype=torch.float64) * 2
    x += torch.where(torch.rand((R, n), generator=g) < 5 / n, 6.0, 0.0)
    if dtype == FIELD:
        return ref.embed((x * 2**16).round().long(), p)
    return torch.where(torch.rand((R, n), generator=g) < banned, -math.inf, x).to(dtype)


def _u(R, seed):
    u = torch.rand(R, generator=torch.Generator().manual_seed(seed))
    u[0] = 0.0
    return u


def _check(x, u, p=P, t=1.0, k=0, top_p=1.0, least=0.0, **kw):
    import paper_2609_10264_amd as mvk
    R = len(x)
    print(f"sample {tuple(x.shape)} {x.dtype} t={t if not torch.is_tensor(t) else 'own'}", flush=True)
    up = lambda v: v.cuda() if torch.is_tensor(v) else v  # noqa: E731
    probs = torch.full((R,), -7.0, device="cuda")
    got = mvk.sample(x.cuda(), u.cuda(), temperature=up(t), top_k=up(k), top_p=up(top_p), min_p=up(least),
                     field_scale=2.0**-16, probs=probs, p=p, **kw)
    assert got.dtype == torch.int32 and got.shape == (R,)
    values = ref.lift(x, 2.0**-16, p)
    for r in range(R):
        at = lambda v: float(v[r]) if torch.is_tensor(v) else v  # noqa: E731
        want, prob = steps_ref.token(values[r], float(u[r]), at(t), int(at(k)), at(top_p), at(least))
        assert int(got[r]) == want, (r, int(got[r]), want)
        # one rounding to 32 bits, weights in multiples of 2^-44
        assert abs(float(probs[r]) - prob) <= 2.0**-24 * prob * 1.001 + len(values[r]) * 2.0**-45
    return got


SETTINGS = [dict(), dict(t=0.7), dict(t=0.0), dict(k=1), dict(k=7), dict(k=40, t=1.4), dict(top_p=0.5), dict(top_p=0.95, t=0.8),
            dict(top_p=0.0), dict(least=0.1), dict(least=1.0), dict(k=30, top_p=0.8, least=0.05, t=1.2), dict(k=10**9, top_p=1.5)]


@pytest.mark.parametrize("dtype", [BF, HF, F32, FIELD])
@pytest.mark.parametrize("how", range(len(SETTINGS)))
def test_settings(dtype, how):
    for n in (1000, 333):
        _check(_logits(12, n, dtype, how), _u(12, how + 50), **SETTINGS[how])


@pytest.mark.parametrize("n", [1, 2, 3, 7, 8, 9, 31, 255, 256, 257, 1023, 1024, 1025, 4095, 4096, 4097, 8191, 8193, 16385, 32768, 40003])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_lengths(n, dtype):
    x = _logits(3, n, dtype, n, banned=0.0)
    _check(x, _u(3, n))
    _check(x, _u(3, n + 1), k=max(1, n // 3), top_p=0.9)


def test_a_large_vocabulary():
    x = _logits(2, 131071, F32, 3)
    _check(x, _u(2, 1), k=1000, top_p=0.97)
    _check(x, _u(2, 2))
    _check(x, _u(2, 3), top_p=0.999, t=3.0)


@pytest.mark.parametrize("p", [P, BB])
def test_fields(p):
    x = _logits(6, 700, FIELD, 9, p)
    x[0, 5], x[0, 6], x[0, 7] = p // 2, p // 2 + 1, p - 1  # the largest, the smallest, -1
    _check(x, _u(6, 1), p=p, k=20, top_p=0.9)
    _check(x, _u(6, 2), p=p, t=0.0)


def test_everybody_has_settings_of_their_own():
    R = 64
    g = torch.Generator().manual_seed(4)
    t = torch.rand(R, generator=g) * 2
    t[::7] = 0.0
    k = torch.randint(-2, 60, (R,), generator=g).to(torch.int32)
    top_p, least = torch.rand(R, generator=g) * 1.2, torch.rand(R, generator=g) * 0.3 - 0.1
    x = _logits(R, 900, BF, 8)
    _check(x, _u(R, 5), t=t, k=k, top_p=top_p, least=least)
    _check(x, _u(R, 6), t=t, k=25, top_p=0.9, least=least)


def test_ties():
    """All alike, and few different values: borders of every setting fall within ties."""
    for n in (8, 100, 5000):
        x = torch.zeros((9, n), dtype=F32)
        u = torch.arange(9) / 8 * (1 - 2.0**-24)
        _check(x, u)
        _check(x, u, k=max(1, n // 4))
        _check(x, u, top_p=0.5)
        _check(x, u, t=0.0)
        x = torch.randint(0, 3, (9, n), generator=torch.Generator().manual_seed(n)).to(BF)
        _check(x, u, k=n // 2, top_p=0.75)
        _check(x, u, k=n // 3 + 1)
        _check(x, u, top_p=0.9, t=0.3)


def test_borders_of_the_random_number():
    """Eight alike: u = i / 8 is the beginning of token i, and less by a bit the end of token i - 1."""
    import paper_2609_10264_amd as mvk
    x = torch.zeros((17, 8), device="cuda")
    u = torch.tensor([i / 8 for i in range(8)] + [i / 8 - 2.0**-24 for i in range(1, 9)] + [0.99999994])
    want = list(range(8)) + list(range(8)) + [7]
    assert mvk.sample(x, u.cuda()).tolist() == want
    far = torch.tensor([-0.5, 1.0, 2.0, math.nan, math.inf, -math.inf])
    assert mvk.sample(x[:6], far.cuda()).tolist() == [0, 7, 7, 0, 7, 0]


def test_zeros_of_either_sign_are_ties():
    import paper_2609_10264_amd as mvk
    x = torch.tensor([[-0.0, 0.0, -0.0, 0.0]]).cuda()
    for dtype in (F32, BF, HF):
        assert mvk.sample(x.to(dtype), torch.tensor([0.9]).cuda(), top_k=2).tolist() == [1]
        assert mvk.sample(x.to(dtype), torch.tensor([0.9]).cuda(), temperature=0.0).tolist() == [0]


@pytest.mark.parametrize("dtype", [BF, HF, F32])
def test_not_finite_logits(dtype):
    x = _logits(8, 300, dtype, 3)
    x[0] = -math.inf
    x[1] = math.nan
    x[2] = -math.inf
    x[2, 217] = -3.0
    x[3, 5] = math.inf
    x[4, 5], x[4, 250], x[4, 251] = math.inf, math.inf, math.inf
    x[5, ::2] = math.nan
    x[6, :299] = math.nan
    for how in (dict(), dict(k=5, top_p=0.9), dict(t=0.0), dict(top_p=0.3), dict(least=0.5), dict(t=math.inf), dict(k=2)):
        got = _check(x, _u(8, 7), **how)
        assert got[:2].tolist() == [-1, -1] and int(got[2]) == 217 and int(got[3]) == 5


def test_far_settings():
    x = _logits(4, 300, F32, 3)
    nan = math.nan
    want = _check(x, _u(4, 7))
    import paper_2609_10264_amd as mvk
    got = mvk.sample(x.cuda(), _u(4, 7).cuda(), top_k=-5, top_p=nan, min_p=nan)
    assert torch.equal(got, want)
    assert torch.equal(mvk.sample(x.cuda(), _u(4, 7).cuda(), temperature=nan), _check(x, _u(4, 7), t=0.0))
    _check(x, _u(4, 8), t=1e-30)
    _check(x, _u(4, 8), t=1e30)
    _check(x, _u(4, 8), least=7.0)
    _check(x, _u(4, 8), top_p=-1.0)


def test_rows_and_strides():
    import paper_2609_10264_amd as mvk
    for R in (1, 2, 300, 3000):
        x = _logits(R, 130, BF, R)
        _check(x, _u(R, R), k=9)
    x = _logits(5, 400, F32, 1)
    wide = torch.full((5, 500), 50.0)
    for lead in (8, 3):
        wide[:, lead:lead + 400] = x
        got = mvk.sample(wide.cuda()[:, lead:lead + 400], _u(5, 1).cuda(), top_k=40)
        assert torch.equal(got, _check(x, _u(5, 1), k=40))
    assert mvk.sample(x[:0].cuda(), torch.zeros(0, device="cuda")).shape == (0,)
    one = x[:1].cuda().expand(4, 400)  # one row of logits, four numbers
    assert torch.equal(mvk.sample(one, _u(4, 2).cuda()), _check(x[:1].repeat(4, 1), _u(4, 2)))


@pytest.mark.parametrize("dtype", [BF, F32, FIELD])
def test_neighbours_in_a_large_vocabulary(dtype):
    """What is kept lies close together, in values and in the vocabulary."""
    n = 200003
    g = torch.Generator().manual_seed(1)
    x = torch.rand((4, n), generator=g) * -20 - 8
    x[0, 5000:5100] = torch.rand(100, generator=g)
    x[1, 131072:131272] = torch.rand(200, generator=g)
    x[2, :] = -30.0
    x[2, 70000:70090] = 1.0
    x[2, 7] = 60.0  # far above: the others share a bin of values
    x[3, 199903:] = 3.0 + torch.rand(100, generator=g) * 1e-3
    x = ref.embed((x.double() * 2**16).round().long()) if dtype == FIELD else x.to(dtype)
    for u in (0.0, 0.37, 0.81, 1 - 2.0**-24):
        for how in (dict(k=90), dict(k=300, top_p=0.7), dict(top_p=0.6), dict(least=0.3), dict(k=80, t=30.0, top_p=0.9)):
            _check(x, torch.full((4,), u), **how)


@pytest.mark.parametrize("dtype", [F32, FIELD])
@pytest.mark.parametrize("far", [3.0, 1000.0, 16000.0])
def test_values_close_together_below_one_far_above(dtype, far):
    """More than a thousand in one bin of values: their order bit by bit."""
    n = 3000
    x = torch.rand((3, n), generator=torch.Generator().manual_seed(2), dtype=torch.float64)
    x[:, 1234] = far
    x = ref.embed((x * 2**16).round().long()) if dtype == FIELD else x.to(dtype)
    u = torch.tensor([0.1, 0.5, 0.9999])
    for how in (dict(k=200), dict(k=900, t=1e4), dict(k=900, t=1e4, top_p=0.33), dict(top_p=0.4, t=1e4), dict(least=0.9, t=1e4)):
        _check(x, u, **how)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("k", [1399, 1400, 1401, 2047, 2048, 2049, 5000, 29999])
def test_more_than_the_list_holds(dtype, k):
    """By the row: the number kept, with ties at the border (in bfloat16 many), and top-p within it."""
    x = torch.randn((2, 30000), generator=torch.Generator().manual_seed(k)).to(dtype)
    _check(x, torch.tensor([0.3, 0.95]), k=k)
    _check(x, torch.tensor([0.3, 0.95]), k=k, top_p=0.9, t=5.0)
    _check(x, torch.tensor([0.3, 0.95]), k=k, top_p=0.1, least=0.2)


def test_all_alike_beyond_the_list():
    x = torch.full((3, 20000), -4.5)
    u = torch.tensor([0.0, 0.5, 1 - 2.0**-24])
    assert _check(x, u, k=7000).tolist() == [0, 3500, 6999]
    assert _check(x, u, top_p=0.25).tolist() == [0, 2500, 4999]
    _check(x, u, k=9000, top_p=0.25)
    _check(x, u, least=1.0)
    _check(x, u, k=3)


@pytest.mark.parametrize("least", [0.0, 1e-3, 0.5])
def test_smallest_probability_alone(least):
    for n, spread in ((50000, 0.3), (50000, 4.0), (70, 1.0)):
        x = torch.randn((3, n), generator=torch.Generator().manual_seed(n)) * spread
        _check(x, torch.tensor([0.0, 0.6, 0.99]), least=least)


@pytest.mark.parametrize("R,n", [(3, 1000), (40, 20000)])
def test_in_a_graph_and_on_two_streams(R, n):
    import paper_2609_10264_amd as mvk
    x, u = _logits(R, n, BF, 2).cuda(), _u(R, 3).cuda()
    out, probs = torch.zeros(R, dtype=torch.int32, device="cuda"), torch.zeros(R, device="cuda")

    def call(out, probs, stream=None):
        mvk.sample(x, u, temperature=0.9, top_k=300, top_p=0.9, min_p=0.01, out=out, probs=probs, stream=stream)

    call(out, probs)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    others = [(torch.zeros_like(out), torch.zeros_like(probs)) for _ in streams]
    torch.cuda.synchronize()
    for _ in range(5):  # in flight together
        for s, o in zip(streams, others):
            call(*o, stream=s)
    torch.cuda.synchronize()
    for o, q in others:
        assert torch.equal(o, out) and torch.equal(q, probs)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=streams[0]):
        call(out, probs)
    for i in range(4):
        x.copy_(_logits(R, n, BF, 20 + i))
        u.copy_(_u(R, 30 + i))
        out.fill_(-9)
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        call(out, probs)
        assert torch.equal(got, out)


def test_refusals():
    import paper_2609_10264_amd as mvk
    x, u = torch.zeros((4, 64), device="cuda"), torch.zeros(4, device="cuda")
    for bad in (dict(u=u[:2]), dict(u=u.half()), dict(out=u), dict(probs=u.half()), dict(temperature=u[:2]),
                dict(top_k=u), dict(top_p=u.cpu()), dict(logits=x[0]), dict(logits=x.t()), dict(logits=x.int()),
                dict(u=torch.zeros(8, device="cuda")[::2])):
        with pytest.raises(ValueError):
            mvk.sample(**{"logits": x, "u": u, **bad})
    with pytest.raises(TypeError):
        mvk.sample(x.cpu(), u)
    with pytest.raises(TypeError):
        mvk.sample(x.double(), u)
    tok = torch.zeros(4, dtype=torch.int32, device="cuda")
    for bad in (dict(probs=u), dict(out=tok, top_k=tok), dict(out=tok, probs=tok.view(F32)), dict(logits=x.int(), field_scale=0.0),
                dict(probs=x[0, :4]), dict(logits=x[:, :0])):
        with pytest.raises(mvk.MvkError):
            mvk.sample(**{"logits": x, "u": u, **bad})


@pytest.mark.parametrize("dtype", [BF, F32, FIELD])
@pytest.mark.parametrize("spread", [0.02, 2.2, 60.0])
def test_prefixes_that_no_list_holds(dtype, spread):
    """By bins of values, then by digits: narrow and wide rows, and one whose values lie far below its
    first few."""
    n = 40000
    x = torch.randn((4, n), generator=torch.Generator().manual_seed(3), dtype=torch.float64) * spread
    x[1] -= 9 * spread
    x[1, 100:103] = 9 * spread
    x[2] = x[2].sign() * 3.0 * spread  # two values
    x[3, ::2] = x[3, 1]
    x = ref.embed((x * 2**16).round().long()) if dtype == FIELD else x.to(dtype)
    u = torch.tensor([0.0, 0.3, 0.9, 0.999])
    for how in (dict(top_p=0.7, t=spread), dict(k=9000, t=spread), dict(k=25000, top_p=0.5, t=3 * spread),
                dict(k=9000, least=0.3, t=spread), dict(k=9000, top_p=0.99, t=1e6), dict(top_p=0.999, t=0.01 * spread)):
        _check(x, u, **how)
        _check(x.flip(0), u, **how)
