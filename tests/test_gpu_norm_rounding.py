"""The stream that mvk_block_norm leaves in 16 bits beside field elements, which are
computed in 64: rounded once, not by way of 32 bits."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


BF, HF, F32, FIELD = torch.bfloat16, torch.float16, torch.float32, torch.int32


def nearest(x, dtype):
    """Doubles rounded once to `dtype`, ties to even, as doubles."""
    bits, least = {BF: (8, -133), HF: (11, -24)}[dtype]
    step = torch.ldexp(torch.ones_like(x), (torch.frexp(x).exponent - bits).clamp(min=least).double())
    return (x / step).round() * step


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("n", [3, 8, 77, 8200])
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_values_next_to_ties(dtype, n, sign):
    import paper_2609_10264_amd as mvk
    ones = {BF: 128, HF: 1024}[dtype]  # values of `ones` to 2 ones - 1 have a step of one
    g = torch.Generator().manual_seed(5)
    tie = sign * (torch.randint(ones, 2 * ones, (4, n), generator=g).double() + 0.5) / ones
    off = torch.randint(-1, 2, (4, n), generator=g).double()
    want = nearest(tie + off * 2.0**-40, dtype)
    h = torch.zeros((4, n), dtype=dtype, device="cuda")
    mvk.block_norm(off.to(F32).cuda(), tie.to(F32).cuda(), scale=2.0**-40, out_dtype=FIELD, out_scale=2.0**-16, residual_out=h)
    assert torch.equal(h.double().cpu(), want)
    # (the test tells the two apart)
    twice = (tie + off * 2.0**-40).to(F32).to(dtype).double()
    assert not torch.equal(twice, want)


def test_ends_of_half_precision():
    import paper_2609_10264_amd as mvk
    # 65520 is between the largest number and infinity, 2^-25 between zero and the least
    res = torch.tensor([[65520.0, 65520.0, -65520.0, 2.0**-25, 2.0**-25, -(2.0**-25), 0.0, 1.0]], dtype=F32)
    off = torch.tensor([[-1.0, 1.0, 1.0, -1.0, 1.0, -1.0, 1.0, 0.0]], dtype=F32)
    h = torch.zeros((1, 8), dtype=HF, device="cuda")
    mvk.block_norm(off.cuda(), res.cuda(), scale=2.0**-60, out_dtype=FIELD, out_scale=2.0**-10, residual_out=h)
    # (in 64 bits 65520 - 2^-60 is 65520 itself, a tie: to infinity)
    assert h.cpu().tolist() == [[float("inf"), float("inf"), float("-inf"), 0.0, 2.0**-24, -(2.0**-24), 0.0, 1.0]]
    mvk.block_norm(off.cuda(), res.cuda(), scale=2.0**-30, out_dtype=FIELD, out_scale=2.0**-10, residual_out=h)
    assert h.cpu().tolist()[0][:3] == [65504.0, float("inf"), -65504.0]


def test_not_finite_values_stay():
    import paper_2609_10264_amd as mvk
    inf, nan = float("inf"), float("nan")
    res = torch.tensor([[inf, -inf, nan, 3e38, -3e38, 1e-45, 0.0, -0.0]], dtype=F32)
    for dtype, big in ((BF, torch.tensor(3e38, dtype=F32).to(BF).item()), (HF, inf)):
        h = torch.zeros((1, 8), dtype=dtype, device="cuda")
        mvk.block_norm(None, res.cuda(), out_dtype=FIELD, out_scale=1.0, residual_out=h)
        got = h.cpu().float().tolist()[0]
        assert got[:2] == [inf, -inf] and got[2] != got[2] and got[3:5] == [big, -big] and got[5:] == [0.0] * 3, got
