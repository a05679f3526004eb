"""Field elements out of mvk_gated_activation: the value in 32 bits over out_scale, any
positive number, rounded once more only."""
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
ACTS = ["silu", "gelu", "gelu_tanh", "relu"]
U = 2.0**-24


def _check(g, u, act, in_scale, out_scale, p=P):
    """g, u: tensors of one type."""
    import paper_2609_10264_amd as mvk
    y = mvk.gated_activation(g.cuda(), u.cuda(), act=act, field_scale=in_scale, out_dtype=FIELD, out_scale=out_scale, p=p)
    x, v = ref.lift(g, in_scale, p), ref.lift(u, in_scale, p)
    one = float(torch.tensor(out_scale, dtype=F32))  # (the call takes a 32-bit float)
    half = (p - 1) // 2
    exact = (steps_ref.activation(x, act) * v / one).clamp(-half, half)
    # In 32 bits: the argument of the exponential (or of erfc, which falls as exp(-g^2 / 2)) is off by a few
    # roundings relative to its size, and so is what follows by as much and a few more; below the least normal
    # number a product is off by half of 2^-149.
    arg = {"silu": x.abs(), "gelu": x.square(), "gelu_tanh": 1.6 * x.abs() + 0.15 * x.abs()**3, "relu": 0 * x}[act]
    err = (16 + 6 * arg) * U * exact.abs() + 2.0**-150 / one
    got = ref.lift(y.cpu(), 1.0, p)
    bad = (got - exact).abs() > 0.5 + err
    assert not bool(bad.any()), (act, int(bad.sum()), float((got - exact).abs().max()))
    return got


def _values(shape, dtype, seed, spread, p=P):
    x = torch.randn(shape, generator=torch.Generator().manual_seed(seed), dtype=torch.float64) * spread
    return ref.embed((x * 2**16).round().long(), p) if dtype == FIELD else x.to(dtype)


@pytest.mark.parametrize("out_scale", [1e-3, 3e-7, 0.1, 7.0, 2.0**-6])
@pytest.mark.parametrize("n", [5, 8, 77, 1000])
def test_values_of_24_bits_over_any_scale(out_scale, n):
    """Products that 32 bits hold: what is left is one rounding, to the whole number."""
    import paper_2609_10264_amd as mvk
    gen = torch.Generator().manual_seed(3)
    g, u = torch.randint(0, 4096, (9, n), generator=gen), torch.randint(-4096, 4096, (9, n), generator=gen)
    one, half = float(torch.tensor(out_scale, dtype=F32)), (P - 1) // 2
    exact = ((g * u).double() / one).clamp(-half, half)
    for kind in (F32, FIELD):
        x, v = (ref.embed(t) if kind == FIELD else t.to(kind) for t in (g, u))
        y = mvk.gated_activation(x.cuda(), v.cuda(), act="relu", field_scale=1.0, out_dtype=FIELD, out_scale=out_scale)
        assert bool(((ref.lift(y.cpu()) - exact).abs() <= 0.5 + 2.0**-51 * exact.abs()).all())


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("dtype", [BF, HF, F32, FIELD])
@pytest.mark.parametrize("n", [5, 8, 77, 1000])
def test_scales(act, dtype, n):
    g, u = _values((9, n), dtype, 1, 3.0), _values((9, n), dtype, 2, 1.0)
    for out_scale in (2.0**-24, 1e-3, 3e-7, 2.0**-8):
        _check(g, u, act, 2.0**-16, out_scale)


@pytest.mark.parametrize("act", ["silu", "relu"])
@pytest.mark.parametrize("p", [P, BB])
def test_whole_residues_in(act, p):
    gen = torch.Generator().manual_seed(3)
    g, u = (torch.randint(-(p // 2), p // 2 + 1, (7, 300), generator=gen) for _ in range(2))
    _check(ref.embed(g, p), ref.embed(u, p), act, 2.0**-26, 2.0**-20, p)


@pytest.mark.parametrize("out_scale", [2.0**-126, 2.0**-127, 2.0**-128, 1e-40, 1.4e-45])
def test_scales_whose_reciprocal_32_bits_do_not_hold(out_scale):
    g = torch.tensor([[1.0, 3.0, -2.0, 0.75, 7.0, 0.0, 100.0, -1.0, 0.25]], dtype=F32).repeat(3, 1)
    u = (torch.tensor([[1.0], [2.5], [1000.0]], dtype=torch.float64) * out_scale).to(F32).expand(3, 9).contiguous()
    got = _check(g, u, "relu", 1.0, out_scale)
    assert bool((got[0, :5] == torch.tensor([1.0, 3.0, 0.0, 1.0, 7.0])).all()), got[0]
    assert int(got.abs().max()) < (P - 1) // 2
    for act in ACTS:
        _check(g, u, act, 1.0, out_scale)
        _check(g[:, :8].contiguous(), u[:, :8].contiguous(), act, 1.0, out_scale)


def test_ends():
    """What is beyond the field is clamped, a not-a-number is zero."""
    import paper_2609_10264_amd as mvk
    g = torch.tensor([[1e30, 1e30, math.inf, math.nan, -1e30, -800.0, 3e4, 0.0]], dtype=F32)
    u = torch.tensor([[1.0, -1.0, 2.0, 1.0, 1.0, 1e30, 3e4, 5.0]], dtype=F32)
    half = (P - 1) // 2
    for act in ("silu", "gelu", "gelu_tanh", "relu"):
        y = mvk.gated_activation(g.cuda(), u.cuda(), act=act, out_dtype=FIELD, out_scale=2.0**-20)
        assert ref.lift(y.cpu()).tolist() == [[half, -half, half, 0, 0, 0, half, 0]], act
