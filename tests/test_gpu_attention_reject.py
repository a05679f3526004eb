"""A step of the attention block whose responses are rejected leaves the client's
state as it was, and the same step can be made again (stack.run_attention)."""
import pytest
import torch

from tests import attention_ref as ref
from tests.test_gpu_attention_stack import FIELD_SCALE, OUT_SCALE, P, W, Run, _draws, layer  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


@pytest.mark.parametrize("which", ["q", "k", "v", "o"])
def test_a_rejected_step_and_its_repetition(layer, which):  # noqa: F811
    honest, run = Run(layer), Run(layer)
    for r in (honest, run):
        r.step([21, 8], 1000)
        r.step([1, 1], 1100)
    assert torch.equal(run.w, honest.w)

    def tamper(name, yhat):
        if name == which:
            yhat[1] = (yhat[1].long() * 7 + 123456789).remainder(P).to(torch.int32)

    lens, pos, w = list(run.lens), list(run.pos), run.w.clone()
    accept = run.step([5, 1], 1200, tamper=tamper)
    assert 0 in accept[which].tolist()
    assert torch.equal(run.w, w)
    run.lens, run.pos = lens, pos
    run.step([5, 1], 1200)
    honest.step([5, 1], 1200)
    assert torch.equal(run.w, honest.w) and not torch.equal(run.w, w)
    assert torch.equal(run.cache.K, honest.cache.K) and torch.equal(run.cache.V, honest.cache.V)
    for r in (honest, run):
        r.evict(12, 4)
        r.step([1, 1], 1300)
    assert torch.equal(run.w, honest.w)


def test_weights_of_a_wider_tensor(layer):  # noqa: F811
    """Weights that are a part of a larger tensor: their strides are kept, their neighbours left alone."""
    a, b = Run(layer), Run(layer)
    every = torch.full((2, 3, 32, 64), -1.0, device="cuda")
    b.w = every[:, 1, :, 5:53].zero_()
    for r in (a, b):
        r.step([9, 4], 1500)
        r.step([1, 1], 1600)
    assert torch.equal(b.w, a.w) and bool(a.w.any())
    every[:, 1, :, 5:53] = -1.0
    assert bool((every == -1.0).all())
