"""The attention block on another stream than the current one: what the call
itself allocates is not handed out again while that stream still has it to use."""
import pytest
import torch

from tests import attention_ref as ref
from tests.test_gpu_attention_stack import FIELD_SCALE, OUT_SCALE, W, Run, _draws, layer  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def test_memory_of_a_late_stream_is_left_alone(layer):  # noqa: F811
    import paper_2609_10264_amd as mvk
    from paper_2609_10264_amd import stack
    T, new = 29, [21, 8]
    g = torch.Generator().manual_seed(5)
    x = ref.embed(torch.randint(-60, 61, (T, W), generator=g)).cuda()
    positions = torch.cat([torch.arange(c) for c in new]).to(torch.int32).cuda()
    ex, ey = _draws(T, 50)
    side = torch.cuda.Stream()

    def call(run, stream):
        seqs = mvk.Sequences(run.table.cuda(), torch.tensor(new, dtype=torch.int32).cuda(), ref.starts(new).cuda())
        torch.cuda.synchronize()
        if stream is not None:
            with torch.cuda.stream(stream):
                torch.cuda._sleep(200_000_000)  # about 0.1 s: the work below waits for it
        y, res = stack.run_attention(layer, x, ex, ey, run.cache, seqs, positions, run.rot, FIELD_SCALE, OUT_SCALE,
                                     weights=run.w, stream=stream)
        # the current stream asks for memory of the sizes that the call has let go, and writes it
        junk = [torch.full((T, W), 7, dtype=d, device="cuda") for d in (torch.int32, torch.bfloat16) for _ in range(6)]
        junk += [torch.full_like(run.w, 3.0) for _ in range(4)]
        torch.cuda.synchronize()
        assert all(bool((r[1] == 1).all()) for r in res.values())
        return y.clone(), junk

    here, there = Run(layer), Run(layer)
    call(Run(layer), side)  # (the stream's workspaces)
    want, _ = call(here, None)
    got, _ = call(there, side)
    assert torch.equal(got, want) and torch.equal(there.w, here.w)
    assert torch.equal(there.cache.K, here.cache.K) and torch.equal(there.cache.V, here.cache.V)
