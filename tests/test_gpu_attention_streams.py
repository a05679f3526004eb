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


def test_two_streams_at_once():
    """Calls in flight together on two streams, each with its own workspace and counters:
    tiles of several workgroups in both, results as one after the other."""
    import paper_2609_10264_amd as mvk
    from tests.test_gpu_attention import Problem
    problems = [Problem([9000, 70, 700], [1, 1, 1], 16, 2, 128, page=32).device(),
                Problem([5003, 260], [150, 260], 8, 2, 64, page=16, seed=2).device()]

    def call(pr, stream=None):
        lse = torch.zeros(pr.q.shape[:2], device="cuda")
        w = torch.zeros((len(pr.lens), 2, pr.cap), device="cuda")
        out = torch.zeros_like(pr.dq)
        torch.cuda.synchronize()

        def go():
            mvk.paged_attention(pr.dq, pr.cache, pr.seqs, out=out, lse=lse, weights_out=w, stream=stream)
        go()
        torch.cuda.synchronize()
        return out, lse, w, go

    want = [call(pr)[:3] for pr in problems]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [call(pr, s) for pr, s in zip(problems, streams)]
    for _ in range(20):
        for *outs, go in got:
            for _ in range(3):
                go()
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert all(torch.equal(x, y) for x, y in zip(a, b))
            for x in a[:3]:
                x.zero_()
        torch.cuda.synchronize()
