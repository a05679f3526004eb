"""A decoder layer with its values carried through (stack.run_decoder_layer): norms,
delegated projections, rotary positions, a cache in 16 or 8 bits, attention, the
gated activation; prompts, single tokens, an eviction, and the token drawn from
the logits, each step against its definition in 64 bits."""
import math

import pytest
import torch

import synth
from tests import attention_ref as ref
from tests import cache8_ref as c8
from tests import steps_ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


P, W, M = 2**31 - 1, 4096, 11008
TX, TY, ELL = 8, 11, 1
QUERY = {"attn_in": 2.0**-8, "attn_out": 2.0**-10, "mlp_in": 2.0**-8, "mlp_out": 2.0**-8}
FIELD = {"attn_in": 2.0**-16, "attn_out": 2.0**-19, "mlp_in": 2.0**-16, "mlp_out": 2.0**-18}
VOCAB = 1000


def _dev(a):
    return torch.from_numpy(a.astype("int32")).cuda()


@pytest.fixture(scope="module")
def layer():
    import paper_2609_10264_amd as mvk
    from paper_2609_10264_amd import stack

    def code(which, n):
        c = synth.raa_code(900 + which, n, 2)
        return mvk.Code(c["k"], c["r"], *(_dev(c[n]) for n in ("pi1", "pi2", "v1", "v2")))

    cx, cy = {n: code(n, n) for n in (W, M)}, {m: code(m + 1, m) for m in (W, M)}
    g = torch.Generator().manual_seed(3)
    raw = {name: torch.randint(-9, 10, (m, n), generator=g).to(torch.int8) for name, m, n, _ in stack.PROJECTIONS}
    lay = stack.build_layer({k: w.cuda() for k, w in raw.items()}, cx, cy)
    lay.raw = raw
    lay.head = torch.randint(-9, 10, (VOCAB, W), generator=g).to(torch.int8)
    return lay


def _draws(T, seed):
    from paper_2609_10264_amd import stack
    ex, ey = {}, {}
    for i, group in enumerate(stack.INPUTS):
        ex[group] = tuple(_dev(a) for a in synth.sparse(seed + i, T, 2 * stack.input_width(group), TX))
    for i, (name, m, _, _) in enumerate(stack.PROJECTIONS):
        ey[name] = tuple(_dev(a) for a in synth.sparse(seed + 10 + i, ELL, 2 * m, TY))
    return ex, ey


class Run:
    def __init__(self, layer, cache, dtype, after):
        import paper_2609_10264_amd as mvk
        self.layer, self.dtype = layer, dtype
        self.table = torch.tensor([[3, 0, 5], [1, 4, 2]], dtype=torch.int32)
        self.cache = mvk.KVCache.allocate(6, 32, 16, 128, dtype=cache)
        self.w = torch.zeros((2, 32, 48), device="cuda")
        self.rot = mvk.rotary_table(128, 4096)
        self.lens, self.pos = [0, 0], [0, 0]
        g = torch.Generator().manual_seed(8)
        names = ("attn_in", "mlp_in") + (("attn_out", "mlp_out") if after else ())
        self.norms = {n: mvk.Norm((1 + 0.2 * torch.randn(W, generator=g)).cuda()) for n in names}

    def args(self, new, seed):
        import paper_2609_10264_amd as mvk
        T = sum(new)
        g = torch.Generator().manual_seed(seed)
        h = (torch.randn((T, W), generator=g)).to(self.dtype).cuda()
        positions = torch.cat([torch.arange(p, p + c) for p, c in zip(self.pos, new)]).to(torch.int32).cuda()
        lens = [n + c for n, c in zip(self.lens, new)]
        seqs = mvk.Sequences(self.table.cuda(), torch.tensor(lens, dtype=torch.int32).cuda(), ref.starts(new).cuda(),
                             max_new=max(new))
        ex, ey = _draws(T, seed)
        return (self.layer, h, ex, ey, self.cache, seqs, positions, self.rot, self.norms, QUERY, FIELD), lens

    def query(self, res, name, group, ex):
        """The plaintext query of a projection: its masked one less the mask of its noise."""
        import paper_2609_10264_amd as mvk
        xhat = res[name][2]
        mask = mvk.encode(self.layer.keys[name], torch.zeros_like(xhat), *ex[group])
        return ref.lift(((xhat.long() - mask.long()) % P).to(torch.int32).cpu())

    def near(self, got, want, scale, rel, what):
        """Whole numbers of `scale`: half of one, and what the value before was off by, relative to the largest."""
        err = 0.5 + rel * want.abs().max() / scale
        assert bool(((got - want / scale).abs() <= err).all()), (what, float((got - want / scale).abs().max()), float(err))

    def step(self, new, seed):
        from paper_2609_10264_amd import stack
        args, lens = self.args(new, seed)
        T, h, ex, positions = sum(new), args[1].cpu().double(), args[2], args[6]
        self.lens, self.pos = lens, [p + c for p, c in zip(self.pos, new)]
        before = self.w.cpu()
        out, res = stack.run_decoder_layer(*args, weights=self.w)
        torch.cuda.synchronize()
        assert out.dtype == self.dtype and all(bool((r[1] == 1).all()) for r in res.values())
        norm = {k: (n.weight.cpu(), None, "rms", 1e-6) for k, n in self.norms.items()}
        x = {}
        for name, _, _, group in stack.PROJECTIONS:  # every projection is the product of its query
            if group not in x:
                x[group] = self.query(res, name, group, ex)
            assert torch.equal(ref.lift(res[name][0].cpu()), x[group] @ self.layer.raw[name].double().t()), name
        y = {name: ref.lift(res[name][0].cpu(), FIELD[group]) for name, _, _, group in stack.PROJECTIONS}
        # the query of q, k, v is the norm, the nearest whole number
        want = steps_ref.norm(h, *norm["attn_in"]) / QUERY["attn_in"]
        assert bool(((x["attn_in"] - want).abs() <= 0.5 + 2.0**-30 * want.abs()).all())
        # attention over what the cache holds
        rows = self.rot.cpu()[positions.cpu().long()]
        q, k = (ref.rotate(y[n].view(T, 32, 128), rows, "half") for n in "qk")
        K, V = self.values()
        t = 0
        for s, c in enumerate(new):
            for i in range(c):
                e = lens[s] - c + i
                pg = int(self.table[s, e // 16])
                for pool, row in ((K, k[t]), (V, y["v"].view(T, 32, 128)[t])):
                    got = pool[pg, :, e % 16].double()
                    if self.cache.k_exp is not None:
                        assert torch.equal(got, c8.worth(*c8.hold(row, self.cache.K.dtype), self.cache.K.dtype))
                    else:
                        assert bool(((got - row).abs() <= 2.0**-8 * row.abs() * 1.01 + 2.0**-20 * row.abs().max()).all())
                t += 1
        r = ref.Attention(q.to(torch.bfloat16), K, V, self.table, torch.tensor(lens), ref.starts(new), w_in=before,
                          out_dtype=torch.float32)
        err = 0.5 + (2 * r.o_err + 2.0**-7 * r.o.abs().max()) / QUERY["attn_out"]
        assert bool(((x["attn_out"].view(T, 32, 128) - r.o / QUERY["attn_out"]).abs() <= err).all())
        # the stream between the blocks, and the query of up and gate
        after = norm.get("attn_out")
        mlp, mid = steps_ref.block(y["o"], h, norm["mlp_in"], after, None, 1.0)
        self.near(x["mlp_in"], mlp, QUERY["mlp_in"], 2.0**-30, "query of up and gate")
        self.near(x["mlp_out"], steps_ref.activation(y["gate"], "silu") * y["up"], QUERY["mlp_out"], 2.0**-18, "query of down")
        u = steps_ref.ROUND[self.dtype]
        _, want = steps_ref.block(y["down"], mid, None, norm.get("mlp_out"), None, 1.0)
        # (the stream is rounded twice to its type, between the blocks and here)
        assert bool(((out.cpu().double() - want).abs() <= 2.01 * u * (mid.abs() + want.abs()) + 2.0**-18 * want.abs().max()).all())
        for s, n in enumerate(lens):
            total = self.w[s, :, :n].double().sum().item() - before[s, :, :n - new[s]].double().sum().item()
            assert abs(total - 32 * new[s]) < 1e-2
        return out

    def values(self):
        if self.cache.k_exp is None:
            return self.cache.K.cpu(), self.cache.V.cpu()
        kind = self.cache.K.dtype
        return tuple(c8.worth(x.view(torch.int8).cpu(), e.cpu(), kind).to(torch.bfloat16)
                     for x, e in ((self.cache.K, self.cache.k_exp), (self.cache.V, self.cache.v_exp)))

    def evict(self, budget):
        import paper_2609_10264_amd as mvk
        seqs = mvk.Sequences(self.table.cuda(), torch.tensor(self.lens, dtype=torch.int32).cuda())
        dst = mvk.KVCache.allocate(6, 32, 16, 128, dtype=self.cache.K.dtype)
        w = torch.zeros_like(self.w)
        _, lens = mvk.cache_evict(self.cache, seqs, self.w, dst, self.table.cuda(), budget, recent=4, sinks=1, weights_out=w)
        self.cache, self.w, self.lens = dst, w, lens.tolist()

    def answer(self, h, seed):
        """The final norm, the logits of the last product and the tokens drawn from them."""
        import paper_2609_10264_amd as mvk
        x, _ = mvk.block_norm(None, h, before=self.norms["attn_in"], out_dtype=mvk.FIELD, out_scale=QUERY["attn_in"])
        logits = mvk.server_eval(mvk.pack_weights(self.layer.head.cuda()), x)
        u = torch.rand(len(h), generator=torch.Generator().manual_seed(seed))
        scale = 2.0**-16
        token = mvk.sample(logits, u.cuda(), temperature=0.7, top_k=40, top_p=0.9, field_scale=scale)
        want = ref.lift(x.cpu()) @ self.layer.head.double().t()
        assert torch.equal(ref.lift(logits.cpu()), want)
        for r in range(len(h)):
            assert int(token[r]) == steps_ref.token(want[r] * scale, float(u[r]), 0.7, 40, 0.9, 0.0)[0]


@pytest.mark.parametrize("cache,dtype,after", [(torch.bfloat16, torch.float32, False), (c8.E4M3, torch.bfloat16, True),
                                               (c8.I8, torch.float32, True)])
def test_prompt_tokens_eviction_and_the_answer(layer, cache, dtype, after):
    run = Run(layer, cache, dtype, after)
    run.step([21, 8], 1000)
    run.step([1, 1], 1100)
    run.evict(12)
    assert run.lens == [12, 9]
    h = run.step([2, 1], 1200)
    run.answer(h, 5)


def test_a_rejected_layer_leaves_the_weights_and_may_be_repeated(layer):
    from paper_2609_10264_amd import stack
    run = Run(layer, c8.E4M3, torch.float32, False)
    run.step([9, 4], 2000)
    args, _ = run.args([1, 2], 2100)
    before, h = run.w.clone(), args[1].clone()

    def tamper(name, yhat):
        if name == "down":
            yhat[1, 77] = (yhat[1, 77] + 5) % P

    _, res = stack.run_decoder_layer(*args, weights=run.w, tamper=tamper)
    assert res["down"][1].tolist() == [1, 0, 1] and res["o"][1].tolist() == [1, 1, 1]
    assert torch.equal(run.w, before) and torch.equal(args[1], h)
    run.step([1, 2], 2100)
    assert not torch.equal(run.w, before)


def test_on_another_stream_and_in_a_graph(layer):
    from paper_2609_10264_amd import stack
    run, other, third = (Run(layer, c8.I8, torch.float32, False) for _ in range(3))
    for r in (run, other, third):
        r.step([5, 3], 3000)
    want, _ = stack.run_decoder_layer(*run.args([1, 1], 3100)[0], weights=run.w)
    side = torch.cuda.Stream()
    args = other.args([1, 1], 3100)[0]
    torch.cuda.synchronize()
    got, _ = stack.run_decoder_layer(*args, weights=other.w, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(got, want) and torch.equal(other.w, run.w)
    args = third.args([1, 1], 3100)[0]
    w0 = third.w.clone()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        out, _ = stack.run_decoder_layer(*args, weights=third.w)
    for _ in range(3):
        third.w.copy_(w0)
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(third.w, run.w)
    assert math.isfinite(float(out.abs().max()))
