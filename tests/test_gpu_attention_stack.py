"""The attention block of a delegated layer with its values carried through
(stack.run_attention): projections by delegation, rotary positions and cache,
attention, the output projection; a prompt, single tokens, an eviction, and more
tokens after it."""
import pytest
import torch

import synth
from tests import attention_ref as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


P, W = 2**31 - 1, 4096
TX, TY, ELL = 16, 31, 2
FIELD_SCALE, OUT_SCALE = 2.0**-16, 2.0**-6


def _dev(a):
    return torch.from_numpy(a.astype("int32")).cuda()


@pytest.fixture(scope="module")
def layer():
    import paper_2609_10264_amd as mvk
    from paper_2609_10264_amd import stack

    def code(which):
        c = synth.raa_code(700 + which, W, 2)
        return mvk.Code(c["k"], c["r"], *(_dev(c[n]) for n in ("pi1", "pi2", "v1", "v2")))

    cx, cy = code(0), code(1)
    g = torch.Generator().manual_seed(3)
    lay = stack.Layer()
    lay.raw = {}
    for name in ("q", "k", "v", "o"):
        w = torch.randint(-9, 10, (W, W), generator=g).to(torch.int8)
        lay.raw[name] = w
        lay.keys[name] = mvk.keygen(mvk.Key.allocate(W, W, cx, cy), w.cuda())
        lay.W[name] = mvk.pack_weights(w.cuda())
    return lay


def _draws(T, seed):
    ex, ey = {}, {}
    for i, group in enumerate(("attn_in", "attn_out")):
        ex[group] = tuple(_dev(a) for a in synth.sparse(seed + i, T, 2 * W, TX))
    for i, name in enumerate(("q", "k", "v", "o")):
        ey[name] = tuple(_dev(a) for a in synth.sparse(seed + 10 + i, ELL, 2 * W, TY))
    return ex, ey


class Run:
    """Two sequences with a cache, and the same steps in 64 bits."""

    def __init__(self, layer):
        import paper_2609_10264_amd as mvk
        self.layer = layer
        self.page = 16
        self.table = torch.tensor([[3, 0, 5], [1, 4, 2]], dtype=torch.int32)
        self.cache = mvk.KVCache.allocate(6, 32, self.page, 128)
        self.w = torch.zeros((2, 32, 48), device="cuda")
        self.rot = mvk.rotary_table(128, 4096)
        self.lens = [0, 0]
        self.pos = [0, 0]  # positions go on where evictions shorten the cache

    def step(self, new, seed, tamper=None):
        import paper_2609_10264_amd as mvk
        from paper_2609_10264_amd import stack
        T = sum(new)
        self.lens = [n + c for n, c in zip(self.lens, new)]
        g = torch.Generator().manual_seed(seed)
        x = torch.randint(-60, 61, (T, W), generator=g)
        positions = torch.cat([torch.arange(p, p + c) for p, c in zip(self.pos, new)]).to(torch.int32)
        self.pos = [p + c for p, c in zip(self.pos, new)]
        q_start = ref.starts(new)
        seqs = mvk.Sequences(self.table.cuda(), torch.tensor(self.lens, dtype=torch.int32).cuda(), q_start.cuda(),
                             max_new=max(new))
        before = self.w.cpu()
        ex, ey = _draws(T, seed)
        yo, res = stack.run_attention(self.layer, ref.embed(x).cuda(), ex, ey, self.cache, seqs, positions.cuda(),
                                      self.rot, FIELD_SCALE, OUT_SCALE, weights=self.w, tamper=tamper)
        torch.cuda.synchronize()
        accept = {n: r[1].cpu() for n, r in res.items()}
        if tamper is not None:
            return accept
        assert all(bool((a == 1).all()) for a in accept.values())
        # q, k, v are the products; the cache has the rotated keys and the values
        y = {n: x.double() @ self.layer.raw[n].double().t() for n in "qkv"}
        for n in "qkv":
            assert torch.equal(ref.lift(res[n][0].cpu()), y[n])
        val = {n: (y[n] * FIELD_SCALE).view(T, 32, 128) for n in "qkv"}
        rows = self.rot.cpu()[positions.long()]
        q, k = ref.rotate(val["q"], rows, "half"), ref.rotate(val["k"], rows, "half")
        K, V = self.cache.K.cpu(), self.cache.V.cpu()
        t = 0
        for s, c in enumerate(new):
            for i in range(c):
                e = self.lens[s] - c + i
                pg = int(self.table[s, e // self.page])
                for pool, want in ((K, k[t]), (V, val["v"][t])):
                    got = pool[pg, :, e % self.page].double()
                    assert bool(((got - want).abs() <= 2.0**-8 * want.abs() * 1.01 + 2.0**-20 * val["k"].abs().max()).all())
                t += 1
        # attention over what the cache holds, then o's product of it, exactly
        r = ref.Attention(q.to(torch.bfloat16), K, V, self.table, torch.tensor(self.lens), q_start, w_in=before,
                          out_dtype=torch.float32)
        xo = ref.lift(_unmask(res["o"], self.layer, ex))
        err = 0.5 + (2 * r.o_err + 2.0**-7 * r.o.abs().max()) / OUT_SCALE
        assert bool(((xo.view(T, 32, 128) - r.o / OUT_SCALE).abs() <= err).all())
        assert torch.equal(ref.lift(yo.cpu()), xo @ self.layer.raw["o"].double().t())
        for s, n in enumerate(self.lens):
            total = self.w[s, :, :n].double().sum().item()
            assert abs(total - before[s, :, :n - new[s]].double().sum().item() - 32 * new[s]) < 1e-2
        return accept

    def evict(self, budget, recent):
        import paper_2609_10264_amd as mvk
        seqs = mvk.Sequences(self.table.cuda(), torch.tensor(self.lens, dtype=torch.int32).cuda())
        dst = mvk.KVCache.allocate(6, 32, self.page, 128)
        w = torch.zeros_like(self.w)
        old = self.w.cpu()
        kept, lens = mvk.cache_evict(self.cache, seqs, self.w, dst, self.table.cuda(), budget, recent=recent, sinks=1,
                                     weights_out=w)
        for s, n in enumerate(self.lens):
            for h in (0, 17, 31):
                want = ref.evict(old[s, h, :n].tolist(), n, budget, recent, 1)
                assert kept[s, h].tolist()[:len(want)] == want
        self.cache, self.w, self.lens = dst, w, lens.tolist()


def _unmask(o, layer, ex):
    """The plaintext query of o: its masked one less the mask of its noise (as field elements)."""
    import paper_2609_10264_amd as mvk
    zero = torch.zeros_like(o[2])
    mask = mvk.encode(layer.keys["o"], zero, *ex["attn_out"])
    return ((o[2].long() - mask.long()) % P).to(torch.int32).cpu()


def test_prompt_tokens_eviction_and_more_tokens(layer):
    run = Run(layer)
    run.step([21, 8], 1000)
    run.step([1, 1], 1100)
    run.step([5, 1], 1200)
    run.evict(12, 4)
    assert run.lens == [12, 10]
    run.step([1, 1], 1300)
    run.step([9, 2], 1400)


def test_a_tampered_response_is_rejected(layer):
    run = Run(layer)

    def tamper(name, yhat):
        if name == "k":
            yhat[2, 77] = (yhat[2, 77] + 5) % P

    accept = run.step([3, 2], 2000, tamper=tamper)
    assert accept["k"].tolist() == [1, 1, 0, 1, 1]
    assert accept["q"].tolist() == accept["v"].tolist() == accept["o"].tolist() == [1] * 5
