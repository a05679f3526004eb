"""The rest of the client's token step between the delegated projections, as cases
that can be timed: what a decoder layer needs beside attention, and the token that
answers.

  append   rotary positions on new tokens' queries and keys and the append of keys
           and values to a cache held in 8 bits with one power of two an entry and
           head, read back as the values that it stands for
  attend   attention of each sequence's new tokens over such a cache, with, where
           "weights" is set, the attention weight that every entry has collected
  norm     the end of a block and the beginning of the next: norm of the block's
           result, gate, scale and residual, and the norm of the sum
  gated    an activation of one projection times another
  sample   a token a row by temperature, top-k, top-p and min-p from given random
           numbers

`own` false computes them in elementary torch operations, in 32 bits, and in 64
where a value next to a border or a long sum decides a whole number; `own` true
calls the library.

Layouts: the cache's pools are pages x kv_heads x page x dim, its exponents pages x
kv_heads x page; entry j of sequence s lies in page table[s, j // page] at j % page.
Tokens of all sequences follow one another, q_start (S + 1) says where each begins;
lens counts a sequence's entries, its new tokens included.
"""
import math
import random

import numpy as np
import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32, "e4m3": torch.float8_e4m3fn,
         "i8": torch.int8}
SIZES = {"bf16": 2, "f16": 2, "f32": 4, "field": 4, "e4m3": 1, "i8": 1}
LARGEST = {"e4m3": 448.0, "i8": 127.0}  # of a code
LEAST, MOST = -96, 119  # exponents of an entry
PRIME = 2**31 - 1
FIELD_SCALE = 2.0**-16  # the value of 1 in field elements


# ---------------------------------------------------------------------------
# The cases
# ---------------------------------------------------------------------------
def _append(name, **kw):
    c = dict(name=name, kind="append", S=1, new_lo=1, new_hi=1, ctx_lo=0, ctx_hi=0, heads=32, kv_heads=32, dim=128,
             rot=128, layout="half", source="field", cache="e4m3", page=64, max_pos=32768, slack=False)
    c.update(kw)
    return c


def _attend(name, **kw):
    c = dict(name=name, kind="attend", S=1, new_lo=1, new_hi=1, ctx_lo=0, ctx_hi=0, heads=32, kv_heads=32, dim=128,
             cache="e4m3", page=64, weights=False)
    c.update(kw)
    return c


def _norm(name, **kw):
    c = dict(name=name, kind="norm", T=1, n=4096, source="field", stream="f32", params="f32", out="field", norm="rms",
             after=False, gate="none", scale=1.0, slack=False)
    c.update(kw)
    return c


def _gated(name, **kw):
    c = dict(name=name, kind="gated", T=1, n=11008, source="field", out="f32", act="silu", slack=False)
    c.update(kw)
    return c


def _sample(name, **kw):
    c = dict(name=name, kind="sample", R=1, V=32000, source="bf16", temperature=0.8, top_k=0, top_p=1.0, min_p=0.0,
             per_row=False, greedy=0)
    c.update(kw)
    return c


def listed():
    return [
        # One decrypted token of a 4096-wide layer written to the cache: latency only.
        _append("append_one_token", ctx_lo=2047, ctx_hi=2047),
        # A long prompt of an 8192-wide layer with grouped heads, q, k and v slices of one
        # stacked projection.
        _append("append_prompt_grouped", new_lo=8192, new_hi=8192, heads=64, kv_heads=8, source="bf16", cache="i8",
                slack=True),
        # One token of one sequence over 2048 entries: the smallest call.
        _attend("attend_one_token", ctx_lo=2047, ctx_hi=2047, cache="i8"),
        # Single tokens of 48 sequences of very different lengths, grouped heads: a serving step.
        _attend("attend_tokens_ragged", S=48, ctx_lo=130, ctx_hi=32767, heads=64, kv_heads=8, page=32),
        # Chunks and single tokens mixed, odd lengths, a narrow head, small pages, collected weights.
        _attend("attend_mixed_weights", S=21, new_lo=1, new_hi=701, ctx_lo=0, ctx_hi=5003, heads=28, kv_heads=4, dim=80,
                cache="i8", page=16, weights=True),
        # A chunk of 512 tokens of one long context, grouped heads: the largest.
        _attend("attend_chunk_long", new_lo=512, new_hi=512, ctx_lo=16000, ctx_hi=16000, heads=64, kv_heads=8),
        # Between attention and the feed-forward part of a 4096-wide layer, eight tokens:
        # decrypted result in, query of the next projection out.
        _norm("norm_stack_step", T=8),
        # A prompt of an 8192-wide layer with norms on both sides of the block and a gate a channel.
        _norm("norm_prompt_both", T=8192, n=8192, source="bf16", stream="bf16", params="bf16", out="bf16", after=True,
              gate="channel"),
        # Eight tokens of an 11008-wide feed-forward part as they come out of decryption.
        _gated("gated_stack_step", T=8),
        # A prompt through it, both halves slices of one stacked projection.
        _gated("gated_prompt", T=8192, source="bf16", out="bf16", slack=True),
        # The next token of one sequence.
        _sample("sample_one", top_k=50, top_p=0.9),
        # A serving batch over a large odd vocabulary with everybody's own settings, from decrypted logits.
        _sample("sample_batch_own", R=64, V=131071, source="field", top_k=400, top_p=0.95, min_p=0.02, per_row=True, greedy=5),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["append", "attend", "attend", "norm", "gated", "sample", "sample"])
    kv_heads = rng.choice([1, 2, 4, 5, 8, 16, 32])
    group = rng.choice([1, 1, 2, 4, 6, 7, 8]) if kv_heads <= 8 else 1
    dim = rng.choice([64, 80, 96, 128, 128, 128])
    common = dict(kv_heads=kv_heads, dim=dim, cache=rng.choice(["e4m3", "i8"]), page=rng.choice([16, 32, 64, 128]))
    while True:
        S = _log(rng, 1, 64)
        single = rng.random() < 0.4
        new_hi = 1 if single else _log(rng, 2, 8192)
        new_lo = 1 if single else _log(rng, 1, new_hi)
        ctx_hi = _log(rng, 1, 32768)
        ctx_lo = rng.choice([0, ctx_hi, _log(rng, 1, ctx_hi)])
        both = dict(S=S, new_lo=new_lo, new_hi=new_hi, ctx_lo=ctx_lo, ctx_hi=ctx_hi, heads=kv_heads * group, **common)
        floats = ["bf16", "bf16", "f16", "f32"]
        if kind == "append":
            c = _append("", rot=rng.choice([dim, dim, dim // 2]), layout=rng.choice(["half", "interleaved"]),
                        source=rng.choice(["field", "bf16", "f16", "f32"]), max_pos=65536, slack=rng.random() < 0.5,
                        **both)
            fits = work(c)["bytes"] <= 300e6 and S * (new_hi + ctx_hi) * kv_heads * dim <= 1e9
        elif kind == "attend":
            c = _attend("", weights=rng.random() < 0.3, **both)
            pad = S * new_hi * c["heads"] * (new_hi + ctx_hi)  # scores of the padded plain form
            fits = work(c)["flops"] <= 2.5e11 and pad <= 1.1e9 and S * (new_hi + ctx_hi) * kv_heads * dim <= 1e9
        elif kind == "norm":
            n = rng.choice([_log(rng, 64, 16384), 8 * _log(rng, 8, 2048)])
            c = _norm("", T=_log(rng, 1, 16384), n=n, source=rng.choice(["field"] + floats), stream=rng.choice(floats),
                      params=rng.choice(["f32", "bf16"]), out=rng.choice(["field"] + floats),
                      norm=rng.choice(["rms", "rms", "layer"]), after=rng.random() < 0.4,
                      gate=rng.choice(["none", "channel", "token"]), scale=rng.choice([1.0, 0.25, 1.5]),
                      slack=rng.random() < 0.4)
            fits = work(c)["bytes"] <= 500e6
        elif kind == "gated":
            n = rng.choice([_log(rng, 64, 32768), 8 * _log(rng, 8, 4096)])
            c = _gated("", T=_log(rng, 1, 16384), n=n, source=rng.choice(["field"] + floats), out=rng.choice(floats),
                       act=rng.choice(["silu", "gelu", "gelu_tanh", "relu"]), slack=rng.random() < 0.4)
            fits = work(c)["bytes"] <= 500e6
        else:
            V = _log(rng, 1000, 200000)
            c = _sample("", R=_log(rng, 1, 256), V=V, source=rng.choice(["field", "bf16", "f16", "f32"]),
                        temperature=rng.choice([0.6, 1.0, 1.3]), top_k=rng.choice([0, 1, 50, _log(rng, 1, V)]),
                        top_p=rng.choice([1.0, 0.5, 0.9, 0.95]), min_p=rng.choice([0.0, 0.0, 0.05]),
                        per_row=rng.random() < 0.5, greedy=rng.choice([0, 1]))
            fits = c["R"] * V <= 8.3e6 and c["greedy"] <= c["R"]
        if fits:
            del c["name"]
            return c


def _spread(lo, hi, n):
    """n lengths from lo to hi, even in their logarithm."""
    if n == 1:
        return [hi]
    a, b = math.log(lo + 1), math.log(hi + 1)
    return [int(round(math.exp(a + (b - a) * i / (n - 1)))) - 1 for i in range(n)]


def _lengths(case):
    """(entries, new tokens) of every sequence; long contexts go with short chunks."""
    S = case["S"]
    ctx = _spread(case["ctx_lo"], case["ctx_hi"], S)
    new = _spread(case["new_lo"], case["new_hi"], S)[::-1]
    return [(n + c, c) for n, c in zip(ctx, new)]


# ---------------------------------------------------------------------------
# Inputs, from the seed alone
# ---------------------------------------------------------------------------
def _pages(lens, page):
    return [max(1, -(-n // page)) for n in lens]


def _table(lens, page, width, order):
    """S x width page numbers: every sequence's pages, scattered over the pool; 0 beyond."""
    used = _pages(lens, page)
    rows, at = [], 0
    for n in used:
        rows.append(order[at:at + n] + [0] * (width - n))
        at += n
    return torch.tensor(rows, dtype=torch.int32, device="cuda")


def _int(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _embed(x):
    """Integers as field elements."""
    return torch.where(x < 0, x + PRIME, x).to(torch.int32)


def _values(g, shape, kind, slack=0, spread=1.0):
    """Projection-like values of a type or as decrypted fixed-point numbers; with slack a slice of a wider row,
    as a stacked projection leaves it."""
    wide = shape[:-1] + (shape[-1] + 2 * slack,)
    x = torch.randn(wide, device="cuda", generator=g) * spread
    x = _embed((x / FIELD_SCALE).round().to(torch.int64)) if kind == "field" else x.to(TYPES[kind])
    return x[..., slack:slack + shape[-1]]


def _heads(g, T, H, D, kind, slack):
    return _values(g, (T, H * D), kind, D if slack else 0).unflatten(1, (H, D))


def prepare(case, seed):
    rng = random.Random(int(seed))
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    s = dict(case=case)
    if case["kind"] == "norm":
        T, n, p = case["T"], case["n"], TYPES[case["params"]]
        s["x"] = _values(g, (T, n), case["source"], 8 if case["slack"] else 0)
        s["stream"] = _values(g, (T, n), case["stream"], 0, 3.0)
        names = ["weight", "after"] + (["bias", "after_bias"] if case["norm"] == "layer" else [])
        for name in names:
            s[name] = ((0.0 if "bias" in name else 1.0) + 0.3 * torch.randn(n, device="cuda", generator=g)).to(p)
        rows = {"none": None, "channel": (n,), "token": (T, n)}[case["gate"]]
        s["gate"] = torch.randn(rows, device="cuda", generator=g).to(p) if rows else None
        s["stream_out"] = torch.zeros((T, n), dtype=TYPES[case["stream"]], device="cuda")
        s["out"] = torch.zeros((T, n), dtype=TYPES.get(case["out"], torch.int32), device="cuda")
        return s
    if case["kind"] == "gated":
        T, n = case["T"], case["n"]
        if case["slack"]:
            both = _values(g, (T, 2 * n), case["source"], 0, 2.0)
            s["gate"], s["up"] = both[:, :n], both[:, n:]
        else:
            s["gate"], s["up"] = (_values(g, (T, n), case["source"], 0, 2.0) for _ in range(2))
        s["out"] = torch.zeros((T, n), dtype=TYPES[case["out"]], device="cuda")
        return s
    if case["kind"] == "sample":
        R, V = case["R"], case["V"]
        # a model's logits: a wide middle and a few tokens far above it
        x = 2.2 * torch.randn((R, V), device="cuda", generator=g)
        x += torch.where(torch.rand((R, V), device="cuda", generator=g) < 30 / V, 9.0, 0.0)
        # some tokens are forbidden (a grammar's mask); field elements have no infinity
        if case["source"] == "field":
            s["logits"] = _embed((x / FIELD_SCALE).round().to(torch.int64))
        else:
            banned = torch.rand((R, V), device="cuda", generator=g) < 0.05
            s["logits"] = torch.where(banned, -math.inf, x).to(TYPES[case["source"]])
        s["u"] = torch.rand(R, device="cuda", generator=g)
        s["temperature"], s["top_k"], s["top_p"], s["min_p"] = (case[k] for k in ("temperature", "top_k", "top_p", "min_p"))
        if case["per_row"]:
            f = torch.rand((3, R), device="cuda", generator=g)
            s["temperature"] = case["temperature"] * (0.7 + 0.6 * f[0])
            s["temperature"][:case["greedy"]] = 0.0
            s["top_k"] = (torch.rand(R, device="cuda", generator=g) * 2 * case["top_k"]).to(torch.int32)
            s["top_p"] = (case["top_p"] * (0.9 + 0.1 * f[1])) if case["top_p"] < 1 else torch.ones(R, device="cuda")
            s["min_p"] = case["min_p"] * f[2]
        s["out"] = torch.zeros(R, dtype=torch.int32, device="cuda")
        s["probs"] = torch.zeros(R, device="cuda")
        return s
    pairs = _lengths(case)
    rng.shuffle(pairs)
    lens, new = [n for n, _ in pairs], [c for _, c in pairs]
    page, hk, h, d, kind = case["page"], case["kv_heads"], case["heads"], case["dim"], case["cache"]
    width = max(_pages(lens, page))
    count = sum(_pages(lens, page))
    order = list(range(count + 1))
    rng.shuffle(order)
    T, S = sum(new), case["S"]
    s.update(lens=_int(lens), table=_table(lens, page, width, order), max_new=max(new), max_len=max(lens))
    s["q_start"] = _int([sum(new[:i]) for i in range(len(new) + 1)])
    s["seq"] = torch.repeat_interleave(torch.arange(S, device="cuda"), _int(new).long())
    # what earlier tokens wrote lies in the cache (and what earlier sequences left, in the places not in use)
    for name in ("K", "V"):
        x = torch.randn((count + 1, hk, page, d), device="cuda", generator=g)
        if name == "K" and case["kind"] == "attend":
            # keys with some entries that many queries look at, as trained heads have
            x = torch.where(torch.rand((count + 1, hk, page, 1), device="cuda", generator=g) < 0.02, x * 2, x)
        s[name], s[name + "e"] = _quantise(x, kind)
    if case["kind"] == "append":
        s["q"], s["k"], s["v"] = (_heads(g, T, n, d, case["source"], case["slack"]) for n in (h, hk, hk))
        s["positions"] = torch.cat([torch.arange(n - c, n, device="cuda") for n, c in pairs]).to(torch.int32)
        half = case["rot"] // 2
        freq = 10000.0 ** (-torch.arange(half, device="cuda", dtype=torch.float64) / half)
        angle = torch.arange(case["max_pos"], device="cuda", dtype=torch.float64)[:, None] * freq
        s["rot_table"] = torch.cat([angle.cos(), angle.sin()], 1).float()
        s["q_out"] = torch.zeros((T, h, d), dtype=torch.bfloat16, device="cuda")
        s["k_out"], s["v_out"] = (torch.zeros((T, hk, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    else:
        s["q"] = _values(g, (T, h, d), "bf16")
        if case["weights"]:
            s["w"] = torch.rand((S, hk, width * page), device="cuda", generator=g) ** 8
            s["w_out"] = torch.zeros_like(s["w"])
    return s


# ---------------------------------------------------------------------------
# The library's operators
# ---------------------------------------------------------------------------
def _run_own(s):
    import paper_2609_10264_amd as mvk

    case = s["case"]
    scale = FIELD_SCALE if case.get("source") == "field" else None
    if case["kind"] == "norm":
        after = mvk.Norm(s["after"], s.get("after_bias"), kind=case["norm"]) if case["after"] else None
        y, h = mvk.block_norm(s["x"], s["stream"], before=mvk.Norm(s["weight"], s.get("bias"), kind=case["norm"]),
                              after=after, gate=s["gate"], scale=case["scale"], field_scale=scale, out=s["out"],
                              out_scale=FIELD_SCALE if case["out"] == "field" else None, residual_out=s["stream_out"])
        return {"y": y, "stream": h}
    if case["kind"] == "gated":
        return {"y": mvk.gated_activation(s["gate"], s["up"], act=case["act"], field_scale=scale, out=s["out"])}
    if case["kind"] == "sample":
        token = mvk.sample(s["logits"], s["u"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"],
                           min_p=s["min_p"], field_scale=scale, out=s["out"], probs=s["probs"])
        return {"token": token, "prob": s["probs"]}
    cache = mvk.KVCache(s["K"], s["V"], s["Ke"], s["Ve"])
    seqs = mvk.Sequences(s["table"], s["lens"], s["q_start"], max_new=s["max_new"])
    if case["kind"] == "append":
        q = mvk.rotary_append(s["q"], s["k"], s["v"], s["positions"], s["rot_table"], cache, seqs,
                              layout=case["layout"], field_scale=scale, out=s["q_out"])
        k, v = mvk.cache_read(cache, seqs, k_out=s["k_out"], v_out=s["v_out"])
        return {"q": q, "k": k, "v": v}
    if not case["weights"]:
        return {"o": mvk.paged_attention(s["q"], cache, seqs)}
    o = mvk.paged_attention(s["q"], cache, seqs, weights=s["w"], weights_out=s["w_out"])
    return {"o": o, "w": s["w_out"]}


# ---------------------------------------------------------------------------
# The same in elementary operations
# ---------------------------------------------------------------------------
def _lift(x, dtype=torch.float32):
    """Centred residues (or floats) in `dtype`."""
    if x.dtype != torch.int32:
        return x.to(dtype)
    return torch.where(x > PRIME // 2, x - PRIME, x).to(dtype) * FIELD_SCALE


def _two(e, dtype):
    """2^e, exactly."""
    return ((e.to(torch.int64) + 1023) << 52).view(torch.float64).to(dtype)


def _quantise(x, kind):
    """Rows of the last axis in 8 bits: (codes, exponents); row = codes * 2^exponent.  The exponent is the least
    in range that lets every finite value fit, the codes are nearest (ties to even)."""
    top = torch.where(x.isfinite(), x.abs(), torch.zeros_like(x)).amax(-1, keepdim=True)
    part, e = torch.frexp(top / LARGEST[kind])
    e = torch.where(part == 0.5, e - 1, e).clamp(LEAST, MOST)
    e = torch.where(top > 0, e, torch.full_like(e, LEAST))
    y = (x * _two(-e, x.dtype)).clamp(-LARGEST[kind], LARGEST[kind])
    if kind == "i8":
        return y.round().to(torch.int8), e[..., 0].to(torch.int8)
    step = torch.frexp(y).exponent.clamp(min=-5) - 4  # of the last place: 3 bits after the first, least normal 2^-6
    y = (y * _two(-step, y.dtype)).round() * _two(step, y.dtype)
    return y.to(TYPES[kind]), e[..., 0].to(torch.int8)


def _worth(codes, e, dtype=torch.float32):
    return codes.to(dtype) * _two(e[..., None], dtype)


def _rotate(x, cos, sin, rot, layout):
    """x: T x H x D; cos, sin: T x 1 x rot / 2."""
    y = x.clone()
    if layout == "half":
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        y[..., :rot // 2], y[..., rot // 2:rot] = a * cos - b * sin, b * cos + a * sin
    else:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        y[..., 0:rot:2], y[..., 1:rot:2] = a * cos - b * sin, b * cos + a * sin
    return y


def _append_plain(s):
    case, seq = s["case"], s["seq"]
    f64 = torch.float64  # codes are chosen next to borders
    rows = s["rot_table"][s["positions"].long()]
    cos, sin = rows[:, None, :case["rot"] // 2], rows[:, None, case["rot"] // 2:]
    q = _rotate(_lift(s["q"]), cos, sin, case["rot"], case["layout"])
    k = _rotate(_lift(s["k"], f64), cos.to(f64), sin.to(f64), case["rot"], case["layout"])
    new = s["q_start"][1:] - s["q_start"][:-1]
    entry = (torch.arange(len(seq), device=seq.device) - s["q_start"][seq] + (s["lens"] - new)[seq]).long()
    page, at = s["table"][seq, entry // case["page"]].long(), entry % case["page"]
    s["q_out"].copy_(q)
    for name, x in (("K", k), ("V", _lift(s["v"], f64))):
        codes, e = _quantise(x, case["cache"])
        s[name].view(torch.int8)[page, :, at] = codes.view(torch.int8)
        s[name + "e"][page, :, at] = e
        back = s[name].view(torch.int8)[page, :, at].view(codes.dtype)
        s[name.lower() + "_out"].copy_(_worth(back, s[name + "e"][page, :, at]))
    return {"q": s["q_out"], "k": s["k_out"], "v": s["v_out"]}


def _gather(pool, e, table):
    """S x Hk x (width * page) x D in 32 bits."""
    table = table.long()
    x = _worth(pool.view(torch.int8)[table].view(pool.dtype), e[table])
    return x.transpose(1, 2).flatten(2, 3)


def _attend_plain(s):
    case, q_start, lens, seq = s["case"], s["q_start"].long(), s["lens"].long(), s["seq"]
    S, hk, d, c, n = case["S"], case["kv_heads"], case["dim"], s["max_new"], s["max_len"]
    grp = case["heads"] // hk
    dev = lens.device
    new = q_start[1:] - q_start[:-1]
    i, j = torch.arange(c, device=dev), torch.arange(n, device=dev)
    width = -(-n // case["page"])
    k, v = (_gather(s[p], s[p + "e"], s["table"][:, :width])[:, :, :n] for p in ("K", "V"))
    token = (q_start[:-1, None] + i).clamp(max=len(seq) - 1)  # S x c
    q = s["q"][token].float().view(S, c, hk, grp, d).permute(0, 2, 1, 3, 4).reshape(S, hk, c * grp, d)
    x = (q @ k.transpose(2, 3)).mul_(1 / math.sqrt(d)).view(S, hk, c, grp, n)
    seen = (j <= (lens - new)[:, None, None] + i[:, None]) & (i < new[:, None])[:, :, None]  # S x c x n
    x = x.masked_fill_(~seen[:, None, :, None], -math.inf)
    top = x.amax(-1, keepdim=True)
    x = x.sub_(torch.where(top > -math.inf, top, torch.zeros_like(top))).exp_()
    x = x.div_(x.sum(-1, keepdim=True).clamp_(min=1e-30)).view(S, hk, c * grp, n)
    o = (x @ v).view(S, hk, c, grp, d).permute(0, 2, 1, 3, 4).reshape(S, c, hk * grp, d)
    tokens = torch.arange(len(seq), device=dev)
    out = {"o": o[seq, tokens - q_start[seq]].to(s["q"].dtype)}
    if case["weights"]:
        old = s["w"][:, :, :n]
        total = torch.where((j < (lens - new)[:, None])[:, None], old, torch.zeros_like(old)) + x.sum(2)
        s["w_out"][:, :, :n] = torch.where((j < lens[:, None])[:, None], total, s["w_out"][:, :, :n])
        out["w"] = s["w_out"]
    return out


def _normed(x, weight, bias, kind):
    if kind == "layer":
        x = x - x.mean(-1, keepdim=True)
    x = x * (x.square().mean(-1, keepdim=True) + 1e-6).rsqrt() * weight.to(x.dtype)
    return x if bias is None else x + bias.to(x.dtype)


def _norm_plain(s):
    case = s["case"]
    t = torch.float64 if case["out"] == "field" else torch.float32  # a field element is a rounded whole number
    x = _lift(s["x"], t)
    if case["after"]:
        x = _normed(x, s["after"], s.get("after_bias"), case["norm"])
    if s["gate"] is not None:
        x = x * s["gate"].to(t)
    h = s["stream"].to(t) + x * case["scale"]
    s["stream_out"].copy_(h)
    y = _normed(h, s["weight"], s.get("bias"), case["norm"])
    s["out"].copy_(_embed((y / FIELD_SCALE).round().to(torch.int64)) if case["out"] == "field" else y)
    return {"y": s["out"], "stream": s["stream_out"]}


def _gated_plain(s):
    x, act = _lift(s["gate"]), s["case"]["act"]
    if act == "silu":
        y = x / (1 + (-x).exp())
    elif act == "gelu":
        y = 0.5 * x * torch.erfc(x * -math.sqrt(0.5))
    elif act == "gelu_tanh":
        y = 0.5 * x * (1 + torch.tanh(math.sqrt(2 / math.pi) * (x + 0.044715 * x * x * x)))
    else:
        y = x.clamp(min=0)
    s["out"].copy_(y * _lift(s["up"]))
    return {"y": s["out"]}


def _column(v, R, dtype):
    return v.to(dtype)[:, None] if isinstance(v, torch.Tensor) else torch.full((R, 1), v, dtype=dtype, device="cuda")


def _sample_plain(s):
    case = s["case"]
    R, V, f64 = case["R"], case["V"], torch.float64  # long sums, and a border decides the token
    x = _lift(s["logits"], f64)
    t, p, least = (_column(s[k], R, f64) for k in ("temperature", "top_p", "min_p"))
    k = _column(s["top_k"], R, torch.int64)
    by, order = x.sort(dim=-1, descending=True, stable=True)
    rank = torch.arange(V, device=x.device)
    greedy = t <= 0
    w = ((by - by[:, :1]) / torch.where(greedy, torch.ones_like(t), t)).exp()
    w = torch.where(w.isnan(), torch.zeros_like(w), w)
    keep = (rank < torch.where(k > 0, k, V)) & (~greedy | (rank == 0))
    w = w * keep
    before = w.cumsum(-1) - w
    keep &= (p >= 1) | (rank == 0) | (before < p * w.sum(-1, keepdim=True))
    w = w * (keep & (w >= least))
    # in the order of the vocabulary
    w = torch.zeros_like(w).scatter_(1, order, w)
    total = w.cumsum(-1)
    want = s["u"].to(f64)[:, None] * total[:, -1:]
    token = (total <= want).sum(-1, keepdim=True).clamp(max=V - 1)
    s["out"].copy_(token[:, 0])
    s["probs"].copy_((w.gather(1, token) / total[:, -1:])[:, 0])
    return {"token": s["out"], "prob": s["probs"]}


def run(state):
    if own:
        return _run_own(state)
    return {"append": _append_plain, "attend": _attend_plain, "norm": _norm_plain, "gated": _gated_plain,
            "sample": _sample_plain}[state["case"]["kind"]](state)


# ---------------------------------------------------------------------------
# What a pass cannot do without
# ---------------------------------------------------------------------------
def work(case):
    if case["kind"] == "norm":
        T, n, p = case["T"], case["n"], SIZES[case["params"]]
        by = T * n * (SIZES[case["source"]] + 2 * SIZES[case["stream"]] + SIZES[case["out"]])
        rows = (1 + case["after"]) * (2 if case["norm"] == "layer" else 1)
        gate = {"none": 0, "channel": n, "token": T * n}[case["gate"]]
        return {"bytes": by + p * (n * rows + gate), "flops": T * n * (6 + 4 * case["after"] + (case["gate"] != "none"))}
    if case["kind"] == "gated":
        n = case["T"] * case["n"]
        return {"bytes": n * (2 * SIZES[case["source"]] + SIZES[case["out"]]), "flops": 8 * n}
    if case["kind"] == "sample":
        return {"bytes": case["R"] * (case["V"] * SIZES[case["source"]] + 12), "flops": 6 * case["R"] * case["V"]}
    pairs = _lengths(case)
    hk, h, d = case["kv_heads"], case["heads"], case["dim"]
    pages = sum(_pages([n for n, _ in pairs], case["page"]))
    T = sum(c for _, c in pairs)
    if case["kind"] == "append":
        by = T * (h + 2 * hk) * d * SIZES[case["source"]] + T * h * d * 2 + 2 * T * hk * (d * (1 + 2) + 1)
        return {"bytes": by + T * (4 * case["rot"] + 4) + 12 * case["S"], "flops": 3 * T * (h + hk) * case["rot"]}
    seen = sum(c * n - c * (c - 1) // 2 for n, c in pairs if c)
    entries = sum(n for n, c in pairs if c)
    by = 4 * T * h * d + 2 * entries * hk * (d + 1) + 4 * pages + 12 * case["S"]
    if case["weights"]:
        by += 8 * entries * hk
    return {"bytes": by, "flops": 4 * seen * h * d}


# ---------------------------------------------------------------------------
# The same values from the definitions, in 64 bits
# ---------------------------------------------------------------------------
def _number(x):
    """What x stands for, in 64 bits."""
    if x.dtype == torch.int32:
        x = x.long()
        return (x - PRIME * (2 * x > PRIME).long()).double() / 65536
    return x.double()


def _nearest(x, kind):
    """The values that rows of x are held as: the code of the table that is nearest, scaled."""
    if kind == "i8":
        table = torch.arange(-127, 128, dtype=torch.float64, device=x.device)
    else:
        table = torch.arange(256, device=x.device).to(torch.uint8).view(torch.float8_e4m3fn).double()
        table = table[table.isfinite()].unique()
    scale = torch.ones_like(x[..., :1]) * 2.0**LEAST
    top, largest = x.abs().amax(-1, keepdim=True), float(table.max())
    for e in range(LEAST + 1, MOST + 1):
        scale = torch.where(top > largest * scale, 2.0**e, scale)
    y = (x / scale).contiguous()
    hi = torch.searchsorted(table, y).clamp(1, len(table) - 1)
    below, above = table[hi - 1], table[hi]
    # a tie goes to the code whose last bit is clear: every second place of the table, counted from zero
    even = (hi - 1 - int((table == 0).nonzero()[0])) % 2 == 0
    down = (y - below < above - y) | ((y - below == above - y) & even)
    return torch.where(down, below, above) * scale


def _entries(s, name, b):
    """Hk x n x D of sequence b, in 64 bits."""
    n = int(s["lens"][b])
    rows = s["table"][b, :max(1, -(-n // s["case"]["page"]))].long()
    powers = torch.tensor([2.0**e for e in range(LEAST, MOST + 1)], dtype=torch.float64, device="cuda")
    x = s[name].view(torch.int8)[rows].view(s[name].dtype).double() * powers[s[name + "e"][rows].long() - LEAST][..., None]
    return x.transpose(0, 1).flatten(1, 2)[:, :n]


def _unit(x, weight, bias, kind):
    """A row by its length over sqrt(n), about its mean where that is asked for."""
    if kind == "layer":
        x = x - x.sum(1, keepdim=True) / x.shape[1]
    x = x / torch.sqrt((x * x).sum(1, keepdim=True) / x.shape[1] + 1e-6) * weight.double()
    return x if bias is None else x + bias.double()


def _one_token(z, k, p, least, u):
    """(token, probability) of one row of logits over temperature, from the definition."""
    order = np.lexsort((np.arange(len(z)), -z))
    if k is not None:
        order = order[:k]
    w = np.exp(z[order] - z[order[0]])
    if p < 1:
        sums = np.cumsum(w)
        order = order[:1 + int(np.count_nonzero(sums[:-1] < p * sums[-1]))]
        w = w[:len(order)]
    order = np.sort(order[w >= least])
    w = np.exp(z[order] - z.max())
    sums = np.cumsum(w)
    at = int(np.searchsorted(sums, u * sums[-1], side="right"))
    return order[min(at, len(order) - 1)], w[min(at, len(order) - 1)] / sums[-1]


def exact(case, seed):
    s = prepare(case, seed)
    f64 = torch.float64
    if case["kind"] == "norm":
        x = _number(s["x"])
        if case["after"]:
            x = _unit(x, s["after"], s.get("after_bias"), case["norm"])
        h = s["stream"].double() + case["scale"] * (x if s["gate"] is None else s["gate"].double() * x)
        y = _unit(h, s["weight"], s.get("bias"), case["norm"])
        if case["out"] == "field":
            y = (y * 65536).round().long()
            y = (y + PRIME * (y < 0).long()).to(torch.int32)
        return {"y": y, "stream": h}
    if case["kind"] == "gated":
        x, act = _number(s["gate"]), case["act"]
        if act == "silu":
            y = x * torch.sigmoid(x)
        elif act == "gelu":
            y = x * torch.special.ndtr(x)
        elif act == "gelu_tanh":
            y = x * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (x + 0.044715 * x**3))
        else:
            y = torch.relu(x)
        return {"y": y * _number(s["up"])}
    if case["kind"] == "sample":
        x, u = _number(s["logits"]).cpu().numpy(), s["u"].double().cpu().numpy()
        R = case["R"]
        t, k, p, least = (s[n].double().cpu().numpy() if isinstance(s[n], torch.Tensor) else np.full(R, float(s[n]))
                          for n in ("temperature", "top_k", "top_p", "min_p"))
        got = []
        for r in range(R):
            if t[r] <= 0:
                got.append((int(np.argmax(x[r])), 1.0))
            else:
                got.append(_one_token(x[r] / t[r], int(k[r]) if k[r] > 0 else None, p[r], least[r], u[r]))
        return {"token": _int([int(a) for a, _ in got]), "prob": torch.tensor([float(b) for _, b in got], dtype=f64)}
    starts, lens = s["q_start"].tolist(), s["lens"].tolist()
    if case["kind"] == "append":
        half, rot = case["rot"] // 2, case["rot"]
        # the rotation as a product of complex numbers
        turn = torch.complex(s["rot_table"][:, :half].double(), s["rot_table"][:, half:].double())[s["positions"].long()]

        def rotated(x):
            x = _number(x)
            by_halves = case["layout"] == "half"
            pairs = x[..., :rot].unflatten(-1, (2, half)).transpose(-1, -2) if by_halves else x[..., :rot].unflatten(-1, (half, 2))
            z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn[:, None])
            return torch.cat([(z.transpose(-1, -2) if by_halves else z).flatten(-2), x[..., rot:]], -1)

        return {"q": rotated(s["q"]), "k": _nearest(rotated(s["k"]), case["cache"]), "v": _nearest(_number(s["v"]), case["cache"])}
    h, hk, d = case["heads"], case["kv_heads"], case["dim"]
    grp = h // hk
    out = torch.zeros((starts[-1], h, d), dtype=f64, device="cuda")
    w = s["w_out"].double() if case["weights"] else None
    for b in range(case["S"]):
        n, c = lens[b], starts[b + 1] - starts[b]
        if not c or not n:
            continue
        K, V = _entries(s, "K", b), _entries(s, "V", b)
        hidden = torch.ones((c, n), dtype=torch.bool, device="cuda").triu(n - c + 1)
        if w is not None:
            w[b, :, :n - c] = s["w"][b, :, :n - c].double()
        for head in range(h):
            x = s["q"][starts[b]:starts[b + 1], head].double() @ K[head // grp].t() / math.sqrt(d)
            prob = torch.softmax(x.masked_fill_(hidden, -math.inf), -1)
            out[starts[b]:starts[b + 1], head] = prob @ V[head // grp]
            if w is not None:
                w[b, head // grp, :n] += prob.sum(0)
    return {"o": out} if w is None else {"o": out, "w": w}
