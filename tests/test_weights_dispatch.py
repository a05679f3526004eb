"""Which form of the collected weights' kernel a call launches: a workgroup's groups
of waves, which hold more of the card, only where rows of one sequence follow one
another for longer than all the work takes (the library's host side; nothing is
computed).  The sizes are those that both forms were timed at."""
from tests.test_attention_dispatch import STRUCTS
from tests.test_host_dispatch import host  # noqa: F401

FORM = """
def threads(T, count, entries, max_new, heads=32, kv_heads=8, dim=128, wide=1, page=64):
    cache, sq = kv(kv_heads, dim, 0, page), seqs(count, -(-entries // page) * wide, max_new)
    cap = sq.width * page
    q, out = rows(ptr(), 0, heads, dim), rows(ptr(), 0, heads, dim)
    call = lambda: lib.mvk_paged_attention(ref(q), T, heads, ref(cache), ref(sq), 0.1, ref(out), 1.0, None, None, ptr(),  # noqa
                                           kv_heads * cap, cap, None)
    call()
    rec.rec_reset()
    assert call() == 0 and rec.rec_count() == 2
    g = (ctypes.c_uint32 * 3)()
    rec.rec_grid(1, g)
    return g[2]
"""
# (tokens, sequences, entries of the longest, most new tokens)
SHORT = {"48 sequences of 32 new": (48 * 32, 48, 4000, 32), "a chunk beside 47 tokens": (256 + 47, 48, 4256, 256),
         "48 single tokens": (48, 48, 4000, 1), "8 sequences of 25 new": (200, 8, 4096, 25)}
LONG = {"a chunk of 256": (256, 1, 6256, 256), "a prompt of 2048": (2048, 1, 2048, 2048),
        "4 prompts of 2048": (8192, 4, 2048, 2048), "a chunk of 1000 beside 20 of 32": (1640, 21, 4000, 1000)}


def _all(host, cases, **kw):  # noqa: F811
    body = "".join(f"result[{name!r}] = threads(*{c}, **{kw})\n" for name, c in cases.items())
    return host(STRUCTS + FORM + body)


def test_short_chains(host):  # noqa: F811
    for dim in (64, 80, 128):
        for wide in (1, 4, 32):
            out = _all(host, SHORT, dim=dim, wide=wide)
            assert set(out.values()) == {256}, (dim, wide, out)


def test_long_chains(host):  # noqa: F811
    for dim in (64, 128):
        out = _all(host, LONG, dim=dim)
        assert set(out.values()) == {1024}, (dim, out)


def test_work_that_fills_the_card(host):  # noqa: F811
    cases = {"16 of 64 new": (1024, 16, 4096, 64), "16 of 512 new": (8192, 16, 4096, 512),
             "16 prompts of 2048": (16 * 2048, 16, 2048, 2048), "8 of 256 new": (2048, 8, 4096, 256)}
    assert set(_all(host, cases).values()) == {256}


def test_what_the_caller_does_not_know(host):  # noqa: F811
    """Without a bound of a sequence's new tokens they count as spread evenly."""
    cases = {"48 of 32 new": (48 * 32, 48, 4000, 48 * 32), "16 of 256 new": (4096, 16, 4096, 4096),
             "said to be one": (4096, 4, 4096, 1)}
    assert set(_all(host, cases).values()) == {256}


def test_heads_above_128(host):  # noqa: F811
    """Two groups take less memory of a compute unit there than one group's keys."""
    out = _all(host, {"48 sequences of 32 new": SHORT["48 sequences of 32 new"], **LONG}, dim=256)
    assert set(out.values()) == {512}, out
    few = {k: SHORT[k] for k in ("a chunk beside 47 tokens", "48 single tokens")}
    assert set(_all(host, few, dim=256).values()) == {256}
    wide = {"48 sequences of 32 new": SHORT["48 sequences of 32 new"]}
    assert set(_all(host, wide, dim=256, wide=32).values()) == {256}
