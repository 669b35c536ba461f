"""What the calls on a cache in pages and the verification of drafted tokens refuse, and the sizes they tell: decided on the host, without a GPU.  The oracle against closed forms."""
import ctypes as C

import numpy as np
import pytest

from oracle import paged
from paper_2609_06172_b200 import binding as tb

A = 4096                                                   # an address that nothing reads: every call here returns before it would


@pytest.fixture(params=["extension", "ctypes"], autouse=True)
def way(request, monkeypatch):
    """Every call both ways: through the extension, which serves integers and what has an address, and through ctypes."""
    tb.lib()
    if request.param == "ctypes":
        monkeypatch.setattr(tb, "_fast", tb._General())


def cfg(**over):
    c = dict(L=1, d=256, Hq=8, Hkv=2, Dh=64, F=1, V=1, E=0, topk=0, B=4, max_len=256, TK=32, rope_base=10000.0, eps=1e-5)
    return tb.ModelCfg(**{**c, **over})


def refused(code, f, *args, **kw):
    with pytest.raises(tb.TgpError) as e:
        f(*args, **kw)
    assert e.value.code == code, e.value


PLAN = ("length", "add", "table", "held", "free", "n_free", "start", "end", "slot", "pos")
APPEND = ("q32", "k32", "v32", "qb", "k_pages", "v_pages", "cos", "sin", "slot", "pos")
ATTN = ("qb", "k_pages", "v_pages", "ob", "table", "start", "end")
VERIFY = ("logits", "draft_logits", "tokens", "start", "u", "u_draw", "out", "n_out")


def plan(c=None, B=4, n_pages=10, T=5, **at):
    tb.k_page_plan(*(at.get(n, A) for n in PLAN), c or cfg(), B, n_pages, T)


def append(c=None, T=5, n_pages=10, **at):
    tb.k_rope_kv_paged(*(at.get(n, A) for n in APPEND), c or cfg(), T, n_pages)


def attn(c=None, B=4, T=5, q_max=2, kv_max=200, n_pages=10, window=0, sinks=0, scratch=A, **at):
    tb.k_attn_paged(*(at.get(n, A) for n in ATTN), c or cfg(), B, T, q_max, kv_max, n_pages, window, sinks, scratch)


def verify(B=4, T=5, V=100, temperature=None, scratch=A, **at):
    tb.k_verify(*(at.get(n, A) for n in VERIFY), B, T, V, temperature, scratch)


@pytest.mark.parametrize("call,names,wide", [(plan, PLAN, ()), (append, APPEND, APPEND[:8]), (attn, ATTN, ATTN[:4]), (verify, VERIFY, ())])
def test_missing_and_misaligned_arguments(call, names, wide):
    for n in names:
        if n != "draft_logits":
            refused(tb.E_INVAL, call, **{n: None})
        refused(tb.E_INVAL, call, **{n: A + 2})
        if n in wide:
            refused(tb.E_INVAL, call, **{n: A + 8})


def test_workspaces_are_needed():
    for call in (attn, verify):
        refused(tb.E_INVAL, call, scratch=None)
        refused(tb.E_INVAL, call, scratch=A + 8)
    refused(tb.E_INVAL, verify, temperature=A + 1)


def test_shapes_that_are_refused():
    for call in (append, attn):
        for bad in (dict(Dh=32), dict(Dh=96), dict(Dh=256), dict(TK=0), dict(Hkv=0), dict(Hq=7), dict(Hq=0), dict(max_len=0)):
            refused(tb.E_INVAL, call, cfg(**bad))
        refused(tb.E_INVAL, call, n_pages=0)
    refused(tb.E_INVAL, attn, cfg(TK=24))
    refused(tb.E_INVAL, attn, cfg(TK=8))
    refused(tb.E_INVAL, attn, cfg(Hq=258, Hkv=2))          # more query heads of a KV head than a tile has rows
    refused(tb.E_INVAL, attn, B=5)                         # more sequences than the model's
    refused(tb.E_INVAL, attn, kv_max=257)
    refused(tb.E_INVAL, plan, cfg(TK=0))
    refused(tb.E_INVAL, plan, cfg(max_len=0))
    refused(tb.E_INVAL, plan, B=5)
    refused(tb.E_INVAL, plan, n_pages=0)
    refused(tb.E_INVAL, verify, V=0)


def test_sizes_beyond_the_stated_ones():
    big = tb.PAGED_MAX_B + 1
    refused(tb.E_TOO_LARGE, plan, cfg(B=big), B=big)
    refused(tb.E_TOO_LARGE, attn, cfg(B=big), B=big)
    refused(tb.E_TOO_LARGE, verify, B=big)
    for call in (plan, append, attn):
        refused(tb.E_TOO_LARGE, call, n_pages=1 << 26)     # 2^31 positions
        refused(tb.E_TOO_LARGE, call, T=1 << 31)
        refused(tb.E_TOO_LARGE, call, cfg(max_len=1 << 31))
    refused(tb.E_TOO_LARGE, attn, cfg(Hkv=8), n_pages=(1 << 23))                       # rows of a head
    refused(tb.E_TOO_LARGE, attn, cfg(Hkv=8, B=1024, max_len=1 << 22), B=1024, kv_max=1 << 22)
    refused(tb.E_TOO_LARGE, verify, V=tb.SAMPLE_MAX_V + 1)
    refused(tb.E_TOO_LARGE, verify, T=32768)


def test_calls_with_nothing_to_do():
    append(T=0)
    for nothing in (dict(B=0), dict(T=0), dict(q_max=0), dict(kv_max=0)):
        attn(**nothing)
    verify(B=0)


def test_bytes_of_workspaces():
    for bad in (dict(Dh=80), dict(TK=8), dict(Hkv=3)):
        refused(tb.E_INVAL, tb.k_attn_paged_scratch_bytes, cfg(**bad), 4, 5, 2, 200)
    refused(tb.E_INVAL, tb.k_attn_paged_scratch_bytes, cfg(), 5, 5, 2, 200)
    refused(tb.E_INVAL, tb.k_attn_paged_scratch_bytes, cfg(), 4, 5, 2, 257)
    # a call of less needs no more
    c = cfg(Hq=32, Hkv=8, Dh=128, B=64, max_len=16384, TK=16)
    sizes = [tb.k_attn_paged_scratch_bytes(c, B, B * S, S, 16384) for S in (1, 4, 40) for B in (1, 3, 64)]
    assert all(s <= tb.k_attn_paged_scratch_bytes(c, 64, 64 * 40, 40, 16384) for s in sizes)
    assert tb.k_verify_scratch_bytes(0, 10) >= 16
    assert tb.k_verify_scratch_bytes(100, 128256) > tb.k_verify_scratch_bytes(99, 128256) > tb.k_verify_scratch_bytes(99, 32000)
    refused(tb.E_INVAL, tb.k_verify_scratch_bytes, 1, 0)
    refused(tb.E_TOO_LARGE, tb.k_verify_scratch_bytes, 32768, 10)
    n, l = tb._U64(), tb.lib()
    assert l.tgp_k_attn_paged_scratch_bytes(None, 1, 1, 1, 1, C.byref(n)) == l.tgp_k_attn_paged_scratch_bytes(C.byref(cfg()), 1, 1, 1, 1, None) == l.tgp_k_verify_scratch_bytes(1, 1, None) == tb.E_INVAL


def test_null_configurations():
    l = tb.lib()
    assert l.tgp_k_page_plan(*[A] * 10, None, 1, 1, 1, None) == tb.E_INVAL
    assert l.tgp_k_rope_kv_paged(*[A] * 10, None, 1, 1, None) == tb.E_INVAL
    assert l.tgp_k_attn_paged(*[A] * 7, None, 1, 1, 1, 1, 1, 0, 0, A, None) == tb.E_INVAL


def test_other_kinds_of_arguments_are_the_same_call():
    refused(tb.E_INVAL, plan, B=np.uint32(5))
    refused(tb.E_INVAL, attn, kv_max=np.int64(257))
    with pytest.raises((TypeError, C.ArgumentError)):
        attn(window=0.5)
    with pytest.raises((TypeError, C.ArgumentError)):
        tb.k_attn_paged(*[A] * 7, "cfg", 1, 1, 1, 1, 1, 0, 0, A)


# ---- the oracle against closed forms ----

def test_oracle_plan():
    p = paged.Pages(3, 4, 16, 6, [5, 4, 3, 2, 1, 0])
    start, end, slot, pos = p.plan([0, 0, 0], [5, 1, 4], 12)
    assert list(start) == [0, 5, 6, 10] and list(end) == [5, 1, 4] and p.lists == [[0, 1], [2], [3]] and p.stack == [5, 4]
    assert list(slot) == [0, 1, 2, 3, 4, 8, 12, 13, 14, 15, -1, -1] and list(pos) == [0, 1, 2, 3, 4, 0, 0, 1, 2, 3, -1, -1]
    before = [list(x) for x in p.lists], list(p.stack)
    p.plan([5, 1, 4], [4, 4, 0], 12)                       # taken ...
    assert p.lists == [[0, 1, 4], [2, 5], [3]] and p.stack == []
    p.plan([5, 1, 4], [0, 0, 0], 12)                       # ... and taken back
    assert (p.lists, p.stack) == before
    start, *_ = p.plan([5, 1, 4], [8, 4, 5], 12)           # two pages for the first, none left for the others
    assert list(start) == [0, 8, 8, 8] and p.lists == [[0, 1, 4, 5], [2], [3]]
    start, *_ = p.plan([0, 1, 4], [0, 4, 5], 8)            # the first has ended; the third's rows are too many
    assert list(start) == [0, 0, 4, 4] and p.lists == [[], [2, 0], [3]]
    start, end, *_ = p.plan([0, -1, 17], [17, 1, 0], 8)    # lengths that make no sense
    assert list(start) == [0, 0, 0, 0] and list(end) == [0, -1, 17] and p.lists == [[], [2, 0], [3]]


def test_oracle_attention():
    rng = np.random.default_rng(1)
    V = rng.standard_normal((2, 9, 64))
    o, *_ = paged.attention(rng.standard_normal((3, 4, 64)), np.ones((2, 9, 64)), V, 6, window=3, sinks=2)
    assert np.allclose(o[1, 3], V[1, [0, 1, 5, 6, 7]].mean(0)) and np.allclose(o[0, 0], V[0, [0, 1, 4, 5, 6]].mean(0))
    o, *_ = paged.attention(rng.standard_normal((1, 4, 64)), np.ones((2, 9, 64)), V, 8, there=np.arange(9) == 3)
    assert np.allclose(o[0, 0], V[0, 3])
    assert not paged.attention(rng.standard_normal((1, 4, 64)), np.ones((2, 9, 64)), V, 8, there=np.zeros(9, bool))[0].any()


def test_oracle_verification_gives_the_targets_distribution():
    """Drafted from q, verified against p: the first token is distributed as p, on a grid of random numbers."""
    p, q = np.array([0.5, 0.2, 0.3, 0.0]), np.array([0.25, 0.5, 0.125, 0.125])
    x, y = np.stack([np.log(p + 1e-300)] * 2), np.stack([np.log(q)] * 2)
    mass = np.zeros(4)
    grid = (np.arange(400) + 0.5) / 400
    for d in range(4):
        for u in grid:
            out = paged.verify(x, y, [d], [u, 0.5], 0.5)
            if len(out) == 2:
                mass[d] += q[d] / 400
            else:
                for v in (np.arange(40) + 0.5) / 40:
                    mass[paged.verify(x, y, [d], [u, 0.5], v)[0]] += q[d] / 400 / 40
    assert np.allclose(mass, p, atol=5e-3)
    assert paged.verify(x, None, [1], [0.19, 0], 0.1) == [1, 0] and paged.verify(x, None, [1], [0.21, 0], 0.1) == [0] and paged.verify(x, None, [1], [0.21, 0], 0.7) == [2]
    assert paged.verify(x, y, [0], [0, 0], 0.9, temperature=0.0) == [0, 0] and paged.verify(x, y, [1], [0, 0], 0.9, temperature=0.0) == [0]
    x[:, 3] = -np.inf
    assert paged.verify(x, x, [3], [0.5, 0], 0.9) == [2]   # nothing is left of p - p: a token of p


def test_a_row_is_one_sequences_at_most():
    """Starts of any numbers: no row is claimed twice, so no line of rows is longer than the arrays; and starts that ascend are taken as they are."""
    rng = np.random.default_rng(2)
    for T in (1, 7, 100, 32767):
        for B in (1, 2, 5, 400):
            for wild in (False, True):
                for _ in range(20):
                    start = rng.integers(0, T + 1, B + 1)
                    if wild:
                        start = np.where(rng.random(B + 1) < 0.2, rng.choice([-1, T + 1, 2 ** 31 - 1, -2 ** 31], B + 1), start)
                    used = np.zeros(T, int)
                    for first, n in paged.rows(start, T):
                        used[first:first + n] += 1
                        assert n >= 0 and (n == 0 or 0 <= first < first + n <= T)
                    assert used.max() <= 1
                    start = np.sort(rng.integers(0, T + 1, B + 1))
                    assert paged.rows(start, T) == [(s, e - s) for s, e in zip(start, start[1:])]
    assert paged.rows([0, 9, 0, 9, 0, 9], 9) == [(0, 9), (9, 0), (0, 0), (9, 0), (0, 0)]
    assert paged.rows([0, 5, 2, 7, 6, 9], 9) == [(0, 5), (5, 0), (2, 0), (7, 0), (6, 0)] and paged.rows([0, 50, 2, 7], 9) == [(0, 0), (50, 0), (2, 5)]


def test_oracle_a_row_of_nothing_takes_no_token():
    x = np.full((3, 5), -np.inf)
    x[1] = np.nan
    for t in (0.0, -1.0, np.nan, 1.0):
        for r in (0, 1):
            assert paged.verify(x[[r, 2]], None, [0], [0.0, 0.0], 0.5, t) == [0]
