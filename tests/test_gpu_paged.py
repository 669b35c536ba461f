"""A cache in pages on the GPU - plan, append, attention - against plain 64-bit arithmetic (oracle/paged.py), at the sizes and values where they can go wrong."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from oracle import paged  # noqa: E402
from oracle.forward import bf16_round  # noqa: E402
from paper_2609_06172_b200 import binding as tb  # noqa: E402

DEV = "cuda:0"
HALF_BF16 = 2.0 ** -8                                      # half a step, relative to the value


def config(Hq=8, Hkv=2, Dh=64, B=2, max_len=256, TK=32):
    return tb.ModelCfg(L=1, d=Hq * Dh, Hq=Hq, Hkv=Hkv, Dh=Dh, F=1, V=1, E=0, topk=0, B=B, max_len=max_len, TK=TK, rope_base=10000.0, eps=1e-5)


def ints(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)


def f64(t):
    return t.double().cpu().numpy()


# ---- the plan of a step ----

class Server:
    """Device arrays of a plan beside the oracle's lists."""

    def __init__(self, B, P, max_len, n_pages, T, seed=0):
        order = np.random.default_rng(seed).permutation(n_pages)
        self.c, self.T, self.n_pages = config(B=B, max_len=max_len, TK=P), T, n_pages
        self.oracle = paged.Pages(B, P, max_len, n_pages, [int(p) for p in order])
        self.table, self.held, self.free, self.n_free = ints(np.full((B, self.oracle.W), -1)), ints(np.zeros(B)), ints(order), ints([n_pages])

    def step(self, length, add):
        B, T = len(length), self.T
        out = [torch.full((n + 1,), -7, dtype=torch.int32, device=DEV) for n in (B + 1, B, T, T)]
        tb.k_page_plan(ints(length), ints(add), self.table, self.held, self.free, self.n_free, *out, self.c, B, self.n_pages, T)
        got = [t.cpu().numpy() for t in out]
        want = self.oracle.plan([int(n) for n in length], [int(a) for a in add], T)
        for name, g, w in zip(("start", "end", "slot", "pos"), got, want):
            assert g[-1] == -7 and np.array_equal(g[:-1], w), (name, np.flatnonzero(g[:-1] != w)[:5])
        assert np.array_equal(self.table.cpu().numpy(), self.oracle.table())
        assert np.array_equal(self.held.cpu().numpy(), [len(x) for x in self.oracle.lists])
        assert np.array_equal(self.free.cpu().numpy(), self.oracle.behind) and int(self.n_free) == len(self.oracle.stack)
        return want


@pytest.mark.parametrize("B,P,max_len,n_pages,T", [(1, 16, 100, 3, 40), (7, 16, 200, 40, 60), (61, 32, 300, 200, 500), (300, 1, 50, 4000, 3000), (33, 48, 1000, 300, 20000), (1500, 16, 90, 3000, 9000),
                                                   (4096, 64, 64, 4000, 5000), (5, 100, 10 ** 6, 50, 70000)])
def test_plans(B, P, max_len, n_pages, T):
    """Sequences grow, are taken back, end and come, with too few pages and too few rows at times, and with lengths that make no sense."""
    rng = np.random.default_rng(B)
    s = Server(B, P, max_len, n_pages, T, seed=B)
    length, most = np.zeros(B, int), min(max_len, 4 * n_pages * P // B + 1)
    for turn in range(8):
        add = rng.integers(0, max(2, min(most, 2 * T // B)), B) * (rng.random(B) < 0.7)
        add = np.where(length + add > max_len, 0, add)
        ended = rng.random(B) < 0.15
        length, add = np.where(ended, 0, length), np.where(ended & (rng.random(B) < 0.5), 0, add)
        wrong = rng.random(B) < 0.05
        kind = rng.integers(0, 3, B)
        asked_len = np.where(wrong & (kind == 0), -5, length)
        asked_add = np.where(wrong & (kind == 1), -1, np.where(wrong & (kind == 2), 2 ** 31 - 1 if max_len < 2 ** 30 else -3, add))
        start, *_ = s.step(asked_len, asked_add)
        rows = np.diff(start)
        length = np.where(wrong, length, length + np.where(rows > 0, np.maximum(0, rows - rng.integers(0, 4, B)), 0))          # some rows are taken back
        # a sequence that was not served keeps its pages: so does its length
        length = np.where(~wrong & (rows == 0) & ended, 0, length)


def test_a_step_taken_back_leaves_the_stack():
    s = Server(20, 16, 500, 300, 2000)
    length = np.arange(20) * 7
    s.step(np.zeros(20, int), length)
    before = s.free.clone(), s.table.clone(), int(s.n_free)
    s.step(length, np.arange(20)[::-1] * 5)
    assert int(s.n_free) < before[2]
    s.step(length, np.zeros(20, int))
    assert torch.equal(s.table, before[1]) and int(s.n_free) == before[2] and torch.equal(s.free[:before[2]], before[0][:before[2]])


def test_a_plan_of_numbers_that_cannot_be():
    """What is on the device is not trusted: counts beyond the arrays write nothing outside them."""
    B, n_pages, T, W = 4, 6, 30, 8
    c = config(B=B, max_len=W * 16, TK=16)
    guard = torch.full((3, 64), -9, dtype=torch.int32, device=DEV)
    table, free = guard[0], guard[1]
    table[:B * W] = ints(np.arange(B * W) - 3)
    held, n_free = ints([2 ** 31 - 1, -2 ** 31, 9, 3]), ints([2 ** 31 - 1])
    out = [torch.zeros(n, dtype=torch.int32, device=DEV) for n in (B + 1, B, T, T)]
    tb.k_page_plan(ints([0, 5, 0, 40]), ints([0, 3, 1, 8]), table, held, free, n_free, *out, c, B, n_pages, T)
    torch.cuda.synchronize()
    assert (table[B * W:] == -9).all() and (free[n_pages:] == -9).all() and 0 <= int(n_free) <= n_pages
    slot = out[2].cpu().numpy()
    assert ((slot >= -1) & (slot < n_pages * 16)).all()


# ---- append ----

@pytest.mark.parametrize("Hq,Hkv,Dh,TK,rows", [(8, 2, 64, 16, [(1, 0)]), (8, 2, 128, 48, [(3, 30), (0, 9), (70, 0)]), (1, 1, 64, 1, [(5, 3)]), (71, 1, 64, 16, [(1, 100), (2, 15)]),
                                               (32, 8, 128, 64, [(1, p) for p in range(0, 300, 7)]), (6, 2, 128, 7, [(9, 5), (1, 6)])])
def test_append_has_the_bits_of_the_append_to_tiles(Hq, Hkv, Dh, TK, rows):
    rng = np.random.default_rng(Hq)
    end = max(p + n for n, p in rows)
    c = config(Hq, Hkv, Dh, len(rows), end, TK)
    n_pages = sum(-(-(p + n) // TK) for n, p in rows) + 2
    order = iter(rng.permutation(n_pages))
    table = [[int(next(order)) for _ in range(-(-(p + n) // TK))] for n, p in rows]
    at = [(b, p + i) for b, (n, p) in enumerate(rows) for i in range(n)]
    T = len(at) + 3                                        # three rows without a place: no slot, a position behind the model's, a slot behind the pages
    slot = [table[b][p // TK] * TK + p % TK for b, p in at] + [-1, 0, n_pages * TK]
    pos = [p for _, p in at] + [0, end, 0]
    q, k, v = (torch.randn(T, H * Dh, device=DEV) for H in (Hq, Hkv, Hkv))
    cos, sin = (torch.empty(end, Dh // 2, device=DEV) for _ in range(2))
    tb.k_rope_tables(Dh, end, 10000.0, cos, sin)
    kp, vp = (torch.full((n_pages, Hkv, TK, Dh), 7.0, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    qb = torch.full((T, Hq * Dh), 7.0, dtype=torch.bfloat16, device=DEV)
    tb.k_rope_kv_paged(q, k, v, qb, kp, vp, cos, sin, ints(slot), ints(pos), c, T, n_pages)
    want_k, want_v, want_q = torch.full_like(kp, 7.0), torch.full_like(vp, 7.0), torch.full_like(qb, 7.0)
    one = config(Hq, Hkv, Dh, 1, end, end)
    for t, (b, p) in enumerate(at):                        # row by row into a tile of all positions
        kt, vt = (torch.empty(1, Hkv, end, Dh, dtype=torch.bfloat16, device=DEV) for _ in range(2))
        tb.k_rope_kv(q[t:], k[t:], v[t:], want_q[t:], [kt], [vt], cos, sin, one, 1, 1, p)
        want_k[table[b][p // TK], :, p % TK], want_v[table[b][p // TK], :, p % TK] = kt[0, :, p], vt[0, :, p]
    assert torch.equal(kp, want_k) and torch.equal(vp, want_v) and torch.equal(qb, want_q)


# ---- attention ----

class Batch:
    """A ragged batch over pages of random values: rows [(new rows, length behind them)], unseen positions hold NaN."""

    def __init__(self, Hq, Hkv, Dh, TK, rows, seed=0, std=1.0, spare=2, max_len=None):
        rng = np.random.default_rng(seed)
        self.rows, self.B, self.T = rows, len(rows), sum(n for n, _ in rows)
        self.kv_max, self.q_max = max(max(e for _, e in rows), 1), max(max(n for n, _ in rows), 1)
        self.c = config(Hq, Hkv, Dh, self.B, max_len or self.kv_max, TK)
        W = -(-(max_len or self.kv_max) // TK)
        self.n_pages = sum(-(-e // TK) for _, e in rows) + spare
        order = iter(rng.permutation(self.n_pages))
        self.table = np.full((self.B, W), -1)
        self.k, self.v = (np.full((self.n_pages, Hkv, TK, Dh), np.nan, np.float32) for _ in range(2))
        for b, (_, e) in enumerate(rows):
            for i in range(-(-e // TK)):
                self.table[b, i] = next(order)
                used = min(TK, e - i * TK)
                self.k[self.table[b, i], :, :used], self.v[self.table[b, i], :, :used] = (bf16_round((rng.standard_normal((Hkv, used, Dh)) * std).astype(np.float32)) for _ in range(2))
        self.q = bf16_round((rng.standard_normal((self.T + 1, Hq, Dh)) * std).astype(np.float32))
        self.start = np.concatenate(([0], np.cumsum([n for n, _ in rows])))
        self.end = np.array([e for _, e in rows])

    def cache(self, b):
        """Keys and values of a sequence, [Hkv, length, Dh], and which of its positions exist."""
        e, P = self.rows[b][1], self.c.TK
        pages = self.table[b, :-(-e // P)]
        there = np.repeat((pages >= 0) & (pages < self.n_pages), P)[:e]
        pages = np.clip(pages, 0, self.n_pages - 1)
        return (*(x[pages].transpose(1, 0, 2, 3).reshape(self.c.Hkv, -1, self.c.Dh)[:, :e].astype(np.float64) for x in (self.k, self.v)), there)

    def device(self):
        to = lambda x: torch.from_numpy(x).to(DEV).bfloat16()                                          # noqa: E731
        return dict(q=to(self.q), k=to(self.k), v=to(self.v), table=ints(self.table), start=ints(self.start), end=ints(self.end))

    def scratch(self):
        n = tb.k_attn_paged_scratch_bytes(self.c, self.B, self.T, self.q_max, self.kv_max)
        t = torch.full((n + 64,), 0xff, dtype=torch.uint8, device=DEV)                                 # NaN: nothing of it is read before it is written
        t[n:] = 77                                         # nothing may be written behind it
        return t, n

    def run(self, window=0, sinks=0, dev=None, stream=None):
        d = dev or self.device()
        o = torch.full((self.T + 1, self.c.Hq * self.c.Dh), 7.0, dtype=torch.bfloat16, device=DEV)
        scratch, n = self.scratch()
        tb.k_attn_paged(d["q"], d["k"], d["v"], o, d["table"], d["start"], d["end"], self.c, self.B, self.T, self.q_max, self.kv_max, self.n_pages, window, sinks, scratch, stream)
        torch.cuda.synchronize()
        assert (scratch[n:] == 77).all() and (o[self.T] == 7).all() and tb.k_attn_status() == 0
        return f64(o[:self.T]).reshape(self.T, self.c.Hq, self.c.Dh)

    def check(self, window=0, sinks=0, got=None, some=None):
        got = self.run(window, sinks) if got is None else got
        for b, (n, e) in enumerate(self.rows):
            K, V, there = self.cache(b)
            for lo in range(0, n):
                if some and lo not in (0, n - 1) and (lo * 7919 + b) % some:
                    continue
                t = self.start[b] + lo
                want, mean, most = paged.attention(self.q[t:t + 1].astype(np.float64), K, V, e - n + lo, window, sinks, there)
                within(got[t:t + 1], want, mean, most)
        return got


def within(got, want, mean, most):
    """What attention may be off by, relative to the weighted mean of |V|: the weights' rounding to bf16 (each off by half a step, in the numerator and in the sum that divides it, where that is of the rounded
    ones), the output's (half a bf16 step of the value), the score's sum in fp32 - at most 40 additions, of which the tensor cores truncate, so a step of 2^-23 each, of the largest
    sum of |q k|, which moves a weight by as much, in the numerator and in the denominator - and 2^-20 for exponentials and the sums of the weights."""
    rel = 2 * HALF_BF16 + 2 * 40 * 2.0 ** -23 * most[..., None] + 2.0 ** -20
    tol = HALF_BF16 * np.abs(want) * (1 + rel) + rel * mean + 1e-30
    with np.errstate(invalid="ignore"):
        same = np.isfinite(want) & (np.abs(got - want) <= tol) | ~np.isfinite(want) & ((got == want) | np.isnan(got) & np.isnan(want))
    assert same.all(), (np.argwhere(~same)[:5], np.nanmax(np.abs(got - want)), np.nanmax(np.abs(got - want) / tol))


SHAPES = [(8, 2, 64, 16), (4, 4, 128, 32), (32, 8, 128, 64), (8, 1, 128, 16), (5, 1, 64, 48), (16, 1, 64, 128), (6, 2, 128, 80), (3, 3, 64, 16)]
VIEWS = [(0, 0), (1, 0), (40, 4), (17, 20), (1000, 3)]


@pytest.mark.parametrize("window,sinks", VIEWS)
@pytest.mark.parametrize("Hq,Hkv,Dh,TK", SHAPES)
def test_single_tokens(Hq, Hkv, Dh, TK, window, sinks):
    Batch(Hq, Hkv, Dh, TK, [(1, e) for e in (1, 2, 15, 16, 17, 63, 64, 65, 300, 1000)] + [(0, 50), (0, 0), (1, 129)], seed=Hq + TK).check(window, sinks)


@pytest.mark.parametrize("window,sinks", VIEWS)
@pytest.mark.parametrize("Hq,Hkv,Dh,TK", SHAPES)
def test_drafted_tokens(Hq, Hkv, Dh, TK, window, sinks):
    """Rows of one tile, of two and of the other kernel's, beside one another."""
    Batch(Hq, Hkv, Dh, TK, [(2, 2), (1, 30), (3, 200), (5, 5), (5, 77), (0, 10), (8, 64), (4, 333), (9, 40), (1, 600)], seed=Hq).check(window, sinks)


@pytest.mark.parametrize("window,sinks", VIEWS)
@pytest.mark.parametrize("Hq,Hkv,Dh,TK", SHAPES)
def test_prompts(Hq, Hkv, Dh, TK, window, sinks):
    """Whole prompts, chunks behind a cache, and single tokens beside them."""
    Batch(Hq, Hkv, Dh, TK, [(33, 33), (1, 200), (128, 128), (129, 300), (64, 1064), (0, 7), (257, 260), (1, 1)], seed=Hq).check(window, sinks, some=9)


def test_many_query_heads_of_a_kv_head():
    Batch(128, 1, 64, 16, [(1, 100), (2, 64), (1, 1)], seed=1).check()
    Batch(64, 1, 128, 16, [(1, 100), (3, 64)], seed=2).check(20, 2)
    Batch(33, 1, 64, 32, [(1, 300), (1, 64)], seed=3).check()
    Batch(200, 2, 64, 64, [(1, 70), (4, 64)], seed=4).check()


@pytest.mark.parametrize("lengths,Hq,Hkv,Dh", [([30000], 8, 2, 128), ([9, 20000, 1, 5000], 32, 8, 64), ([700] * 40, 8, 8, 128), ([16 * i + 1 for i in range(200)], 4, 1, 64)])
def test_contexts_split_over_many(lengths, Hq, Hkv, Dh):
    b = Batch(Hq, Hkv, Dh, 16, [(1, e) for e in lengths], seed=5)
    one = b.check(some=3)
    assert np.array_equal(one, b.run())                    # the same bits, whoever arrives last


@pytest.mark.parametrize("window,sinks", [(0, 0), (1000, 4)])
@pytest.mark.parametrize("rows", [[(5, 6000), (1, 3000)], [(5 if b % 3 else 1, 300 + 7 * b) for b in range(40)], [(0, 9), (4, 900), (0, 0), (8, 17)]])
def test_drafts_over_contexts_split_over_many(rows, window, sinks):
    """Stretches within a KV head's keys, short and long, and those that cross from one to the next."""
    b = Batch(32, 8, 128, 16, rows, seed=19)
    one = b.check(window, sinks, some=7)
    assert np.array_equal(one, b.run(window, sinks))


def test_more_sequences_than_a_launch_takes():
    Batch(4, 1, 64, 16, [(b % 3, 3 + b % 40) for b in range(2500)], seed=6).check(some=5)


@pytest.mark.parametrize("rows", [[(1, 300), (1, 70)], [(4, 300), (3, 70)], [(150, 300), (33, 70), (1, 129)]])
def test_missing_pages_are_not_seen(rows):
    b = Batch(8, 2, 128, 16, rows, seed=7)
    rng = np.random.default_rng(7)
    drop = rng.random(b.table.shape) < 0.4
    b.table = np.where(drop, rng.choice([-1, b.n_pages, 2 ** 31 - 1, -2 ** 31], b.table.shape), b.table)
    b.check(some=5)
    b.check(50, 3, some=5)
    b.table[:] = -1                                        # nothing is left: zeros
    assert not b.run().any() and not b.run(20, 1).any()


@pytest.mark.parametrize("rows", [[(1, 300), (1, 70)], [(4, 300), (3, 70), (2, 40)], [(150, 300), (40, 70), (1, 129)]])
def test_pages_before_a_window_are_not_read(rows):
    b = Batch(8, 2, 64, 16, rows, seed=8)
    for i, (n, e) in enumerate(rows):
        low = max(0, e - n - 30 + 1) // 16
        b.table[i, 1:low] = np.where(np.arange(1, max(low, 1)) % 2, -1, 2 ** 31 - 1)                  # page 0 holds the first positions
    got = b.run(30, 5)
    full = Batch(8, 2, 64, 16, rows, seed=8)
    full.check(30, 5, got=got, some=7)


@pytest.mark.parametrize("value", [np.nan, np.inf, -np.inf])
@pytest.mark.parametrize("Dh", [64, 128])
def test_what_is_no_number_reaches_the_rows_that_see_it_alone(value, Dh):
    """Keys and values that are no numbers, in positions that some rows of a sequence see and others do not: of drafted tokens, and of prompts."""
    for rows in ([(4, 120), (3, 40)], [(100, 160), (40, 40)]):
        for window, sinks in ((0, 0), (25, 3)):
            b = Batch(4, 2, Dh, 16, rows, seed=9)
            for i, (n, e) in enumerate(rows):
                for p in (e - 1, e - n // 2 - 1, max(0, e - n - 24)):
                    page = b.table[i, p // 16]
                    b.v[page, 0, p % 16, 5::7] = value
                    b.v[page, 1, p % 16, 3] = value
            b.check(window, sinks)
    b = Batch(4, 2, Dh, 16, [(4, 50), (60, 90)], seed=10)
    for i, p in ((0, 48), (1, 70)):
        b.k[b.table[i, p // 16], 1, p % 16, 3] = np.nan
    b.check()


def test_scores_of_minus_infinity_weigh_nothing():
    b = Batch(4, 2, 64, 16, [(1, 100), (3, 50), (70, 200), (1, 20)], seed=11)
    b.q[:, :, 0] = 1.0
    for i, (n, e) in enumerate(b.rows):
        for p in range(0, e, 2 if i < 3 else 1):           # every other key; of the last sequence every one: nothing is left
            b.k[b.table[i, p // 16], :, p % 16, 0] = -np.inf
    got = b.check()
    assert not got[b.start[3]].any()


def test_large_scores_and_equal_keys():
    b = Batch(8, 2, 64, 32, [(1, 500), (3, 100), (130, 400)], seed=12, std=8.0)
    b.check(some=11)
    b = Batch(8, 2, 128, 32, [(1, 500), (3, 100), (130, 400)], seed=13)
    b.k[~np.isnan(b.k)] = 0.0
    b.check(some=11)


def test_sequences_beyond_the_bounds_are_idle():
    """Lengths, rows and starts on the device that the call was not told of."""
    b = Batch(8, 2, 64, 16, [(1, 40), (2, 60), (3, 50), (40, 90), (1, 30)], seed=14)
    d = b.device()
    good = b.run(dev=d)
    for end in ([40, 61, 50, 90, 30], [40, -3, 50, 90, 30], [40, 1, 50, 90, 30], [40, 2 ** 31 - 1, 50, 90, 30]):
        b.kv_max = 90 if end[1] != 61 else 60
        bad = end[1] != 61
        d["end"] = ints(end if bad else [40, 61, 50, 60, 30])
        got = b.run(dev=d)
        assert not got[1:3].any() and np.array_equal(got[3:6], good[3:6])
    b.kv_max = 90
    d["end"] = ints(b.end)
    b.q_max = 39                                           # the prompt has more rows than the call says
    got = b.run(dev=d)
    assert not got[6:46].any()
    b.q_max = 40
    for start in ([0, 1, 3, 6, 47, 48], [0, 1, 3, 6, 46, 40], [-1, 1, 3, 6, 46, 47], [0, 2 ** 31 - 1, 3, 6, 46, 47]):
        d["start"] = ints(start)
        got = b.run(dev=d)
        assert np.array_equal(got[3:6], good[3:6])         # the third sequence is what it was


def test_far_pages_of_a_large_cache():
    """Byte offsets beyond 2^32: the pages in use lie at the end of the arrays."""
    b = Batch(8, 8, 128, 64, [(1, 200), (5, 100), (60, 130)], seed=15)
    shift = 40000                                          # pages of 128 KB
    d = b.device()
    for x in ("k", "v"):
        far = torch.zeros((shift + b.n_pages, *d[x].shape[1:]), dtype=torch.bfloat16, device=DEV)
        far[shift:] = d[x]
        d[x] = far
    d["table"] = torch.where(d["table"] >= 0, d["table"] + shift, d["table"])
    near = b.run()
    b.n_pages += shift
    assert np.array_equal(b.run(dev=d), near)


def test_another_stream_and_a_captured_call():
    """A captured step is replayed with other lengths, rows and pages; a second graph shares the workspace."""
    first = Batch(8, 2, 64, 16, [(2, 300), (1, 100), (40, 90), (0, 0)], seed=16, max_len=400)
    other = Batch(8, 2, 64, 16, [(1, 17), (3, 399), (0, 50), (39, 60)], seed=17, max_len=400)
    stream = torch.cuda.Stream()
    T, n_pages = 43, max(first.n_pages, other.n_pages)

    def padded(b):
        d = b.device()
        for x in ("k", "v"):
            d[x] = torch.cat((d[x], d[x].new_full((n_pages - b.n_pages, *d[x].shape[1:]), float("nan"))))
        return d

    d, e = padded(first), padded(other)
    scratch = torch.empty(tb.k_attn_paged_scratch_bytes(first.c, 4, T, 40, 400), dtype=torch.uint8, device=DEV)
    outs = [torch.zeros(T, 512, dtype=torch.bfloat16, device=DEV) for _ in range(2)]

    def call(o, window):
        tb.k_attn_paged(d["q"], d["k"], d["v"], o, d["table"], d["start"], d["end"], first.c, 4, T, 40, 400, n_pages, window, 4, scratch, stream)

    graphs = []
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        call(outs[0], 0)
        for o, window in zip(outs, (0, 50)):
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=stream):
                call(o, window)
            graphs.append(g)
    for b, source in ((first, None), (other, e), (first, padded(first))):
        if source:
            for x in d:
                d[x][:len(source[x])].copy_(source[x])
        torch.cuda.synchronize()
        for _ in range(2):
            for g in graphs:
                g.replay()
        torch.cuda.synchronize()
        for o, window in zip(outs, (0, 50)):
            b.check(window, 4, got=f64(o[:b.T]).reshape(b.T, 8, 64), some=5)


def test_a_wait_that_runs_out_ends_the_call():
    """The first tile's second V block is never loaded: the kernel returns by itself, names a wait that ran out - the roles that depend on the load (3: a load, 1: S, whose
    next keys are not asked for either, 2: P V) begin to wait within microseconds of one another - and stores nothing of that tile; the next call is right."""
    b = Batch(8, 2, 128, 64, [(64, 300)], seed=18)
    d = b.device()
    want = b.run(dev=d)
    o = torch.full((b.T, 1024), 7.0, dtype=torch.bfloat16, device=DEV)
    scratch, _ = b.scratch()
    tb.k_wait_test(2_000_000, 1)
    try:
        tb.k_attn_paged(d["q"], d["k"], d["v"], o, d["table"], d["start"], d["end"], b.c, 1, b.T, b.q_max, b.kv_max, b.n_pages, 0, 0, scratch)
        torch.cuda.synchronize()
        assert tb.k_attn_status() in (1, 2, 3)
    finally:
        tb.k_wait_test(0, 0)
        tb.k_status_clear()
    got = f64(o).reshape(b.T, 8, 128)
    assert (got[32:, :4] == 7).all() and np.array_equal(got[:32], want[:32]) and np.array_equal(got[32:, 4:], want[32:, 4:])          # (the last tile is the grid's first)
    assert np.array_equal(b.run(dev=d), want)


def test_graphs_that_share_a_scratch_and_calls_at_once():
    """Two captured calls with one scratch replayed in turn, then two streams with a scratch each at the same time."""
    batches = [Batch(8, 2, 128, 64, [(64, 300), (1, 900), (3, 77), (70, 70)], seed=20), Batch(8, 2, 128, 64, [(1, 700), (2, 90), (0, 5)], seed=21)]
    want, devs = [b.run(30, 2) for b in batches], [b.device() for b in batches]
    outs = [torch.zeros(b.T, 1024, dtype=torch.bfloat16, device=DEV) for b in batches]
    shared = max((b.scratch()[0] for b in batches), key=len)

    def call(i, scratch, stream):
        b, d = batches[i], devs[i]
        tb.k_attn_paged(d["q"], d["k"], d["v"], outs[i], d["table"], d["start"], d["end"], b.c, b.B, b.T, b.q_max, b.kv_max, b.n_pages, 30, 2, scratch, stream)

    def right():
        torch.cuda.synchronize()
        ok = [np.array_equal(f64(o).reshape(w.shape), w) for o, w in zip(outs, want)]
        for o in outs:
            o.zero_()
        torch.cuda.synchronize()
        return ok

    graphs, stream = [], torch.cuda.Stream()
    for i in range(2):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[i], stream=stream):
            call(i, shared, stream)
    for order in ((0, 1), (1, 0), (0, 0, 1, 1)):
        for i in order:
            graphs[i].replay()
        assert right() == [True, True]
    scratches, streams = [b.scratch()[0] for b in batches], [torch.cuda.Stream() for _ in batches]
    torch.cuda.synchronize()
    for turn in range(5):
        for _ in range(8):
            for i in (turn % 2, 1 - turn % 2):
                call(i, scratches[i], streams[i])
        assert right() == [True, True]
    assert tb.k_attn_status() == 0


@pytest.mark.parametrize("rows", [[(64, 300)], [(1300, 1300), (1, 40)]])
def test_a_scratch_is_good_for_the_next_call_when_a_wait_ran_out(rows):
    """Fewer tiles than the GPU takes at a time, and more: those that a CTA leaves when it gives up are counted all the same."""
    b = Batch(32, 8, 64, 64, rows, seed=22)
    d, (scratch, _) = b.device(), b.scratch()
    want, o = b.run(dev=d), torch.zeros(b.T, 2048, dtype=torch.bfloat16, device=DEV)
    call = lambda: tb.k_attn_paged(d["q"], d["k"], d["v"], o, d["table"], d["start"], d["end"], b.c, b.B, b.T, b.q_max, b.kv_max, b.n_pages, 0, 0, scratch)          # noqa: E731
    for withheld in (0, 1, 3):
        tb.k_wait_test(2_000_000, withheld)
        try:
            call()
            torch.cuda.synchronize()
            assert tb.k_attn_status() in (1, 2, 3, 4)             # (4: the warp that finds tiles waited for room for the next)
        finally:
            tb.k_wait_test(0, 0)
            tb.k_status_clear()
        for _ in range(2):
            o.zero_()
            call()
            torch.cuda.synchronize()
            assert tb.k_attn_status() == 0 and np.array_equal(f64(o).reshape(want.shape), want)


def assert_bits(got, want, rows):
    """Equal bits (in 64 bits, so NaN as NaN) of these rows, which are numbers."""
    rows = np.asarray(rows)
    assert np.isfinite(want[rows]).all() and np.array_equal(got[rows], want[rows]), np.argwhere(got[rows] != want[rows])[:5]


OF_ITS_OWN = [[(33, 300), (50, 420), (1, 200), (41, 41)], [(4, 300), (3, 170), (1, 200), (2, 900)], [(2, 40), (60, 700), (4, 90), (5, 333)], [(1, 500), (1, 90), (1, 700)]]


@pytest.mark.parametrize("window,sinks", [(0, 0), (60, 4)])
@pytest.mark.parametrize("rows", OF_ITS_OWN)
def test_a_rows_bits_do_not_depend_on_what_other_sequences_hold(rows, window, sinks):
    """Queries and values of one sequence made large or no numbers: the others, of the same lengths, keep their bits."""
    for Dh in (64, 128):
        b = Batch(8, 2, Dh, 16, rows, seed=23, std=2.0)
        want = b.run(window, sinks)
        for change in range(len(rows)):
            others = [t for i in range(len(rows)) if i != change for t in range(b.start[i], b.start[i + 1])]
            for value in (1e3, np.nan, np.inf):
                o = Batch(8, 2, Dh, 16, rows, seed=23, std=2.0)
                o.q[o.start[change]:o.start[change + 1]] *= value
                pages = o.table[change][o.table[change] >= 0]
                o.v[pages] *= value
                assert_bits(o.run(window, sinks), want, others)


@pytest.mark.parametrize("window,sinks", [(0, 0), (60, 4)])
@pytest.mark.parametrize("rows", OF_ITS_OWN)
def test_a_rows_bits_do_not_depend_on_other_queries(rows, window, sinks):
    """Of the same sequence: another token's, another head's."""
    for Dh in (64, 128):
        b = Batch(8, 2, Dh, 16, rows, seed=24, std=2.0)
        q, want = b.q.copy(), b.run(window, sinks)
        for value in (1e3, np.nan):
            b.q = q.copy()
            b.q[1::3] *= value
            assert_bits(b.run(window, sinks), want, [t for t in range(b.T) if t % 3 != 1])
            b.q = q.copy()
            b.q[:, 1::3] *= value
            assert_bits(b.run(window, sinks)[:, [0, 2, 3, 5, 6]], want[:, [0, 2, 3, 5, 6]], range(b.T))


@pytest.mark.parametrize("value", [np.nan, np.inf])
@pytest.mark.parametrize("rows", OF_ITS_OWN)
def test_a_rows_bits_do_not_depend_on_values_that_it_does_not_see(rows, value):
    """Keys and values behind a row, or before its window, that other rows of the sequence see."""
    for Dh in (64, 128):
        b = Batch(8, 2, Dh, 16, rows, seed=25, std=2.0)
        for window, sinks in ((0, 0), (60, 4)):
            want = b.run(window, sinks)
            for back in (0, 1):                                  # what the last row alone sees; with a window, what the first row alone sees
                o = Batch(8, 2, Dh, 16, rows, seed=25, std=2.0)
                keep = []
                for i, (n, e) in enumerate(rows):
                    first = e - n
                    p = first - window + 1 if back else e - 1
                    if n < 2 or (back and (not window or p < sinks)):
                        keep += range(b.start[i], b.start[i + 1])
                        continue
                    page = o.table[i, p // 16]
                    o.v[page, :, p % 16, 3::5] = value
                    o.k[page, :, p % 16, 7] = np.nan
                    keep += range(b.start[i] + 1, b.start[i + 1]) if back else range(b.start[i], b.start[i + 1] - 1)
                assert_bits(o.run(window, sinks), want, keep)


def test_a_step_of_the_engine_is_not_told_of_a_wait_over_pages():
    """A wait of the attention over pages that ran out is its caller's to see (tgp_k_attn_status): a planned pass, which has no pages, goes on."""
    import seeded_inputs as si
    from conftest import MACHINE
    from paper_2609_06172_b200.runner import Runner, pinned_pool
    from paper_2609_06172_b200.session import Session
    b = Batch(8, 2, 128, 64, [(64, 300)], seed=28)
    d, (scratch, _) = b.device(), b.scratch()
    o = torch.zeros(b.T, 1024, dtype=torch.bfloat16, device=DEV)
    tb.k_wait_test(2_000_000, 1)
    try:
        tb.k_attn_paged(d["q"], d["k"], d["v"], o, d["table"], d["start"], d["end"], b.c, 1, b.T, b.q_max, b.kv_max, b.n_pages, 0, 0, scratch)
        torch.cuda.synchronize()
    finally:
        tb.k_wait_test(0, 0)
    try:
        assert tb.k_attn_status() in (1, 2, 3)
        cfg = si.CONFIGS[1]
        lay = si.build_layout(cfg)
        pool = pinned_pool(lay.pool_bytes)
        si.fill_pool(lay, pool.numpy())
        s = Session(lay, MACHINE, pool_base=pool.data_ptr(), pool_flags=tb.POOL_PINNED)
        s.plan(T=1)
        r = Runner(s, cfg.B * cfg.S)
        assert r.step(tb.PREFILL, si.prompt_tokens(cfg), cfg.S, want_stats=True).n_launches > 0
        s.close()
        assert tb.k_attn_status() in (1, 2, 3)
    finally:
        tb.k_status_clear()


def test_large_values():
    """|V| * kv_max up to 2^88 stays finite, with scores that grow as far as they can without another reference: V times a power of two is the result times it."""
    for rise in (0.0, 10.5, 24.0):                               # times log2(e): 15.1 and 34.6; weights of 2^16 (few rows) and, over 32 keys, 2^40 (prompts) move the reference
        b = Batch(4, 2, 64, 16, [(1, 400), (3, 350), (90, 400), (1, 8)], seed=26)
        b.q[:, :, 1:] *= 0.01
        b.q[:, :, 0] = 8.0
        for i, (n, e) in enumerate(b.rows):
            for p in range(e):
                b.k[b.table[i, p // 16], :, p % 16, 0] = 0.0 if p < 64 else rise
        b.check(some=11)
        d = b.device()
        d["v"] = d["v"] * 2.0 ** 76                              # of |V| up to some 4.5 * 2^76, by 400 keys
        assert d["v"].nan_to_num(0.0).abs().max().item() * 400 <= 2.0 ** 88
        b.check(got=b.run(dev=d) * 2.0 ** -76, some=11)


@pytest.mark.parametrize("bounds", [dict(q_max=0), dict(kv_max=0), dict(q_max=0, kv_max=0)])
def test_bounds_of_nothing_leave_the_rows_as_they_are(bounds):
    b = Batch(8, 2, 64, 16, [(1, 40), (2, 60)], seed=27)
    for name, value in bounds.items():
        setattr(b, name, value)
    assert (b.run() == 7).all()
