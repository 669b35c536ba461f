"""Requests served over a cache in pages, as its operators would be used together: the plan of a step, append and attention of two layers (one with a window) that share a table, and the verification of what
a draft proposed - requests that come, are prefilled in chunks beside the others' single and drafted tokens, run out of pages, end, and leave their place to the next.  Every step is captured once and replayed,
and checked from what the GPU had before it."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from oracle import paged  # noqa: E402
from paper_2609_06172_b200 import binding as tb  # noqa: E402

DEV = "cuda:0"
HALF_BF16 = 2.0 ** -8                                      # half a step, relative to the value
B, HQ, HKV, DH, TK, MAX, T, V, D, F = 5, 8, 2, 64, 16, 200, 64, 640, 512, 768
N_PAGES, CHUNK, DRAFTS = 26, 24, 3
VIEWS = [(0, 0), (30, 4)]                                  # window and first positions of the layers


def bf16(x):
    return torch.from_numpy(np.ascontiguousarray(x)).to(DEV).bfloat16()


def ints(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)


def within(got, want, mean, most):
    """As the attention's own tests have it: weights rounded to bf16 in numerator and sum, the output's rounding, 40 additions in fp32 of a score, a step each."""
    rel = 2 * HALF_BF16 + 2 * 40 * 2.0 ** -23 * most[..., None] + 2.0 ** -20
    assert (np.abs(got - want) <= HALF_BF16 * np.abs(want) * (1 + rel) + rel * mean + 1e-30).all()


class Model:
    """Two layers, and a draft that proposes by the last token alone."""

    def __init__(self):
        rng = np.random.default_rng(4)
        self.c = tb.ModelCfg(L=2, d=D, Hq=HQ, Hkv=HKV, Dh=DH, F=F, V=V, E=0, topk=0, B=B, max_len=MAX, TK=TK, rope_base=10000.0, eps=1e-5)
        w = lambda n, k: bf16(rng.standard_normal((n, k)) * k ** -0.5)                                 # noqa: E731
        self.layers = [dict(q=w(HQ * DH, D), k=w(HKV * DH, D), v=w(HKV * DH, D), o=w(D, HQ * DH), g=w(F, D), u=w(F, D), d=w(D, F)) for _ in VIEWS]
        self.embed, self.lm, self.gain = bf16(rng.standard_normal((V, D))), w(V, D) * 2, bf16(1 + 0.1 * rng.standard_normal(D))
        self.cos, self.sin = (torch.empty(MAX, DH // 2, device=DEV) for _ in range(2))
        tb.k_rope_tables(DH, MAX, 10000.0, self.cos, self.sin)
        f, h = (lambda *s: torch.zeros(*s, device=DEV)), (lambda *s: torch.zeros(*s, dtype=torch.bfloat16, device=DEV))
        n = lambda *s: torch.zeros(*s, dtype=torch.int32, device=DEV)                                  # noqa: E731
        # what the host writes before a step
        self.length, self.add, self.tokens, self.rows, self.judged, self.u, self.u_draw = n(B), n(B), n(T), torch.zeros(T, dtype=torch.int64, device=DEV), n(B + 1), f(T), f(B)
        self.fed = n(T)
        self.temperature = f(B)
        # the cache, and what a step leaves
        self.pages = [(h(N_PAGES, HKV, TK, DH), h(N_PAGES, HKV, TK, DH)) for _ in VIEWS]
        self.table, self.held, self.free, self.n_free = torch.full((B, -(-MAX // TK)), -1, dtype=torch.int32, device=DEV), n(B), n(N_PAGES), n(1)
        self.start, self.end, self.slot, self.pos, self.out, self.n_out = n(B + 1), n(B), n(T), n(T), n(T), n(B)
        self.x, self.h, self.act, self.g32, self.u32 = f(T, D), h(T, D), h(T, F), f(T, F), f(T, F)
        self.parts = [dict(q=f(T, HQ * DH), k=f(T, HKV * DH), v=f(T, HKV * DH), qb=h(T, HQ * DH), o=h(T, HQ * DH)) for _ in VIEWS]
        self.logits, self.draft, self.drafted_from = f(T, V), f(T, V), h(T, D)
        self.attn_scratch = torch.full((tb.k_attn_paged_scratch_bytes(self.c, B, T, T, MAX),), 0xff, dtype=torch.uint8, device=DEV)
        self.verify_scratch = torch.full((tb.k_verify_scratch_bytes(T, V),), 0xff, dtype=torch.uint8, device=DEV)

    def step(self, stream=None):
        tb.k_page_plan(self.length, self.add, self.table, self.held, self.free, self.n_free, self.start, self.end, self.slot, self.pos, self.c, B, N_PAGES, T, stream)
        tb.k_embed(self.embed, self.tokens, self.x, T, D, V, stream)
        for w, p, (kp, vp), (window, sinks) in zip(self.layers, self.parts, self.pages, VIEWS):
            tb.k_rmsnorm(self.x, D, self.gain, self.h, T, D, 1e-5, stream)
            tb.k_gemm_group(self.h, [w["q"], w["k"], w["v"]], [p["q"], p["k"], p["v"]], T, [HQ * DH, HKV * DH, HKV * DH], D, [HQ * DH, HKV * DH, HKV * DH], False, stream)
            tb.k_rope_kv_paged(p["q"], p["k"], p["v"], p["qb"], kp, vp, self.cos, self.sin, self.slot, self.pos, self.c, T, N_PAGES, stream)
            tb.k_attn_paged(p["qb"], kp, vp, p["o"], self.table, self.start, self.end, self.c, B, T, CHUNK, MAX, N_PAGES, window, sinks, self.attn_scratch, stream)
            tb.k_gemm(p["o"], w["o"], self.x, T, D, HQ * DH, D, 0, True, stream)
            tb.k_rmsnorm(self.x, D, self.gain, self.h, T, D, 1e-5, stream)
            tb.k_gemm_group(self.h, [w["g"], w["u"]], [self.g32, self.u32], T, [F, F], D, [F, F], False, stream)
            tb.k_swiglu(self.g32, self.u32, self.act, T * F, stream)
            tb.k_gemm(self.act, w["d"], self.x, T, D, F, D, 0, True, stream)
        # only rows that a token is asked of, one sequence's behind the other's
        tb.k_rmsnorm(torch.index_select(self.x, 0, self.rows), D, self.gain, self.h, T, D, 1e-5, stream)
        tb.k_gemm(self.h, self.lm, self.logits, T, V, D, V, 0, False, stream)
        torch.index_select(self.embed, 0, self.fed.long(), out=self.drafted_from)
        tb.k_gemm(self.drafted_from, self.lm, self.draft, T, V, D, V, 0, False, stream)
        tb.k_verify(self.logits, self.draft, self.fed, self.judged, self.u, self.u_draw, self.out, self.n_out, B, T, V, self.temperature, self.verify_scratch, stream)

    def propose(self, token, rng, temperature):
        """What the draft draws behind a token, on the GPU."""
        out = []
        for _ in range(DRAFTS):
            logits, drawn = torch.empty(1, V, device=DEV), torch.empty(1, dtype=torch.int32, device=DEV)
            tb.k_gemm(self.embed[token:token + 1].contiguous(), self.lm, logits, 1, V, D, V, 0, False)
            tb.k_sample(logits, torch.tensor([rng.random()], device=DEV, dtype=torch.float32), drawn, 1, V, torch.tensor([temperature], device=DEV))
            token = int(drawn)
            out.append(token)
        return out


class Request:
    def __init__(self, rng, temperature):
        self.prompt, self.asks, self.t = [int(x) for x in rng.integers(0, V, rng.integers(3, 90))], int(rng.integers(4, 30)), temperature
        self.kept, self.answer, self.drafts = 0, [], True     # positions in the cache


@pytest.mark.parametrize("seed,temperatures", [(0, [0.0]), (1, [1.0, 0.7, 0.0])])
def test_requests_that_come_and_go(seed, temperatures):
    rng = np.random.default_rng(seed)
    m = Model()
    order = rng.permutation(N_PAGES)
    m.free.copy_(ints(order))
    m.n_free.fill_(N_PAGES)
    oracle = paged.Pages(B, TK, MAX, N_PAGES, [int(p) for p in order])
    waiting = [Request(rng, temperatures[i % len(temperatures)]) for i in range(9)]
    place, one = [None] * B, tb.ModelCfg(L=1, d=D, Hq=HQ, Hkv=HKV, Dh=DH, F=F, V=V, E=0, topk=0, B=1, max_len=MAX, TK=MAX, rope_base=10000.0, eps=1e-5)
    line = [[tuple(torch.zeros(1, HKV, MAX, DH, dtype=torch.bfloat16, device=DEV) for _ in range(2)) for _ in range(B)] for _ in VIEWS]          # each sequence's cache once more, in one tile
    stream, graph = torch.cuda.Stream(), None
    ended = unserved = taken = refused = 0
    for turn in range(200):
        for b in range(B):
            if place[b] is None and waiting:
                place[b] = waiting.pop()
        if not any(place):
            break
        # what each asks for: a chunk of its prompt, or its last token and what the draft proposes (after a step without pages: fewer)
        asked = []
        for b, r in enumerate(place):
            if r is None:
                asked.append([])
            elif r.kept < len(r.prompt):
                asked.append(r.prompt[r.kept:r.kept + (CHUNK if r.drafts else 1)])
            else:
                last = (r.prompt + r.answer)[-1]
                asked.append([last] + (m.propose(last, rng, r.t) if r.drafts else []))
        kept = [r.kept if r else 0 for r in place]
        start, end, slot, pos = oracle.plan(kept, [len(a) for a in asked], T)
        fed, rows, judged, tokens = [], [], [0], np.zeros(T, int)
        for b, r in enumerate(place):
            n = start[b + 1] - start[b]
            tokens[start[b]:start[b + 1]] = asked[b][:n]
            if n and kept[b] + n > len(r.prompt):            # drafts
                rows += range(start[b], start[b + 1])
                fed += asked[b]
            elif n and kept[b] + n == len(r.prompt):         # the end of a prompt
                rows.append(start[b + 1] - 1)
                fed.append(asked[b][-1])
            judged.append(len(rows))
        u, u_draw = rng.random(T).astype(np.float32), rng.random(B).astype(np.float32)
        for to, x in ((m.length, kept), (m.add, [len(a) for a in asked]), (m.tokens, tokens), (m.rows, rows + [0] * (T - len(rows))), (m.fed, fed + [0] * (T - len(fed))), (m.judged, judged),
                      (m.temperature, [r.t if r else 1.0 for r in place]), (m.u, u), (m.u_draw, u_draw)):
            to.copy_(torch.tensor(np.asarray(x)))
        if graph is None:
            state = [t.clone() for t in (m.table, m.held, m.free, m.n_free)]
            torch.cuda.synchronize()
            with torch.cuda.stream(stream):
                m.step(stream)
                for t, s in zip((m.table, m.held, m.free, m.n_free), state):
                    t.copy_(s)
                graph = torch.cuda.CUDAGraph()
                with torch.cuda.graph(graph, stream=stream):
                    m.step(stream)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert tb.k_attn_status() == 0
        # ---- the plan ----
        assert all(np.array_equal(t.cpu().numpy(), x) for t, x in ((m.start, start), (m.end, end), (m.slot, slot), (m.pos, pos), (m.table, oracle.table())))
        assert int(m.n_free) == len(oracle.stack) and np.array_equal(m.held.cpu().numpy(), [len(x) for x in oracle.lists])
        # ---- the cache and the attention of each layer ----
        for p, (kp, vp), tiles, (window, sinks) in zip(m.parts, m.pages, line, VIEWS):
            for b in range(B):
                lo, n = int(start[b]), int(start[b + 1] - start[b])
                if not n:
                    continue
                kt, vt = tiles[b]
                qb = torch.empty(n, HQ * DH, dtype=torch.bfloat16, device=DEV)
                tb.k_rope_kv(p["q"][lo:], p["k"][lo:], p["v"][lo:], qb, [kt], [vt], m.cos, m.sin, one, 1, n, kept[b])
                mine, e = torch.tensor(oracle.lists[b], device=DEV), int(end[b])
                K, W = (x[mine].transpose(0, 1).reshape(HKV, -1, DH)[:, :e] for x in (kp, vp))
                assert torch.equal(K, kt[0, :, :e]) and torch.equal(W, vt[0, :, :e]) and torch.equal(qb, p["qb"][lo:lo + n])
                f64 = lambda x: x.double().cpu().numpy()                                               # noqa: E731
                within(f64(p["o"][lo:lo + n]).reshape(n, HQ, DH), *paged.attention(f64(qb).reshape(n, HQ, DH), f64(K), f64(W), e - n, window, sinks))
        # ---- what the requests go on with ----
        x, y, got, n_got = (t.cpu().numpy() for t in (m.logits, m.draft, m.out, m.n_out))
        for b, r in enumerate(place):
            lo, hi, n = judged[b], judged[b + 1], int(start[b + 1] - start[b])
            want = paged.verify(x[lo:hi], y[lo:hi], fed[lo + 1:hi], u[lo:hi], u_draw[b], float(np.float32(r.t))) if hi > lo else []
            assert list(got[lo:hi]) == want + [-1] * (hi - lo - len(want)) and n_got[b] == len(want)
            if r is None:
                continue
            unserved += n == 0
            r.drafts = n > 0
            if kept[b] + n <= len(r.prompt):
                r.kept += n
            else:
                r.kept += int(n_got[b])
                taken, refused = taken + len(want) - 1, refused + n - len(want)
            r.answer += [int(g) for g in got[lo:lo + n_got[b]]]
            if len(r.answer) >= r.asks or r.kept + DRAFTS + 1 > MAX:
                assert all(0 <= g < V for g in r.answer)
                place[b], ended = None, ended + 1
        if not any(start[b + 1] > start[b] for b in range(B)):
            place[next(b for b in range(B) if place[b])] = None                     # all pages are held by sequences that need more: one gives up
            ended += 1
    assert ended == 9 and not waiting and taken > 0 and refused > 0 and unserved > 0
    # the last ones give their pages back
    for t in (m.length, m.add):
        t.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert int(m.n_free) == N_PAGES and sorted(m.free.cpu().tolist()) == list(range(N_PAGES)) and (m.table == -1).all()


def test_nothing_is_read_before_it_is_written():
    """Append, attention and a product in a row without a pause, over inputs that change from turn to turn: the bits of the same calls with the GPU waited for between them.  (The kernels are launched while those before
    them run: each has to wait for what it reads, the one for few rows beside the one for prompts, too.)"""
    rng = np.random.default_rng(8)
    rows = [(300, 1500), (1, 800), (1, 40), (5, 70), (0, 9), (90, 90)]
    n, P, T_, W = len(rows), 32, sum(r for r, _ in rows), 47
    c = tb.ModelCfg(L=1, d=D, Hq=HQ, Hkv=HKV, Dh=DH, F=1, V=1, E=0, topk=0, B=n, max_len=1500, TK=P, rope_base=10000.0, eps=1e-5)
    order = iter(rng.permutation(100))
    table = np.full((n, W), -1)
    for b, (_, e) in enumerate(rows):
        table[b, :-(-e // P)] = [next(order) for _ in range(-(-e // P))]
    at = [(b, e - r + i) for b, (r, e) in enumerate(rows) for i in range(r)]
    slot, pos = ints([table[b, p // P] * P + p % P for b, p in at]), ints([p for _, p in at])
    start, end = ints(np.concatenate(([0], np.cumsum([r for r, _ in rows])))), ints([e for _, e in rows])
    cos, sin = (torch.empty(1500, DH // 2, device=DEV) for _ in range(2))
    tb.k_rope_tables(DH, 1500, 10000.0, cos, sin)
    sets = [[torch.randn(T_, H * DH, device=DEV) for H in (HQ, HKV, HKV)] for _ in range(3)]
    tables = [ints(table), ints(np.where(np.arange(W) % 2, table, -1)), ints(table)]
    weight = bf16(rng.standard_normal((256, HQ * DH)) * 0.05)
    scratch = torch.empty(tb.k_attn_paged_scratch_bytes(c, n, T_, 300, 1500), dtype=torch.uint8, device=DEV)
    first = [torch.randn(100, HKV, P, DH, device=DEV).bfloat16() for _ in range(2)]

    def turns(wait):
        kp, vp = (x.clone() for x in first)
        q, k, v = (torch.empty_like(x) for x in sets[0])
        now = torch.empty_like(tables[0])
        qb, o = (torch.zeros(T_, HQ * DH, dtype=torch.bfloat16, device=DEV) for _ in range(2))
        outs = [torch.empty(T_, 256, device=DEV) for _ in range(12)]
        torch.cuda.synchronize()
        for i, out in enumerate(outs):
            for to, x in zip((q, k, v, now), (*sets[i % 3], tables[i % 3])):
                to.copy_(x)
            wait()
            tb.k_rope_kv_paged(q, k, v, qb, kp, vp, cos, sin, slot, pos, c, T_, 100)
            wait()
            tb.k_attn_paged(qb, kp, vp, o, now, start, end, c, n, T_, 300, 1500, 100, (0, 200)[i % 2], 0, scratch)
            wait()
            tb.k_gemm(o, weight, out, T_, 256, HQ * DH, 256, 0, False)
            wait()
        torch.cuda.synchronize()
        return outs

    want, got = turns(torch.cuda.synchronize), turns(lambda: None)
    assert all(torch.equal(a, b) for a, b in zip(want, got)) and not torch.equal(want[0], want[1])


def test_verification_waits_for_its_logits():
    """The same of a product, the verification of what it gives and a copy of the answer."""
    rng = np.random.default_rng(9)
    n, rows, V_ = 7, 21, 9001
    hidden = [bf16(rng.standard_normal((rows, D))) for _ in range(6)]
    weight = bf16(rng.standard_normal((V_, D)) * 0.15)
    tokens = [ints(rng.integers(0, V_, rows)) for _ in range(3)]
    starts = [ints([0, 5, 6, 9, 9, 15, 20, 21]), ints([0, 3, 6, 9, 12, 15, 18, 21])]
    us = [torch.rand(rows, device=DEV) * 0.2 for _ in range(3)]
    draws, t = torch.rand(n, device=DEV), torch.tensor([1.0, 0.7, 0.0, 1.0, 1.3, 2.0, 0.5], device=DEV)
    scratch = torch.empty(tb.k_verify_scratch_bytes(rows, V_), dtype=torch.uint8, device=DEV)

    def turns(wait):
        x, y = (torch.zeros(rows, V_, device=DEV) for _ in range(2))
        tok, start, u, out, count = torch.zeros_like(tokens[0]), torch.zeros_like(starts[0]), torch.zeros_like(us[0]), torch.zeros(rows, dtype=torch.int32, device=DEV), torch.zeros(n, dtype=torch.int32, device=DEV)
        answers = [(torch.empty_like(out), torch.empty_like(count)) for _ in range(12)]
        torch.cuda.synchronize()
        for i, (a, b) in enumerate(answers):
            for to, v in ((tok, tokens[i % 3]), (start, starts[i % 2]), (u, us[(i + 1) % 3])):
                to.copy_(v)
            wait()
            tb.k_gemm(hidden[i % 6], weight, x, rows, V_, D, V_, 0, False)
            tb.k_gemm(hidden[(i + 2) % 6], weight, y, rows, V_, D, V_, 0, False)
            wait()
            tb.k_verify(x, y if i % 4 else None, tok, start, u, draws, out, count, n, rows, V_, t, scratch)
            wait()
            a.copy_(out)
            b.copy_(count)
            wait()
        torch.cuda.synchronize()
        return answers

    want, got = turns(torch.cuda.synchronize), turns(lambda: None)
    assert all(torch.equal(a, b) for x, y in zip(want, got) for a, b in zip(x, y)) and len({tuple(a.tolist()) for a, _ in want}) > 3
