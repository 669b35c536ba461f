"""Verification of drafted tokens on the GPU against plain 64-bit arithmetic (oracle/paged.py).

A weight and a sum over the vocabulary are off by some 2^-41 of themselves, a comparison or a border of the draw by little more: for the seeds here none lies so near."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from oracle import paged  # noqa: E402
from paper_2609_06172_b200 import binding as tb  # noqa: E402

DEV = "cuda:0"


def dev(x, t):
    return None if x is None else torch.from_numpy(np.ascontiguousarray(x, t)).to(DEV)


def run(x, y, tokens, start, u, u_draw, temperature=None, T=None):
    B, V = len(start) - 1, x.shape[1]
    T = len(x) if T is None else T
    out, n_out = (torch.full((n + 1,), -7, dtype=torch.int32, device=DEV) for n in (T, B))
    n = tb.k_verify_scratch_bytes(T, V)
    scratch = torch.full((n + 64,), 0xff, dtype=torch.uint8, device=DEV)
    scratch[n:] = 77
    tb.k_verify(dev(x, np.float32), dev(y, np.float32), dev(tokens, np.int32), dev(start, np.int32), dev(u, np.float32), dev(u_draw, np.float32), out, n_out, B, T, V,
                dev(temperature, np.float32), scratch)
    torch.cuda.synchronize()
    assert (scratch[n:] == 77).all() and int(out[T]) == -7 and int(n_out[B]) == -7
    return out.cpu().numpy()[:T], n_out.cpu().numpy()[:B]


def check(x, y, tokens, n, u, u_draw, temperature=None):
    """n: rows of each sequence, one behind the other; returns how many tokens each goes on with."""
    x, y = np.asarray(x, np.float32), None if y is None else np.asarray(y, np.float32)
    u, u_draw = np.asarray(u, np.float32), np.asarray(u_draw, np.float32)
    start = np.concatenate(([0], np.cumsum(n)))
    out, n_out = run(x, y, tokens, start, u, u_draw, temperature)
    for b in range(len(n)):
        lo, hi = start[b], start[b + 1]
        t = 1.0 if temperature is None else float(np.float32(temperature[b]))
        want = paged.verify(x[lo:hi], None if y is None else y[lo:hi], tokens[lo + 1:hi], u[lo:hi], u_draw[b], t) if n[b] else []
        assert list(out[lo:hi]) == want + [-1] * (n[b] - len(want)) and n_out[b] == len(want), (b, list(out[lo:hi]), want)
    assert (out[start[-1]:] == -7).all()
    return n_out


def drafts(rng, n, V, spread=2.0, away=0.5, temperature=None):
    """Logits of a target and a draft near it, and tokens drawn from the draft."""
    T = int(np.sum(n))
    x = (rng.standard_normal((T, V)) * spread).astype(np.float32)
    y = (x + rng.standard_normal((T, V)) * away).astype(np.float32)
    seq = np.repeat(np.arange(len(n)), n)
    t = np.ones(T) if temperature is None else np.asarray(temperature, float)[seq]
    drawn = [paged.draw(paged.softmax(y[r], t[r]), rng.random()) if t[r] > 0 else int(np.argmax(y[r])) for r in range(T)]
    return x, y, np.concatenate(([rng.integers(V)], drawn[:-1])).astype(np.int32) if T else np.zeros(0, np.int32)


@pytest.mark.parametrize("V", [1, 2, 31, 513, 4096, 4097, 8192, 8193, 32000, 128256])
@pytest.mark.parametrize("with_draft", [True, False])
def test_vocabularies(V, with_draft):
    rng = np.random.default_rng(V)
    n = [5, 1, 3, 2, 5, 8] if V < 10000 else [5, 1, 3]
    x, y, tokens = drafts(rng, n, V)
    check(x, y if with_draft else None, tokens, n, rng.random(len(x)), rng.random(len(n)))


@pytest.mark.parametrize("B", [1, 2, 37, 75, 150, 400])
def test_sequences_with_temperatures_of_their_own(B):
    rng = np.random.default_rng(B)
    n = rng.integers(0, 6, B)
    t = rng.choice([0.0, 0.5, 1.0, 1.7, -1.0, np.nan], B)
    x, y, tokens = drafts(rng, n, 5001, temperature=np.where(t > 0, t, 0))
    got = check(x, y, tokens, n, rng.random(len(x)), rng.random(B), t)
    assert B < 30 or (got == n).sum() and (got < n).sum()  # some drafts are taken whole, some are not


def test_flat_rows():
    """Thousands of tokens of a like weight: the sums have to be right to far beyond 32 bits."""
    rng = np.random.default_rng(3)
    n = [3] * 40
    x, y, tokens = drafts(rng, n, 50000, spread=0.1, away=0.1)
    check(x, y, tokens, n, rng.random(len(x)), rng.random(40))
    check(x, None, tokens, n, rng.random(len(x)), rng.random(40))


def test_random_numbers_at_their_ends():
    rng = np.random.default_rng(4)
    n = [4] * 8
    x, y, tokens = drafts(rng, n, 5000)
    ends = np.array([0.0, 1 - 2.0 ** -24, 1.0, -1.0, 2.0, 0.5, 1e-30, 0.25])
    for u in (0.0, 0.999, 1.0):
        check(x, y, tokens, n, np.full(32, u), ends)
        check(x, None, tokens, n, np.full(32, u), ends)
    out, n_out = run(x, y, tokens, np.arange(9) * 4, np.full(32, np.nan, np.float32), np.full(8, np.nan, np.float32))              # NaN is 0
    want = run(x, y, tokens, np.arange(9) * 4, np.zeros(32, np.float32), np.zeros(8, np.float32))
    assert np.array_equal(out, want[0]) and np.array_equal(n_out, want[1])


def test_logits_that_are_infinite_or_no_numbers():
    rng = np.random.default_rng(5)
    V, n = 6000, [4] * 9
    x, y, tokens = drafts(rng, n, V)
    x[::5, ::3] = -np.inf
    x[1::5, ::2] = np.nan
    y[2::5, 1::2] = -np.inf
    y[3::5, 5::7] = np.nan
    x[0:4] = -np.inf                                       # nothing else
    x[4:8, :] = np.nan
    y[8:12] = -np.inf                                      # a draft without a distribution: whatever the target may give is taken
    x[12:16, 77] = np.inf
    x[16:20, [5, 99, 100]] = np.inf
    y[20:24, 50] = np.inf
    x[24:28] = 3e38 * np.sign(x[24:28])
    for t in (None, np.full(9, 0.3), np.full(9, 1e-30), np.full(9, 1e30), np.full(9, np.inf), np.zeros(9)):
        for u in (0.01, 0.5):
            check(x, y, tokens, n, np.full(36, u), rng.random(9), t)
            check(x, None, tokens, n, np.full(36, u), rng.random(9), t)


def test_likeliest_tokens_of_equal_logits():
    V = 20000
    x = np.zeros((6, V), np.float32)
    x[1, [700, 9000]] = 1.0
    x[2, [9000, 15000]] = 1.0
    tokens = np.array([3, 0, 700, 9000, 15000, 0])
    check(x, None, tokens, [6], np.zeros(6), [0.5], [0.0])
    check(x, None, [3, 0, 9000, 9000, 15000, 0], [6], np.zeros(6), [0.5], [0.0])


def test_a_draft_that_is_the_target():
    """p - q is nothing: every token is taken, and where the random number says otherwise a token of p follows."""
    rng = np.random.default_rng(6)
    n = [3, 3, 4]
    x, _, tokens = drafts(rng, n, 9000, away=0.0)
    assert list(check(x, x, tokens, n, np.full(10, 0.999), rng.random(3))) == n
    check(x, x, tokens, n, np.ones(10), rng.random(3))


def test_tokens_outside_the_vocabulary_are_not_taken():
    rng = np.random.default_rng(7)
    x, y, tokens = drafts(rng, [3, 3, 3], 700)
    tokens[[1, 4, 8]] = [-1, 700, 2 ** 31 - 1]
    check(x, y, tokens, [3, 3, 3], np.zeros(9), rng.random(3))
    check(x, None, tokens, [3, 3, 3], np.zeros(9), rng.random(3))
    check(x, y, tokens, [3, 3, 3], np.zeros(9), rng.random(3), np.zeros(3))


def test_rows_that_do_not_lie_in_the_arrays():
    rng = np.random.default_rng(8)
    x, y, tokens = drafts(rng, [3, 3, 3], 700)
    u, v = rng.random(9), rng.random(3)
    good, n_good = run(x, y, tokens, [0, 3, 6, 9], u, v)
    for start, lost in (([-1, 3, 6, 9], [0]), ([0, 3, 6, 10], [2]), ([0, 3, 3, 3], [1, 2]), ([0, 3, 6, 2], [2]), ([0, 2 ** 31 - 1, 3, 6], [0, 1])):
        out, n_out = run(x, y, tokens, start, u, v)
        for b in range(3):
            rows = slice(3 * b, 3 * b + 3)
            if b in lost:
                assert n_out[b] == 0
            elif start[1] == 2 ** 31 - 1:                  # the third sequence has the rows of the second
                assert n_out[b] >= 1 and out[3] >= 0 and (out[:3] == -7).all() and (out[6:] == -7).all()
            else:
                assert n_out[b] == n_good[b] and np.array_equal(out[rows], good[rows])
        if start[1] != 2 ** 31 - 1:
            assert all((out[3 * b:3 * b + 3] == -7).all() for b in lost)


def test_a_captured_call():
    rng = np.random.default_rng(9)
    sets = []
    for n in ([5, 1, 3], [2, 2, 0], [1, 8, 0]):
        x, y, tokens = drafts(rng, n, 9001)
        pad = 9 - len(x)
        sets.append((n, *(np.concatenate((a, np.zeros((pad, *a.shape[1:]), a.dtype))) for a in (x, y, tokens)), rng.random(9).astype(np.float32), rng.random(3).astype(np.float32)))
    args = [dev(a, a.dtype) for a in sets[0][1:]]
    start, t = dev([0, 5, 6, 9], np.int32), dev([1.0, 0.7, 1.3], np.float32)
    out, n_out = torch.zeros(9, dtype=torch.int32, device=DEV), torch.zeros(3, dtype=torch.int32, device=DEV)
    scratch = torch.empty(tb.k_verify_scratch_bytes(9, 9001), dtype=torch.uint8, device=DEV)
    stream, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    call = lambda: tb.k_verify(args[0], args[1], args[2], start, args[3], args[4], out, n_out, 3, 9, 9001, t, scratch, stream)          # noqa: E731
    with torch.cuda.stream(stream):
        call()
        with torch.cuda.graph(g, stream=stream):
            call()
    for n, x, y, tokens, u, v in sets + sets[:1]:
        first = np.concatenate(([0], np.cumsum(n)))
        for to, a in zip(args, (x, y, tokens, u, v)):
            to.copy_(torch.from_numpy(a))
        start.copy_(torch.from_numpy(first.astype(np.int32)))
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        got, counts = out.cpu().numpy(), n_out.cpu().numpy()
        for b, temp in enumerate((1.0, float(np.float32(0.7)), float(np.float32(1.3)))):
            lo, hi = first[b], first[b + 1]
            want = paged.verify(x[lo:hi], y[lo:hi], tokens[lo + 1:hi], u[lo:hi], v[b], temp) if n[b] else []
            assert list(got[lo:hi]) == want + [-1] * (n[b] - len(want)) and counts[b] == len(want)


@pytest.mark.parametrize("start", [[0, 9, 0, 9, 0, 9], [0, 5, 2, 7, 6, 9], [3, 6, 0, 3, 6, 9], [0, 50, 2, 7, 7, 9], [0, 9, 9, 1, 4, 9], [-5, 4, 1, 8, 8, 8], [2, 2, 5, 4, 4, 9], [0, 3, 9, -1, 3, 9]])
def test_rows_that_several_sequences_claim(start):
    """They are the first one's: a sequence that begins before the start of one before it has none."""
    rng = np.random.default_rng(12)
    x, y, tokens = drafts(rng, [9], 5000)
    u, v, t = rng.random(9).astype(np.float32), rng.random(5).astype(np.float32), np.array([1.0, 0.0, 0.8, 1.0, 1.5], np.float32)
    for draft in (y, None):
        out, n_out = run(x, draft, tokens, start, u, v, t)
        left = np.full(9, -7)
        for b, (lo, n) in enumerate(paged.rows(start, 9)):
            rows = slice(lo, lo + n)
            want = paged.verify(x[rows], None if draft is None else y[rows], tokens[lo + 1:lo + n], u[rows], v[b], float(t[b])) if n else []
            left[lo:lo + n] = want + [-1] * (n - len(want))
            assert n_out[b] == len(want)
        assert list(out) == list(left)


@pytest.mark.parametrize("B", [255, 256, 257, 700, 2000])
def test_many_sequences_with_starts_that_fall(B):
    """Beyond one turn of the counts: sequences behind one that claims the rows to the end, or that begin before others."""
    rng = np.random.default_rng(B)
    T, V = 600, 33
    x, y, tokens = drafts(rng, [T], V)
    u, v = rng.random(T).astype(np.float32), rng.random(B).astype(np.float32)
    start = np.minimum(np.arange(B + 1) * 2 // 5, T)
    start[rng.integers(0, B, B // 9)] -= rng.integers(1, 40, B // 9)
    for start in (start, np.tile([0, T], B // 2 + 1)[:B + 1], np.where(np.arange(B + 1) == 200, T, start)):
        out, n_out = run(x, y, tokens, start, u, v)
        left = np.full(T, -7)
        for b, (lo, n) in enumerate(paged.rows(start, T)):
            rows = slice(lo, lo + n)
            want = paged.verify(x[rows], y[rows], tokens[lo + 1:lo + n], u[rows], v[b]) if n else []
            left[lo:lo + n] = want + [-1] * (n - len(want))
            assert n_out[b] == len(want)
        assert list(out) == list(left)


@pytest.mark.parametrize("t", [1e37, np.inf])
def test_an_infinite_logit_late_in_a_row_of_a_high_temperature(t):
    """More parts of rows than CTAs, so that threads meet the infinite logit behind others of its row, where a temperature's span is beyond the largest number."""
    rng = np.random.default_rng(10)
    V, n = 128256, [5] * 12
    x, y = (rng.standard_normal((60, V)).astype(np.float32) for _ in range(2))
    tokens = rng.integers(0, V, 60)
    for r in range(60):
        x[r, 4096 * (1 + 7 * r % 31) + 5 + r] = np.inf
        if r % 3 == 0:
            y[r, 4096 * (1 + 5 * r % 31) + 77] = np.inf
    tokens[1::4] = [int(np.argmax(x[r])) for r in range(0, 60, 4)]                 # some are the only ones that the target has
    got = check(x, y, tokens, n, rng.random(60), rng.random(12), np.full(12, t))
    assert (got > 1).any()
    check(x, None, tokens, n, rng.random(60), rng.random(12), np.full(12, t))


@pytest.mark.parametrize("t", [0.0, -1.0, np.nan, 1.0])
@pytest.mark.parametrize("V", [700, 9000])
def test_a_row_of_nothing_takes_no_token(V, t):
    """Not token 0 either, which is what it gives."""
    rng = np.random.default_rng(11)
    x, y, tokens = drafts(rng, [4] * 4, V)
    x[0], x[5], x[10], x[15] = -np.inf, np.nan, np.where(np.arange(V) % 2, np.nan, -np.inf), -np.inf
    for r in (0, 4, 5, 8, 9, 10):
        tokens[r + 1] = 0                                        # also behind rows that have other tokens
    x[[4, 8, 9], 0] = 50.0                                       # there it is the likeliest
    for draft in (y, None):
        got = check(x, draft, tokens, [4] * 4, np.zeros(16), rng.random(4), np.full(4, t))
        assert list(got[:3]) == [1, 2, 3]


@pytest.mark.parametrize("V", [300, 5000])
@pytest.mark.parametrize("t", [1.0, 0.0])
def test_long_drafts(V, t):
    """Rows are judged 32 at a time: first refusals in the first, second and third turn, at their ends, and none."""
    rng = np.random.default_rng(13)
    stop = {70: 64, 40: 35, 33: None, 32: 30, 31: None, 34: 32, 65: None, 100: 31, 97: 95, 64: 63}
    n = list(stop)
    x, _, tokens = drafts(rng, n, V, away=0.0, temperature=np.full(len(n), t))
    y, start = x.copy(), np.concatenate(([0], np.cumsum(n)))
    for lo, (rows, i) in zip(start, stop.items()):
        if i is not None and i + 1 < rows:
            x[lo + i, tokens[lo + i + 1]] = -np.inf
    for draft in (y, None) if t == 0 else (y,):
        got = check(x, draft, tokens, n, np.full(len(x), 0.9), rng.random(len(n)), np.full(len(n), t))
        assert list(got) == [rows if i is None or i + 1 == rows else i + 1 for rows, i in stop.items()]
